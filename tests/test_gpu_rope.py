"""GPU parity of fa_rope_fwd and fa_rope_bwd against the definition, angles as exact products: one axis and several, both ways of pairing,
every width that the kernel moves at once, channels that pass through, slices, far and negative positions, in place, packed.

Tolerances: sine and cosine rounded to float32 and two float32 roundings (4 2^-24 of |x1| + |x2| together), then the type's own rounding, half a
step of |y| (half precision: 2^-25 where it is subnormal)."""
import numpy as np
import pytest

from oracle import qcache_oracle as orc
from paper_2307_08691_amd import binding

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from qcaches import TYPES, f64, gpu, ints  # noqa: E402


def frequencies(n):
    return (10000.0**(-np.arange(n) / n)).astype(np.float32)


def bound(x, y, pairs, neighbours, dtype):
    first = np.arange(pairs) * (2 if neighbours else 1)
    second = first + (1 if neighbours else pairs)
    size = np.zeros(x.shape)
    size[..., first] = size[..., second] = np.abs(x[..., first]) + np.abs(x[..., second])
    e = torch.finfo(TYPES[dtype]).eps / 2
    return 4 * size / 2**24 + e * np.abs(y) * (1 + 2**-10) + (2.0**-25 if dtype == "f16" else 0.0) * (size > 0)


def check(dtype, B, N, hq, hkv, d, pairs, axes, neighbours, inverse=False, fused=False, far=100, out=None, seed=0):
    r = np.random.default_rng(seed + d + pairs + N)
    heads = hq + hkv
    X = gpu(r.normal(size=(B, N, heads, d)), TYPES[dtype])
    Q, K = X[:, :, :hq], X[:, :, hq:]
    if not fused:
        Q, K = Q.contiguous(), K.contiguous()
    if not hkv:
        K = None
    pos = r.integers(-far, far + 1, size=(axes, B, N))
    axis = r.integers(0, axes, size=pairs)
    f = frequencies(pairs)
    call = binding.fa_rope_bwd if inverse else binding.fa_rope_fwd
    p = ints(pos.tolist())
    Qo, Ko = call(Q, K, p[0] if axes == 1 else p, gpu(f), None if axes == 1 else ints(axis.tolist()), neighbours)
    for x, y in ((Q, Qo), (K, Ko)):
        if x is None:
            assert y is None
            continue
        x, y = f64(x), f64(y)
        want = orc.rotate(x, pos, f, axis, neighbours, inverse)
        assert (np.abs(y - want) <= bound(x, want, pairs, neighbours, dtype)).all()
        assert np.array_equal(y[..., 2 * pairs:], x[..., 2 * pairs:])
    return Qo, Ko


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("neighbours", [False, True])
@pytest.mark.parametrize("B,N,hq,hkv,d,pairs,axes", [
    (1, 1, 1, 0, 8, 1, 1),      # the smallest call: one pair, elements one by one
    (2, 3, 4, 2, 64, 32, 1),
    (1, 5, 5, 1, 128, 64, 3),
    (3, 2, 2, 2, 72, 36, 2),    # four at once
    (2, 2, 3, 1, 72, 18, 2),    # two at once, half of the channels pass through
    (1, 7, 3, 3, 96, 17, 4),    # an odd number of pairs
    (2, 1, 32, 8, 256, 128, 3),
    (1, 2, 1, 1, 256, 40, 1),
])
def test_rotation(dtype, neighbours, B, N, hq, hkv, d, pairs, axes):
    for inverse in (False, True):
        for fused in (False, True):
            check(dtype, B, N, hq, hkv, d, pairs, axes, neighbours, inverse, fused)


@pytest.mark.parametrize("far", [10**6, 2**31 - 1])
def test_far_positions(far):
    check("f32", 2, 9, 2, 1, 64, 32, 2, False, far=far)
    check("f32", 2, 9, 2, 1, 64, 32, 1, True, inverse=True, far=far)


def test_axes_that_are_none_read_no_other_memory():
    X = gpu(np.random.default_rng(1).normal(size=(1, 4, 2, 16)).astype(np.float32))
    pos, f = ints([[[1, 2, 3, 4]], [[5, 6, 7, 8]]]), gpu(frequencies(8))
    a = binding.fa_rope_fwd(X, None, pos, f, ints([-3, 0, 1, 2, 99, 1, 0, 2**31 - 1]))[0]
    assert torch.equal(a, binding.fa_rope_fwd(X, None, pos, f, ints([0, 0, 1, 1, 1, 1, 0, 1]))[0])


@pytest.mark.parametrize("neighbours", [False, True])
def test_in_place_into_slices_packed_and_shared_positions(neighbours):
    r = np.random.default_rng(2)
    X = gpu(r.normal(size=(2, 6, 9, 64)), torch.bfloat16)
    pos, f = ints(r.integers(0, 99, size=(2, 1, 6)).tolist()), gpu(frequencies(24))
    axis = ints([0] * 10 + [1] * 14)
    shared = pos.expand(2, 2, 6)  # (the same positions for both sequences)
    want = binding.fa_rope_fwd(X[:, :, :4].contiguous(), X[:, :, 4:6].contiguous(), shared.contiguous(), f, axis, neighbours)
    got = binding.fa_rope_fwd(X[:, :, :4], X[:, :, 4:6], shared, f, axis, neighbours)
    assert all(torch.equal(a, b) and a.is_contiguous() for a, b in zip(got, want))
    flat = binding.fa_rope_fwd(X[1, :, :4], X[1, :, 4:6], pos[:, 0], f, axis, neighbours)
    assert all(torch.equal(a, b[1]) for a, b in zip(flat, want))
    wide = torch.zeros(2, 6, 9, 64, dtype=torch.bfloat16, device="cuda")
    q, k = binding.fa_rope_fwd(X[:, :, :4], X[:, :, 4:6], shared, f, axis, neighbours, Qout=wide[:, :, 5:], Kout=wide[:, :, 1:3])
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and (wide[:, :, [0, 3, 4]] == 0).all()
    x = X.clone()
    q, k = binding.fa_rope_fwd(x[:, :, :4], x[:, :, 4:6], shared, f, axis, neighbours, Qout=x[:, :, :4], Kout=x[:, :, 4:6])
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(x[:, :, 6:], X[:, :, 6:])


def test_slices_that_are_not_aligned():
    """Rows that begin at odd elements: moved one by one, with the same results."""
    X = gpu(np.random.default_rng(3).normal(size=(2, 3, 5, 73)), torch.float16)
    pos, f = ints([[1, 2, 3], [4, 5, 6]]), gpu(frequencies(32))
    want = binding.fa_rope_fwd(X[..., 1:65].contiguous(), None, pos, f)[0]
    assert torch.equal(binding.fa_rope_fwd(X[..., 1:65], None, pos, f)[0], want)


def test_gradient_of_a_rotation_of_learned_tensors():
    """<w, rotate(x)> in float32: its gradient is fa_rope_bwd of w, against differences (the rotation is linear: a step of 1/2 has no error of
    its own; the sums of 64 products round by 2^-18 at most)."""
    r = np.random.default_rng(4)
    x, w = (gpu(r.normal(size=(1, 2, 1, 32)).astype(np.float32)) for _ in range(2))
    pos, f, axis = ints([[[3, 70]], [[1, 9]]]), gpu(frequencies(16)), ints([0, 1] * 8)
    for neighbours in (False, True):
        g = binding.fa_rope_bwd(w, None, pos, f, axis, neighbours)[0]
        y = binding.fa_rope_fwd(x, None, pos, f, axis, neighbours)[0].double()
        for i in range(2):
            for t in range(32):
                z = x.clone()
                z[0, i, 0, t] += 0.5
                d = (w.double() * (binding.fa_rope_fwd(z, None, pos, f, axis, neighbours)[0].double() - y)).sum() / 0.5
                assert abs(float(d) - float(g[0, i, 0, t])) < 2**-16


def test_more_tokens_than_workgroups_and_elements_past_31_bits():
    """2^20 + 5 packed tokens of 33 heads of 64 in place: as the same tokens by themselves."""
    T, f = 2**20 + 5, gpu(frequencies(32))
    X = torch.zeros(T, 33, 64, dtype=torch.bfloat16, device="cuda")
    pos = torch.arange(T, dtype=torch.int32, device="cuda")
    at = torch.tensor([0, 1, 7, 2**20 - 1, 2**20, 2**20 + 4], device="cuda")
    X[at] = gpu(np.random.default_rng(5).normal(size=(6, 33, 64)), torch.bfloat16)
    want = binding.fa_rope_fwd(X[at], None, pos[at], f)[0]
    got = binding.fa_rope_fwd(X, None, pos, f, Qout=X)[0]
    assert got is X and torch.equal(X[at], want)
    X[at] = 0
    assert not X.any()
