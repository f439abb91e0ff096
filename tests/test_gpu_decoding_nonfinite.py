"""GPU: infinities and NaN in the operators of a decoding batch and in the split-key forward beside them. What a query, or a key that it
sees, makes NaN in a row's softmax stays NaN in the result: no share of the keys drops out silently, and rows that do not see it keep
their values. And verification of drafts at inverse temperatures from the smallest to the largest float32."""
import numpy as np
import pytest

from paper_2307_08691_amd import binding
from oracle import decoding_oracle as dec
from test_gpu_decoding import TYPES, Cache, check_verify, distributions, f64, gpu, ints, rng

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


class Prefix:
    """A call of fa_prefix_fwd whose inputs can be spoiled."""

    def __init__(self, dtype, d, B, nq, hq, hkv, n_p, slots, lens, page=0, seed=0):
        r = rng(seed + d + n_p)
        self.cache = Cache(r, dtype, B, slots, hkv, d, page, lens)
        self.Q = gpu(r.normal(size=(B, nq, hq, d)), TYPES[dtype])
        self.Kp, self.Vp = (gpu(r.normal(size=(n_p, hkv, d)), TYPES[dtype]) for _ in range(2))
        self.lens, self.d, self.G = lens, d, hq // hkv

    def __call__(self, causal=True):
        O, L = binding.fa_prefix_fwd(self.Q, self.Kp, self.Vp, self.cache.K, self.cache.V, self.d**-0.5, causal, seqlens_k=ints(self.lens),
                                     block_table=self.cache.table)
        torch.cuda.synchronize()
        return O, L.transpose(1, 2)  # [B, Nq, Hq, d], [B, Nq, Hq]

    def sizes(self):
        """sum_c p_c |v_c|"""
        values, self.Vp, self.cache.V = (self.Vp, self.cache.V), self.Vp.abs(), self.cache.V.abs()
        O, _ = self()
        self.Vp, self.cache.V = values
        return O


def same_but(got, clean, size, spoiled, apart):
    """Rows `spoiled` [B, Nq, Hq] are NaN throughout, rows `apart` from them (other heads or sequences, which no workgroup has together
    with a spoiled one) keep their bits. The rest may take their exponentials against another reference: P is rounded anew (e of every p |v|,
    whose sum `size` is, half precision's subnormal P by up to 2^-25 of the row's largest), O too, the exponentials' arguments in float32."""
    e, (O, L), (cO, cL) = torch.finfo(clean[0].dtype).eps / 2, got, clean
    assert O[spoiled].isnan().all() and L[spoiled].isnan().all()
    assert torch.equal(O[apart], cO[apart]) and torch.equal(L[apart], cL[apart])
    rest = ~spoiled
    O, cO, size = (x[rest].double() for x in (O, cO, size))
    small = 4096 * 5.0 / 2**25 if e < 2**-8 else 0.0  # (at most 4096 keys, |v| below 5)
    assert ((O - cO).abs() <= 3 * e * (size + cO.abs()) + small).all()
    assert ((L - cL)[rest].abs() <= 5e-5).all()


# rows of a head: one narrow item, wide items with rows of several sequences, wide own items; several shares of the prefix
SHAPES = [(2, 1, 8, 2, 3000, 200, [200, 70]), (40, 1, 8, 2, 3000, 100, [100, 1] * 20), (2, 70, 4, 2, 1500, 300, [300, 150])]


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f16", 128), ("bf16", 128), ("f16", 64)])
@pytest.mark.parametrize("B,nq,hq,hkv,n_p,slots,lens", SHAPES)
def test_prefix_keys_that_are_nan(dtype, d, B, nq, hq, hkv, n_p, slots, lens):
    p = Prefix(dtype, d, B, nq, hq, hkv, n_p, slots, lens)
    clean, size = p(), p.sizes()
    head = torch.arange(hq, device="cuda").expand(B, nq, hq) // p.G
    for key in (0, 777, n_p - 1):  # one key of the prefix, in one head: all rows of that head's group
        x = p.Kp[key, hkv - 1].clone()
        p.Kp[key, hkv - 1, 3] = NAN
        same_but(p(), clean, size, head == hkv - 1, head != hkv - 1)
        p.Kp[key, hkv - 1] = x
    # an own key: the rows of its sequence that see it
    n = lens[1]
    for key in (0, n - 1):
        x = p.cache.K[1, key, 0].clone()
        p.cache.K[1, key, 0, d - 1] = NAN
        r = torch.arange(nq, device="cuda")[None, :, None]
        seq = torch.arange(B, device="cuda")[:, None, None]
        same_but(p(), clean, size, (head == 0) & (seq == 1) & (r + n - nq >= key), (head != 0) | (seq != 1))
        p.cache.K[1, key, 0] = x
    # a query: its row alone
    p.Q[1, nq - 1, 1, 5] = NAN
    row = torch.zeros((B, nq, hq), dtype=torch.bool, device="cuda")
    row[1, nq - 1, 1] = True
    same_but(p(), clean, size, row, head != 0)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("B,nq,hq,hkv,n_p,slots,lens", SHAPES)
def test_prefix_keys_that_are_infinite(dtype, B, nq, hq, hkv, n_p, slots, lens):
    """A key with one infinite element scores +inf or -inf by the query's sign there: the first makes the row NaN, the second is a weight of 0."""
    d = 64
    p = Prefix(dtype, d, B, nq, hq, hkv, n_p, slots, lens)
    clean = p()
    key, g = 1234, 1
    p.Kp[key, g, 7] = INF
    O, L = p()
    head = torch.arange(hq, device="cuda").expand(B, nq, hq) // p.G
    up = (head == g) & (p.Q[..., 7] > 0)
    assert torch.equal(O[head != g], clean[0][head != g]) and torch.equal(L[head != g], clean[1][head != g])
    assert O[up].isnan().all() and L[up].isnan().all()
    # the others: as if the key were not there (bounds as for finite inputs)
    keep = [i for i in range(n_p) if i != key]
    eO, eL, A, M = dec.prefix_forward(f64(p.Q), f64(p.Kp)[keep], f64(p.Vp)[keep], *p.cache.rows, lens, d**-0.5, True)
    eL, M = eL.transpose(0, 2, 1), M.transpose(0, 2, 1)
    down = ((head == g) & (p.Q[..., 7] < 0)).cpu().numpy()
    e = torch.finfo(TYPES[dtype]).eps / 2
    score = M * d / 2**24 + (M + np.abs(eL) + 8) / 2**21
    assert down.any() and (np.abs(f64(L) - eL)[down] <= score[down]).all()
    small = (n_p + slots) * 4.0 / 2**25 if dtype == "f16" else 0.0
    tol = e * (A + np.abs(eO)) * (1 + 2 * e) + A * 4 * score[..., None] + small
    assert (np.abs(f64(O) - eO)[down] <= tol[down]).all()


def test_prefix_of_nan_queries_alone():
    """A row that is NaN in every share, one of them empty; shares beyond those that the merge holds at once (more than 17)."""
    for n_p, slots, lens in ((3000, 64, [0]), (5000, 2000, [2000]), (0, 64, [64])):
        p = Prefix("bf16", 64, 1, 1, 2, 1, n_p, slots, lens)
        clean, size = p(), p.sizes()
        p.Q[0, 0, 1] = NAN
        row = torch.tensor([[[False, True]]], device="cuda")
        same_but(p(), clean, size, row, torch.zeros_like(row))


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f16", 128)])
@pytest.mark.parametrize("nq,splits", [(1, 1), (1, 4), (1, 11), (40, 1), (40, 4)])  # few rows, and blocks of them; the result itself, and shares
def test_split_keys_that_are_nan(dtype, d, nq, splits):
    r = rng(nq + splits)
    B, hq, hkv, n = 2, 4, 2, 1500
    Q = gpu(r.normal(size=(B, nq, hq, d)), TYPES[dtype])
    K, V = (gpu(r.normal(size=(B, n, hkv, d)), TYPES[dtype]) for _ in range(2))

    def call(V=V):
        O, L = binding.fa_kvcache_fwd(Q, K, V, d**-0.5, True, seqlens_k=ints([n, n - 300]), num_splits=splits)
        torch.cuda.synchronize()
        return O, L.transpose(1, 2)

    clean, size = call(), call(V.abs())[0]
    head = torch.arange(hq, device="cuda").expand(B, nq, hq) // (hq // hkv)
    seq = torch.arange(B, device="cuda")[:, None, None]
    for key in (0, 800):
        x = K[1, key, 0].clone()
        K[1, key, 0, 9] = NAN
        same_but(call(), clean, size, (head == 0) & (seq == 1), (head != 0) | (seq != 1))
        K[1, key, 0] = x
    Q[0, nq - 1, 3, 0] = NAN
    row = torch.zeros((B, nq, hq), dtype=torch.bool, device="cuda")
    row[0, nq - 1, 3] = True
    same_but(call(), clean, size, row, (head != 1) | (seq != 0))


@pytest.mark.parametrize("nq,hq", [(2, 4), (60, 4), (300, 4)])  # rows in registers, in LDS, streaming
@pytest.mark.parametrize("causal", [False, True])
def test_weights_rows_without_a_logsumexp_add_nothing(nq, hq, causal):
    """LSE = -inf takes a row out, whatever its query holds."""
    r = rng(nq)
    K = gpu(r.normal(size=(2, 500, 2, 64)), torch.bfloat16)
    Q = gpu(r.normal(size=(2, nq, hq, 64)), torch.bfloat16)
    _, L = binding.fa_kvcache_fwd(Q, K, K, 0.125, causal)
    out = rng(1).random((2, hq, nq)) < 0.3
    out[0, 1, nq // 2] = True
    L[torch.from_numpy(out).cuda()] = -INF
    want = torch.zeros((2, 2, 500), device="cuda")
    binding.fa_cache_weights(Q, K, L, want, 0.125, causal)
    for bad in (NAN, INF):
        Q[torch.from_numpy(out).cuda().transpose(1, 2)] = bad
        W = torch.zeros_like(want)
        binding.fa_cache_weights(Q, K, L, W, 0.125, causal)
        assert want.isfinite().all() and torch.equal(W, want)


@pytest.mark.parametrize("inv_t", [1e-42, 1e-30, 1e3, 1e6, 1e14, 1e16, 1e18, 1e20, 2.4e38, float(np.finfo(np.float32).max)])
@pytest.mark.parametrize("q_type", [torch.float32, None])
def test_verify_extreme_temperatures(inv_t, q_type):
    """From even to the largest logit alone (how greedy decoding is asked for): two equal largest ones share the draw, -inf stays out."""
    r = rng(31)
    l, q, drafts = distributions(r, 12, 3, 9000)
    l[:, :, ::7] = -np.inf
    top = l.max(-1) + 0.5
    for i in (1000, 8001):
        np.put_along_axis(l, np.full((12, 4, 1), i), top[..., None], 2)
    l[3, 0] = -np.inf
    l[4] += 1e4  # (far from 0)
    drafts[:6, 0], drafts[::2, 1] = 1000, 8001
    u = r.random((12, 4)).astype(np.float32)
    for type_ in (torch.float32, torch.bfloat16):
        check_verify(drafts, None if q_type is None else q, l, u, True, inv_t, q_type, type_)
