"""The definitions of caches in 4 or 8 bits and of rotary positions against brute force and what follows from them."""
import numpy as np
import pytest

from oracle import qcache_oracle as orc


@pytest.mark.parametrize("bits", [4, 8])
def test_every_value_goes_to_the_nearest_element_of_the_smallest_scale_that_fits(bits):
    r = np.random.default_rng(bits)
    x = r.normal(size=(200, 64)) * np.exp2(r.integers(-60, 60, size=(200, 1)))
    x[0], x[1, :32], x[2, 5] = 0, 1e-45, 7.0
    codes, scales = orc.quantise(x, bits)
    y = orc.values(codes, scales, bits)
    g = orc.grid(bits)
    both = np.concatenate([-g[::-1], g])
    for i in range(len(x)):
        for b in range(2):
            v, s = x[i, 32 * b:32 * b + 32], 2.0**(int(scales[i, b]) - 127)
            top = np.abs(v).max()
            assert top <= orc.LARGEST[bits] * s
            assert scales[i, b] == 16 or top > orc.LARGEST[bits] * s / 2
            near = np.abs(both[None] * s - v[:, None]).min(1)
            assert (np.abs(y[i, 32 * b:32 * b + 32] - v) <= near).all()


@pytest.mark.parametrize("bits", [4, 8])
def test_halves_go_to_even_codes_and_elements_stay(bits):
    g = orc.grid(bits)
    block = np.zeros(32)
    for k in range(len(g)):
        block[:] = 0
        block[0], block[1], block[2] = g[-1], g[k], -g[k]  # (the largest element: the scale is 1)
        codes, scales = orc.quantise(block, bits)
        assert scales[0] == 127 and (codes[:3] == [len(g) - 1, k, k + (8 if bits == 4 else 128)]).all()
        if k + 1 < len(g):
            block[1] = (g[k] + g[k + 1]) / 2
            assert orc.quantise(block, bits)[0][1] == k + k % 2


@pytest.mark.parametrize("bits", [4, 8])
@pytest.mark.parametrize("bad", [np.inf, -np.inf, np.nan])
def test_a_block_with_something_that_is_no_number_is_none(bits, bad):
    x = np.ones((2, 64))
    x[1, 40] = bad
    codes, scales = orc.quantise(x, bits)
    assert scales.tolist() == [[scales[0, 0]] * 2, [scales[0, 0], 255]] and (codes[1, 32:] == 0).all()
    assert np.isnan(orc.values(codes, scales, bits)[1, 32:]).all() and (orc.values(codes, scales, bits)[:, :32] == 1).all()


def test_packing():
    codes, _ = orc.quantise(np.arange(-16.0, 16.0), 4)
    p = orc.packed(codes, 4)
    assert p.shape == (16,) and ((p & 15) == codes[0::2]).all() and ((p >> 4) == codes[1::2]).all()


@pytest.mark.parametrize("neighbours", [False, True])
def test_rotation(neighbours):
    r = np.random.default_rng(3)
    x, pos = r.normal(size=(2, 3, 2, 24)), r.integers(-50, 50, size=(3, 2, 3))
    f, axis = np.float32(10.0)**-np.arange(8, dtype=np.float32), r.integers(0, 3, size=8)
    y = orc.rotate(x, pos, f, axis, neighbours)
    assert np.allclose((y**2).sum(-1), (x**2).sum(-1)) and (y[..., 16:] == x[..., 16:]).all()
    assert np.allclose(orc.rotate(y, pos, f, axis, neighbours, inverse=True), x)
    assert np.allclose(orc.rotate(x, 0 * pos, f, axis, neighbours), x)
    # products of queries and keys go by the difference of their positions alone
    q, k = r.normal(size=(1, 1, 1, 16)), r.normal(size=(1, 1, 1, 16))
    dot = lambda a, b: (orc.rotate(q, np.full((3, 1, 1), a), f, axis, neighbours) * orc.rotate(k, np.full((3, 1, 1), b), f, axis, neighbours)).sum()  # noqa: E731
    assert np.isclose(dot(7, 3), dot(1007, 1003))
    # the gradient of <w, rotate(x)> is the rotation of w by the opposite angle: against differences (the rotation is linear: any step will do)
    w, g = r.normal(size=x.shape), np.zeros(x.shape)
    for at in np.ndindex(*x.shape):
        z = x.copy()
        z[at] += 0.5
        g[at] = (w * (orc.rotate(z, pos, f, axis, neighbours) - y)).sum() / 0.5
    assert np.allclose(g, orc.rotate(w, pos, f, axis, neighbours, inverse=True))


def test_far_positions_lose_nothing():
    x = np.zeros((1, 1, 1, 2))
    x[..., 0] = 1
    y = orc.rotate(x, np.full((1, 1, 1), 355 * 5), np.float32([1.0]), [0], False)  # 355 / 113 is pi to 2.7e-7
    a = 355 * 5 - 113 * 5 * np.pi
    assert np.isclose(y[0, 0, 0, 0], -np.cos(a), atol=1e-12) and np.isclose(y[0, 0, 0, 1], -np.sin(a), atol=1e-12)
