"""How fa_prefix_fwd cuts a prefix over workgroups, read off the workspace that it asks for: a function of the sizes, on the host."""
import pytest

from paper_2307_08691_amd import binding as fa

CUS = 256


def prefix_shares(rows, hkv, n_p, d=128):
    """`rows` packed rows a key/value head, of sequences with 64 own slots (one share of those)."""
    row = rows * hkv * (d + 1) * 4
    return fa.fa_prefix_fwd_workspace_bytes(rows, hkv, hkv, 1, n_p, 64, d) // row - 1


LENGTHS = sorted({64, 100, *(1024 * i + j for i in list(range(1, 64)) + [64, 96, 128, 129, 160, 192, 256, 257, 512, 1000] for j in (-1, 0, 1))})


@pytest.mark.parametrize("hkv", [1, 2, 3, 4, 8, 16, 32])
@pytest.mark.parametrize("rows", [1, 32, 33, 128, 129, 500])
def test_prefix_shares_grow_with_the_prefix(hkv, rows):
    """Shares of 1024 keys (up to a block of 64 more, where they do not divide evenly), up to one item a compute unit; shorter ones, 16 at most,
    while half of the chip has no item. Never fewer than a shorter prefix has, but by that rounding."""
    units = hkv * -(-rows // (32 if rows <= 32 else 128))
    least = 0
    for n in LENGTHS:
        s = prefix_shares(rows, hkv, n)
        assert 1 <= s <= max(16, -(-CUS // units))
        per = -(-n // s)  # keys of a share
        assert per <= max(1024 + 64, -(-n * units // CUS) + 64) or s >= min(16, -(-CUS // 2 // units))
        assert s >= 0.8 * least
        least = max(least, s)
        assert units * s >= min(CUS, units * (n // 1024)) * 0.8
