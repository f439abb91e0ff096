"""GPU parity of fa_prefix_fwd where its loops over shares and page numbers go round again: more shares of a row than the merge holds at
once, and shares of more pages than a wavefront looks up together. Oracle and tolerances: test_gpu_decoding."""
import pytest

from test_gpu_decoding import check_prefix

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f16", 128)])
@pytest.mark.parametrize("n_p,slots,page", [(5000, 2000, 0), (5000, 0, 64), (40001, 2000, 64)])
def test_prefix_of_more_shares_than_the_merge_holds(dtype, d, n_p, slots, page):
    """16 shares of 5000 shared keys and eight of 2000 own ones, or one (17, as many as are held); 37 of 40001."""
    check_prefix(dtype, d, 1, 1, 2, 1, n_p, slots or 64, page, [slots or 1], prefix_page=page)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f16", 128)])
@pytest.mark.parametrize("less", [0, 31, 8256 - 8193])  # the last share: whole, off a tile's edge, one key past the pages looked up first
def test_prefix_of_own_shares_of_many_pages(dtype, d, less):
    """66048 own keys in eight shares of 8256: a wavefront takes every fourth tile of 32 keys, and looks 64 pages up at once."""
    check_prefix(dtype, d, 1, 1, 2, 1, 100, 66048, 64, [66048 - less])
