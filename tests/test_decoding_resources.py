"""What the compiler made of the kernels of a decoding batch: no scratch memory, no spills (direct-to-LDS copies are ordered by counting,
which a spill would upset), and LDS that fits."""
import concurrent.futures

import pytest

from test_kernel_resources import resource_remarks

SOURCES = ["fa_prefix.hip", "fa_cache.hip", "fa_weights.hip", "fa_verify.hip"]


@pytest.fixture(scope="module")
def remarks():
    with concurrent.futures.ThreadPoolExecutor(4) as ex:
        return {k: v for part in ex.map(resource_remarks, SOURCES) for k, v in part.items()}


def test_every_kernel_was_seen_and_none_spills(remarks):
    names = " ".join(remarks)
    for k in ("prefix_items_kernel", "prefix_merge_kernel", "append_kernel", "evict_select_kernel", "evict_move_kernel", "weights_step_kernel",
              "weights_prompt_kernel", "verify_stats_kernel", "verify_sums_kernel", "verify_draw_kernel"):
        assert k in names
    bad = {k: v for k, v in remarks.items() if v.get("ScratchSize [bytes/lane]", 0) or v.get("VGPRs Spill", 0)}
    assert not bad, bad
    assert max(v.get("LDS Size [bytes/block]", 0) for v in remarks.values()) <= 160 * 1024
