"""Every kernel of a decoding batch that its sources define is among those whose resources are checked: none uses scratch memory or
spills vector registers (scalar registers may go into lanes of vector ones: that touches no memory)."""
import concurrent.futures
import os
import re

from paper_2307_08691_amd import build as fa_build
from test_decoding_resources import SOURCES
from test_kernel_resources import resource_remarks


def test_every_kernel_of_the_sources_is_built_and_needs_no_scratch():
    text = "".join(open(os.path.join(fa_build.CSRC, s)).read() for s in SOURCES)
    # (what stands between __global__ and the name: launch bounds and attributes)
    names = set(re.findall(r"__global__[^;{]*?void\s+(\w+)\s*\(", text))
    assert len(names) == text.count("__global__") and {"weights_rows_kernel", "evict_lengths_kernel"} <= names
    with concurrent.futures.ThreadPoolExecutor(4) as ex:
        remarks = {k: v for part in ex.map(resource_remarks, SOURCES) for k, v in part.items()}
    for n in names:
        built = [v for k, v in remarks.items() if n in k]
        assert built, n
        assert all(v["ScratchSize [bytes/lane]"] == 0 and v["VGPRs Spill"] == 0 for v in built), n
