"""What the compiler made of the kernels of caches in 4 or 8 bits and of rotary positions: every one that the sources define is built, none uses
scratch memory or spills, LDS fits."""
import concurrent.futures
import os
import re

from paper_2307_08691_amd import build as fa_build
from test_kernel_resources import resource_remarks

SOURCES = ["fa_qcache.hip", "fa_qattend.hip", "fa_qattend_wide.hip", "fa_rope.hip"]


def test_every_kernel_is_built_and_needs_no_scratch():
    text = "".join(open(os.path.join(fa_build.CSRC, s)).read() for s in SOURCES)
    names = set(re.findall(r"__global__[^;{]*?void\s+(\w+)\s*\(", text))
    assert len(names) == text.count("__global__") and {"qappend_kernel", "qread_kernel", "rope_kernel"} <= names
    with concurrent.futures.ThreadPoolExecutor(4) as ex:
        remarks = {k: v for part in ex.map(resource_remarks, SOURCES) for k, v in part.items()}
    for n in names:
        built = [v for k, v in remarks.items() if n in k]
        assert built, n
        assert all(v["ScratchSize [bytes/lane]"] == 0 and v["VGPRs Spill"] == 0 for v in built), n
    assert max(v.get("LDS Size [bytes/block]", 0) for v in remarks.values()) <= 160 * 1024
