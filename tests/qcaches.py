"""Caches in 4 or 8 bits on the GPU beside what they hold in float64, for the tests of the operators on them."""
import json
import subprocess
import sys

import numpy as np
import torch

from oracle import qcache_oracle as orc
from paper_2307_08691_amd import binding

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def gpu(x, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(x)).cuda()
    return t if dtype is None else t.to(dtype)


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Cache:
    """A QCache of the given lengths, in slabs (page 0) or in pages in any order. Wherever no sequence holds a key the codes are noise and
    the scales 255, NaN. K, V: what the slots stand for, [B, slots, Hkv, d]."""

    def __init__(self, r, B, slots, hkv, d, page, lens, k_bits, v_bits, spare=3, data=None):
        self.page, self.slots, self.B, self.lens, self.bits = page, slots, B, lens, (k_bits, v_bits)
        self.order = None
        n, rows = B, slots
        if page:
            per = -(-slots // page)
            self.order, n, rows = r.permutation(B * per + spare)[:B * per].reshape(B, per), B * per + spare, page
        self.table = ints(self.order.tolist()) if page else None
        tensors, self.rows = [], []
        for i, bits in enumerate((k_bits, v_bits)):
            x = data[i] if data is not None else r.normal(size=(B, slots, hkv, d)) * np.exp2(r.integers(-2, 3, size=(B, slots, hkv, 1)))
            codes, scales = orc.quantise(x, bits)
            for b in range(B):
                scales[b, lens[b]:] = 255
                codes[b, lens[b]:] = r.integers(0, 256, size=codes[b, lens[b]:].shape)
            self.rows.append(orc.values(codes & (15 if bits == 4 else 255), scales, bits))
            codes = orc.packed(codes & (15 if bits == 4 else 255), bits)
            for t in (codes, scales):
                t = t.transpose(0, 2, 1, 3)  # [B, Hkv, slots, ..]
                pool = np.full((n, hkv, rows, t.shape[3]), 255, np.uint8)
                if page:
                    for b in range(B):
                        for p in range(per):
                            part = t[b, :, p * page:(p + 1) * page]
                            pool[self.order[b, p], :, :part.shape[1]] = part
                else:
                    pool[:] = t
                tensors.append(gpu(pool))
        self.q = binding.QCache(*tensors)
        self.more = dict(seqlens_k=ints(lens), block_table=self.table)
        if page:
            self.more["max_seqlen_k"] = slots

    def held(self, q=None):
        """The four tensors of a cache of this shape as the slots of the sequences have them, [B, slots, Hkv, ..] each."""
        out = []
        for t in q or self.q:
            t = t.cpu().numpy()
            if self.page:
                t = np.stack([np.concatenate([t[p] for p in self.order[b]], 1)[:, :self.slots] for b in range(self.B)])
            out.append(t.transpose(0, 2, 1, 3))
        return out


# Batches whose sequences are long and many, so that a workgroup has tens of thousands of keys of one: (d, K's and V's bits, queries, query heads, sequences, page,
# most slots), 8 key/value heads.
LONG = [
    (128, 4, 4, 1, 32, 96, 64, 10240),   # 16 rows, tiles of 32 keys
    (64, 4, 4, 1, 16, 96, 64, 17536),    # ... of 64
    (128, 8, 8, 4, 32, 64, 256, 10240),  # 512 workgroups, one tile on its way
    (128, 4, 4, 5, 32, 64, 64, 10240),   # 32 rows
    (64, 8, 4, 3, 64, 64, 256, 10240),
    (128, 4, 4, 40, 32, 32, 64, 10240),  # 128 rows, two blocks
    (64, 8, 8, 32, 32, 64, 256, 10240),  # ... one
]


def long_lengths(B, slots):
    return [slots - 37 * (b % 5) for b in range(B)]


def longest_segment(lens, nq, group, hkv, rows, chunk, workgroups):
    """Keys of the longest part of a sequence that one workgroup has: the chunks of all (sequence, head, block of rows) under the causal rule, one
    after the other, in equal runs."""
    blocks = -(-nq * group // rows)
    units = []
    for n in lens:
        for _ in range(hkv):
            for k in range(blocks):
                last = (min((k + 1) * rows, nq * group) - 1) // group
                units.append(-(-max(0, min(n, n - nq + last + 1)) // chunk))
    total = sum(units)
    run, more = divmod(total, workgroups)
    cuts = np.cumsum([0] + [run + (w < more) for w in range(workgroups)])
    ends = np.cumsum([0] + units)
    points = np.unique(np.concatenate([cuts, ends]))
    return int(np.diff(points).max()) * chunk


GRIDS = """
import ctypes, json, sys
sys.path.insert(0, sys.argv[1])
recorder = ctypes.CDLL(sys.argv[2], mode=ctypes.RTLD_GLOBAL)
recorder.recorded.restype = ctypes.c_char_p
from paper_2307_08691_amd import binding
out = []
for args in json.load(sys.stdin):
    assert binding.fa_qcache_fwd_raw(*args) == 0
    out.append([int(line.split("|")[1]) for line in recorder.recorded().decode().splitlines()])
json.dump(out, sys.stdout)
"""


def grids(calls):
    """[arguments of fa_qcache_fwd_raw] -> per call the workgroups of its launches, seen without a GPU (launches.py; the kernels have no names outside)."""
    import launches
    r = subprocess.run([sys.executable, "-c", GRIDS, launches.ROOT, launches.recorder()], input=json.dumps(calls), capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    return json.loads(r.stdout)
