"""The operators between a layer's projections and its attention when the cache is held in 4 or 8 bits, as cases that can be timed and compared.

New queries and keys are rotated by their positions (one axis for text; time, height and width for images and video), keys and values are
quantised into the cache as they are written, and attention reads that cache; what it holds can be read back in 16 bits.

Cache: blocks of 32 consecutive channels of a row share a scale byte e, 2^(e - 127); the elements are E2M1 (4 bits, two a byte, the even
channel in the low half) or E4M3 (8 bits). Codes [pages, Hkv, page, d * bits / 8] and scales [pages, Hkv, page, d / 32], or slabs
[B, Hkv, slots, ..]. The scale is the smallest power of two that leaves no element above 1.75 * 2^2 (E2M1: 7, which rounds to 6)
or 1.75 * 2^8 (E4M3: 448), e = 16 at least; a block that holds an infinity or a NaN has e = 255, which makes all of it NaN.

`path` says which operator a case takes:
  rope     fa_rope_fwd, fa_rope_bwd: queries and keys rotated by positions of one or several axes, and the gradient
  append   fa_qcache_append: new keys and values quantised into slabs or pages, and the values that the cache now stands for
  read     fa_qcache_read: a range of every sequence's slots, or whole sequences packed one after the other, in 16 bits
  attend   fa_qcache_fwd: new queries against the cache

`own` says whether run() calls the library (True) or computes the operators in their plain form (False).
"""
import math
import random

import torch

own = False

DEVICE = torch.device("cuda" if torch.cuda.is_available() else "cpu")
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZES = {"bf16": 2, "f16": 2, "f32": 4}


def listed():
    return [
        # One decoding step of a serving batch, positions of one axis: latency.
        dict(name="rope_step", path="rope", dtype="bf16", B=64, N=1, Hq=32, Hkv=8, d=128, rot=128, axes=1, style="halves", grad=False, fused=True, far=100000),
        # Two clips of video among text, 8192 tokens each, queries and keys as slices of the projection's output.
        dict(name="rope_video", path="rope", dtype="bf16", B=2, N=8192, Hq=32, Hkv=8, d=128, rot=128, axes=3, style="halves", grad=False, fused=True, far=20000),
        # Training on images: the gradient of rows and columns, neighbouring channels paired, an odd number of patches, single precision.
        dict(name="rope_image_grad", path="rope", dtype="f32", B=8, N=1531, Hq=16, Hkv=16, d=64, rot=64, axes=2, style="pairs", grad=True, fused=False, far=0),
        # One decoding step of the serving batch: a key and a value a head and sequence go into their page, in 4 bits.
        dict(name="append_step", path="append", dtype="bf16", B=64, Nq=1, cap=2048, page=256, lens_seed=1, Hkv=8, d=128, k_bits=4, v_bits=4, fused=True),
        # Four prompts of an odd length enter slabs, keys in 8 bits and values in 4, half precision.
        dict(name="append_prompt", path="append", dtype="f16", B=4, Nq=1531, cap=4096, page=0, lens_seed=2, Hkv=16, d=64, k_bits=8, v_bits=4, fused=False),
        # The last 200 slots of a few sequences for a re-scoring pass: latency.
        dict(name="read_window", path="read", dtype="f16", B=4, N=200, cap=2048, page=0, lens_seed=3, Hkv=8, d=64, k_bits=8, v_bits=8),
        # Sixteen sequences of up to 4096 keys come back packed, for the attention of a prompt in 16 bits.
        dict(name="read_packed", path="read", dtype="bf16", B=16, N=0, cap=4096, page=64, lens_seed=4, Hkv=8, d=128, k_bits=4, v_bits=4),
        # A few users with short caches: latency.
        dict(name="attend_small", path="attend", dtype="bf16", B=4, Nq=1, cap=2048, page=0, lens_seed=5, Hq=32, Hkv=8, d=128, k_bits=4, v_bits=4),
        # The serving batch: 64 paged caches of up to 8192 keys in 4 bits.
        dict(name="attend_batch", path="attend", dtype="bf16", B=64, Nq=1, cap=8192, page=256, lens_seed=6, Hq=32, Hkv=8, d=128, k_bits=4, v_bits=4),
        # One user with a very long document, keys in 8 bits and values in 4.
        dict(name="attend_long", path="attend", dtype="bf16", B=1, Nq=1, cap=131072, page=64, lens_seed=7, Hq=32, Hkv=8, d=128, k_bits=8, v_bits=4),
        # Four drafted tokens and the last one for each of 16 sequences, a key/value head a query head, 8 bits, half precision.
        dict(name="attend_draft", path="attend", dtype="f16", B=16, Nq=5, cap=4096, page=64, lens_seed=8, Hq=16, Hkv=16, d=64, k_bits=8, v_bits=8),
        # The next 512 tokens of four long prompts against what the cache holds of them.
        dict(name="attend_prompt", path="attend", dtype="bf16", B=4, Nq=512, cap=8192, page=256, lens_seed=9, Hq=32, Hkv=8, d=128, k_bits=4, v_bits=4),
    ]


# ---------------------------------------------------------------------------------------------
# more cases of the same ranges

def _log_int(rng, lo, hi):
    """An integer in lo .. hi, uniform over the logarithm; odd ones as likely as even ones."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _heads(rng, most=32):
    hkv = rng.choice([h for h in (1, 2, 4, 8, 16) if h <= most])
    return hkv * rng.choice([g for g in (1, 2, 4, 8) if hkv * g <= most]), hkv


def _draw_once(rng):
    path = rng.choice(["rope", "rope", "append", "append", "read", "read", "attend", "attend", "attend", "attend"])
    hq, hkv = _heads(rng)
    if path == "rope":
        d = rng.choice([64, 72, 96, 128, 256])
        axes = rng.choice([1, 1, 2, 3])
        rot = rng.choice([d, d, d // 2])
        return dict(path=path, dtype=rng.choice(["bf16", "bf16", "f16", "f32"]), B=_log_int(rng, 1, 64), N=_log_int(rng, 1, 8192), Hq=hq, Hkv=hkv, d=d,
                    rot=rot, axes=axes, style=rng.choice(["halves", "halves", "pairs"]), grad=rng.random() < 0.4, fused=rng.random() < 0.5,
                    far=rng.choice([0, 1000, 1000000]))
    unit = rng.choice([0, 64, 256])
    c = dict(path=path, dtype=rng.choice(["bf16", "f16"]), lens_seed=rng.randrange(1 << 30), page=unit, Hkv=hkv, d=rng.choice([64, 128]),
             k_bits=rng.choice([4, 4, 8]), v_bits=rng.choice([4, 4, 8]))
    step = unit or 1

    def slots(lo, hi):
        return -(-_log_int(rng, lo, hi) // step) * step

    if path == "append":
        c.update(B=_log_int(rng, 1, 96), Nq=rng.choice([1, 1, 5, _log_int(rng, 16, 2048)]), fused=rng.random() < 0.5)
        c["cap"] = -(-max(c["Nq"], slots(64, 4096)) // step) * step
    elif path == "read":
        c.update(B=_log_int(rng, 1, 64), cap=slots(64, 8192))
        c["N"] = rng.choice([0, _log_int(rng, 1, c["cap"])])
        c["d"] = rng.choice([64, 128, 96, 256])
    else:
        c.update(Hq=hq, B=_log_int(rng, 1, 96), cap=slots(64, 131072), Nq=rng.choice([1, 1, 1, 2, 5, 16, _log_int(rng, 33, 1024)]))
        if c["Nq"] > c["cap"]:
            c["Nq"] = 1
    return c


def draw(rng):
    limit = {}
    for c in listed():
        w = work(c)
        limit[c["path"]] = [max(a, b) for a, b in zip(limit.get(c["path"], [0, 0]), (w["bytes"], w["flops"]))]
    while True:
        c = _draw_once(rng)
        w = work(c)
        if w["bytes"] <= limit[c["path"]][0] and w["flops"] <= limit[c["path"]][1]:
            return c


# ---------------------------------------------------------------------------------------------
# shapes

def _lengths(case):
    """Cached keys of each sequence, the new ones among them."""
    r = random.Random(case["lens_seed"])
    least = max(case.get("Nq", 1), case["cap"] // 64, 1)
    lens = [r.randint(min(case["cap"], least), case["cap"]) for _ in range(case["B"])]
    lens[0] = case["cap"]  # the longest sequence is what the cache was sized for
    return lens


def _seen(nq, nk):
    """Visible (query, key) pairs of one head under the causal rule."""
    return nq * nk - nq * (nq - 1) // 2


def _row_bytes(case):
    """Codes and scales of a key and its value, one head."""
    return case["d"] * (case["k_bits"] + case["v_bits"]) // 8 + case["d"] // 16


def work(case):
    e, d, B = SIZES[case["dtype"]], case["d"], case["B"]
    if case["path"] == "rope":
        tokens, heads = B * case["N"], case["Hq"] + case["Hkv"]
        return {"bytes": 2 * e * tokens * heads * d + 4 * case["axes"] * tokens, "flops": 3 * tokens * heads * case["rot"]}
    hkv, lens = case["Hkv"], _lengths(case)
    if case["path"] == "append":  # (new rows in; codes, scales and the values that they stand for out)
        return {"bytes": B * case["Nq"] * hkv * (2 * e * d + _row_bytes(case) + 2 * e * d), "flops": 0}
    if case["path"] == "read":
        rows = sum(min(case["N"], n) if case["N"] else n for n in lens)
        return {"bytes": rows * hkv * (_row_bytes(case) + 2 * e * d), "flops": 0}
    nq, hq = case["Nq"], case["Hq"]
    return {"bytes": hkv * _row_bytes(case) * sum(lens) + 2 * e * B * nq * hq * d + 4 * B * nq * hq,
            "flops": 4 * hq * d * sum(_seen(nq, n) for n in lens)}


# ---------------------------------------------------------------------------------------------
# quantising and back, in elementary operations

_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _quantise(x, bits):
    """float32 [..., d] -> codes uint8 [..., d * bits / 8], scales uint8 [..., d / 32]."""
    blocks = x.reshape(*x.shape[:-1], -1, 32)
    top = blocks.abs().amax(-1)
    whole = torch.isfinite(blocks).all(-1)
    # (exponent, one more where the significand is above 1.75: the largest element lies between 3.5 and 7, or 224 and 448)
    e = ((top.view(torch.int32) + 0x1fffff) >> 23) - (2 if bits == 4 else 8)
    e = e.clamp_min(16)
    y = blocks * ((254 - e) << 23).view(torch.float32)[..., None]  # (powers of two: exact)
    y = torch.where(whole[..., None], y, 0.0)
    if bits == 8:
        codes = y.to(torch.float8_e4m3fn).view(torch.uint8).reshape(*x.shape)
    else:  # to the nearest, halves to the even code
        a = y.abs()
        c = torch.signbit(y).to(torch.uint8) << 3
        for i, t in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
            c += a >= t if i % 2 else a > t
        c = c.reshape(*x.shape[:-1], -1, 2)
        codes = c[..., 0] | c[..., 1] << 4
    return codes.contiguous(), torch.where(whole, e, 255).to(torch.uint8)


def _values(codes, scales):
    """What codes and scales stand for, float32 [..., d]."""
    d = 32 * scales.shape[-1]
    if codes.shape[-1] == d:
        x = codes.view(torch.float8_e4m3fn).float()
    else:
        t = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), device=codes.device)
        pairs = torch.stack([t.repeat(16), t.repeat_interleave(16)], 1)  # of a byte: low half, high half
        x = pairs.index_select(0, codes.reshape(-1).int()).reshape(*codes.shape[:-1], d)
    s = torch.where(scales == 255, math.nan, (scales.int() << 23).view(torch.float32))
    return (x.reshape(*scales.shape, 32) * s[..., None]).reshape(*scales.shape[:-1], d)


# ---------------------------------------------------------------------------------------------
# inputs

def _randn(g, shape, dtype):
    return torch.randn(shape, generator=g, device=DEVICE).to(dtype)


def _slices(g, B, N, heads, d, dtype, fused):
    """Tensors [B, N, h, d] for h in heads: slices of one projection's output, or tensors of their own."""
    if not fused:
        return [_randn(g, (B, N, h, d), dtype) for h in heads]
    return list(_randn(g, (B, N, sum(heads), d), dtype).split(heads, 2))


def _cache(g, case):
    """(K codes, K scales, V codes, V scales) and the page table (None: slabs): pages handed out in any order, some not in use. Keys have
    channels of uneven size, as rotated keys do."""
    B, cap, page, hkv, d = case["B"], case["cap"], case["page"], case["Hkv"], case["d"]
    n, slots = (B * (cap // page) + 3, page) if page else (B, cap)
    out = []
    for bits, spread in ((case["k_bits"], 0.5), (case["v_bits"], 0.0)):
        size = torch.exp(spread * torch.randn(d, generator=g, device=DEVICE))
        codes = torch.empty((n, hkv, slots, d * bits // 8), dtype=torch.uint8, device=DEVICE)
        scales = torch.empty((n, hkv, slots, d // 32), dtype=torch.uint8, device=DEVICE)
        each = max(1, (1 << 27) // (hkv * slots * d))
        for i in range(0, n, each):
            x = torch.randn((min(each, n - i), hkv, slots, d), generator=g, device=DEVICE) * size
            codes[i:i + each], scales[i:i + each] = _quantise(x, bits)
        out += [codes, scales]
    table = None
    if page:
        table = torch.randperm(n, generator=g, device=DEVICE)[:n - 3].reshape(B, -1).int()
    return tuple(out), table


def _positions(g, case):
    """int32 [axes, B, N]: tokens of one axis from anywhere on; with two, rows and columns of an image; with three, pieces of text (all
    axes alike) between clips of frames, rows and columns."""
    B, N, axes = case["B"], case["N"], case["axes"]
    start = torch.randint(0, case["far"] + 1, (B, 1), generator=g, device=DEVICE, dtype=torch.int64)
    i = torch.arange(N, device=DEVICE)
    if axes == 1:
        return (start + i)[None].int().contiguous()
    wide = max(1, round(math.sqrt(N / (4 if axes == 3 else 1))))
    row, col = i // wide, i % wide
    if axes == 2:
        return (torch.stack([row, col])[:, None] + start).int().contiguous()
    frame, row = row // wide, row % wide
    text = (i // 97) % 5 == 0
    p = torch.stack([torch.where(text, i, frame), torch.where(text, i, row), torch.where(text, i, col)])
    return (p[:, None] + start).int().contiguous()


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    path, dtype, B, d = case["path"], TYPES[case["dtype"]], case["B"], case["d"]
    s = dict(path=path)
    if path == "rope":
        pairs = case["rot"] // 2
        s["Q"], s["K"] = _slices(g, B, case["N"], [case["Hq"], case["Hkv"], case["Hkv"]] if case["fused"] else [case["Hq"], case["Hkv"]], d, dtype,
                                 case["fused"])[:2]
        # (frequencies fall from 1 to 1 / 10000; the axes take pairs in runs, the first axis a shorter one)
        s["inv_freq"] = (10000.0 ** (-torch.arange(pairs, device=DEVICE, dtype=torch.float64) / pairs)).float()
        runs = {1: [pairs], 2: [pairs // 2, pairs - pairs // 2], 3: [pairs // 4, (pairs - pairs // 4) // 2, pairs - pairs // 4 - (pairs - pairs // 4) // 2]}
        s["axis"] = torch.cat([torch.full((n,), a, dtype=torch.int32) for a, n in enumerate(runs[case["axes"]])]).to(DEVICE)
        s.update(positions=_positions(g, case), pairs=pairs, neighbours=case["style"] == "pairs", grad=case["grad"])
        return s
    lens = _lengths(case)
    s["cache"], s["table"] = _cache(g, case)
    s.update(lens=torch.tensor(lens, dtype=torch.int32, device=DEVICE), cap=case["cap"], scale=1 / math.sqrt(d), dtype=dtype)
    if path == "append":
        heads = [2 * case["Hkv"]] if case["fused"] else []
        s["Kn"], s["Vn"] = _slices(g, B, case["Nq"], heads + [case["Hkv"], case["Hkv"]], d, dtype, case["fused"])[-2:]
    elif path == "read":
        rows = (B, case["N"]) if case["N"] else (sum(lens),)
        s["K"], s["V"] = (torch.zeros((*rows, case["Hkv"], d), dtype=dtype, device=DEVICE) for _ in range(2))
        if case["N"]:
            s["first"] = (s["lens"] - case["N"]).clamp_min(0)
        else:
            s["cu"] = torch.tensor([0] + lens, dtype=torch.int32, device=DEVICE).cumsum(0).int()
    else:
        s["Q"] = _randn(g, (B, case["Nq"], case["Hq"], d), dtype)
    return s


# ---------------------------------------------------------------------------------------------
# the operators in their plain form

def _plain_rope(s):
    # (angles in 64 bits: far positions)
    a = s["positions"].double().index_select(0, s["axis"]).permute(1, 2, 0) * s["inv_freq"].double()
    cos, sin = torch.cos(a).float()[:, :, None], torch.sin(a).float()[:, :, None]
    if s["grad"]:
        sin = -sin
    n, out = s["pairs"], []
    for x in (s["Q"], s["K"]):
        f = x.float()
        x1, x2 = (f[..., 0:2 * n:2], f[..., 1:2 * n:2]) if s["neighbours"] else (f[..., :n], f[..., n:2 * n])
        y1, y2 = x1 * cos - x2 * sin, x1 * sin + x2 * cos
        y = torch.stack([y1, y2], -1).flatten(-2) if s["neighbours"] else torch.cat([y1, y2], -1)
        out.append(torch.cat([y, f[..., 2 * n:]], -1).to(x.dtype))
    return {"Q": out[0], "K": out[1]}


def _at(s, b, c):
    """Index of slots c of sequences b (of one shape) into the first and third dimension of the cache's tensors."""
    if s["table"] is None:
        return b, c
    page = s["cache"][0].shape[2]
    return s["table"][b, c // page].long(), c % page


def _plain_append(s):
    B, nq = s["Kn"].shape[:2]
    c = (s["lens"][:, None] - nq + torch.arange(nq, device=DEVICE)).long()
    page, slot = _at(s, torch.arange(B, device=DEVICE)[:, None].expand_as(c), c)
    out = {}
    for name, new, codes, scales in (("K", s["Kn"], *s["cache"][:2]), ("V", s["Vn"], *s["cache"][2:])):
        q, e = _quantise(new.float(), 8 if codes.shape[3] == new.shape[3] else 4)
        codes[page, :, slot] = q
        scales[page, :, slot] = e
        out.update({name: _values(q, e).to(new.dtype), name + "codes": codes, name + "scales": scales})
    return out


def _plain_read(s):
    B = s["lens"].shape[0]
    if s["K"].dim() == 4:
        c = s["first"][:, None].long() + torch.arange(s["K"].shape[1], device=DEVICE)
        b = torch.arange(B, device=DEVICE)[:, None].expand_as(c)
        held = c < s["lens"][:, None]
        c = torch.where(held, c, 0)
    else:
        i = torch.arange(s["K"].shape[0], device=DEVICE)
        b = torch.bucketize(i, s["cu"][1:].long(), right=True)
        c = i - s["cu"].long()[b]
        held = c < s["lens"][b]
    page, slot = _at(s, b, c)
    for x, codes, scales in ((s["K"], *s["cache"][:2]), (s["V"], *s["cache"][2:])):
        x.copy_(torch.where(held[..., None, None], _values(codes[page, :, slot], scales[page, :, slot]).to(x.dtype), x))
    return {"K": s["K"], "V": s["V"]}


def _whole(s, codes, scales):
    """The slots of all sequences, float32 [B, Hkv, cap, d]."""
    x = _values(codes, scales)
    if s["table"] is None:
        return x
    B, per = s["table"].shape
    x = x.index_select(0, s["table"].reshape(-1)).reshape(B, per, *x.shape[1:]).transpose(1, 2)
    return x.reshape(B, x.shape[1], s["cap"], -1)


def _plain_attend(s):
    B, nq, hq, d = s["Q"].shape
    hkv, cap = s["cache"][0].shape[1], s["cap"]
    q = s["Q"].float().reshape(B, nq, hkv, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, -1, d)
    x = torch.matmul(q, _whole(s, *s["cache"][:2]).transpose(2, 3).contiguous()) * s["scale"]
    last = s["lens"][:, None] - nq + torch.arange(nq, device=DEVICE)  # query r stands at position r + length - Nq
    see = torch.arange(cap, device=DEVICE) <= last.repeat_interleave(hq // hkv, 1)[:, None, :, None]
    x = x.masked_fill_(~see, -math.inf)
    m = x.amax(-1, keepdim=True)
    x = torch.exp(x.sub_(m))
    z = x.sum(-1, keepdim=True)
    o = torch.matmul(x, _whole(s, *s["cache"][2:])) / z
    o = o.reshape(B, hkv, nq, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(B, nq, hq, d).to(s["Q"].dtype)
    lse = (m + torch.log(z)).reshape(B, hkv, nq, hq // hkv).transpose(2, 3).reshape(B, hq, nq)
    return {"O": o, "LSE": lse.contiguous()}


# ---------------------------------------------------------------------------------------------

def _own(s):
    from paper_2307_08691_amd import binding as fa
    if s["path"] == "rope":
        rotate = fa.fa_rope_bwd if s["grad"] else fa.fa_rope_fwd
        Q, K = rotate(s["Q"], s["K"], s["positions"], s["inv_freq"], s["axis"], neighbours=s["neighbours"])
        return {"Q": Q, "K": K}
    if s["path"] == "append":
        K, V = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (s["Kn"], s["Vn"]))
        fa.fa_qcache_append(s["Kn"], s["Vn"], s["cache"], seqlens_k=s["lens"], block_table=s["table"], Kout=K, Vout=V)
        c = s["cache"]
        return {"K": K, "V": V, "Kcodes": c[0], "Kscales": c[1], "Vcodes": c[2], "Vscales": c[3]}
    if s["path"] == "read":
        fa.fa_qcache_read(s["cache"], s["K"], s["V"], seqlens_k=s["lens"], block_table=s["table"], first=s.get("first"), cu_seqlens=s.get("cu"))
        return {"K": s["K"], "V": s["V"]}
    O, L = fa.fa_qcache_fwd(s["Q"], s["cache"], s["scale"], True, seqlens_k=s["lens"], block_table=s["table"])
    return {"O": O, "LSE": L}


def run(state):
    if own:
        return _own(state)
    return {"rope": _plain_rope, "append": _plain_append, "read": _plain_read, "attend": _plain_attend}[state["path"]](state)


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits

def _decoded(codes, scales):
    """Elements from their sign, exponent and significand bits, float64 [..., d]."""
    d = 32 * scales.shape[-1]
    if codes.shape[-1] == d:
        bits, bias, c = 3, 7, codes.long()
        sign = c >> 7
    else:
        bits, bias = 1, 1
        c = torch.stack([codes & 15, codes >> 4], -1).reshape(*codes.shape[:-1], d).long()
        sign = c >> 3
    exponent = (c >> bits) & ((1 << (4 if bits == 3 else 2)) - 1)
    part = (c & ((1 << bits) - 1)).double() / 2 ** bits
    x = torch.where(exponent == 0, part * 2.0 ** (1 - bias), (1 + part) * torch.exp2((exponent - bias).double()))
    x = torch.where(sign == 1, -x, x)
    return x * torch.exp2(scales.double() - 127).repeat_interleave(32, -1)


def _exact_rope(case, s):
    turn = torch.polar(torch.ones((), dtype=torch.float64, device=DEVICE),
                       torch.stack([s["positions"][a].double() * f for a, f in zip(s["axis"].tolist(), s["inv_freq"].double())], -1))
    if case["grad"]:
        turn = turn.conj()
    out, n = {}, case["rot"] // 2
    first = torch.arange(n, device=DEVICE) * (2 if case["style"] == "pairs" else 1)
    second = first + (1 if case["style"] == "pairs" else n)
    for name in ("Q", "K"):
        y = s[name].double()
        z = torch.complex(y[..., first], y[..., second]) * turn[:, :, None]
        y[..., first], y[..., second] = z.real, z.imag
        out[name] = y
    return out


def _exact_append(case, s):
    """The nearest element of every value's block, found among all of them."""
    out = {k: None for k in ("K", "V", "Kcodes", "Kscales", "Vcodes", "Vscales")}
    for name, bits in (("K", case["k_bits"]), ("V", case["v_bits"])):
        x = s[name + "n"].double()
        blocks = x.reshape(-1, 32)
        top = blocks.abs().amax(1, keepdim=True)
        most = 7.0 if bits == 4 else 448.0
        scale = torch.exp2(torch.ceil(torch.log2(top / most)).clamp_min(16 - 127))
        scale = torch.where(top > most * scale, 2 * scale, torch.where(top <= most * scale / 2, scale / 2, scale)).clamp_min(2.0 ** (16 - 127))
        y = blocks / scale
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp_min(1.0 if bits == 4 else 2.0 ** -6))) - (1 if bits == 4 else 3))
        y = torch.round(y / step) * step  # (halves to even; past the largest element there is none)
        out[name] = (y.clamp(-6, 6) if bits == 4 else y).mul(scale).reshape(x.shape)
    return out


def _slots(case, s, codes, scales, b, lo, hi):
    """Slots lo .. hi - 1 of sequence b, float64 [Hkv, hi - lo, d]."""
    if not case["page"]:
        return _decoded(codes[b, :, lo:hi], scales[b, :, lo:hi])
    page = case["page"]
    pages = s["table"][b, lo // page:-(-hi // page)].tolist()
    x = torch.cat([_decoded(codes[p], scales[p]) for p in pages], 1)
    return x[:, lo % page:lo % page + hi - lo]


def exact(case, seed):
    s = prepare(case, seed)
    path = case["path"]
    if path == "rope":
        return _exact_rope(case, s)
    if path == "append":
        return _exact_append(case, s)
    lens = _lengths(case)
    if path == "read":
        out = {}
        for name, codes, scales in (("K", *s["cache"][:2]), ("V", *s["cache"][2:])):
            x = torch.zeros(s[name].shape, dtype=torch.float64, device=DEVICE)
            at = 0
            for b, n in enumerate(lens):
                if case["N"]:
                    lo = max(0, n - case["N"])
                    x[b, :n - lo] = _slots(case, s, codes, scales, b, lo, n).transpose(0, 1)
                else:
                    x[at:at + n] = _slots(case, s, codes, scales, b, 0, n).transpose(0, 1)
                    at += n
            out[name] = x
        return out
    nq, hq, group = case["Nq"], case["Hq"], case["Hq"] // case["Hkv"]
    out = {"O": torch.zeros(s["Q"].shape, dtype=torch.float64, device=DEVICE), "LSE": torch.zeros((case["B"], hq, nq), dtype=torch.float64, device=DEVICE)}
    for b, n in enumerate(lens):
        keys, values = _slots(case, s, *s["cache"][:2], b, 0, n), _slots(case, s, *s["cache"][2:], b, 0, n)
        hidden = torch.ones((nq, n), dtype=torch.bool, device=DEVICE).triu(n - nq + 1)
        for h in range(hq):
            x = (s["Q"][b, :, h].double() @ keys[h // group].T * s["scale"]).masked_fill(hidden, -math.inf)
            out["LSE"][b, h] = torch.logsumexp(x, 1)
            out["O"][b, :, h] = torch.exp(x - out["LSE"][b, h][:, None]) @ values[h // group]
    return out
