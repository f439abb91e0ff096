"""The operators with which a batch decodes on caches that it keeps small, as cases that can be timed and compared.

A batch of continuations of one prompt: new keys and values are appended to each sequence's cache, the new queries attend to the
shared prompt and to the sequence's own keys, the attention weight that every cached key has drawn is accumulated, what drew least
is evicted, and drafted tokens are verified against the target's probabilities.

`path` says which operator a case takes:
  prefix   fa_prefix_fwd: new queries against a prefix that all sequences share and each sequence's own cache
  append   fa_cache_append: new keys and values into slabs or pages, with their weights and positions
  weights  fa_cache_weights: attention weight per cached key, accumulated
  evict    fa_cache_evict: caches cut to a budget
  verify   fa_verify_drafts: drafted tokens accepted or replaced, from given random numbers

`own` says whether run() calls the library (True) or computes the operators in their plain form (False).
"""
import math
import random

import torch

own = False

DEVICE = torch.device("cuda" if torch.cuda.is_available() else "cpu")
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def listed():
    return [
        # A few continuations of a prompt of 2048 tokens, each with a short answer so far: latency.
        dict(name="prefix_small", path="prefix", dtype="bf16", B=4, Nq=1, Np=2048, cap=256, page=0, lens_seed=1, Hq=32, Hkv=8, d=128),
        # A full serving batch on one system prompt of 8192 tokens, up to 1024 own tokens each in pages.
        dict(name="prefix_batch", path="prefix", dtype="bf16", B=64, Nq=1, Np=8192, cap=1024, page=256, lens_seed=2, Hq=32, Hkv=8, d=128),
        # Four drafted tokens and the last one for each of 16 sequences, one key/value head a query head, an odd prefix, half precision.
        dict(name="prefix_draft", path="prefix", dtype="f16", B=16, Nq=5, Np=12345, cap=2048, page=64, lens_seed=3, Hq=16, Hkv=16, d=64),
        # One decoding step of the serving batch: a key and a value a head and sequence go into their page.
        dict(name="append_step", path="append", dtype="bf16", B=64, Nq=1, cap=8192, page=256, lens_seed=4, Hkv=8, d=128),
        # Four prompts of an odd length enter slabs.
        dict(name="append_prompt", path="append", dtype="bf16", B=4, Nq=1531, cap=8192, page=0, lens_seed=5, Hkv=8, d=128),
        # The weights of one decoding step for a few users: latency.
        dict(name="weights_small", path="weights", dtype="bf16", B=4, Nq=1, cap=2048, page=0, lens_seed=6, Hq=32, Hkv=8, d=128),
        # The weights of one decoding step of the serving batch, 64 paged caches of up to 8192 keys.
        dict(name="weights_step", path="weights", dtype="bf16", B=64, Nq=1, cap=8192, page=256, lens_seed=7, Hq=32, Hkv=8, d=128),
        # The weights that two prompts of 2048 tokens give their own keys.
        dict(name="weights_prompt", path="weights", dtype="f16", B=2, Nq=2048, cap=2048, page=0, lens_seed=8, Hq=16, Hkv=16, d=64),
        # Every step of a serving batch that lives on 2048 keys a sequence: a few too many, a few go.
        dict(name="evict_step", path="evict", dtype="bf16", B=64, cap=2112, page=64, lens_seed=9, budget=2048, sinks=4, recent=512, Hkv=8, d=128, step=True),
        # After a prompt: caches of up to 8192 keys are cut to 1024.
        dict(name="evict_prompt", path="evict", dtype="bf16", B=8, cap=8192, page=0, lens_seed=10, budget=1024, sinks=4, recent=256, Hkv=8, d=128, step=False),
        # Four drafts for each of four sequences, probabilities of 32000 tokens in single precision: latency.
        dict(name="verify_small", path="verify", dtype="f32", B=4, k=4, V=32000, logits=False, drafts="probs"),
        # The serving batch: four drafts a sequence, the target's bfloat16 logits over 131072 tokens, the drafts' probabilities.
        dict(name="verify_batch", path="verify", dtype="bf16", B=64, k=4, V=131072, logits=True, drafts="probs"),
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
    path = rng.choice(["prefix", "prefix", "append", "weights", "weights", "evict", "verify", "verify"])
    hq, hkv = _heads(rng)
    c = dict(path=path, dtype=rng.choice(["bf16", "f16"]), lens_seed=rng.randrange(1 << 30), page=rng.choice([0, 64, 256]), Hq=hq, Hkv=hkv,
             d=rng.choice([64, 128]))
    unit = c["page"] or 1
    if path == "prefix":
        c.update(B=_log_int(rng, 1, 96), Nq=rng.choice([1, 1, 1, 2, 5, 8, 16]), Np=_log_int(rng, 64, 16384),
                 cap=-(-_log_int(rng, 64, 4096) // unit) * unit)
    elif path == "append":
        del c["Hq"]
        c.update(B=_log_int(rng, 1, 96), Nq=rng.choice([1, 1, 5, _log_int(rng, 16, 2048)]), cap=256 * _log_int(rng, 8, 32))
    elif path == "weights":
        if rng.random() < 0.7:
            c.update(B=_log_int(rng, 1, 96), Nq=rng.choice([1, 1, 5, 16]), cap=-(-_log_int(rng, 256, 8192) // unit) * unit)
        else:
            n = _log_int(rng, 64, 2048)
            c.update(B=_log_int(rng, 1, 4), Nq=n, cap=-(-n * rng.choice([1, 1, 2]) // unit) * unit)
    elif path == "evict":
        del c["Hq"]
        step, budget = rng.random() < 0.5, _log_int(rng, 128, 4096)
        c.update(B=_log_int(rng, 1, 64), budget=budget, sinks=rng.choice([0, 4]), recent=rng.randint(0, budget // 2), step=step,
                 cap=-(-(budget + 64 if step else round(budget * rng.uniform(1.5, 8))) // unit) * unit)
    else:
        c = dict(path=path, dtype=rng.choice(["f32", "bf16", "f16"]), B=_log_int(rng, 1, 64), k=rng.choice([1, 2, 4, 7]),
                 V=_log_int(rng, 1000, 131072), logits=rng.random() < 0.6, drafts=rng.choice(["probs", "probs", "none"]))
        if not c["logits"]:
            c["dtype"] = "f32"
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
    if case["path"] == "evict":
        if case["step"]:  # one to a few new tokens since the last call; some sequences are still below the budget
            return [case["budget"] + r.randint(1, 8) if r.random() < 0.9 else r.randint(1, case["budget"]) for _ in range(case["B"])]
        lens = [r.randint(min(case["budget"], case["cap"] // 2), case["cap"]) for _ in range(case["B"])]
    elif case["path"] == "weights" and case["Nq"] > 16:
        lens = [r.randint(case["Nq"], case["cap"]) for _ in range(case["B"])]
    else:
        lo = min(case["cap"], max(case["Nq"], case["cap"] // 64))
        lens = [r.randint(lo, case["cap"]) for _ in range(case["B"])]
    lens[0] = case["cap"]  # the longest sequence is what the cache was sized for
    return lens


def _seen(nq, nk):
    """Visible (query, key) pairs of one head under the causal rule."""
    return nq * nk - nq * (nq - 1) // 2


def work(case):
    path = case["path"]
    if path == "verify":
        B, k, V, e = case["B"], case["k"], case["V"], 4 if case["dtype"] == "f32" else 2
        # As logits every row of the target is read for its normaliser, else the one that is drawn from; and that one of the drafts.
        rows = B * (k + 1) if case["logits"] else B
        return {"bytes": rows * V * e + (B * V * 4 if case["drafts"] == "probs" else 0), "flops": 4 * rows * V}
    B, hkv, d, lens = case["B"], case["Hkv"], case["d"], _lengths(case)
    if path == "prefix":
        nq, hq, n = case["Nq"], case["Hq"], case["Np"]
        pairs = sum(_seen(nq, x) + nq * n for x in lens)
        return {"bytes": 4 * hkv * d * (n + sum(lens)) + 4 * B * nq * hq * d + 4 * B * nq * hq, "flops": 4 * hq * d * pairs}
    if path == "append":
        return {"bytes": 8 * B * case["Nq"] * hkv * d + 8 * B * case["Nq"] * hkv, "flops": 0}
    if path == "weights":
        nq, hq = case["Nq"], case["Hq"]
        return {"bytes": (2 * hkv * d + 8 * hkv) * sum(lens) + 2 * B * nq * hq * d + 4 * B * nq * hq,
                "flops": 2 * hq * d * sum(_seen(nq, x) for x in lens)}
    # Of n slots over the budget the kept ones that lie past it move; weights spread evenly over the slots, besides the newest.
    moved = sum((x - case["budget"]) * min(1.0, case["budget"] / x) for x in lens if x > case["budget"])
    return {"bytes": round(8 * hkv * moved * d + 8 * hkv * (sum(lens) + sum(min(x, case["budget"]) for x in lens))), "flops": 0}


# ---------------------------------------------------------------------------------------------
# inputs

def _randn(g, shape, dtype):
    return torch.randn(shape, generator=g, device=DEVICE).to(dtype)


def _cache(g, case, n=2):
    """n pools (or slabs) of the keys, values of a batch and the page table (None: slabs), as an engine has them: pages handed out in
    any order, some not in use, and sequences that own pages up to their capacity."""
    B, cap, page, hkv, d, dtype = case["B"], case["cap"], case["page"], case["Hkv"], case["d"], TYPES[case["dtype"]]
    if not page:
        return [_randn(g, (B, cap, hkv, d), dtype) for _ in range(n)], None
    per = cap // page
    pools = [_randn(g, (B * per + 3, page, hkv, d), dtype) for _ in range(n)]
    return pools, torch.randperm(B * per + 3, generator=g, device=DEVICE)[:B * per].reshape(B, per).int()


def _rows(pool, table, cap):
    """The first cap slots of every sequence, [B, cap, Hkv, d]."""
    if table is None:
        return pool[:, :cap]
    page = pool.shape[1]
    c = torch.arange(cap, device=pool.device)
    return pool.reshape(-1, *pool.shape[2:])[table[:, c // page].long() * page + c % page]


def _visible(lens, nq, cap):
    """[B, Nq, cap]: query r stands at position r + length - Nq of its sequence's keys."""
    c = torch.arange(cap, device=lens.device)
    r = torch.arange(nq, device=lens.device)
    return c <= (lens[:, None] - nq + r)[:, :, None]


def _heads_first(x, hkv):
    """[B, N, H, d] -> float32 [B, Hkv, N * H / Hkv, d], row r * G + h."""
    B, n, h, d = x.shape
    return x.float().reshape(B, n, hkv, h // hkv, d).permute(0, 2, 1, 3, 4).reshape(B, hkv, n * (h // hkv), d)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    path = case["path"]
    s = dict(path=path)
    if path == "verify":
        B, k, V = case["B"], case["k"], case["V"]
        logits = 3.0 * torch.randn((B, k + 1, V), generator=g, device=DEVICE)
        # (the draft model's logits are the target's with an error of their own; drafts are drawn from the drafts' probabilities)
        near = logits[:, :k] + 0.7 * torch.randn((B, k, V), generator=g, device=DEVICE)
        q = torch.softmax(near, -1)
        noise = -torch.log(-torch.log(torch.rand((B, k, V), generator=g, device=DEVICE).clamp_(1e-20, 1 - 6e-8)))
        tokens = (near + noise).argmax(-1).int()
        del near, noise
        if case["drafts"] == "none":
            tokens, q = torch.where(torch.rand((B, k), generator=g, device=DEVICE) < 0.6, logits[:, :k].argmax(-1).int(), tokens), None
        s.update(tokens=tokens, q=q, target=(logits if case["logits"] else torch.softmax(logits, -1)).to(TYPES[case["dtype"]]), logits=case["logits"],
                 uniform=torch.rand((B, k + 1), generator=g, device=DEVICE), inv_t=1.25 if case["logits"] else 1.0)
        return s
    B, hkv, d, cap, dtype = case["B"], case["Hkv"], case["d"], case["cap"], TYPES[case["dtype"]]
    lens = torch.tensor(_lengths(case), dtype=torch.int32, device=DEVICE)
    s.update(lens=lens, cap=cap, scale=1 / math.sqrt(d))
    if path == "prefix":
        (s["K"], s["V"]), s["table"] = _cache(g, case)
        s["Kp"], s["Vp"] = (_randn(g, (case["Np"], hkv, d), dtype) for _ in range(2))
        s["Q"] = _randn(g, (B, case["Nq"], case["Hq"], d), dtype)
        return s
    if path == "append":
        (s["K"], s["V"]), s["table"] = _cache(g, case)
        s["Kn"], s["Vn"] = (_randn(g, (B, case["Nq"], hkv, d), dtype) for _ in range(2))
        s["weights"] = -torch.log(torch.rand((B, hkv, cap), generator=g, device=DEVICE).clamp_min(1e-9))
        s["positions"] = torch.arange(cap, device=DEVICE, dtype=torch.int32).expand(B, hkv, cap).contiguous()
        s["first"] = lens - case["Nq"] + torch.randint(0, 5000, (B,), generator=g, device=DEVICE, dtype=torch.int32)
        return s
    if path == "weights":
        (s["K"],), s["table"] = _cache(g, case, 1)
        s["Q"] = _randn(g, (B, case["Nq"], case["Hq"], d), dtype)
        # (what a step or two before this one left: of the size that this one adds)
        s["weights"] = -torch.log(torch.rand((B, hkv, cap), generator=g, device=DEVICE).clamp_min(1e-9)) * (case["Nq"] * case["Hq"] / hkv / cap)
        # (the logsumexp that the attention over these keys left)
        s["LSE"] = torch.logsumexp(_scores(s), -1).reshape(B, hkv, case["Nq"], -1).transpose(2, 3).reshape(B, case["Hq"], case["Nq"])
        return s
    (s["K"], s["V"]), s["table"] = _cache(g, case)
    # weights as attention leaves them: a few keys with much, most with little; slots in the order that earlier evictions left
    s["weights"] = torch.exp(2 * torch.randn((B, hkv, cap), generator=g, device=DEVICE))
    order = torch.rand((B, hkv, cap), generator=g, device=DEVICE)
    order = torch.where(torch.arange(cap, device=DEVICE) < lens[:, None, None], order, 2 + order)  # (slots in use have the first positions)
    s["positions"] = (order.argsort(-1).argsort(-1) if case["step"] else torch.arange(cap, device=DEVICE).expand(B, hkv, cap)).int().contiguous()
    s.update(budget=case["budget"], sinks=case["sinks"], recent=case["recent"], weights_out=torch.zeros_like(s["weights"]),
             positions_out=torch.zeros_like(s["positions"]), lens_out=torch.zeros_like(lens))
    return s


# ---------------------------------------------------------------------------------------------
# the operators in their plain form

def _scores(s):
    """float32 [B, Hkv, Nq * G, cap], -inf where a key is not visible."""
    B, nq, hq = s["Q"].shape[:3]
    hkv = s["K"].shape[2]
    k = _rows(s["K"], s["table"], s["cap"]).float().permute(0, 2, 3, 1).contiguous()
    x = torch.matmul(_heads_first(s["Q"], hkv), k) * s["scale"]
    see = _visible(s["lens"], nq, s["cap"]).repeat_interleave(hq // hkv, 1)
    return x.masked_fill(~see[:, None], -math.inf)


def _plain_prefix(s):
    B, nq, hq, d = s["Q"].shape
    hkv, n = s["K"].shape[2], s["Kp"].shape[0]
    q = _heads_first(s["Q"], hkv)
    rows = q.shape[2]
    shared = q.transpose(0, 1).reshape(hkv, B * rows, d)
    a = torch.matmul(shared, s["Kp"].float().permute(1, 2, 0).contiguous()) * s["scale"]
    a = a.reshape(hkv, B, rows, n).transpose(0, 1)
    b = _scores(s)
    m = torch.maximum(a.amax(-1, keepdim=True), b.amax(-1, keepdim=True))
    a, b = torch.exp(a - m), torch.exp(b - m)
    z = a.sum(-1, keepdim=True) + b.sum(-1, keepdim=True)
    o = torch.matmul(a.transpose(0, 1).reshape(hkv, B * rows, n), s["Vp"].float().transpose(0, 1).contiguous())
    o = o.reshape(hkv, B, rows, d).transpose(0, 1) + torch.matmul(b, _rows(s["V"], s["table"], s["cap"]).float().transpose(1, 2).contiguous())
    o = (o / z).reshape(B, hkv, nq, hq // hkv, d).permute(0, 2, 1, 3, 4).reshape(B, nq, hq, d).to(s["Q"].dtype)
    lse = (m + torch.log(z)).reshape(B, hkv, nq, hq // hkv).transpose(2, 3).reshape(B, hq, nq)
    return {"O": o, "LSE": lse.contiguous()}


def _slots(s, c):
    """Where slots c [B, n] of every sequence lie among all rows of the pool (or of the slabs)."""
    if s["table"] is None:
        return torch.arange(c.shape[0], device=c.device)[:, None] * s["K"].shape[1] + c
    page = s["K"].shape[1]
    return s["table"].gather(1, c // page).long() * page + c % page


def _plain_append(s):
    B, nq = s["Kn"].shape[:2]
    c = (s["lens"][:, None] - nq + torch.arange(nq, device=DEVICE)).long()
    at = _slots(s, c).reshape(-1)
    for cache, new in ((s["K"], s["Kn"]), (s["V"], s["Vn"])):
        cache.view(-1, *cache.shape[2:])[at] = new.reshape(-1, *new.shape[2:])
    c = c[:, None].expand(-1, s["weights"].shape[1], -1)
    s["weights"].scatter_(2, c, 0.0)
    s["positions"].scatter_(2, c, (s["first"][:, None] + torch.arange(nq, device=DEVICE, dtype=torch.int32))[:, None].expand_as(c).contiguous())
    return {k: s[k] for k in ("K", "V", "weights", "positions")}


def _plain_weights(s):
    B, hq, nq = s["LSE"].shape
    hkv = s["K"].shape[2]
    lse = s["LSE"].reshape(B, hkv, hq // hkv, nq).transpose(2, 3).reshape(B, hkv, -1, 1)
    s["weights"] += torch.exp(_scores(s) - lse).sum(2)
    return {"weights": s["weights"]}


def _plain_evict(s):
    w, pos, budget = s["weights"], s["positions"], s["budget"]
    slot = torch.arange(s["cap"], device=DEVICE)
    held = slot < s["lens"][:, None, None]
    top = torch.where(held, pos, -1).amax(-1, keepdim=True) + 1
    safe = (pos < s["sinks"]) | (pos >= top - s["recent"])
    key = torch.where(held, torch.where(safe, math.inf, w), -math.inf)
    rank = key.sort(dim=-1, descending=True, stable=True).indices.argsort(-1)
    keep = held & (rank < budget)
    # what each of the first `budget` slots holds afterwards: itself, or the kept slots past the budget in their order
    movers = torch.where(keep & (slot >= budget), slot, s["cap"]).sort(-1).values
    free = held & ~keep & (slot < budget)
    nth = (free.cumsum(-1) - 1).clamp_min(0)
    source = torch.where(free, movers.gather(-1, nth), slot).clamp_max(s["cap"] - 1)
    first = held & (slot < budget)
    for new, old in ((s["weights_out"], w), (s["positions_out"], pos)):
        new.copy_(torch.where(first, old.gather(-1, source), new))
    b, g, c = free.nonzero(as_tuple=True)
    frm = source[b, g, c]
    for cache in (s["K"], s["V"]):
        if s["table"] is None:
            cache[b, c, g] = cache[b, frm, g]
        else:
            page, t = cache.shape[1], s["table"].long()
            cache[t[b, c // page], c % page, g] = cache[t[b, frm // page], frm % page, g]
    s["lens_out"].copy_(s["lens"].clamp_max(budget))
    return {k: s[k] for k in ("K", "V", "weights_out", "positions_out", "lens_out")}


def _plain_verify(s):
    # (in 64 bits: which token is drawn goes by where a running sum passes the random number)
    x, u = s["tokens"].long(), s["uniform"].double()
    B, k = x.shape
    p = s["target"].double()
    if s["logits"]:
        p = torch.softmax(p * s["inv_t"], -1)
    px = p[:, :k].gather(2, x[:, :, None])[:, :, 0]
    qx = torch.ones_like(px) if s["q"] is None else s["q"].gather(2, x[:, :, None])[:, :, 0].double()
    accepted = (u[:, :k] * qx < px).int().cumprod(1).sum(1)
    b = torch.arange(B, device=DEVICE)
    p, at = p[b, accepted], accepted.clamp_max(k - 1)
    if s["q"] is None:
        q = torch.zeros_like(p).scatter_(1, x[b, at][:, None], 2.0)
    else:
        q = s["q"][b, at].double()
    r = torch.where((accepted < k)[:, None], (p - q).clamp_min(0), p)
    r = torch.where(r.sum(1, keepdim=True) > 0, r, p)
    c = r.cumsum(1)
    some = (r > 0).long() * torch.arange(1, r.shape[1] + 1, device=DEVICE)
    drawn = torch.minimum((c <= u[:, k:] * c[:, -1:]).sum(1), some.amax(1) - 1)
    i = torch.arange(k + 1, device=DEVICE)
    out = torch.cat([x, x[:, :1]], 1)
    out = torch.where(i < accepted[:, None], out, torch.where(i == accepted[:, None], drawn[:, None], -1))
    return {"tokens": out.int(), "accepted": accepted.int()}


# ---------------------------------------------------------------------------------------------

def _own(s):
    from paper_2307_08691_amd import binding as fa
    path = s["path"]
    if path == "prefix":
        O, L = fa.fa_prefix_fwd(s["Q"], s["Kp"], s["Vp"], s["K"], s["V"], s["scale"], True, seqlens_k=s["lens"], block_table=s["table"])
        return {"O": O, "LSE": L}
    if path == "append":
        fa.fa_cache_append(s["Kn"], s["Vn"], s["K"], s["V"], s["lens"], block_table=s["table"], weights=s["weights"], positions=s["positions"],
                           first_position=s["first"])
        return {k: s[k] for k in ("K", "V", "weights", "positions")}
    if path == "weights":
        fa.fa_cache_weights(s["Q"], s["K"], s["LSE"], s["weights"], s["scale"], True, seqlens_k=s["lens"], block_table=s["table"])
        return {"weights": s["weights"]}
    if path == "evict":
        fa.fa_cache_evict(s["K"], s["V"], s["weights"], s["positions"], s["lens"], s["budget"], s["sinks"], s["recent"], block_table=s["table"],
                          weights_out=s["weights_out"], positions_out=s["positions_out"], seqlens_out=s["lens_out"])
        return {k: s[k] for k in ("K", "V", "weights_out", "positions_out", "lens_out")}
    tokens, accepted = fa.fa_verify_drafts(s["tokens"], s["q"], s["target"], s["uniform"], logits=s["logits"], inv_temperature=s["inv_t"])
    return {"tokens": tokens, "accepted": accepted}


def run(state):
    if own:
        return _own(state)
    return {"prefix": _plain_prefix, "append": _plain_append, "weights": _plain_weights, "evict": _plain_evict, "verify": _plain_verify}[state["path"]](state)


def exact(case, seed):
    """The definition, sequence by sequence and head by head in 64 bits. Cut and appended caches, lengths and tokens are moved or whole
    values and have none."""
    path = case["path"]
    if path not in ("prefix", "weights"):
        return None
    s = prepare(case, seed)
    hkv, hq, nq = case["Hkv"], case["Hq"], case["Nq"]
    group = hq // hkv
    out = {"O": torch.zeros(s["Q"].shape, dtype=torch.float64, device=DEVICE), "LSE": torch.zeros((case["B"], hq, nq), dtype=torch.float64, device=DEVICE)}
    total = s["weights"].double() if path == "weights" else None
    for b, n in enumerate(_lengths(case)):
        keys, values = s["K"], s.get("V")
        if case["page"]:
            pages = s["table"][b].tolist()
            keys = torch.cat([keys[p] for p in pages])[:n]
            values = torch.cat([values[p] for p in pages])[:n] if path == "prefix" else None
        else:
            keys, values = keys[b, :n], values[b, :n] if path == "prefix" else None
        hidden = torch.ones((nq, n), dtype=torch.bool, device=DEVICE).triu(n - nq + 1)
        for h in range(hq):
            kv = h // group
            q = s["Q"][b, :, h].double()
            x = (q @ keys[:, kv].double().T * s["scale"]).masked_fill(hidden, -math.inf)
            if path == "weights":
                total[b, kv, :n] += torch.exp(x - s["LSE"][b, h].double()[:, None]).sum(0)
                continue
            x = torch.cat([q @ s["Kp"][:, kv].double().T * s["scale"], x], 1)
            out["LSE"][b, h] = torch.logsumexp(x, 1)
            out["O"][b, :, h] = torch.exp(x - out["LSE"][b, h][:, None]) @ torch.cat([s["Vp"][:, kv], values[:, kv]]).double()
    return {"weights": total} if path == "weights" else out
