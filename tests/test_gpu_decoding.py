"""GPU parity of the operators of a decoding batch (fa_prefix_fwd, fa_cache_append, fa_cache_weights, fa_cache_evict,
fa_verify_drafts) against their definitions in float64: lengths of 0 and 1, one row and many, slabs and pages, lengths off every tile
edge, what no call may read filled with NaN, rows that see nothing, caches past 2^31 elements, other streams, captured graphs.

Tolerances count roundings. e = half a step of the element type (2^-8 bfloat16, 2^-11 half precision). O: P rounded to the type (e
of every p |v|) and O itself (e of |O|), each score off by d 2^-24 of its sum of |q k| and by a few float32 roundings of itself, and
half precision's P by up to 2^-25 of the row's largest where it is subnormal. LSE and weights: the scores' part alone. Moved rows,
positions, lengths and tokens are exact."""
import numpy as np
import pytest

from paper_2307_08691_amd import binding
from oracle import decoding_oracle as dec

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}


def rng(seed):
    return np.random.default_rng(seed)


def gpu(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype).cuda()


def f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


class Cache:
    """Keys and values [B, slots, Hkv, d] of the given lengths on the GPU, in slabs (page 0) or in pages in any order; NaN wherever no
    sequence holds a key."""

    def __init__(self, r, dtype, B, slots, hkv, d, page, lens, spare=3):
        self.page, self.slots, self.B, self.lens = page, slots, B, lens
        data = [gpu(r.normal(size=(B, slots, hkv, d)), TYPES[dtype]) for _ in range(2)]
        for x in data:
            for b in range(B):
                x[b, lens[b]:] = float("nan")
        self.rows = [f64(x) for x in data]
        self.table = None
        if page:
            per = -(-slots // page)
            order = r.permutation(B * per + spare)[:B * per].reshape(B, per)
            pools = []
            for x in data:
                pool = torch.full((B * per + spare, page, hkv, d), float("nan"), dtype=x.dtype, device="cuda")
                whole = torch.full((B, per * page, hkv, d), float("nan"), dtype=x.dtype, device="cuda")
                whole[:, :slots] = x
                pool[torch.from_numpy(order.reshape(-1)).cuda()] = whole.reshape(B * per, page, hkv, d)
                pools.append(pool)
            data, self.table = pools, ints(order.tolist())
        self.K, self.V = data

    def read(self, x):
        """What the slots of every sequence hold now, [B, slots, Hkv, d]."""
        if not self.page:
            return x
        return torch.stack([x[self.table[b].long()].reshape(-1, *x.shape[2:])[:self.slots] for b in range(self.B)])


def check_prefix(dtype, d, B, nq, hq, hkv, n_p, slots, page, lens, causal=True, prefix_page=0, seed=0, scale=None, call=None):
    r = rng(seed + d + nq + n_p)
    scale = scale or d**-0.5
    cache = Cache(r, dtype, B, slots, hkv, d, page, lens)
    Q = gpu(r.normal(size=(B, nq, hq, d)), TYPES[dtype])
    Kp, Vp = (gpu(r.normal(size=(n_p, hkv, d)), TYPES[dtype]) for _ in range(2))
    kp, vp, more = Kp, Vp, {}
    if prefix_page:
        per = -(-n_p // prefix_page)
        order = r.permutation(per + 2)[:per]
        pools = [torch.full((per + 2, prefix_page, hkv, d), float("nan"), dtype=TYPES[dtype], device="cuda") for _ in range(2)]
        for pool, x in zip(pools, (Kp, Vp)):
            for i, at in enumerate(order):
                part = x[i * prefix_page:(i + 1) * prefix_page]
                pool[at, :len(part)] = part
        (kp, vp), more = pools, dict(prefix_table=ints(order.tolist()), prefix_len=n_p)
    if cache.table is not None:
        more["max_seqlen_k"] = slots
    call = call or (lambda *x, **y: binding.fa_prefix_fwd(*x, **y))
    O, L = call(Q, kp, vp, cache.K, cache.V, scale, causal, seqlens_k=ints(lens), block_table=cache.table, **more)
    torch.cuda.synchronize()
    assert not binding.fa_prefix_fwd_workspace_bytes(B, hq, hkv, nq, n_p, slots, d) % 256
    eO, eL, A, M = dec.prefix_forward(f64(Q), f64(Kp), f64(Vp), *cache.rows, lens, scale, causal)
    e = torch.finfo(TYPES[dtype]).eps / 2
    L, O = f64(L), f64(O)
    none = eL == -np.inf
    assert (L[none] == -np.inf).all() and (O.transpose(0, 2, 1, 3)[none] == 0).all()
    score = np.where(none, 0, M * d / 2**24 + (M + np.abs(np.where(none, 0, eL)) + 8) / 2**21)
    assert (np.abs(L[~none] - eL[~none]) <= score[~none]).all()
    small = (n_p + slots) * 4.0 / 2**25 if dtype == "f16" else 0.0  # (|v| below 4 where it counts)
    tol = e * (A + np.abs(eO)) * (1 + 2 * e) + A * 4 * score.transpose(0, 2, 1)[..., None] + small
    assert (np.abs(O - eO) <= tol).all(), np.max(np.abs(O - eO) / np.maximum(tol, 1e-30))
    return O, L


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,nq,hq,hkv,n_p,slots,page,lens", [
    (1, 1, 1, 1, 1, 1, 0, [1]),                           # the smallest call
    (3, 1, 8, 2, 700, 300, 0, [300, 1, 0]),               # 12 rows a head: one row tile against the prefix
    (5, 1, 32, 4, 1000, 200, 64, [200, 64, 65, 0, 1]),    # 40 rows: the wide form, its last wavefronts empty
    (20, 2, 16, 2, 515, 130, 64, [(7 * i) % 129 + 2 for i in range(20)]),  # 320 rows: three blocks of rows
    (2, 9, 8, 2, 333, 200, 0, [200, 9]),                  # 36 own rows: two narrow items
    (2, 70, 4, 1, 129, 500, 128, [500, 70]),              # 280 own rows: wide items under the causal rule
    (150, 1, 2, 1, 200, 70, 0, [(11 * i) % 71 for i in range(150)]),  # more sequences than are ranked by length
])
def test_prefix(dtype, d, B, nq, hq, hkv, n_p, slots, page, lens):
    check_prefix(dtype, d, B, nq, hq, hkv, n_p, slots, page, lens)


@pytest.mark.parametrize("nq,lens", [(1, [100, 0, 37]), (3, [100, 3, 1]), (40, [100, 40, 12])])
def test_prefix_without_causal_rule_and_with_more_queries_than_keys(nq, lens):
    """Causal: queries before the first own key see the prefix alone."""
    for causal in (False, True):
        check_prefix("bf16", 64, 3, nq, 4, 2, 90, 100, 0, lens, causal=causal)


@pytest.mark.parametrize("nq", [1, 20])
def test_prefix_of_no_keys(nq):
    """Np = 0 is the cache alone; rows that see no key at all are empty."""
    check_prefix("bf16", 128, 3, nq, 8, 2, 0, 80, 0, [80, 0, 5], causal=True)
    check_prefix("f16", 64, 3, nq, 8, 2, 0, 80, 64, [0, 0, 0], causal=False)


@pytest.mark.parametrize("n_p,prefix_page,page", [(1000, 64, 64), (513, 128, 0), (64, 64, 64), (1, 256, 256)])
def test_prefix_in_pages(n_p, prefix_page, page):
    check_prefix("bf16", 128, 4, 1, 16, 4, n_p, 190, page, [190, 64, 1, 130], prefix_page=prefix_page)
    check_prefix("f16", 64, 12, 3, 4, 1, n_p, 190, page, [190] * 12, prefix_page=prefix_page)


EDGES = [700, 1, 32, 33, 127, 128, 129, 160, 161, 256, 257, 288, 289, 384, 385, 415, 511, 512, 513, 640, 641, 672, 673, 699]


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f16", 128), ("bf16", 128)])
@pytest.mark.parametrize("page", [0, 64])
def test_prefix_of_many_sequences(dtype, d, page):
    """So many that each has its cache to itself: one to six tiles a wavefront, ends on and off the tiles' edges."""
    lens = (EDGES * 3)[:64]
    check_prefix(dtype, d, 64, 1, 8, 8, 300, 700, page, lens)


def test_prefix_of_spread_scores():
    """The softmax's reference advances (and is left behind by up to 2^8 or 2^20) when scores spread widely."""
    for dtype in ("bf16", "f16"):
        check_prefix(dtype, 64, 40, 1, 4, 1, 3000, 100, 0, [50] * 40, scale=1.5)


def test_prefix_equals_the_cache_that_begins_with_it():
    r = rng(5)
    B, hq, hkv, d, n_p, slots = 6, 8, 2, 128, 384, 128
    lens = [1, 2, 64, 65, 127, 128]
    cache = Cache(r, "bf16", B, slots, hkv, d, 0, lens)
    Q, Kp, Vp = (gpu(r.normal(size=s), torch.bfloat16) for s in ((B, 1, hq, d), (n_p, hkv, d), (n_p, hkv, d)))
    O, L = binding.fa_prefix_fwd(Q, Kp, Vp, cache.K, cache.V, d**-0.5, True, seqlens_k=ints(lens))
    K, V = (torch.cat([p.expand(B, -1, -1, -1), x], 1).contiguous() for p, x in ((Kp, cache.K), (Vp, cache.V)))
    eO, eL = binding.fa_kvcache_fwd(Q, K, V, d**-0.5, True, seqlens_k=ints([n + n_p for n in lens]))
    torch.testing.assert_close(L, eL, rtol=0, atol=2e-6)
    torch.testing.assert_close(O.float(), eO.float(), rtol=2**-7, atol=2**-9)


def test_prefix_on_another_stream_and_in_a_graph():
    r = rng(6)
    B, hq, hkv, d, n_p, slots = 8, 16, 4, 64, 600, 192
    lens = ints([100] * B)
    cache = Cache(r, "bf16", B, slots, hkv, d, 64, [slots] * B)
    Q = gpu(r.normal(size=(B, 1, hq, d)), torch.bfloat16)
    Kp, Vp = (gpu(r.normal(size=(n_p, hkv, d)), torch.bfloat16) for _ in range(2))
    out = [torch.empty_like(Q), torch.empty((B, hq, 1), device="cuda")]

    def call():
        return binding.fa_prefix_fwd(Q, Kp, Vp, cache.K, cache.V, 0.125, True, seqlens_k=lens, block_table=cache.table, O=out[0], LSE=out[1])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for n in (3, 192, 64):
        lens.fill_(n)
        Q.copy_(gpu(r.normal(size=(B, 1, hq, d)), torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        O, L = (x.clone() for x in out)
        eO, eL = binding.fa_prefix_fwd(Q, Kp, Vp, cache.K, cache.V, 0.125, True, seqlens_k=lens, block_table=cache.table)
        assert torch.equal(O, eO) and torch.equal(L, eL)


# ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("B,nq,hkv,d,slots,page,lens", [
    (1, 1, 1, 8, 1, 0, [1]),
    (4, 1, 8, 128, 200, 64, [200, 1, 64, 65]),
    (3, 130, 2, 64, 300, 0, [300, 130, 200]),
    (3, 5, 3, 256, 130, 128, [130, 5, 128]),
    (3, 5, 2, 72, 100, 0, [3, 104, 0]),  # slots before the first and past the last: dropped
])
def test_append(dtype, B, nq, hkv, d, slots, page, lens):
    r = rng(B + nq + d)
    cache = Cache(r, dtype, B, slots, hkv, d, page, [slots] * B)
    Kn, Vn = (gpu(r.normal(size=(B, nq, hkv, d)), TYPES[dtype]) for _ in range(2))
    W, P = gpu(r.random((B, hkv, slots)), torch.float32), ints(r.integers(0, 99, (B, hkv, slots)).tolist())
    first = ints([1000 * b + 7 for b in range(B)])
    eK, eV, eW, eP = (x.clone() for x in (cache.read(cache.K), cache.read(cache.V), W, P))
    other = [x.isnan().sum().item() for x in (cache.K, cache.V)]
    for b in range(B):
        for i in range(nq):
            s = lens[b] - nq + i
            if 0 <= s < slots:
                eK[b, s], eV[b, s], eW[b, :, s], eP[b, :, s] = Kn[b, i], Vn[b, i], 0.0, 1000 * b + 7 + i
    binding.fa_cache_append(Kn, Vn, cache.K, cache.V, ints(lens), block_table=cache.table, weights=W, positions=P, first_position=first)
    torch.cuda.synchronize()
    assert torch.equal(cache.read(cache.K), eK) and torch.equal(cache.read(cache.V), eV)
    assert torch.equal(W, eW) and torch.equal(P, eP)
    assert other == [x.isnan().sum().item() for x in (cache.K, cache.V)]  # (the pages that nobody owns)


def test_append_alone():
    """Neither weights nor positions, or positions that are the slots; lengths left out."""
    r = rng(3)
    cache = Cache(r, "bf16", 2, 64, 2, 64, 64, [64, 64])
    Kn, Vn = (gpu(r.normal(size=(2, 3, 2, 64)), torch.bfloat16) for _ in range(2))
    binding.fa_cache_append(Kn, Vn, cache.K, cache.V, block_table=cache.table)
    assert torch.equal(cache.read(cache.K)[:, 61:], Kn) and torch.equal(cache.read(cache.V)[:, 61:], Vn)
    P = ints(np.zeros((2, 2, 64)).tolist())
    binding.fa_cache_append(Kn, Vn, cache.K, cache.V, ints([3, 10]), block_table=cache.table, positions=P)
    assert P[0, 1, :4].tolist() == [0, 1, 2, 0] and P[1, 0, 6:11].tolist() == [0, 7, 8, 9, 0]


# ---------------------------------------------------------------------------------------------

def check_weights(dtype, d, B, nq, hq, hkv, slots, page, lens, causal=True, queries=None, scale=None, junk_lse=False):
    r = rng(B + nq + d + slots)
    scale = scale or d**-0.5
    cache = Cache(r, dtype, B, slots, hkv, d, page, lens)
    Q = gpu(r.normal(size=(B, nq, hq, d)), TYPES[dtype])
    _, L, _, _ = dec.prefix_forward(f64(Q), np.zeros((0, hkv, d)), np.zeros((0, hkv, d)), *cache.rows, lens, scale, causal)
    L = gpu(L, torch.float32)
    if queries is not None:  # what does not count may hold anything
        for b in range(B):
            Q[b, queries[b]:] = float("nan")
            L[b, :, queries[b]:] = float("nan")
    W0 = r.random((B, hkv, slots)) / slots
    W = gpu(W0, torch.float32)
    W0 = f64(W)
    binding.fa_cache_weights(Q, cache.K, L, W, scale, causal, seqlens_k=ints(lens), block_table=cache.table,
                             queries=None if queries is None else ints(queries))
    torch.cuda.synchronize()
    W = f64(W)
    w, err = dec.key_weights(np.nan_to_num(f64(Q)), cache.rows[0], np.nan_to_num(f64(L), nan=0.0, neginf=-np.inf), lens, scale, causal, queries)
    for b in range(B):
        n = lens[b]
        assert (W[b, :, n:] == W0[b, :, n:]).all()
        tol = 2 * err[b] + (w[b] + W0[b, :, :n]) * (nq * (hq // hkv) + 8) / 2**24
        assert (np.abs(W[b, :, :n] - W0[b, :, :n] - w[b]) <= tol).all(), (b, np.max(np.abs(W[b, :, :n] - W0[b, :, :n] - w[b]) / np.maximum(tol, 1e-30)))


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,nq,hq,hkv,slots,page,lens", [
    (1, 1, 1, 1, 1, 0, [1]),
    (4, 1, 32, 8, 1100, 64, [1100, 1, 0, 513]),   # one row tile, several workgroups a head
    (3, 8, 8, 2, 200, 0, [200, 8, 40]),           # 32 rows: the most that the step kernel takes
    (3, 9, 8, 2, 200, 64, [200, 9, 33]),          # 36 rows: the prompt kernel
    (2, 300, 4, 2, 300, 0, [300, 300]),           # a prompt among its own keys
    (2, 67, 6, 2, 600, 128, [600, 67]),           # three heads a group: rows off the tiles' edges
    (11, 1, 4, 2, 260, 64, [260, 1, 2, 33, 64, 65, 96, 97, 128, 129, 200]),  # eight sequences, and three
    (9, 5, 12, 1, 150, 0, [150, 5, 6, 31, 32, 33, 64, 65, 149]),             # 60 rows
    (2, 150, 6, 2, 200, 64, [200, 150]),          # 450 rows, three heads a group: the prompt kernel
    (1, 33, 16, 1, 50, 0, [40]),                  # 528 rows, one query past a tile
])
def test_weights(dtype, d, B, nq, hq, hkv, slots, page, lens):
    check_weights(dtype, d, B, nq, hq, hkv, slots, page, lens)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f16", 128), ("bf16", 128)])
@pytest.mark.parametrize("B,nq,hq,hkv,slots,page,lens", [
    (64, 1, 8, 8, 700, 64, (EDGES * 3)[:64]),    # 512 keys a workgroup: up to four tiles a wavefront
    (48, 3, 16, 8, 700, 0, (EDGES * 2)[:48]),    # (queries before the first key among them)
    (16, 2, 8, 8, 700, 0, EDGES[:16]),           # 256
    (24, 5, 64, 8, 800, 64, EDGES),              # 40 rows, 384
])
def test_weights_of_many_sequences(dtype, d, B, nq, hq, hkv, slots, page, lens):
    check_weights(dtype, d, B, nq, hq, hkv, slots, page, lens)


@pytest.mark.parametrize("nq", [3, 50, 140])
def test_weights_of_accepted_queries_without_causal_rule_and_of_rows_without_keys(nq):
    lens = [120, min(nq, 120), 1, 0]
    check_weights("bf16", 64, 4, nq, 4, 2, 120, 0, lens)  # (sequence 2: queries before the first key, with L = -inf)
    check_weights("bf16", 64, 4, nq, 4, 2, 120, 0, lens, causal=False)
    check_weights("f16", 128, 4, nq, 4, 2, 120, 64, [120, 120, 60, 90], queries=[nq, 1, 0, 2])
    check_weights("bf16", 64, 4, nq, 4, 2, 120, 0, [120, 120, 60, 90], queries=[nq - 1, 1, nq, 2], causal=False)


@pytest.mark.parametrize("nq", [1, 12, 300])
def test_weights_take_a_logsumexp_of_any_strides(nq):
    r = rng(nq)
    Q, K = gpu(r.normal(size=(2, nq, 4, 64)), torch.bfloat16), gpu(r.normal(size=(2, 320, 2, 64)), torch.bfloat16)
    _, L = binding.fa_kvcache_fwd(Q, K, K, 0.125, True)
    got = []
    for x in (L, L.transpose(1, 2).contiguous().transpose(1, 2), L.permute(2, 1, 0).contiguous().permute(2, 1, 0), L.repeat(1, 1, 2)[..., :nq]):
        W = torch.zeros((2, 2, 320), device="cuda")
        binding.fa_cache_weights(Q, K, x, W, 0.125, True)
        got.append(W)
    assert all(torch.equal(got[0], x) for x in got[1:]) and (got[0] > 0).all()


def test_weights_do_not_see_what_is_masked():
    """Infinities and NaN in keys that no counted query sees stay out of every sum."""
    for nq in (3, 40):
        r = rng(nq)
        K = gpu(r.normal(size=(1, 200, 1, 64)), torch.bfloat16)
        Q = gpu(r.normal(size=(1, nq, 2, 64)), torch.bfloat16)
        L = torch.full((1, 2, nq), 5.0, device="cuda")
        W = torch.zeros((1, 1, 200), device="cuda")
        binding.fa_cache_weights(Q, K, L, W, 0.125, True, seqlens_k=ints([150]), queries=ints([1]))
        clean = W.clone()
        K[0, 150 - nq + 1:, :, ::2] = float("inf")
        K[0, 150 - nq + 1:, :, 1::2] = float("nan")
        W.zero_()
        binding.fa_cache_weights(Q, K, L, W, 0.125, True, seqlens_k=ints([150]), queries=ints([1]))
        assert torch.equal(W, clean) and W[0, 0, 150 - nq].item() > 0 and (W[0, 0, 150 - nq + 1:] == 0).all()


# ---------------------------------------------------------------------------------------------

def check_evict(dtype, B, hkv, d, slots, page, lens, budget, sinks, recent, weights=None, in_place=False, positions=None):
    r = rng(B + d + slots + budget)
    cache = Cache(r, dtype, B, slots, hkv, d, page, lens)
    w = r.exponential(size=(B, hkv, slots)) if weights is None else weights(r, (B, hkv, slots))
    pos = np.argsort(r.random((B, hkv, slots)), -1) if positions is None else positions
    W, P, n = gpu(w, torch.float32), ints(pos.tolist()), ints(lens)
    w = f64(W)
    oK, oV = (f64(cache.read(x)) for x in (cache.K, cache.V))
    out = {} if in_place else dict(weights_out=torch.full_like(W, -7), positions_out=torch.full_like(P, -7), seqlens_out=torch.full_like(n, -7))
    Wo, Po, no = binding.fa_cache_evict(cache.K, cache.V, W, P, n, budget, sinks, recent, block_table=cache.table, **out)
    torch.cuda.synchronize()
    if in_place:
        assert Wo is W and Po is P and no is n
    else:
        assert np.array_equal(f64(W), w, equal_nan=True) and n.tolist() == lens
    assert no.tolist() == [min(x, budget) for x in lens]
    K, V, Wo, Po = f64(cache.read(cache.K)), f64(cache.read(cache.V)), f64(Wo), Po.cpu().numpy()
    for b in range(B):
        for g in range(hkv):
            src = dec.kept_slots(w[b, g], pos[b, g], lens[b], budget, sinks, recent)
            m = len(src)
            assert np.array_equal(Po[b, g, :m], pos[b, g, src])
            assert np.array_equal(Wo[b, g, :m], w[b, g, src], equal_nan=True)
            assert np.array_equal(K[b, :m, g], oK[b, src, g], equal_nan=True) and np.array_equal(V[b, :m, g], oV[b, src, g], equal_nan=True)
            assert np.array_equal(K[b, m:, g], oK[b, m:, g], equal_nan=True)
            if in_place:
                assert np.array_equal(Wo[b, g, m:], w[b, g, m:], equal_nan=True) and np.array_equal(Po[b, g, m:], pos[b, g, m:])
            else:
                assert (Wo[b, g, m:] == -7).all() and (Po[b, g, m:] == -7).all()


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,hkv,d,slots,page,lens,budget,sinks,recent", [
    (1, 1, 8, 2, 0, [2], 1, 0, 0),
    (3, 2, 64, 200, 0, [200, 100, 101], 100, 4, 20),
    (4, 2, 128, 300, 64, [300, 0, 65, 1], 64, 0, 64),
    (2, 3, 72, 2500, 0, [2500, 2047], 1000, 4, 100),
    (2, 1, 8, 5000, 0, [5000, 4100], 4050, 4, 100),     # 1024 threads, eight keys a lane in registers
    (1, 2, 64, 9000, 128, [8999], 8000, 1, 7),          # 32 keys a lane in registers
    (1, 2, 8, 33000, 0, [32999], 500, 1, 7),            # keys formed anew
    (2, 1, 256, 2048, 64, [2048, 1500], 17, 4, 4),
])
def test_evict(B, hkv, d, slots, page, lens, budget, sinks, recent, in_place):
    check_evict("bf16" if d != 64 else "f16", B, hkv, d, slots, page, lens, budget, sinks, recent, in_place=in_place)


@pytest.mark.parametrize("slots", [700, 8500, 33000])
def test_evict_equal_and_odd_weights(slots):
    """Ties go to the lower slot; zeros of both signs are one; NaN is less than everything, infinities count; few distinct values."""
    lens, some = [slots, slots - 333], [0.0, -0.0, np.nan, np.inf, -np.inf, 1.0, -1.0, 1e-42]
    for weights in (lambda r, s: np.zeros(s), lambda r, s: r.choice(some, s), lambda r, s: np.full(s, np.nan), lambda r, s: 1 + r.integers(0, 3, s) * 2.0**-23):
        check_evict("bf16", 2, 2, 8, slots, 0, lens, slots // 3, 2, 5, weights=weights, in_place=True)


def test_evict_of_protected_positions_beyond_the_budget():
    """Positions that are not all different may protect more slots than there are to keep: the lowest slots of them stay."""
    pos = np.zeros((1, 1, 300), int)
    check_evict("bf16", 1, 1, 8, 300, 0, [300], 50, 1, 0, positions=pos)
    pos = np.full((1, 1, 300), 2**31 - 1)
    check_evict("bf16", 1, 1, 8, 300, 0, [300], 50, 0, 1, positions=pos)
    check_evict("bf16", 1, 1, 8, 300, 0, [300], 50, 0, 0, positions=pos)
    check_evict("bf16", 1, 1, 8, 300, 0, [300], 50, 0, 5, positions=-pos - 1)


@pytest.mark.parametrize("slots,page,lens,budget", [(362, 0, [300, 361, 362, 1], 298), (2112, 64, [2049, 2056, 2111, 100], 2048), (5000, 0, [4500, 4999], 3000),
                                                    (9000, 0, [8200, 8999], 500), (33000, 0, [32768, 32900], 500)])
def test_evict_does_not_look_past_a_length(slots, page, lens, budget):
    """Slots past a length hold whatever an earlier use left there, newer positions than any key's and the largest weights among it."""
    r = rng(slots)
    B, hkv = len(lens), 2
    pos = np.argsort(r.random((B, hkv, slots)), -1)
    w = r.exponential(size=(B, hkv, slots))
    for b, n in enumerate(lens):
        pos[b, :, :n] = np.argsort(r.random((hkv, n)), -1)
        pos[b, :, n:] = 10**6 + np.arange(slots - n)
        w[b, :, n:] = 1e30
    for in_place in (False, True):
        check_evict("bf16", B, hkv, 64, slots, page, lens, budget, 4, budget // 4, weights=lambda r, s: w, in_place=in_place, positions=pos)


# ---------------------------------------------------------------------------------------------

def distributions(r, B, k, V, spread=3.0):
    logits = spread * r.normal(size=(B, k + 1, V))
    near = logits[:, :k] + 0.7 * r.normal(size=(B, k, V))
    q = np.exp(near - near.max(-1, keepdims=True))
    q /= q.sum(-1, keepdims=True)
    drafts = (near + r.gumbel(size=near.shape)).argmax(-1)
    return logits, q, drafts


def check_verify(drafts, q, target, uniform, logits, inv_t, q_type, type_, pad=0):
    def wide(x, dtype):  # rows that are slices of wider ones
        t = torch.full((*x.shape[:2], x.shape[2] + pad), float("nan"), dtype=dtype, device="cuda")
        t[..., :x.shape[2]] = torch.from_numpy(x)
        return t[..., :x.shape[2]]
    T, D = wide(target, type_), None if q is None else wide(q, q_type)
    u = gpu(uniform, torch.float32)
    tokens, accepted = binding.fa_verify_drafts(ints(drafts.tolist()) if drafts.shape[1] else torch.zeros(drafts.shape, dtype=torch.int32, device="cuda"),
                                                D, T, u, logits=logits, inv_temperature=inv_t)
    torch.cuda.synchronize()
    et, ea, margin = dec.verify(drafts, None if q is None else f64(D), f64(T), f64(u), logits, float(np.float32(inv_t)))
    # (an input on the border of a decision would be no test: float32 settles acceptances, float64 draws)
    assert margin > 1e-9
    assert accepted.tolist() == ea.tolist()
    assert tokens.tolist() == et.tolist()


@pytest.mark.parametrize("q_type,type_,logits", [
    (torch.float32, torch.float32, False), (torch.float32, torch.bfloat16, True), (torch.bfloat16, torch.float16, True),
    (torch.float16, torch.bfloat16, False), (torch.float32, torch.float32, True), (None, torch.float32, True), (None, torch.float16, False)])
@pytest.mark.parametrize("B,k,V,pad", [(1, 1, 1, 0), (6, 4, 7, 1), (5, 3, 4096, 0), (4, 7, 4097, 3), (16, 2, 20001, 0)])
def test_verify(q_type, type_, logits, B, k, V, pad):
    r = rng(B + k + V)
    l, q, drafts = distributions(r, B, k, V)
    p = np.exp(l - l.max(-1, keepdims=True))
    target = l if logits else p / p.sum(-1, keepdims=True)
    if q_type is None:
        drafts = np.where(r.random((B, k)) < 0.7, l[:, :k].argmax(-1), drafts)
    check_verify(drafts, None if q_type is None else q, target, r.random((B, k + 1)), logits, 1.3 if logits else 1.0, q_type, type_, pad)


@pytest.mark.parametrize("q_type", [torch.float32, torch.bfloat16, torch.float16, None])
@pytest.mark.parametrize("type_", [torch.float32, torch.bfloat16, torch.float16])
def test_verify_types(q_type, type_):
    """Every pair of types, as logits and as probabilities, over more segments than a wavefront has lanes."""
    r = rng(21)
    l, q, drafts = distributions(r, 3, 5, 140001)
    p = np.exp(l - l.max(-1, keepdims=True))
    for logits, target in ((True, l), (False, p / p.sum(-1, keepdims=True))):
        check_verify(drafts, None if q_type is None else q, target, r.random((3, 6)), logits, 0.9 if logits else 1.0, q_type, type_)


def test_verify_without_drafts_and_with_absent_ones():
    r = rng(8)
    l, q, drafts = distributions(r, 6, 3, 500)
    check_verify(drafts[:, :0], None, l[:, :1], r.random((6, 1)), True, 0.8, None, torch.float32)
    drafts[0, 0], drafts[1, 2], drafts[2, 1], drafts[3, 0] = -1, -1, 500, 2**31 - 1
    check_verify(drafts, q, l, r.random((6, 4)), True, 1.0, torch.float32, torch.float32)
    check_verify(drafts, None, l, r.random((6, 4)), True, 1.0, None, torch.float32)


def test_verify_masked_logits():
    """Logits of -inf (top-k, a grammar) are probabilities of 0, whole rows of them leave no token."""
    r = rng(9)
    l, q, drafts = distributions(r, 8, 3, 9000)
    l = np.where(r.random(l.shape) < 0.99, -np.inf, l)
    l[0], l[1, 0, 4000:] = -np.inf, -np.inf
    check_verify(drafts, q, l, r.random((8, 4)), True, 1.0, torch.float32, torch.bfloat16)


def test_verify_random_numbers_at_the_ends():
    """uniform = 0 draws the first token of weight above 0, the largest below 1 one at the end; p = q accepts everything."""
    r = rng(10)
    _, q, drafts = distributions(r, 4, 3, 5000)
    p = np.concatenate([q, q[:, :1]], 1)
    p[:, 3, :7] = 0
    u = np.zeros((4, 4), np.float32)
    u[:, :3] = np.nextafter(np.float32(1), np.float32(0))
    u[2:, 3] = np.nextafter(np.float32(1), np.float32(0))
    args = [gpu(x, torch.float32) for x in (q, p, u)]
    tokens, accepted = binding.fa_verify_drafts(ints(drafts.tolist()), *args)
    assert accepted.tolist() == [3] * 4 and tokens[:, :3].tolist() == drafts.tolist()
    assert tokens[:2, 3].tolist() == [7, 7] and (tokens[2:, 3] > 4000).all() and (tokens[2:, 3] < 5000).all()


def test_verify_many_draws_follow_the_target():
    """What is drawn, over random numbers that cover the unit interval evenly, is the target's distribution."""
    n, V = 4096, 50
    r = rng(11)
    p = r.dirichlet(np.ones(V)).astype(np.float32)
    u = ((np.arange(n) + 0.5) / n).astype(np.float32)[:, None]
    tokens, _ = binding.fa_verify_drafts(torch.zeros((n, 0), dtype=torch.int32, device="cuda"), None, gpu(p, torch.float32).expand(n, 1, V).contiguous(),
                                         gpu(u, torch.float32))
    count = np.bincount(tokens[:, 0].cpu().numpy(), minlength=V)
    assert np.abs(count / n - p / p.sum()).max() <= 2 / n


def test_caches_past_32_bit_offsets():
    """A pool of pages whose last rows lie past 2^31 elements (and 2^32 bytes): every operator addresses it in 64 bits."""
    page, hkv, d, hq = 256, 8, 128, 16
    pages = 2**31 // (page * hkv * d) + 8
    r = rng(12)
    K, V = (torch.empty((pages, page, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = ints([[pages - 1, pages - 3], [pages - 2, pages - 5]])
    small = Cache(r, "bf16", 2, 512, hkv, d, 0, [512, 512])
    for big, x in ((K, small.K), (V, small.V)):
        for b in range(2):
            for i in range(2):
                big[table[b, i].item()] = x[b, 256 * i:256 * i + 256]
    Q, Kp, Vp = (gpu(r.normal(size=s), torch.bfloat16) for s in ((2, 1, hq, d), (100, hkv, d), (100, hkv, d)))
    lens = ints([512, 300])
    a = binding.fa_prefix_fwd(Q, Kp, Vp, K, V, 0.1, True, seqlens_k=lens, block_table=table)
    b = binding.fa_prefix_fwd(Q, Kp, Vp, small.K, small.V, 0.1, True, seqlens_k=lens)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    Kn, Vn = (gpu(r.normal(size=(2, 1, hkv, d)), torch.bfloat16) for _ in range(2))
    W = [gpu(r.random((2, hkv, 512)), torch.float32)] * 1
    W = [W[0], W[0].clone()]
    P = [torch.arange(512, dtype=torch.int32, device="cuda").expand(2, hkv, 512).contiguous() for _ in range(2)]
    n = [lens, lens.clone()]
    for i, (k, v, t) in enumerate(((K, V, table), (small.K, small.V, None))):
        binding.fa_cache_append(Kn, Vn, k, v, n[i], block_table=t, weights=W[i], positions=P[i])
        binding.fa_cache_weights(Q, k, a[1], W[i], 0.1, True, seqlens_k=n[i], block_table=t)
        binding.fa_cache_evict(k, v, W[i], P[i], n[i], 200, 4, 30, block_table=t)
    assert torch.equal(W[0], W[1]) and torch.equal(P[0], P[1]) and n[0].tolist() == n[1].tolist() == [200, 200]
    for big, x in ((K, small.K), (V, small.V)):
        for s in range(2):
            assert torch.equal(big[table[s, 0].item()], x[s, :256])
            assert torch.equal(big[table[s, 1].item()], x[s, 256:])


def test_a_step_in_a_graph():
    """Append, attend, weigh, verify, evict, captured once: every replay equals the eager calls on the same state."""
    r = rng(13)
    B, nq, hq, hkv, d, slots, n_p, V, budget = 4, 3, 8, 2, 64, 128, 200, 3000, 100
    cache = Cache(r, "bf16", B, slots, hkv, d, 0, [slots] * B)
    lens = ints([90, 98, 3, 50])
    first = ints([190, 298, 3, 50])
    W, P = torch.zeros((B, hkv, slots), device="cuda"), torch.arange(slots, dtype=torch.int32, device="cuda").expand(B, hkv, slots).contiguous()
    Kp, Vp = (gpu(r.normal(size=(n_p, hkv, d)), torch.bfloat16) for _ in range(2))
    new = [gpu(r.normal(size=s), torch.bfloat16) for s in ((B, nq, hq, d), (B, nq, hkv, d), (B, nq, hkv, d))]
    l, q, drafts = distributions(r, B, nq - 1, V)
    target, probs, tokens, u = gpu(l, torch.bfloat16), gpu(q, torch.float32), ints(drafts.tolist()), gpu(r.random((B, nq)), torch.float32)

    def step():
        Q, Kn, Vn = new
        lens.add_(nq)
        binding.fa_cache_append(Kn, Vn, cache.K, cache.V, lens, weights=W, positions=P, first_position=first)
        O, L = binding.fa_prefix_fwd(Q, Kp, Vp, cache.K, cache.V, 0.125, True, seqlens_k=lens)
        out, acc = binding.fa_verify_drafts(tokens, probs, target, u, logits=True)
        ok = acc + 1
        binding.fa_cache_weights(Q, cache.K, L, W, 0.125, True, seqlens_k=lens, queries=ok)
        lens.add_(ok - nq)
        first.add_(ok)
        binding.fa_cache_evict(cache.K, cache.V, W, P, lens, budget, 4, 20)
        return O, L, out, acc

    state = [cache.K, cache.V, lens, first, W, P]
    start = [x.clone() for x in state]

    def back(to):
        for x, y in zip(state, to):
            x.copy_(y)

    step()
    torch.cuda.synchronize()
    back(start)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    back(start)
    for i in range(4):
        for x in new + [target]:
            x.copy_(gpu(r.normal(size=tuple(x.shape)), torch.bfloat16))
        u.copy_(gpu(r.random((B, nq)), torch.float32))
        before = [x.clone() for x in state]
        graph.replay()
        torch.cuda.synchronize()
        got, after = [x.clone() for x in out], [x.clone() for x in state]
        back(before)
        for x, y in zip(step(), got):
            assert torch.equal(x, y)
        for x, y in zip(state, after):
            assert torch.equal(x.nan_to_num(9) if x.is_floating_point() else x, y.nan_to_num(9) if y.is_floating_point() else y)
