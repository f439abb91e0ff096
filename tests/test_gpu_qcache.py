"""GPU parity of the operators on caches in 4 or 8 bits (fa_qcache_append, fa_qcache_read, fa_qcache_fwd) against their definitions in
float64: lengths of 0 and 1, one row and many, slabs and pages, lengths off every tile edge, what no call may read made NaN, rows that see
nothing, keys and values that are NaN where a row does and does not see them, strides, other streams, captured graphs.

What is quantised and read back is exact. Attention: e = half a step of the element type (2^-8 bfloat16, 2^-11 half precision); O: P rounded
to the type (e of every p |v|) and O itself (e of |O|), each score off by d 2^-24 of its sum of |q k| and by a few float32
roundings of itself, and half precision's P by up to 2^-25 of the row's largest where it is subnormal. LSE: the scores' part alone."""
import numpy as np
import pytest

from oracle import decoding_oracle as dec
from oracle import qcache_oracle as orc
from paper_2307_08691_amd import binding

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from qcaches import LONG, Cache, TYPES, f64, gpu, ints, long_lengths  # noqa: E402

BITS = [(4, 4), (8, 4), (4, 8), (8, 8)]


def rng(seed):
    return np.random.default_rng(seed)


# ---- append

def check_append(dtype, d, B, nq, hkv, slots, page, lens, k_bits, v_bits, fused, values=None, outs=True, seed=0):
    r = rng(seed + d + nq)
    cache = Cache(r, B, slots, hkv, d, page, [max(0, n - nq) for n in lens], k_bits, v_bits)
    before = cache.held()
    if values is None:
        values = r.normal(size=(2, B, nq, hkv, d)) * np.exp2(r.integers(-8, 8, size=(2, B, nq, hkv, 1)))
    new = [gpu(x, TYPES[dtype]) for x in values]
    if fused:  # slices of one tensor, with other things between them
        wide = torch.full((B, nq, 3 * hkv + 1, d), float("nan"), dtype=TYPES[dtype], device="cuda")
        wide[:, :, hkv:2 * hkv], wide[:, :, 2 * hkv:3 * hkv] = new
        new = [wide[:, :, hkv:2 * hkv], wide[:, :, 2 * hkv:3 * hkv]]
    Ko, Vo = (torch.full((B, nq, hkv, d), 7.0, dtype=TYPES[dtype], device="cuda") for _ in range(2)) if outs else (None, None)
    more = dict(cache.more, seqlens_k=ints(lens))
    assert binding.fa_qcache_append(*new, cache.q, Kout=Ko, Vout=Vo, **more) is cache.q
    torch.cuda.synchronize()
    after = cache.held()
    for i, bits in enumerate((k_bits, v_bits)):
        x = f64(new[i])
        codes, scales = orc.quantise(x, bits)
        want = [before[2 * i].copy(), before[2 * i + 1].copy()]
        out = np.full(x.shape, 7.0)
        for b in range(B):
            for q in range(nq):
                c = lens[b] - nq + q
                if 0 <= c < slots:
                    want[0][b, c], want[1][b, c] = orc.packed(codes[b, q], bits), scales[b, q]
                    out[b, q] = orc.values(codes[b, q], scales[b, q], bits)
        assert (after[2 * i] == want[0]).all() and (after[2 * i + 1] == want[1]).all()
        if outs:
            out = f64(torch.from_numpy(out).to(TYPES[dtype]))  # (exact, but past the type's range: infinite)
            assert np.array_equal(f64((Ko, Vo)[i]), out, equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("k_bits,v_bits", BITS)
@pytest.mark.parametrize("d,B,nq,hkv,slots,page,lens,fused", [
    (32, 1, 1, 1, 1, 0, [1], False),                    # the smallest call
    (64, 3, 1, 2, 130, 0, [130, 1, 66], True),          # a step, an odd number of slots
    (128, 3, 7, 8, 192, 64, [192, 66, 7], True),        # across pages
    (96, 2, 131, 3, 300, 128, [300, 131], False),       # a prompt, d of three blocks
    (256, 2, 2, 1, 64, 64, [2, 64], False),
])
def test_append(dtype, k_bits, v_bits, d, B, nq, hkv, slots, page, lens, fused):
    check_append(dtype, d, B, nq, hkv, slots, page, lens, k_bits, v_bits, fused)


@pytest.mark.parametrize("page", [0, 64])
def test_append_drops_rows_without_a_slot(page):
    """More new rows than the length counts, lengths of no cache, and outputs left alone there."""
    check_append("bf16", 64, 5, 3, 2, 100, page, [2, 101, 0, -5, 3], 4, 8, False)
    check_append("f16", 64, 5, 3, 2, 100, page, [2, 101, 0, 100, 1], 8, 4, True, outs=False)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("bits", [4, 8])
def test_append_of_every_number(dtype, bits):
    """All 16-bit numbers, in blocks of their own and in the company of larger ones; halves, subnormals, zeros of both signs."""
    every = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(TYPES[dtype])
    x = every.double().numpy()
    alone = x[np.isfinite(x)].reshape(-1, 32)
    mixed = np.repeat(x[np.isfinite(x)][:, None], 32, 1)
    mixed[:, 1:] = np.exp2(rng(1).integers(-14, 15, size=(len(mixed), 1)))  # (each with a block mate of any size)
    both = np.concatenate([alone, mixed])
    n = len(both) // 8 * 8
    values = both[:n].reshape(1, n // 8, 4, 64)
    check_append(dtype, 64, 1, n // 8, 4, n // 8, 0, [n // 8], bits, 12 - bits, False, values=np.stack([values, values[:, ::-1]]))


@pytest.mark.parametrize("bits", [4, 8])
def test_append_of_what_is_no_number(bits):
    v = rng(5).normal(size=(2, 2, 3, 2, 96))
    v[0, 0, 1, 1, 40], v[0, 1, 2, 0, 95], v[1, 1, 0, 0, 0] = np.inf, np.nan, -np.inf
    check_append("bf16", 96, 2, 3, 2, 70, 0, [70, 3], bits, 12 - bits, False, values=v)


def test_append_rounds_in_place():
    r = rng(6)
    K, V = (gpu(r.normal(size=(2, 5, 2, 64)), torch.bfloat16) for _ in range(2))
    k, v = K.clone(), V.clone()
    a, b = Cache(r, 2, 64, 2, 64, 0, [0, 0], 4, 8), Cache(r, 2, 64, 2, 64, 0, [0, 0], 4, 8)
    Ko, Vo = torch.empty_like(K), torch.empty_like(V)
    binding.fa_qcache_append(K, V, a.q, seqlens_k=ints([5, 6]), Kout=Ko, Vout=Vo)
    binding.fa_qcache_append(k, v, b.q, seqlens_k=ints([5, 6]), Kout=k, Vout=v)
    assert torch.equal(k, Ko) and torch.equal(v, Vo) and not torch.equal(K, Ko)


# ---- read

@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("k_bits,v_bits", BITS)
@pytest.mark.parametrize("d,hkv,slots,page", [(32, 1, 1, 0), (64, 2, 130, 0), (128, 8, 192, 64), (96, 3, 300, 128), (256, 1, 70, 64)])
def test_read(dtype, k_bits, v_bits, d, hkv, slots, page):
    r = rng(d + slots)
    lens = [slots, 0, 1, (slots + 1) // 2]
    c = Cache(r, 4, slots, hkv, d, page, lens, k_bits, v_bits)
    for N, first in ((slots, None), (slots + 3, [0, 0, 0, 0]), (max(1, slots // 3), [slots - 1, 5, -2, 1])):
        K, V = (torch.full((4, N, hkv, d), 7.0, dtype=TYPES[dtype], device="cuda") for _ in range(2))
        out = binding.fa_qcache_read(c.q, K, V, first=None if first is None else ints(first), **c.more)
        assert out[0] is K and out[1] is V
        for got, rows in ((K, c.rows[0]), (V, c.rows[1])):
            want = np.full(got.shape, 7.0)
            for b in range(4):
                for i in range(N):
                    slot = i + (first[b] if first else 0)
                    if 0 <= slot < lens[b]:
                        want[b, i] = rows[b, slot]
            assert np.array_equal(f64(got), want)
    # packed: more rows than a sequence holds, fewer, none; rows past the last sequence; offsets past the outputs
    takes = [min(slots, 3), 2, 1, (slots + 1) // 2]
    cu = np.concatenate([[0], np.cumsum(takes)])
    for T in (cu[-1], cu[-1] + 5, max(1, cu[-1] - 1)):
        K, V = (torch.full((int(T), hkv, d), 7.0, dtype=TYPES[dtype], device="cuda") for _ in range(2))
        binding.fa_qcache_read(c.q, K, V, cu_seqlens=ints(cu.tolist()), **c.more)
        for got, rows in ((K, c.rows[0]), (V, c.rows[1])):
            want = np.full(got.shape, 7.0)
            for b in range(4):
                for i in range(min(takes[b], lens[b])):
                    if cu[b] + i < T:
                        want[cu[b] + i] = rows[b, i]
            assert np.array_equal(f64(got), want)


def test_read_of_no_lengths_is_all_slots_and_blocks_without_numbers_are_nan():
    c = Cache(rng(8), 2, 66, 2, 64, 0, [66, 66], 4, 8)
    c.q.Kscales[1, 0, 5, 1] = 255
    c.q.Vscales[0, 1, 65, 0] = 255
    K, V = (torch.zeros((2, 66, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    binding.fa_qcache_read(c.q, K, V)
    c.rows[0][1, 5, 0, 32:] = c.rows[1][0, 65, 1, :32] = np.nan
    assert np.array_equal(f64(K), c.rows[0], equal_nan=True) and np.array_equal(f64(V), c.rows[1], equal_nan=True)


def test_read_of_windows_longer_than_the_cache():
    """Wherever the window begins, the rows that have a slot are found, and no others written."""
    first = [0, -1, -63, -64, -65, -430, -499, -500, 69, 70, -2**31, 2**31 - 1, 5]
    lens = [70] * (len(first) - 1) + [0]
    c = Cache(rng(20), len(first), 70, 2, 64, 0, lens, 4, 8)
    K, V = (torch.full((len(first), 500, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    binding.fa_qcache_read(c.q, K, V, first=ints(first), **c.more)
    for got, rows in ((K, c.rows[0]), (V, c.rows[1])):
        want = np.full(got.shape, 7.0)
        for b in range(len(first)):
            lo, hi = max(0, -first[b]), min(500, lens[b] - first[b])
            if lo < hi:
                want[b, lo:hi] = rows[b, first[b] + lo:first[b] + hi]
        assert np.array_equal(f64(got), want)


# ---- attention

def check(dtype, d, B, nq, hq, hkv, slots, page, lens, k_bits, v_bits, causal=True, seed=0, scale=None, cache=None, Q=None, call=None):
    r = rng(seed + d + nq + slots)
    scale = scale or d**-0.5
    cache = cache or Cache(r, B, slots, hkv, d, page, lens, k_bits, v_bits)
    Q = gpu(r.normal(size=(B, nq, hq, d)), TYPES[dtype]) if Q is None else Q
    call = call or binding.fa_qcache_fwd
    O, L = call(Q, cache.q, scale, causal, **cache.more)
    torch.cuda.synchronize()
    none = np.zeros((0, hkv, d))
    rows = [[np.nan_to_num(x[b][:lens[b]], nan=0.0) for b in range(B)] for x in cache.rows]
    eO, eL, A, M = dec.prefix_forward(f64(Q), none, none, *rows, lens, scale, causal)
    e = torch.finfo(TYPES[dtype]).eps / 2
    L, O = f64(L), f64(O)
    empty = eL == -np.inf
    assert (L[empty] == -np.inf).all() and (O.transpose(0, 2, 1, 3)[empty] == 0).all()
    score = np.where(empty, 0, M * d / 2**24 + (M + np.abs(np.where(empty, 0, eL)) + 8) / 2**21)
    nan = np.isnan(L) if any(np.isnan(x[b][:lens[b]]).any() for x in cache.rows for b in range(B)) else np.zeros(L.shape, bool)
    ok = ~empty & ~nan
    assert (np.abs(L[ok] - eL[ok]) <= score[ok]).all()
    small = slots * 4.0 / 2**25 * np.abs(np.concatenate([x.reshape(-1) for x in rows[1]] + [np.zeros(1)])).max() if dtype == "f16" else 0.0
    tol = e * (A + np.abs(eO)) * (1 + 2 * e) + A * 4 * score.transpose(0, 2, 1)[..., None] + small
    good = ~np.isnan(O)
    assert (np.abs(O - eO)[good] <= np.broadcast_to(tol, O.shape)[good]).all()
    if not any(np.isnan(x[b][:lens[b]]).any() for x in cache.rows for b in range(B)):
        assert good.all()
    return O, L


SHAPES = [
    (1, 1, 1, 1, 1, 0, [1]),                                  # the smallest call
    (3, 1, 8, 2, 300, 0, [300, 1, 0]),                        # four rows a head; a cache of one key, an empty one
    (5, 1, 32, 4, 200, 64, [200, 64, 65, 0, 1]),              # pages that end inside tiles
    (2, 4, 16, 2, 1500, 64, [1500, 4]),                       # 32 rows: two tiles of rows, several shares
    (2, 5, 8, 2, 700, 256, [700, 33]),                        # 20 rows: the second tile of rows partly empty
    (2, 9, 8, 2, 200, 0, [200, 9]),                           # 36 rows: a block of 32 and one of four
    (2, 70, 4, 1, 500, 128, [500, 70]),                       # 280 rows under the causal rule
    (150, 1, 2, 1, 70, 0, [(11 * i) % 71 for i in range(150)]),  # many short sequences, some of them empty
    (3, 1, 4, 2, 1100, 64, [1100, 0, 1]),                     # caches that are cut, one of them empty
    (300, 1, 2, 2, 300, 0, [(37 * i) % 300 * (i % 7 > 0) for i in range(300)]),  # more sequences than a workgroup has threads, runs over several
    (2, 130, 4, 2, 1200, 64, [1200, 64]),                     # wide blocks, some of which see no key at all
]


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("k_bits,v_bits", BITS)
@pytest.mark.parametrize("B,nq,hq,hkv,slots,page,lens", SHAPES)
def test_attend(dtype, d, k_bits, v_bits, B, nq, hq, hkv, slots, page, lens):
    check(dtype, d, B, nq, hq, hkv, slots, page, lens, k_bits, v_bits)


@pytest.mark.parametrize("nq,lens", [(1, [100, 0, 37]), (3, [100, 3, 1]), (40, [100, 40, 12])])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_without_causal_rule_and_with_more_queries_than_keys(nq, lens, d):
    for causal in (False, True):
        check("bf16", d, 3, nq, 4, 2, 100, 0, lens, 4, 8, causal=causal)
        check("f16", d, 3, nq, 4, 2, 128, 64, lens, 8, 4, causal=causal)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("k_bits,v_bits", BITS)
def test_attend_with_groups_of_five_and_slabs_of_odd_lengths(d, k_bits, v_bits):
    check("bf16", d, 3, 1, 10, 2, 301, 0, [301, 7, 150], k_bits, v_bits)
    check("f16", d, 3, 7, 10, 2, 301, 0, [301, 7, 150], k_bits, v_bits)
    check("bf16", d, 3, 30, 10, 2, 1277, 0, [1277, 3, 640], k_bits, v_bits)  # wide blocks


EDGES = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 159, 160, 161, 255, 256, 257, 287, 288, 289, 383, 384, 385, 511, 512, 513, 699]


@pytest.mark.parametrize("dtype,d,k_bits,v_bits,page", [("bf16", 128, 4, 4, 0), ("f16", 64, 8, 8, 64), ("bf16", 64, 4, 8, 64), ("f16", 128, 8, 4, 256)])
def test_attend_at_every_edge(dtype, d, k_bits, v_bits, page):
    for nq in (1, 3, 17):
        check(dtype, d, len(EDGES), nq, 4, 1, 768, page, EDGES, k_bits, v_bits)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_attend_over_a_long_cache(dtype):
    """Many shares; page numbers are requested again and again."""
    check(dtype, 64, 1, 1, 4, 1, 20000, 64, [19999], 4, 8)
    check(dtype, 128, 2, 2, 2, 1, 9000, 0, [9000, 8191], 8, 4)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
def test_attend_to_scores_that_grow_and_spread(dtype, d):
    """The running reference has to be advanced, early, late and in single rows."""
    r = rng(9)
    B, nq, hq, hkv, slots = 2, 2, 8, 2, 900
    K = r.normal(size=(B, slots, hkv, d)) * np.linspace(0.1, 6, slots)[None, :, None, None]
    K[1, 500:505] *= 4
    c = Cache(r, B, slots, hkv, d, 0, [900, 777], 8, 8, data=[K, r.normal(size=K.shape)])
    check(dtype, d, B, nq, hq, hkv, slots, 0, [900, 777], 8, 8, cache=c)
    check(dtype, d, B, nq, hq, hkv, slots, 0, [900, 777], 8, 8, cache=c, scale=0.02)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("k_bits,v_bits", BITS)
@pytest.mark.parametrize("nq", [1, 5, 40])
def test_what_a_row_does_not_see_may_be_nan(d, k_bits, v_bits, nq):
    """Blocks that are NaN among the newest keys: the rows before them are as if they were not there, the others get their NaN, a key's in
    the whole row and a value's in the block's channels."""
    hq, hkv, B, slots = 4, 2, 2, 300
    c = Cache(rng(nq + d), B, slots, hkv, d, 64, [300, 171], k_bits, v_bits)
    rows = [x.copy() for x in c.rows]

    def spoil(which, b, slot, g, blk):
        page, at = c.order[b, slot // 64], slot % 64
        c.q[2 * which + 1][int(page), g, at, blk] = 255
        rows[which][b, slot, g, 32 * blk:32 * blk + 32] = np.nan

    spoil(1, 0, 300 - 1, 0, 1)
    if nq > 1:
        spoil(1, 0, 300 - 2, 1, 0)
        spoil(0, 1, 171 - nq // 2, 0, 1)
        spoil(1, 1, 171 - nq // 2, 1, 1)
    c.rows = rows
    lens = [300, 171]
    O, L = check("bf16", d, B, nq, hq, hkv, slots, 64, lens, k_bits, v_bits, cache=c)
    for b in range(B):
        for q in range(nq):
            seen = lens[b] - nq + q + 1
            for h in range(hq):
                g = h // 2
                key = np.isnan(rows[0][b, :seen, g]).any()
                assert np.isnan(L[b, h, q]) == key
                want = np.isnan(rows[1][b, :seen, g]).any(0) | key
                assert (np.isnan(O[b, q, h]) == want).all(), (b, q, h)


def test_a_nan_in_a_query_stays_in_its_row():
    r = rng(11)
    Q = gpu(r.normal(size=(2, 2, 4, 64)), torch.bfloat16)
    Q[1, 0, 2, 5] = float("nan")
    c = Cache(r, 2, 600, 2, 64, 0, [600, 500], 4, 4)
    O, L = (f64(x) for x in binding.fa_qcache_fwd(Q, c.q, 0.125, True, **c.more))
    bad = np.zeros((2, 2, 4), bool)
    bad[1, 0, 2] = True
    assert (np.isnan(O).all(-1) == bad).all() and (np.isnan(O).any(-1) == bad).all() and (np.isnan(L).transpose(0, 2, 1) == bad).all()


def test_nothing_behind_the_rows_is_written_and_the_workspace_is_as_large_as_it_says():
    r = rng(12)
    for B, nq, hq, hkv, slots, d, bits in ((2, 1, 8, 2, 2000, 64, 4), (2, 5, 8, 2, 1100, 64, 8), (2, 40, 8, 2, 900, 64, 4), (2, 1, 8, 2, 64, 64, 4),
                                           (75, 1, 8, 8, 300, 128, 8), (75, 1, 8, 8, 300, 64, 4), (90, 1, 8, 8, 260, 128, 4), (3, 9, 4, 4, 3000, 128, 8)):
        c = Cache(r, B, slots, hkv, d, 0, [slots, 40] + [slots - i for i in range(B - 2)], bits, bits)
        Q = gpu(r.normal(size=(B, nq, hq, d)), torch.bfloat16)
        need = binding.fa_qcache_fwd_workspace_bytes(B, hq, hkv, nq, slots, d)
        ws = torch.full((need + 4096,), 0x5a, dtype=torch.uint8, device="cuda")
        O = torch.full((B * nq * hq * d + 512,), 3.0, dtype=torch.bfloat16, device="cuda")
        L = torch.full((B * nq * hq + 512,), 3.0, device="cuda")
        o, l = O[:-512].view(B, nq, hq, d), L[:-512].view(B, hq, nq)
        binding.fa_qcache_fwd(Q, c.q, 0.125, True, O=o, LSE=l, workspace=ws, **c.more)
        eO, eL = binding.fa_qcache_fwd(Q, c.q, 0.125, True, **c.more)
        assert torch.equal(o, eO) and torch.equal(l, eL)
        assert (O[-512:] == 3).all() and (L[-512:] == 3).all() and (ws[need:] == 0x5a).all()


def test_results_do_not_depend_on_the_run_or_on_noise_in_the_workspace():
    c = Cache(rng(13), 3, 2500, 2, 128, 64, [2500, 1, 777], 4, 4)
    Q = gpu(rng(14).normal(size=(3, 1, 8, 128)), torch.bfloat16)
    need = binding.fa_qcache_fwd_workspace_bytes(3, 8, 2, 1, 2500, 128)
    first = binding.fa_qcache_fwd(Q, c.q, 0.1, True, **c.more)
    for fill in (0, 0x7f, 0xff):
        again = binding.fa_qcache_fwd(Q, c.q, 0.1, True, workspace=torch.full((need,), fill, dtype=torch.uint8, device="cuda"), **c.more)
        assert all(torch.equal(x, y) for x, y in zip(first, again))


def test_other_streams():
    """Two calls at once, each on a stream of its own."""
    c = Cache(rng(15), 2, 3000, 2, 64, 0, [3000, 1234], 8, 4)
    Q = gpu(rng(16).normal(size=(2, 1, 8, 64)), torch.bfloat16)
    want = binding.fa_qcache_fwd(Q, c.q, 0.125, True, **c.more)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for _ in range(5):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(binding.fa_qcache_fwd(Q, c.q, 0.125, True, **c.more))
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for r in got for x, y in zip(r, want))


def test_past_two_gigabytes():
    """Pools whose rows lie past 2^31 bytes and 2^31 elements: only the last pages are used."""
    pages, hkv, page, d = 70000, 2, 256, 64
    q = binding.qcache(pages, hkv, page, d, 8, 4)
    lens = [400, 256]
    table = ints([[pages - 1, pages - 3], [pages - 2, pages - 4]])
    r = rng(17)
    K, V = (gpu(r.normal(size=(2, 256, hkv, d)), torch.bfloat16) for _ in range(2))
    binding.fa_qcache_append(K, V, q, seqlens_k=ints([256, 256]), block_table=table)
    k2, v2 = (gpu(r.normal(size=(2, 144, hkv, d)), torch.bfloat16) for _ in range(2))
    binding.fa_qcache_append(k2, v2, q, seqlens_k=ints([400, 0]), block_table=table)
    rows = []
    for a, b, bits in ((K, k2, 8), (V, v2, 4)):
        x = np.concatenate([f64(a), f64(b)], 1)
        codes, scales = orc.quantise(x, bits)
        rows.append(orc.values(codes, scales, bits))
    k, v = (torch.zeros((2, 400, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    binding.fa_qcache_read(q, k, v, seqlens_k=ints(lens), block_table=table)
    for got, x in ((k, rows[0]), (v, rows[1])):
        assert np.array_equal(f64(got)[0], x[0]) and np.array_equal(f64(got)[1, :256], x[1, :256]) and (f64(got)[1, 256:] == 0).all()
    c = Cache.__new__(Cache)
    c.q, c.rows, c.more = q, rows, dict(seqlens_k=ints(lens), block_table=table)
    check("bf16", d, 2, 1, 4, hkv, 512, page, lens, 8, 4, cache=c)


def test_a_layer_of_a_decoding_batch_in_a_graph():
    """Rotate, quantise into the cache, attend, read back: captured once and replayed with other work between the replays, a step further each
    time. Every replay is the eager run of the same state."""
    r = rng(18)
    B, hq, hkv, d, page, per = 3, 8, 2, 64, 64, 24
    table = ints(r.permutation(B * per).reshape(B, per).tolist())
    lens, pos = ints([1400, 63, 1]), ints([[1399], [62], [0]])
    f = torch.tensor([10000.0**(-i / 32) for i in range(32)], device="cuda")
    cache = binding.qcache(B * per, hkv, page, d, 8, 4)
    prompt = [gpu(r.normal(size=(B, 1400, hkv, d)), torch.bfloat16) for _ in range(2)]
    binding.fa_qcache_append(*prompt, cache, seqlens_k=lens, block_table=table)
    qkv = gpu(r.normal(size=(B, 1, hq + 2 * hkv, d)), torch.bfloat16)
    back = [torch.zeros((B, 16, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    first = ints([0, 0, 0])

    def step(cache):
        q, k = binding.fa_rope_fwd(qkv[:, :, :hq], qkv[:, :, hq:hq + hkv], pos, f)
        kr, vr = torch.empty_like(k), torch.empty_like(k)
        binding.fa_qcache_append(k, qkv[:, :, hq + hkv:], cache, seqlens_k=lens, block_table=table, Kout=kr, Vout=vr)
        O, L = binding.fa_qcache_fwd(q, cache, 0.125, True, seqlens_k=lens, block_table=table)
        binding.fa_qcache_read(cache, *back, seqlens_k=lens, block_table=table, first=first)
        return q, kr, vr, O, L

    twin = binding.QCache(*(t.clone() for t in cache))
    step(binding.QCache(*(t.clone() for t in cache)))
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        out = step(cache)
    for t, was in zip(cache, twin):  # (capturing runs nothing; the graph's cache is as it was)
        assert torch.equal(t, was)
    for i in range(4):
        qkv.copy_(gpu(r.normal(size=tuple(qkv.shape)), torch.bfloat16))
        lens += 1
        pos += 1
        first.copy_(lens - 16)
        g.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (*out, *cache, *back)]
        want = [*step(twin), *twin, *back]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i


@pytest.mark.parametrize("k_bits,v_bits", [(4, 4), (8, 8)])
def test_a_prompt_sees_what_later_steps_see(k_bits, v_bits):
    """The values that append returns are those that attention over the cache uses: a prompt through fa_fwd on them, its cache through
    fa_qcache_fwd, and its cache read back through fa_varlen_cross_fwd, agree to the rounding of O and P (e of |O| twice, e of p |v| twice)."""
    r = rng(19)
    B, n, hq, hkv, d = 2, 300, 8, 2, 64
    Q = gpu(r.normal(size=(B, n, hq, d)), torch.bfloat16)
    K, V = (gpu(r.normal(size=(B, n, hkv, d)), torch.bfloat16) for _ in range(2))
    cache = binding.qcache(B, hkv, n, d, k_bits, v_bits)
    binding.fa_qcache_append(K, V, cache, Kout=K, Vout=V)
    O, L = binding.fa_qcache_fwd(Q, cache, 0.125, True)
    O2, L2 = binding.fa_fwd(Q, K, V, 0.125, True)
    k, v = (torch.zeros((B * n, hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cu = ints([0, n, 2 * n])
    binding.fa_qcache_read(cache, k, v, cu_seqlens=cu)
    assert torch.equal(k.view(B, n, hkv, d), K) and torch.equal(v.view(B, n, hkv, d), V)
    O3, L3 = binding.fa_varlen_cross_fwd(Q.view(B * n, hq, d), k, v, cu, cu, n, n, 0.125, True)
    _, _, A, M = dec.prefix_forward(f64(Q), np.zeros((0, hkv, d)), np.zeros((0, hkv, d)), f64(K), f64(V), [n, n], 0.125, True)
    for o, l in ((O2, L2), (O3.view(B, n, hq, d), L3.view(hq, B, n).transpose(0, 1))):
        score = 2 * (M * d / 2**24 + (M + np.abs(f64(L)) + 8) / 2**21)
        assert (np.abs(f64(l) - f64(L)) <= score).all()
        assert (np.abs(f64(o) - f64(O)) <= 2 * 2.0**-8 * (A + np.abs(f64(O))) * (1 + 2.0**-7) + A * 8 * score.transpose(0, 2, 1)[..., None]).all()


@pytest.mark.parametrize("d", [64, 128])
def test_pages_behind_a_sequence_are_not_looked_up(d):
    """Entries of the table behind the last page that has a key are no pages at all."""
    r, lens = rng(d), [70, 0, 640, 64, 1, 129]
    cache = Cache(r, 6, 640, 2, d, 64, lens, 4, 8)
    short = cache.table.clone()
    for b, n in enumerate(lens):
        short[b, -(-n // 64):] = -2**30
    for nq in (1, 5, 40):
        Q = gpu(r.normal(size=(6, nq, 4, d)), torch.bfloat16)
        for causal in (False, True):
            want = binding.fa_qcache_fwd(Q, cache.q, 0.1, causal, **cache.more)
            got = binding.fa_qcache_fwd(Q, cache.q, 0.1, causal, **{**cache.more, "block_table": short})
            assert all(torch.equal(a, b) for a, b in zip(got, want))
    outs = []
    for table in (cache.table, short):
        K, V = (torch.zeros(6, 700, 2, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        binding.fa_qcache_read(cache.q, K, V, cache.more["seqlens_k"], table)
        k, v = (torch.zeros(sum(lens), 2, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        binding.fa_qcache_read(cache.q, k, v, cache.more["seqlens_k"], table, cu_seqlens=ints([0] + np.cumsum(lens).tolist()))
        q = binding.QCache(*(t.clone() for t in cache.q))
        x = gpu(np.random.default_rng(7).normal(size=(6, 3, 2, d)), torch.bfloat16)
        binding.fa_qcache_append(x, x, q, cache.more["seqlens_k"], table)
        outs.append([K, V, k, v, *q])
    assert all(torch.equal(a, b) for a, b in zip(*outs))


# ---- values past the type's range among keys that only some rows see

def check_beside(dtype, c, Q, lens, causal, infinite, skip=None):
    """O of fa_qcache_fwd where c.rows has the keys and values with what is `infinite` (values as the type has them: infinities, NaN; else 0)
    left out: as if that were zeros in the rows that do not see it, and not finite in those that do (NaN where the key's weight is below the type's
    least number). skip: rows [B, Nq, Hq] left out of the comparison."""
    B, nq, hq, d = Q.shape
    hkv = c.rows[0].shape[2]
    O, L = (f64(x) for x in binding.fa_qcache_fwd(Q, c.q, d**-0.5, causal, **c.more))
    none = np.zeros((0, hkv, d))
    rows = [[x[b][:lens[b]] for b in range(B)] for x in c.rows]
    eO, eL, A, M = dec.prefix_forward(f64(Q), none, none, *rows, lens, d**-0.5, causal)
    e = torch.finfo(TYPES[dtype]).eps / 2
    score = M * d / 2**24 + (M + np.abs(eL) + 8) / 2**21
    tol = e * (A + np.abs(eO)) * (1 + 2 * e) + A * 4 * score.transpose(0, 2, 1)[..., None]
    wrong = []
    for b in range(B):
        for q in range(nq):
            seen = max(0, min(lens[b], lens[b] - nq + q + 1)) if causal else lens[b]
            for h in range(hq):
                if skip is not None and skip[b, q, h]:
                    continue
                g = h * hkv // hq
                x = infinite[b, :seen, g]
                with np.errstate(invalid="ignore"):
                    want = eO[b, q, h] + x.sum(0)
                # (half precision's P, where it is subnormal, as everywhere above: of the largest value in the channel)
                small = c.slots * 4.0 / 2**25 * np.abs(c.rows[1][b, :lens[b], g]).max(0) if dtype == "f16" else 0.0
                finite = np.isfinite(want)
                ok = np.where(finite, np.abs(O[b, q, h] - np.where(finite, want, 0)) <= tol[b, q, h] + small, ~np.isfinite(O[b, q, h]))
                # Sums are float32, over weights against a reference that bfloat16's largest score may outgrow by up to 2^20 before it is
                # advanced: where the values seen sum to 2^128 / 2^20 the sum may pass 2^128 and be infinite (half precision's cannot:
                # 2^8 times the few hundred values below 2^16 stays below 2^33).
                if dtype == "bf16":
                    ok |= ~np.isfinite(O[b, q, h]) & (np.abs(c.rows[1][b, :seen, g]).sum(0) >= 2.0**108)
                if not ok.all() or not abs(L[b, h, q] - eL[b, h, q]) <= score[b, h, q]:
                    wrong.append((b, q, h, np.flatnonzero(~ok).tolist()))
    assert not wrong, wrong[:5]


def put_block(c, which, b, slot, g, blk, values):
    """A block of 32 values into the cache; returns what it stands for."""
    bits = c.bits[which]
    codes, scales = orc.quantise(values, bits)
    row, at = (int(c.order[b, slot // c.page]), slot % c.page) if c.page else (b, slot)
    packed = orc.packed(codes, bits)
    n = len(packed)
    c.q[2 * which][row, g, at, n * blk:n * blk + n] = gpu(packed)
    c.q[2 * which + 1][row, g, at, blk] = int(scales[0])
    return orc.values(codes, scales, bits)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("k_bits,v_bits", BITS)
@pytest.mark.parametrize("nq,page", [(1, 64), (5, 0), (10, 64), (40, 64)])
def test_what_a_row_does_not_see_may_be_past_the_type(dtype, d, k_bits, v_bits, nq, page):
    """The type's largest numbers, which quantised come back as infinities, among the newest values: the rows before them are as if they were not
    there, the others are not finite in that channel and in no other; of an old value every row is. Likewise keys, of which the rows that
    do see them are left out; and E4M3's own NaN codes, which no block of append's has."""
    hq, hkv, B, slots, lens = 4, 2, 2, 300, [300, 171]
    r = rng(nq + d)
    c = Cache(r, B, slots, hkv, d, page, lens, k_bits, v_bits)
    for x in c.rows:
        for b in range(B):
            x[b, lens[b]:] = 0.0  # (no key's)
    Q = gpu(r.normal(size=(B, nq, hq, d)), TYPES[dtype])
    top = torch.finfo(TYPES[dtype]).max
    infinite, skip = np.zeros((B, slots, hkv, d)), np.zeros((B, nq, hq), bool)

    def spoil(b, slot, g, blk, at, other):
        x = np.zeros(32)
        x[at], x[other], x[(at + 2) % 32] = top, -top, top / 4
        x = put_block(c, 1, b, slot, g, blk, x)
        held = f64(torch.from_numpy(x).to(TYPES[dtype]))
        assert np.isinf(held[at]) and np.isinf(held[other]) and np.isfinite(held).sum() == 30
        here = slice(32 * blk, 32 * blk + 32)
        infinite[b, slot, g, here] = np.where(np.isfinite(held), 0, held)
        c.rows[1][b, slot, g, here] = np.where(np.isfinite(held), x, 0)

    spoil(0, 299, 0, 1, 3, 20)
    spoil(1, 5, 0, 0, 31, 0)
    if nq > 1:
        spoil(0, 298, 1, 0, 16, 15)
        spoil(1, 171 - nq // 2, 1, d // 32 - 1, 8, 7)
        x = np.zeros(32)
        x[4] = top
        put_block(c, 0, 1, 171 - nq // 2, 0, 1, x)
        skip[1, nq - nq // 2:, :2] = True  # (query q sees keys up to 171 - nq + q)
    if v_bits == 8:
        slot, g = 300 - max(1, nq // 3), 1
        row, at = (int(c.order[0, slot // page]), slot % page) if page else (0, slot)
        c.q.Vcodes[row, g, at, 35], c.q.Vcodes[row, g, at, 47] = 0x7f, 0xff
        infinite[0, slot, g, [35, 47]] = np.nan
        c.rows[1][0, slot, g, [35, 47]] = 0.0
    check_beside(dtype, c, Q, lens, True, infinite, skip)
    if nq > 1:  # (without the causal rule every row sees every key: the spoilt key is taken back)
        c.rows[0][1, 171 - nq // 2, 0, 32:64] = put_block(c, 0, 1, 171 - nq // 2, 0, 1, r.normal(size=32))
        check_beside(dtype, c, Q, lens, False, infinite)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("d,k_bits,v_bits,nq,hq,B,page,slots", LONG)
def test_attend_where_a_workgroup_has_many_tiles_of_a_sequence(dtype, d, k_bits, v_bits, nq, hq, B, page, slots):
    """More than 64 tiles in a row, for which page numbers are looked up together: they are looked up again. (The sequences' pages, in orders of their own,
    are from one small pool.)"""
    r, hkv, pool = rng(slots + d + nq), 8, 48
    data = [r.normal(size=(pool, page, hkv, d)) for _ in range(2)]
    tensors, held = [], []
    for x, bits in zip(data, (k_bits, v_bits)):
        codes, scales = orc.quantise(x, bits)
        held.append(orc.values(codes, scales, bits))
        tensors += [gpu(t.transpose(0, 2, 1, 3)) for t in (orc.packed(codes, bits), scales)]
    q, lens, order = binding.QCache(*tensors), long_lengths(B, slots), r.integers(0, pool, size=(B, -(-slots // page)))
    Q = gpu(r.normal(size=(B, nq, hq, d)), TYPES[dtype])
    O, L = binding.fa_qcache_fwd(Q, q, d**-0.5, True, seqlens_k=ints(lens), block_table=ints(order.tolist()), max_seqlen_k=slots)
    some = [0, B // 2 + 1, B - 1]
    c = Cache.__new__(Cache)
    c.q, c.more, c.rows = q, {}, [np.stack([x[order[b]].reshape(-1, hkv, d) for b in some]) for x in held]
    check(dtype, d, 3, nq, hq, hkv, slots, page, [lens[b] for b in some], k_bits, v_bits, cache=c, Q=Q[some], call=lambda *a: (O[some], L[some]))
