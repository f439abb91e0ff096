"""Refusals of the operators on caches in 4 or 8 bits and of the rotary positions, at the C ABI and at the tensor level: nothing is
launched, no GPU is touched."""
import pytest

from launches import launches
from paper_2307_08691_amd import binding as fa

torch = pytest.importorskip("torch")

from qcaches import LONG, grids, long_lengths, longest_segment  # noqa: E402

P = 0x10000  # a non-null, 16-byte aligned fake device address; never dereferenced on these paths
BIG = 1 << 40
INF, NAN = float("inf"), float("nan")


def append(Kn=P, Vn=P, Kc=P, Ks=P, Vc=P, Vs=P, Ko=P, Vo=P, lens=P, tab=0, B=2, Hkv=2, Nq=1, Nk=200, d=64, kb=4, vb=8, page=0, pages=0,
           ks=(128, 128, 64), vs=(128, 128, 64), type=fa.FA_TYPE_BF16):
    return fa.fa_qcache_append_raw(Kn, Vn, Kc, Ks, Vc, Vs, Ko, Vo, lens, tab, B, Hkv, Nq, Nk, d, kb, vb, page, pages, ks, vs, type)


def read(Kc=P, Ks=P, Vc=P, Vs=P, K=P, V=P, lens=P, tab=0, first=0, cu=0, B=2, Hkv=2, N=10, Nk=200, d=64, kb=4, vb=8, page=0, pages=0,
         type=fa.FA_TYPE_F16):
    return fa.fa_qcache_read_raw(Kc, Ks, Vc, Vs, K, V, lens, tab, first, cu, B, Hkv, N, Nk, d, kb, vb, page, pages, type)


def attend(Q=P, Kc=P, Ks=P, Vc=P, Vs=P, lens=P, tab=0, O=P, L=P, ws=P, nb=BIG, B=2, Hq=8, Hkv=2, Nq=1, Nk=4000, d=64, kb=4, vb=8, page=0,
           pages=0, scale=0.1, type=fa.FA_TYPE_BF16):
    return fa.fa_qcache_fwd_raw(Q, Kc, Ks, Vc, Vs, lens, tab, O, L, ws, nb, B, Hq, Hkv, Nq, Nk, d, kb, vb, page, pages, scale, True, type)


STRIDES = (512, 512, 64) * 4


def rope(inverse, Q=P, K=P, Qo=P, Ko=P, pos=P, f=P, axis=P, B=2, N=3, Hq=8, Hkv=2, d=64, pairs=32, axes=2, strides=STRIDES, ps=6, pb=3,
         type=fa.FA_TYPE_BF16):
    return fa.fa_rope_raw(inverse, Q, K, Qo, Ko, pos, f, axis, B, N, Hq, Hkv, d, pairs, axes, False, strides, ps, pb, type)


SLOTS = [dict(B=0), dict(Nk=0), dict(Hkv=0), dict(B=1 << 21), dict(Nk=(1 << 30) + 1), dict(tab=P, page=64, pages=3, Nk=200), dict(tab=P, page=64, pages=0)]
PAGES = [dict(tab=P, page=32, pages=100), dict(tab=P, page=96, pages=100), dict(kb=6), dict(vb=16), dict(kb=0)]


def test_append_refusals():
    for name in ("Kn", "Vn", "Kc", "Ks", "Vc", "Vs"):
        assert append(**{name: 0}) == fa.FA_ERR_NULL, name
    for name in ("Kn", "Vn", "Kc", "Vc", "Ko", "Vo"):
        assert append(**{name: P + 8}) == fa.FA_ERR_ALIGN, name
    for name in ("Ks", "Vs", "lens", "tab"):
        assert append(**{name: P + 2}, page=64, pages=100) == fa.FA_ERR_ALIGN, name
    for bad in SLOTS + [dict(Nq=0), dict(d=0), dict(d=-32), dict(ks=(128, 128, 60)), dict(vs=(-128, 128, 64)), dict(ks=(4, 128, 64)),
                        dict(B=1 << 18, Nq=1 << 12)]:
        assert append(**bad) == fa.FA_ERR_SHAPE, bad
    for bad in PAGES + [dict(d=48), dict(d=288), dict(type=fa.FA_TYPE_F32), dict(type=7)]:
        assert append(**bad) == fa.FA_ERR_UNSUPPORTED, bad


def test_read_refusals():
    for name in ("Kc", "Ks", "Vc", "Vs", "K", "V"):
        assert read(**{name: 0}) == fa.FA_ERR_NULL, name
    for name in ("Kc", "Vc", "K", "V"):
        assert read(**{name: P + 8}) == fa.FA_ERR_ALIGN, name
    for name in ("Ks", "Vs", "lens", "first", "cu"):
        assert read(**{name: P + 2}) == fa.FA_ERR_ALIGN, name
    for bad in SLOTS + [dict(N=0), dict(first=P, cu=P), dict(B=1 << 19, N=1 << 12)]:
        assert read(**bad) == fa.FA_ERR_SHAPE, bad
    for bad in PAGES + [dict(d=16), dict(d=260), dict(type=fa.FA_TYPE_F32)]:
        assert read(**bad) == fa.FA_ERR_UNSUPPORTED, bad


def test_how_many_rows_read_takes():
    """Both sides of the limit: below 2^30 rows of all heads in whole workgroups of 64, where packed rows count as many a sequence as its cache has
    slots at most, and windows (which may begin before slot 0) all of theirs."""
    def call(cu, B, Hkv, N, Nk):
        return "fa_qcache_read", [P] * 7 + [0, 0, P if cu else 0, B, Hkv, N, Nk, 64, 4, 8, 0, 0, fa.FA_TYPE_BF16]

    sizes = [(0, 64, 8, 1 << 20, 64, 1 << 23), (1, 64, 8, 1 << 21, 64, 512), (0, 1 << 10, 1 << 8, 65, 1 << 30, 1 << 19),
             (1, 1 << 10, 1 << 8, 1 << 12, 63 * 64, 63 << 18), (0, 1, 1, (1 << 30) - 64, 1 << 30, (1 << 24) - 1),
             (1, 1, 1, (1 << 30) - 64, 1 << 30, (1 << 24) - 1)]
    for (*_, grid), kernels in zip(sizes, launches([call(*x[:-1]) for x in sizes])):
        assert [(k[0].split("<")[0], *k[1:]) for k in kernels] == [("qread_kernel", grid, 1, 256)]
    for cu, B, Hkv, N, Nk in ((0, 1, 1, 1 << 30, 1 << 30), (1, 1, 1, 1 << 30, 1 << 30), (0, 1, 1, (1 << 30) - 63, 1 << 30), (0, 64, 8, 1 << 21, 64),
                              (0, 1 << 10, 1 << 8, 1 << 12, 1 << 12), (1, 1 << 10, 1 << 8, 1 << 13, 1 << 12)):
        assert read(cu=P if cu else 0, B=B, Hkv=Hkv, N=N, Nk=Nk) == fa.FA_ERR_SHAPE


def test_attend_refusals():
    for name in ("Q", "Kc", "Ks", "Vc", "Vs", "O", "L"):
        assert attend(**{name: 0}) == fa.FA_ERR_NULL, name
    for name in ("Q", "Kc", "Vc", "O", "ws"):
        assert attend(**{name: P + 8}) == fa.FA_ERR_ALIGN, name
    for name in ("Ks", "Vs", "L", "lens", "tab"):
        assert attend(**{name: P + 2}, page=64, pages=100) == fa.FA_ERR_ALIGN, name
    for bad in SLOTS[:5] + [dict(tab=P, page=64, pages=3), dict(Nq=0), dict(Hq=7), dict(Hq=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=INF),
                            dict(scale=NAN), dict(B=1 << 20, Nq=64), dict(Hq=1 << 17, Hkv=1 << 17)]:
        assert attend(**bad) == fa.FA_ERR_SHAPE, bad
    for bad in PAGES + [dict(d=96), dict(d=256), dict(d=32), dict(type=fa.FA_TYPE_F32), dict(type=-1)]:
        assert attend(**bad) == fa.FA_ERR_UNSUPPORTED, bad
    need = fa.fa_qcache_fwd_workspace_bytes(2, 8, 2, 1, 4000, 64)
    assert need > 0 and attend(nb=need - 1) == fa.FA_ERR_WORKSPACE and attend(ws=0) == fa.FA_ERR_NULL
    for bad in (dict(B=0), dict(Hq=7), dict(Nq=0), dict(Nk=0), dict(d=96), dict(Nk=(1 << 30) + 1), dict(B=1 << 20, Nq=64)):
        x = dict(B=2, Hq=8, Hkv=2, Nq=1, Nk=4000, d=64, **{k: v for k, v in bad.items() if k not in ("B", "Hq", "Nq", "Nk", "d")})
        x.update(bad)
        assert fa.fa_qcache_fwd_workspace_bytes(*x.values()) == 0, bad
    # more chunks of keys than are counted in 31 bits
    assert attend(B=64, Hq=1 << 10, Hkv=1 << 4, Nq=1 << 10, Nk=1 << 30) == fa.FA_ERR_SHAPE
    # 2^24 rows, but 2^28 with those of the blocks of 16: a merge of more threads than a grid counts
    assert attend(B=1 << 20, Hq=16, Hkv=16, Nq=1, Nk=256) == fa.FA_ERR_SHAPE
    assert fa.fa_qcache_fwd_workspace_bytes(1 << 20, 16, 16, 1, 256, 64) == 0


@pytest.mark.parametrize("d", [64, 128])
def test_workspace_needs(d):
    """None where nothing can be cut: caches of a chunk, and of up to 1024 keys while every head of every sequence has a workgroup of its own;
    else places for two parts of each workgroup, however long the caches are."""
    need = lambda B, Hkv, Nq, Nk: fa.fa_qcache_fwd_workspace_bytes(B, Hkv, Hkv, Nq, Nk, d)  # noqa: E731
    assert need(4, 8, 1, 1024) == need(64, 8, 1, 1024) == need(1000, 8, 1, 128) == need(1, 1, 200, 128) == 0
    assert need(4, 8, 1, 1025) > 0 and need(65, 8, 1, 1024) > 0 and need(1, 1, 200, 129) > 0
    assert need(64, 8, 1, 1 << 20) - need(64, 8, 1, 8192) == 0
    assert need(64, 8, 1, 1 << 20) <= 2 * 768 * 16 * (d + 1) * 4 + 64 * 8 * 8 + 256
    assert need(64, 8, 200, 1 << 20) <= 2 * 512 * 128 * (d + 1) * 4 + 2 * 64 * 8 * 8 + 256


def test_workspace_of_the_largest_batches():
    """Partial results of all workgroups, and eight bytes for every block of rows of every head: the most that the header says."""
    for rows, G, groups, blocks, most in ((16, 16, 768, 1, 22), (32, 64, 512, 2, 34), (128, 128, 512, 1, 72)):
        B = min(1 << 20, (1 << 26) // (rows * blocks))
        need = fa.fa_qcache_fwd_workspace_bytes(B, G, 1, 1, 256, 128)
        assert need == 2 * groups * rows * 129 * 4 + 8 * B * blocks <= most * 10**6
        assert attend(B=B, Hq=G, Hkv=1, Nk=256, d=128, nb=need - 1) == fa.FA_ERR_WORKSPACE
        assert fa.fa_qcache_fwd_workspace_bytes(B, G, 1, 1, 1 << 20 if B < 1 << 18 else 256, 128) == need


def test_the_long_batches_of_the_gpu_tests_are_long():
    """Page numbers are looked up for 64 tiles at a time: a wavefront has more than that (128 rows: the workgroup)."""
    calls = [[P] * 10 + [BIG, B, hq, 8, nq, slots, d, kb, vb, page, slots // page, 0.1, True, fa.FA_TYPE_BF16]
             for d, kb, vb, nq, hq, B, page, slots in LONG]
    for (d, kb, vb, nq, hq, B, page, slots), launched in zip(LONG, grids(calls)):
        rows = 16 if nq * hq // 8 <= 16 else (32 if nq * hq // 8 <= 64 else 128)
        tile = 64 if rows == 128 or (d == 64 and kb + vb == 8) else 32
        chunk = 256 if rows < 128 and tile == 64 else 128
        n = longest_segment(long_lengths(B, slots), nq, hq // 8, 8, rows, chunk, launched[0])
        assert n > 64 * tile * (1 if rows == 128 else 4), (d, kb, vb, nq, n)


@pytest.mark.parametrize("inverse", [False, True])
def test_rope_refusals(inverse):
    for name in ("Q", "Qo", "Ko", "pos", "f"):
        assert rope(inverse, **{name: 0}) == fa.FA_ERR_NULL, name
    assert rope(inverse, strides=None) == fa.FA_ERR_NULL
    for name in ("Q", "K", "Qo", "Ko"):
        assert rope(inverse, **{name: P + 1}) == fa.FA_ERR_ALIGN, name
        assert rope(inverse, **{name: P + 2}, type=fa.FA_TYPE_F32) == fa.FA_ERR_ALIGN, name
    for name in ("pos", "f", "axis"):
        assert rope(inverse, **{name: P + 2}) == fa.FA_ERR_ALIGN, name
    for bad in (dict(B=0), dict(N=0), dict(B=1 << 16, N=1 << 16), dict(Hq=0), dict(Hkv=0), dict(Hq=1 << 20), dict(d=0), dict(pairs=0), dict(pairs=33),
                dict(axes=0), dict(ps=-1), dict(pb=-1), dict(strides=(512, 512, 64) * 3 + (512, -512, 64))):
        assert rope(inverse, **bad) == fa.FA_ERR_SHAPE, bad
    for bad in (dict(d=66), dict(d=264), dict(type=3), dict(type=-1)):
        assert rope(inverse, **bad) == fa.FA_ERR_UNSUPPORTED, bad


# ---- the tensor level (host tensors: the last check of all refuses them, so that everything before it can be seen here)

def cpu_cache(n=2, Hkv=2, slots=128, d=64, **kw):
    return fa.qcache(n, Hkv, slots, d, device="cpu", **kw)


def ints(*x):
    return torch.tensor(x, dtype=torch.int32)


def refused(match, f, *args, **kw):
    with pytest.raises(ValueError, match=match):
        f(*args, **kw)


def test_tensors_of_a_cache():
    c = cpu_cache(k_bits=8)
    assert [tuple(t.shape) for t in c] == [(2, 2, 128, 64), (2, 2, 128, 2), (2, 2, 128, 32), (2, 2, 128, 2)]
    refused("4 or 8 bits", fa.qcache, 1, 1, 64, 64, 2, 4, "cpu")
    refused("4 or 8 bits", fa.qcache, 1, 1, 64, 80, 4, 4, "cpu")
    Q = torch.zeros(2, 1, 8, 64, dtype=torch.bfloat16)
    fwd = lambda cache, **kw: fa.fa_qcache_fwd(Q, cache, 0.1, True, **kw)  # noqa: E731
    refused("must live on the GPU", fwd, c)
    refused("a cache is", fwd, c[:3])
    refused("Kcodes must hold", fwd, (c[0][..., :48], *c[1:]))
    refused("uint8", fwd, (c[0].to(torch.int8), *c[1:]))
    refused("Vscales must have shape", fwd, (*c[:3], c[3][:, :, :64]))
    refused("contiguous", fwd, (c[0].transpose(0, 1), *c[1:]))
    refused("without a block_table", fwd, cpu_cache(n=3))
    refused("slots of a contiguous", fwd, c, max_seqlen_k=100)
    refused("head dimension", fwd, cpu_cache(d=128))
    refused("seqlens_k", fwd, c, seqlens_k=ints(1, 2, 3))
    refused("int32", fwd, c, seqlens_k=torch.tensor([1, 2]))
    refused("block_table must be", fwd, c, block_table=ints(0, 1))
    refused("hold 256 slots", fwd, c, block_table=ints(0, 1).repeat(2, 1), max_seqlen_k=257)
    refused("workspace holds", fwd, cpu_cache(slots=4096), workspace=torch.zeros(16, dtype=torch.uint8))
    refused("bfloat16 or float16", fa.fa_qcache_fwd, Q.float(), c, 0.1, True)


def test_tensors_of_append_and_read():
    c = cpu_cache()
    K = torch.zeros(2, 3, 2, 64, dtype=torch.bfloat16)
    refused("must live on the GPU", fa.fa_qcache_append, K, K, c)
    refused("Vnew must be", fa.fa_qcache_append, K, K.half(), c)
    refused("heads of", fa.fa_qcache_append, K[:, :, :1], K[:, :, :1], c)
    refused("rows of Knew", fa.fa_qcache_append, K.transpose(2, 3).contiguous().transpose(2, 3), K, c)
    refused("multiple of 8", fa.fa_qcache_append, torch.zeros(2, 3, 2, 68, dtype=torch.bfloat16)[..., :64], K, c)
    refused("Kout must have shape", fa.fa_qcache_append, K, K, c, Kout=K[:, :1])
    refused("must live on the GPU", fa.fa_qcache_read, c, K, K)
    refused("V must have shape", fa.fa_qcache_read, c, K, K[:, :1].contiguous())
    refused("exclude each other", fa.fa_qcache_read, c, K[0], K[0], first=ints(0, 0), cu_seqlens=ints(0, 1, 2))
    refused("with cu_seqlens", fa.fa_qcache_read, c, K, K, cu_seqlens=ints(0, 1, 2))
    refused("or .T, Hkv, d. with", fa.fa_qcache_read, c, K[0], K[0])
    refused("first must have shape", fa.fa_qcache_read, c, K, K, first=ints(0))
    refused("heads of", fa.fa_qcache_read, c, K[..., :32], K[..., :32])


@pytest.mark.parametrize("f", [fa.fa_rope_fwd, fa.fa_rope_bwd])
def test_tensors_of_rope(f):
    Q, K = torch.zeros(2, 3, 4, 64), torch.zeros(2, 3, 2, 64)
    pos, inv = torch.zeros(2, 3, dtype=torch.int32), torch.zeros(32)
    refused("must live on the GPU", f, Q, K, pos, inv)
    refused("must live on the GPU", f, Q[0], None, pos[0], inv)
    refused("float32, bfloat16 or float16", f, Q.double(), K, pos, inv)
    refused("K must be", f, Q, K[:1], pos, inv)
    refused("K must be", f, Q, K[0], pos, inv)
    refused("positions must be int32", f, Q, K, pos.long(), inv)
    refused("positions must be int32", f, Q, K, pos[:, :2], inv)
    refused("must be dense", f, Q, K, torch.zeros(2, 6, dtype=torch.int32)[:, ::2], inv)
    refused("half of d at most", f, Q, K, pos, torch.zeros(33))
    refused("axis must have shape", f, Q, K, pos, inv, ints(0, 0))
    refused("must be dense", f, torch.zeros(2, 3, 4, 128)[..., ::2], K, pos, inv)
    refused("Qout must be", f, Q, K, pos, inv, None, False, Q[:, :2])
    refused("places of their own", f, Q, K, pos, inv, None, False, torch.zeros(2, 1, 4, 64).expand(2, 3, 4, 64))
    refused("Kout without K", f, Q, None, pos, inv, None, False, None, K)


def test_dimensions_past_31_bits():
    """Seen before anything is called: tensors that only have a shape."""
    def cache(n, hkv, rows):
        return fa.qcache(n, hkv, rows, 64, device="meta")

    def x(*shape):
        return torch.empty(shape, dtype=torch.bfloat16, device="meta")

    far, f = 2**31 + 1, torch.empty(8, device="meta")
    for call in (lambda: fa.fa_qcache_fwd(x(1, 1, 1, 64), cache(1, 1, far), 1.0, True),
                 lambda: fa.fa_qcache_fwd(x(1, far, 1, 64), cache(1, 1, 64), 1.0, True),
                 lambda: fa.fa_qcache_append(x(1, far, 1, 64), x(1, far, 1, 64), cache(1, 1, 64)),
                 lambda: fa.fa_qcache_read(cache(1, 1, 64), x(1, far, 1, 64), x(1, far, 1, 64)),
                 lambda: fa.fa_rope_fwd(x(1, far, 1, 64), None, torch.empty((1, far), dtype=torch.int32, device="meta"), f)):
        with pytest.raises(ValueError, match=r"2\*\*31"):
            call()
