"""Refusals of the operators of a decoding batch, at the C ABI and at the tensor level: nothing is launched, no GPU is touched."""
import pytest

from paper_2307_08691_amd import binding as fa

P = 0x10000  # a non-null, 16-byte aligned fake device address; never dereferenced on these paths
BIG = 1 << 40
INF, NAN = float("inf"), float("nan")


def prefix(Q=P, Kp=P, Vp=P, ptab=0, K=P, V=P, lens=P, tab=0, O=P, L=P, ws=P, nb=BIG, B=2, Hq=8, Hkv=2, Nq=1, Np=100, Nk=200, d=64, page=0,
           ppages=0, pages=0, scale=0.1, f16=False):
    return fa.fa_prefix_fwd_raw(Q, Kp, Vp, ptab, K, V, lens, tab, O, L, ws, nb, B, Hq, Hkv, Nq, Np, Nk, d, page, ppages, pages, scale, True, 0, f16)


def append(Kn=P, Vn=P, K=P, V=P, lens=P, tab=0, W=P, pos=P, first=P, B=2, Hkv=2, Nq=1, Nk=200, d=64, page=0, pages=0):
    return fa.fa_cache_append_raw(Kn, Vn, K, V, lens, tab, W, pos, first, B, Hkv, Nq, Nk, d, page, pages)


def weights(Q=P, K=P, L=P, lens=P, tab=0, queries=0, W=P, B=2, Hq=8, Hkv=2, Nq=1, Nk=200, d=64, page=0, pages=0, scale=0.1, f16=False):
    return fa.fa_cache_weights_raw(Q, K, L, lens, tab, queries, W, B, Hq, Hkv, Nq, Nk, d, page, pages, Hq * Nq, Nq, 1, scale, True, 0, f16)


def evict(K=P, V=P, W=P, pos=P, lens=P, tab=0, Wo=P, po=P, no=P, ws=P, nb=BIG, B=2, Hkv=2, Nk=200, d=64, budget=100, sinks=4, recent=20,
          page=0, pages=0):
    return fa.fa_cache_evict_raw(K, V, W, pos, lens, tab, Wo, po, no, ws, nb, B, Hkv, Nk, d, budget, sinks, recent, page, pages)


def verify(x=P, q=P, t=P, u=P, tok=P, acc=P, ws=P, nb=BIG, B=2, k=3, V=1000, qs=1000, ts=1000, qt=0, tt=1, logits=True, inv=1.0):
    return fa.fa_verify_drafts_raw(x, q, t, u, tok, acc, ws, nb, B, k, V, qs, ts, qt, tt, logits, inv)


@pytest.mark.parametrize("f16", [False, True])
def test_prefix_refusals(f16):
    def p(**kw):
        return prefix(f16=f16, **kw)
    for name in ("Q", "Kp", "Vp", "K", "V", "O", "L", "ws"):
        assert p(**{name: 0}) == fa.FA_ERR_NULL
    for bad in (dict(B=0), dict(Nq=0), dict(Np=-1), dict(Nk=0), dict(Hq=7), dict(Hkv=0), dict(scale=0.0), dict(scale=NAN), dict(scale=INF),
                dict(tab=P, page=64, pages=3), dict(tab=P, page=64, pages=0), dict(ptab=P, page=64, ppages=1), dict(ptab=P, page=64, ppages=0),
                dict(B=1 << 20, Nq=64), dict(B=1 << 30), dict(Hq=1 << 17, Hkv=1 << 17)):
        assert p(**bad) == fa.FA_ERR_SHAPE, bad
    for bad in (dict(d=96), dict(d=256), dict(d=60), dict(tab=P, page=32, pages=100), dict(tab=P, page=96, pages=100),
                dict(ptab=P, page=48, ppages=100)):
        assert p(**bad) == fa.FA_ERR_UNSUPPORTED, bad
    for name in ("Q", "Kp", "Vp", "K", "V", "O", "L", "ws"):
        assert p(**{name: P + 8}) == fa.FA_ERR_ALIGN
    for name in ("lens", "tab", "ptab"):
        assert p(**{name: P + 2}, page=64, pages=100, ppages=100) == fa.FA_ERR_ALIGN
    need = fa.fa_prefix_fwd_workspace_bytes(2, 8, 2, 1, 100, 200, 64)
    assert need > 0 and p(nb=need - 1) == fa.FA_ERR_WORKSPACE


def test_append_refusals():
    for name in ("Kn", "Vn", "K", "V"):
        assert append(**{name: 0}) == fa.FA_ERR_NULL
        assert append(**{name: P + 8}) == fa.FA_ERR_ALIGN
    for name in ("lens", "W", "pos", "first"):
        assert append(**{name: P + 2}) == fa.FA_ERR_ALIGN
    for bad in (dict(B=0), dict(Nq=0), dict(Nk=0), dict(Hkv=0), dict(d=0), dict(tab=P, page=64, pages=3), dict(B=1 << 20, Nq=1 << 12)):
        assert append(**bad) == fa.FA_ERR_SHAPE, bad
    for bad in (dict(d=12), dict(d=264), dict(tab=P, page=63, pages=100)):
        assert append(**bad) == fa.FA_ERR_UNSUPPORTED, bad


@pytest.mark.parametrize("f16", [False, True])
def test_weights_refusals(f16):
    for name in ("Q", "K", "L", "W"):
        assert weights(**{name: 0}, f16=f16) == fa.FA_ERR_NULL
    for name in ("Q", "K"):
        assert weights(**{name: P + 8}, f16=f16) == fa.FA_ERR_ALIGN
    for name in ("L", "W", "lens", "queries"):
        assert weights(**{name: P + 2}, f16=f16) == fa.FA_ERR_ALIGN
    for bad in (dict(B=0), dict(Nq=0), dict(Nk=0), dict(Hq=7), dict(scale=-1.0), dict(tab=P, page=64, pages=3), dict(Nq=1 << 30)):
        assert weights(**bad, f16=f16) == fa.FA_ERR_SHAPE, bad
    for bad in (dict(d=96), dict(d=256), dict(tab=P, page=16, pages=100)):
        assert weights(**bad, f16=f16) == fa.FA_ERR_UNSUPPORTED, bad


def test_evict_refusals():
    for name in ("K", "V", "W", "pos", "Wo", "po", "no", "ws"):
        assert evict(**{name: 0}) == fa.FA_ERR_NULL
    for name in ("K", "V"):
        assert evict(**{name: P + 8}) == fa.FA_ERR_ALIGN
    for name in ("W", "pos", "Wo", "po", "no", "ws", "lens"):
        assert evict(**{name: P + 2}) == fa.FA_ERR_ALIGN
    for bad in (dict(B=0), dict(Nk=0), dict(budget=0), dict(sinks=-1), dict(recent=-1), dict(sinks=50, recent=51), dict(sinks=2**31 - 1, recent=2**31 - 1),
                dict(tab=P, page=64, pages=3), dict(d=-8)):
        assert evict(**bad) == fa.FA_ERR_SHAPE, bad
    for bad in (dict(d=12), dict(d=512), dict(tab=P, page=100, pages=3)):
        assert evict(**bad) == fa.FA_ERR_UNSUPPORTED, bad
    need = fa.fa_cache_evict_workspace_bytes(2, 2, 200, 100)
    assert need >= 4 * (1 + 2 * 100) * 4 and evict(nb=need - 1) == fa.FA_ERR_WORKSPACE


def test_verify_refusals():
    for name in ("x", "t", "u", "tok", "acc", "ws"):
        assert verify(**{name: 0}) == fa.FA_ERR_NULL
    for name in ("x", "u", "tok", "acc", "q"):
        assert verify(**{name: P + 2}) == fa.FA_ERR_ALIGN
    assert verify(ws=P + 4) == fa.FA_ERR_ALIGN and verify(t=P + 1) == fa.FA_ERR_ALIGN
    for bad in (dict(B=0), dict(k=-1), dict(V=0), dict(V=(1 << 24) + 1, qs=1 << 25, ts=1 << 25), dict(qs=999), dict(ts=999), dict(ts=-1000), dict(inv=0.0),
                dict(inv=NAN), dict(inv=INF), dict(B=1 << 20, k=1)):
        assert verify(**bad) == fa.FA_ERR_SHAPE, bad
    for bad in (dict(tt=3), dict(tt=-1), dict(qt=7)):
        assert verify(**bad) == fa.FA_ERR_UNSUPPORTED, bad
    need = fa.fa_verify_drafts_workspace_bytes(2, 3, 1000)
    assert need > 0 and verify(nb=need - 1) == fa.FA_ERR_WORKSPACE


def test_workspaces_of_senseless_sizes_are_zero():
    assert fa.fa_prefix_fwd_workspace_bytes(0, 8, 2, 1, 100, 200, 64) == 0
    assert fa.fa_prefix_fwd_workspace_bytes(2, 7, 2, 1, 100, 200, 64) == 0
    assert fa.fa_prefix_fwd_workspace_bytes(2, 8, 2, 1, 100, 200, 96) == 0
    assert fa.fa_cache_evict_workspace_bytes(2, 2, 0, 100) == 0
    assert fa.fa_verify_drafts_workspace_bytes(2, -1, 100) == 0


torch = pytest.importorskip("torch")


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def f32(*shape):
    return torch.zeros(shape)


def refused(call, *args, match=None, **kw):
    with pytest.raises(ValueError, match=match):
        call(*args, **kw)


def test_prefix_tensors():
    Q, p, K = bf(2, 1, 8, 64), bf(10, 2, 64), bf(2, 20, 2, 64)
    pool, tab = bf(9, 64, 2, 64), i32(2, 4)

    def call(*a, **kw):
        refused(fa.fa_prefix_fwd, *a, 0.1, True, **kw)
    call(Q, p, p, K, bf(2, 20, 2, 32))
    call(Q, p, p, bf(3, 20, 2, 64), bf(3, 20, 2, 64))
    call(Q, p, bf(9, 2, 64), K, K)
    call(Q, p.half(), p.half(), K, K)
    call(Q, bf(10, 1, 64), bf(10, 1, 64), K, K)
    call(Q, p, p, K, K, prefix_len=11)
    call(Q, p, p, K, K, prefix_len=-1)
    call(Q, p, p, K, K, seqlens_k=i32(3))
    call(Q, p, p, K, K, seqlens_k=torch.zeros(2, dtype=torch.int64))
    call(Q, p, p, pool, pool, block_table=i32(3, 4))
    call(Q, p, p, pool, pool, block_table=tab, max_seqlen_k=257)
    call(Q, p, p, pool, pool, block_table=tab, prefix_table=i32(2), prefix_len=5)
    call(Q, bf(9, 128, 2, 64), bf(9, 128, 2, 64), pool, pool, block_table=tab, prefix_table=i32(2), prefix_len=5)
    call(Q, pool, pool, K, K, prefix_table=i32(2))
    call(Q, pool, pool, K, K, prefix_table=i32(2), prefix_len=129)
    call(Q, pool, pool, K, K, prefix_table=i32(2, 1), prefix_len=5)
    call(Q, p, p, K, K, O=bf(2, 1, 8, 32))
    call(Q.float(), p, p, K, K)
    call(Q.transpose(1, 2), p, p, K, K)
    call(Q, p, p, K, K, match=None)  # (all in order, but on the host)


def test_cache_tensors():
    K, W, pos, n = bf(2, 20, 2, 64), f32(2, 2, 20), i32(2, 2, 20), i32(2)
    pool, tab = bf(9, 64, 2, 64), i32(2, 4)
    new = bf(2, 1, 2, 64)
    ap, we, ev = fa.fa_cache_append, fa.fa_cache_weights, fa.fa_cache_evict
    refused(ap, new, bf(2, 1, 2, 32), K, K, n)
    refused(ap, new, new, bf(2, 20, 1, 64), K, n)
    refused(ap, new, new, K.half(), K.half(), n)
    refused(ap, new, new, K, K, n, weights=f32(2, 2, 21))
    refused(ap, new, new, K, K, n, weights=W, positions=i32(2, 2, 19))
    refused(ap, new, new, K, K, n, positions=pos.float())
    refused(ap, new, new, K, K, n, first_position=i32(3))
    refused(ap, new, new, pool, pool, n, block_table=tab, weights=f32(2, 2, 257))
    refused(ap, new, new, K, K, n)  # on the host
    Q, L = bf(2, 1, 8, 64), f32(2, 8, 1)
    refused(we, Q, K, f32(2, 1, 8), W, 0.1, True, n)
    refused(we, Q, K, L.double(), W, 0.1, True, n)
    refused(we, Q, K, L, f32(2, 2, 21), 0.1, True, n)
    refused(we, Q, K, L, W.double(), 0.1, True, n)
    refused(we, Q, K, L, W, 0.1, True, n, queries=i32(1))
    refused(we, Q, pool, L, W, 0.1, True, n, block_table=i32(2, 0))
    refused(we, Q, K, L, W, 0.1, True, n)  # on the host
    refused(ev, K, K, W, pos, i32(1), 10)
    refused(ev, K, K, W, i32(2, 2, 21), n, 10)
    refused(ev, K, K, f32(2, 1, 20), pos, n, 10)
    refused(ev, K.float(), K.float(), W, pos, n, 10)
    refused(ev, K, K, W, pos, n, 10, weights_out=f32(2, 2, 19))
    refused(ev, K, K, W, pos, n, 10)  # on the host


def test_verify_tensors():
    x, q, t, u = i32(2, 3), f32(2, 3, 50), f32(2, 4, 50), f32(2, 4)
    ve = fa.fa_verify_drafts
    refused(ve, x.long(), q, t, u)
    refused(ve, x, f32(2, 3, 49), t, u)
    refused(ve, x, q, f32(2, 3, 50), u)
    refused(ve, x, q, t, f32(2, 3))
    refused(ve, x, q, t.double(), u)
    refused(ve, x, q, f32(2, 4, 100)[..., ::2], u)
    refused(ve, x, q, f32(4, 2, 50).transpose(0, 1), u)
    refused(ve, x, q, t, u, tokens=i32(2, 3))
    refused(ve, x, q, t, u)  # on the host


def test_slots_beyond_the_limit():
    """A slot and the one a tile further have to fit 32 bits: 2^30 is the most, also of slots in pages that repeat."""
    most = 1 << 30
    paged = dict(tab=P, page=1 << 20, pages=1 << 11)
    for call in (prefix, append, weights, evict):
        assert call(Nk=most + 1, **paged) == fa.FA_ERR_SHAPE
        assert call(Nk=2**31 - 1, **paged) == fa.FA_ERR_SHAPE
    assert prefix(Np=most + 1, ptab=P, page=1 << 20, ppages=1 << 11) == fa.FA_ERR_SHAPE
    # (accepted up to there: what is refused next is the workspace)
    assert prefix(Nk=most, Np=most, ptab=P, ppages=1 << 11, nb=0, **paged) == fa.FA_ERR_WORKSPACE
    assert evict(Nk=most, nb=0, **paged) == fa.FA_ERR_WORKSPACE
