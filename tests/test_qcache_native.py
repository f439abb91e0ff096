"""The native marshalling of the calls on caches in 4 or 8 bits and of the rotary positions: it makes the call that binding.py would make, and
leaves what is not an ordinary call to it."""
import pytest

from paper_2307_08691_amd import binding

torch = pytest.importorskip("torch")

NAMES = {"qcache_append": 8, "qcache_read": 8, "qcache_fwd": 7, "rope": 7}


@pytest.fixture(scope="module")
def host():
    binding._load_host()
    assert binding._host, "the extension module has not been built"
    return binding._host


def test_host_tensors_and_other_objects_are_left_to_the_binding(host):
    x = torch.zeros(1, 64, 2, 64, dtype=torch.bfloat16)
    for name, n in NAMES.items():
        call = getattr(host, name)
        assert call() is None and call(*[x] * n) is None and call(*[None] * n) is None and call(*[True] * n) is None and call(*[(x,) * 4] * n) is None


def calls(page):
    """name -> (the native call's name, a call that returns everything that it returns or writes)"""
    g = torch.Generator(device="cuda").manual_seed(29000)
    t = lambda *s: torch.randn(s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    B, nq, hq, hkv, d, slots = 3, 2, 8, 2, 64, 256
    lens = ints(200, 2, 256)
    table = torch.tensor([[3, 0, 6, 1], [2, 7, 5, 4], [8, 9, 10, 11]], dtype=torch.int32, device="cuda") if page else None
    cache = binding.qcache(12, hkv, 64, d, 8, 4) if page else binding.qcache(B, hkv, slots, d, 8, 4)
    where = dict(seqlens_k=lens, block_table=table)
    binding.fa_qcache_append(t(B, slots, hkv, d), t(B, slots, hkv, d), cache, block_table=table)
    wide, Q, f = t(B, nq, 4 * hkv, d), t(B, nq, hq, d), torch.rand(24, generator=g, device="cuda")
    pos = torch.arange(2 * B * nq, dtype=torch.int32, device="cuda").view(2, B, nq)

    def append(**kw):
        c = binding.QCache(*(x.clone() for x in cache))
        binding.fa_qcache_append(wide[:, :, 1:1 + hkv], wide[:, :, hkv:2 * hkv], c, **where, **kw)
        return (*c, *kw.values())

    def read(packed, **kw):
        K, V = (torch.zeros((40, hkv, d) if packed else (B, 30, hkv, d), dtype=torch.float16, device="cuda") for _ in range(2))
        return binding.fa_qcache_read(cache, K, V, **where, **kw)

    out = {"append": ("qcache_append", append), "append, rounded": ("qcache_append", lambda: append(Kout=torch.zeros_like(wide[:, :, :hkv].contiguous()),
                                                                                                   Vout=torch.zeros_like(wide[:, :, :hkv].contiguous()))),
           "read": ("qcache_read", lambda: read(False, first=ints(180, 0, 3))), "read, packed": ("qcache_read", lambda: read(True, cu_seqlens=ints(0, 30, 32, 39))),
           "fwd": ("qcache_fwd", lambda: binding.fa_qcache_fwd(Q, cache, 0.125, True, **where)),
           "rope": ("rope", lambda: binding.fa_rope_fwd(wide[:, :, :6], wide[:, :, 6:], pos, f, ints(*[0, 1] * 12))),
           "rope, back": ("rope", lambda: binding.fa_rope_bwd(Q, None, pos[0], f, neighbours=True)[:1]),
           "rope, packed": ("rope", lambda: binding.fa_rope_fwd(Q[0], wide[0, :, :2], pos[:, 0], f))}
    if page:
        out["fwd, bounded"] = ("qcache_fwd", lambda: binding.fa_qcache_fwd(Q, cache, 0.125, False, max_seqlen_k=220, **where))
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("page", [False, True])
def test_native_calls_do_what_the_binding_does(host, page, monkeypatch):
    for name, (native, call) in calls(page).items():
        seen = []

        class Watched:
            def __getattr__(self, n):
                f = getattr(host, n)

                def made(*a):
                    r = f(*a)
                    seen.append((n, r is not None))
                    return r
                return made

        monkeypatch.setattr(binding, "_host", Watched())
        got = call()
        assert (native, True) in seen, name
        monkeypatch.setattr(binding, "_host", False)
        want = call()
        assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want)), name


@pytest.mark.gpu
def test_unusual_calls_go_to_the_binding(host):
    """Errors are the binding's own."""
    c = binding.qcache(1, 2, 64, 64)
    Q = torch.zeros(1, 1, 4, 64, dtype=torch.bfloat16, device="cuda")
    assert host.qcache_fwd(Q, c, 0.1, True, None, None, 65) is None
    with pytest.raises(ValueError):
        binding.fa_qcache_fwd(Q, c, 0.1, True, max_seqlen_k=65)
    assert host.qcache_fwd(Q, c, -1.0, True, None, None, 0) is None
    with pytest.raises(binding.FaError):
        binding.fa_qcache_fwd(Q, c, -1.0, True)
    x = torch.zeros(1, 1, 2, 68, dtype=torch.bfloat16, device="cuda")[..., :64]
    assert host.qcache_append(x, x, c, None, None, 0, None, None) is None
    with pytest.raises(ValueError):
        binding.fa_qcache_append(x, x, c)
