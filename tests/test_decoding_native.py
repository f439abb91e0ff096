"""The native marshalling of the calls of a decoding batch: it makes the call that binding.py would make, and leaves what is not an
ordinary call to it."""
import pytest

from paper_2307_08691_amd import binding

torch = pytest.importorskip("torch")

NAMES = ("prefix_fwd", "cache_append", "cache_weights", "cache_evict", "verify_drafts")


@pytest.fixture(scope="module")
def host():
    binding._load_host()
    assert binding._host, "the extension module has not been built"
    return binding._host


def test_host_tensors_and_other_objects_are_left_to_the_binding(host):
    x = torch.zeros(1, 64, 2, 64, dtype=torch.bfloat16)
    for name, args in zip(NAMES, (12, 9, 9, 12, 6)):
        call = getattr(host, name)
        assert call() is None and call(*[x] * args) is None and call(*[None] * args) is None and call(*["x"] * args) is None


def calls(dtype, page):
    """name -> a call on state of its own, which returns everything that it returns or writes"""
    g = torch.Generator(device="cuda").manual_seed(23000)
    t = lambda *s: torch.randn(s, generator=g, device="cuda").to(dtype)  # noqa: E731
    B, nq, hq, hkv, d, slots = 3, 2, 8, 2, 64, 256
    lens = torch.tensor([200, 2, 256], dtype=torch.int32, device="cuda")
    table = torch.tensor([[3, 0, 6, 1], [2, 7, 5, 4], [8, 9, 10, 11]], dtype=torch.int32, device="cuda") if page else None
    K, V = (t(12, 64, hkv, d) if page else t(B, slots, hkv, d) for _ in range(2))
    Q, Kn, Vn, Kp, Vp = t(B, nq, hq, d), t(B, nq, hkv, d), t(B, nq, hkv, d), t(90, hkv, d), t(90, hkv, d)
    W = torch.rand((B, hkv, slots), generator=g, device="cuda")
    P = torch.arange(slots, dtype=torch.int32, device="cuda").expand(B, hkv, slots).contiguous()
    L = torch.rand((B, hq, nq), generator=g, device="cuda") + 4
    x = torch.randint(0, 500, (B, 4), generator=g, device="cuda", dtype=torch.int32)
    q, p = (torch.softmax(torch.randn((B, n, 500), generator=g, device="cuda"), -1) for n in (4, 5))
    u = torch.rand((B, 5), generator=g, device="cuda")

    def prefix(**kw):
        return binding.fa_prefix_fwd(Q, Kp, Vp, K, V, 0.125, True, seqlens_k=lens, block_table=table, **kw)

    def append():
        k, v, w, i = K.clone(), V.clone(), W.clone(), P.clone()
        binding.fa_cache_append(Kn, Vn, k, v, lens, block_table=table, weights=w, positions=i, first_position=lens)
        return k, v, w, i

    def weights():
        return (binding.fa_cache_weights(Q, K, L, W.clone(), 0.125, True, seqlens_k=lens, block_table=table, queries=lens),)

    def evict():
        k, v, w, i, n = K.clone(), V.clone(), W.clone(), P.clone(), lens.clone()
        return (k, v, *binding.fa_cache_evict(k, v, w, i, n, 100, 4, 20, block_table=table))

    out = {"prefix_fwd": prefix, "prefix_fwd, bounded": lambda: prefix(prefix_len=33, **(dict(max_seqlen_k=220) if page else {})), "cache_append": append,
           "cache_weights": weights, "cache_evict": evict, "verify_drafts": lambda: binding.fa_verify_drafts(x, q, p, u),
           "verify_drafts, logits": lambda: binding.fa_verify_drafts(x, None, p.to(dtype), u, logits=True, inv_temperature=0.5)}
    if page:
        out["prefix_fwd, pages"] = lambda: binding.fa_prefix_fwd(Q, K, V, K, V, 0.125, False, seqlens_k=lens, block_table=table,
                                                                 prefix_table=table[0, :2].contiguous(), prefix_len=100)
    return out


@pytest.mark.gpu
@pytest.mark.parametrize("page", [0, 64])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_native_and_python_calls_agree_bitwise(host, dtype, page, monkeypatch):
    class Counting:
        def __init__(self):
            self.native = 0

        def __getattr__(self, name):
            def call(*args):
                r = getattr(host, name)(*args)
                self.native += r is not None
                return r
            return call

    for name, call in calls(dtype, page).items():
        counting = Counting()
        monkeypatch.setattr(binding, "_host", counting)
        a = call()
        assert counting.native == 1, name
        monkeypatch.setattr(binding, "_host", False)
        b = call()
        torch.cuda.synchronize()
        for y, z in zip(a, b):
            assert torch.equal(y, z), name


@pytest.mark.gpu
def test_unusual_calls_are_left_to_the_binding(host):
    """Slices of wider rows, a float64 target, a transposed query: taken by the Python, with its results or its errors."""
    wide = torch.softmax(torch.randn((2, 3, 110), device="cuda"), -1)
    x, u = torch.zeros((2, 2), dtype=torch.int32, device="cuda"), torch.rand((2, 3), device="cuda")
    assert host.verify_drafts(x, None, wide[..., :100], u, False, 1.0) is None
    a = binding.fa_verify_drafts(x, None, wide[..., :100], u)
    b = binding.fa_verify_drafts(x, None, wide[..., :100].contiguous(), u)
    assert all(torch.equal(y, z) for y, z in zip(a, b))
    with pytest.raises(ValueError):
        binding.fa_verify_drafts(x, None, wide.double(), u)
    Q = torch.zeros((2, 4, 3, 64), dtype=torch.bfloat16, device="cuda")
    K = torch.zeros((2, 64, 1, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(ValueError):
        binding.fa_cache_weights(Q.transpose(1, 2), K, torch.zeros((2, 4, 3), device="cuda"), torch.zeros((2, 1, 64), device="cuda"), 0.125, True)
    with pytest.raises(binding.FaError):
        binding.fa_cache_weights(Q, K, torch.zeros((2, 3, 4), device="cuda"), torch.zeros((2, 1, 64), device="cuda"), -1.0, True)
