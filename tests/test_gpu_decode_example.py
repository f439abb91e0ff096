"""The decoding example (examples/decode_batch.py): all operators of a decoding batch as one program uses them. What its caches hold after
many steps is checked against the tokens that it made."""
import importlib.util
import os

import pytest

from paper_2307_08691_amd import binding as fa

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("decode_batch", os.path.join(ROOT, "examples", "decode_batch.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def play(example, budget, steps=40, drafts=3):
    model = example.Model(vocab=400, width=128, heads=8, kv_heads=2, d=64, seed=1)
    prompt = torch.randint(0, 400, (300,), generator=torch.Generator().manual_seed(2)).cuda()
    batch = example.Batch(model, prompt, 5, budget, drafts, recent=16, seed=3)
    text = [[int(prompt[-1])] for _ in range(5)]
    took = torch.zeros(drafts + 1, dtype=torch.int64)
    for _ in range(steps):
        tokens, accepted = batch.step()
        for b, (row, n) in enumerate(zip(tokens.tolist(), accepted.tolist())):
            assert all(0 <= t < 400 for t in row[:n + 1]) and row[n + 1:] == [-1] * (drafts - n)
            text[b] += row[:n + 1]
            took[n] += 1
    return model, prompt, batch, text, took


@pytest.mark.parametrize("budget", [48, 4096])
def test_caches_hold_the_tokens_that_were_made(example, budget):
    model, prompt, batch, text, took = play(example, budget)
    assert (took > 0).sum() >= 2  # (drafts were accepted and rejected)
    start = len(prompt) - 1
    for b in range(5):
        fed = len(text[b]) - 1  # (the newest token has not been fed)
        n = int(batch.lengths[b])
        assert n == min(fed, budget) and int(batch.next_position[b]) == start + fed and int(batch.last[b]) == text[b][-1]
        rows = [x[batch.table[b].long()].reshape(-1, 2, 64)[:n] for x in (batch.K, batch.V)]
        pos = batch.positions[b, :, :n].long() - start
        for g in range(2):
            held = pos[g].tolist()
            assert len(set(held)) == n and min(held) >= 0 and max(held) == fed - 1
            assert set(range(fed - min(batch.recent, fed), fed)) <= set(held)  # the newest stay
            h = model.embedding[torch.tensor([text[b][p] for p in held], device="cuda")]
            for x, y in zip(rows, model.keys_values(h)):
                torch.testing.assert_close(x[:, g].float(), y[:, g].float(), rtol=2**-6, atol=2**-6)
        # every counted query gave its weight to the prompt and to own keys: never more than one a query and head
        total = batch.weights[b, :, :n].double().sum(-1)
        assert (total >= 0).all() and (total <= fed * 4 * (1 + 1e-4)).all()


def test_a_step_attends_to_the_prompt_and_to_what_is_kept(example):
    model, _, batch, _, _ = play(example, 48, steps=30)
    q = model.queries(model.embedding[batch.last]).contiguous()
    O, L = fa.fa_prefix_fwd(q, *batch.prefix, batch.K, batch.V, 0.125, True, seqlens_k=batch.lengths, block_table=batch.table)
    whole = [torch.cat([p.expand(5, -1, -1, -1), torch.stack([x[batch.table[b].long()].reshape(-1, 2, 64) for b in range(5)])], 1).contiguous()
             for p, x in zip(batch.prefix, (batch.K, batch.V))]
    eO, eL = fa.fa_kvcache_fwd(q, *whole, 0.125, True, seqlens_k=batch.lengths + len(batch.prefix[0]))
    torch.testing.assert_close(L, eL, rtol=0, atol=1e-5)
    torch.testing.assert_close(O.float(), eO.float(), rtol=2**-6, atol=2**-8)
