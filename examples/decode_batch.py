"""Decode a batch of answers to one prompt with caches that stay small and drafted tokens.

    python examples/decode_batch.py --sequences 64 --prompt 8192 --budget 128 --drafts 4 --steps 50

A toy model of one attention layer with random weights (there is nothing to learn from its text): the target's logits come from the
embedding and the attention over everything so far, the draft's from the embedding alone. Every step

  drafts k tokens per sequence,
  appends the keys and values of the last token and of the drafts to the sequence's pages       (fa_cache_append),
  attends to the prompt, which is kept once for the whole batch, and to the sequence's own keys  (fa_prefix_fwd),
  accepts the drafts or replaces one, in the target's distribution                              (fa_verify_drafts),
  adds up what the accepted queries looked at                                                   (fa_cache_weights),
  and drops what was looked at least from caches that have outgrown their budget                (fa_cache_evict).

Nothing in a step waits for the GPU: lengths, accepted tokens and page contents stay there.
"""
import argparse
import os
import sys
import time

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2307_08691_amd import binding as fa  # noqa: E402


class Model:
    def __init__(self, vocab, width, heads, kv_heads, d, seed=0, device="cuda", dtype=torch.bfloat16):
        g = torch.Generator(device=device).manual_seed(seed)
        w = lambda *s: (torch.randn(s, generator=g, device=device) / s[0]**0.5).to(dtype)  # noqa: E731
        self.heads, self.kv_heads, self.d, self.vocab = heads, kv_heads, d, vocab
        self.embedding = torch.randn((vocab, width), generator=g, device=device).to(dtype)
        self.wq, self.wk, self.wv = w(width, heads * d), w(width, kv_heads * d), w(width, kv_heads * d)
        self.wo, self.head = w(heads * d, width), 2 * w(width, vocab)

    def keys_values(self, h):
        return (h @ self.wk).unflatten(-1, (self.kv_heads, self.d)), (h @ self.wv).unflatten(-1, (self.kv_heads, self.d))

    def queries(self, h):
        return (h @ self.wq).unflatten(-1, (self.heads, self.d))


class Batch:
    """The state of `sequences` answers to one prompt, in pages of 64 slots."""

    PAGE = 64

    def __init__(self, model, prompt, sequences, budget, drafts, sinks=4, recent=64, seed=0):
        self.model, self.budget, self.drafts, self.sinks, self.recent = model, budget, drafts, sinks, min(recent, budget - sinks)
        device = prompt.device
        self.rng = torch.Generator(device=device).manual_seed(seed)
        # (the prompt's last token is the first that is fed: its key is the batch's own)
        self.prefix = tuple(x.contiguous() for x in model.keys_values(model.embedding[prompt[:-1]]))
        pages = -(-(budget + drafts + 1) // self.PAGE)
        slots = pages * self.PAGE
        shape = (sequences * pages, self.PAGE, model.kv_heads, model.d)
        self.K, self.V = (torch.zeros(shape, dtype=model.wk.dtype, device=device) for _ in range(2))
        order = torch.randperm(sequences * pages, generator=self.rng, device=device)
        self.table = order.reshape(sequences, pages).int()
        self.weights = torch.zeros((sequences, model.kv_heads, slots), device=device)
        self.positions = torch.zeros((sequences, model.kv_heads, slots), dtype=torch.int32, device=device)
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device=device)
        self.next_position = torch.full((sequences,), len(prompt) - 1, dtype=torch.int32, device=device)
        self.last = prompt[-1].expand(sequences, 1).int().contiguous()

    def draft(self):
        """k tokens per sequence drawn from the draft model, and its probabilities."""
        x, tokens, probs = self.last, [], []
        for _ in range(self.drafts):
            q = torch.softmax((self.model.embedding[x[:, 0]] @ self.model.head).float(), -1)
            noise = torch.rand(q.shape, generator=self.rng, device=q.device).clamp_min_(1e-20)
            x = (q / -torch.log(noise)).argmax(-1, keepdim=True).int()
            tokens.append(x)
            probs.append(q)
        return torch.cat(tokens, 1), torch.stack(probs, 1)

    def step(self):
        """One round of drafting and verification -> tokens [B, k + 1] (the new ones, then -1) and how many drafts were accepted [B]."""
        m, k = self.model, self.drafts
        drafts, probs = self.draft()
        h = m.embedding[torch.cat([self.last, drafts], 1)]
        self.lengths += k + 1
        keys, values = m.keys_values(h)
        where = dict(seqlens_k=self.lengths, block_table=self.table)
        fa.fa_cache_append(keys.contiguous(), values.contiguous(), self.K, self.V, weights=self.weights, positions=self.positions,
                           first_position=self.next_position, **where)
        q = m.queries(h).contiguous()
        scale = m.d**-0.5
        out, lse = fa.fa_prefix_fwd(q, *self.prefix, self.K, self.V, scale, True, **where)
        logits = (h + out.flatten(2) @ m.wo) @ m.head
        uniform = torch.rand((len(h), k + 1), generator=self.rng, device=h.device)
        tokens, accepted = fa.fa_verify_drafts(drafts, probs, logits, uniform, logits=True)
        fed = accepted + 1  # the last token and the accepted drafts: what the sequence now holds keys of
        fa.fa_cache_weights(q, self.K, lse, self.weights, scale, True, queries=fed, **where)
        self.lengths += fed - (k + 1)
        self.next_position += fed
        self.last = tokens.gather(1, accepted[:, None].long())
        fa.fa_cache_evict(self.K, self.V, self.weights, self.positions, self.lengths, self.budget, self.sinks, self.recent, block_table=self.table)
        return tokens, accepted


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in dict(sequences=64, prompt=8192, budget=128, drafts=4, steps=50, vocab=32000, width=1024, heads=32, kv_heads=8, d=128).items():
        ap.add_argument("--" + name.replace("_", "-"), type=int, default=value)
    a = ap.parse_args()
    model = Model(a.vocab, a.width, a.heads, a.kv_heads, a.d)
    prompt = torch.randint(0, a.vocab, (a.prompt,), device="cuda")
    batch = Batch(model, prompt, a.sequences, a.budget, a.drafts)
    for _ in range(3):
        batch.step()
    torch.cuda.synchronize()
    start, made = time.perf_counter(), 0
    accepted = [batch.step()[1] for _ in range(a.steps)]
    torch.cuda.synchronize()
    seconds = time.perf_counter() - start
    made = sum(int((x + 1).sum()) for x in accepted)
    print(f"{a.sequences} sequences on a prompt of {a.prompt}: {a.steps} steps, {made} tokens ({made / a.steps / a.sequences:.2f} a step and sequence), "
          f"{1e3 * seconds / a.steps:.2f} ms a step, {made / seconds:.0f} tokens/s; at most {int(batch.lengths.max())} own keys a sequence")


if __name__ == "__main__":
    main()
