"""The operators of a decoding batch from their definitions, in float64 on the CPU: attention over a shared prefix and own keys, attention
weight per cached key, which slots of a cache are kept, which drafted tokens are accepted. Test infrastructure only."""
import numpy as np


def sees(nq, nk, causal):
    """[nq, nk]: query r stands at position r + nk - nq of the keys."""
    c, r = np.arange(nk), np.arange(nq)[:, None]
    return c <= r + nk - nq if causal else np.ones((nq, nk), bool)


def prefix_forward(Q, Kp, Vp, K, V, lens, scale, causal):
    """Q [B,Nq,Hq,d], Kp, Vp [Np,Hkv,d], K, V: per sequence [>= lens[b],Hkv,d] -> O, LSE [B,Hq,Nq], and sum_c p_c |v_c| [B,Nq,Hq,d] with
    the largest sum of |q k| of a row [B,Hq,Nq], by which rounding errors go."""
    B, nq, hq, d = Q.shape
    hkv = Kp.shape[1]
    O, A = np.zeros(Q.shape), np.zeros(Q.shape)
    L, M = np.full((B, hq, nq), -np.inf), np.zeros((B, hq, nq))
    for b in range(B):
        n = int(lens[b])
        for h in range(hq):
            g = h // (hq // hkv)
            k, v = np.concatenate([Kp[:, g], K[b][:n, g]]), np.concatenate([Vp[:, g], V[b][:n, g]])
            see = np.concatenate([np.ones((nq, len(Kp)), bool), sees(nq, n, causal)], 1)
            s = np.where(see, scale * (Q[b, :, h] @ k.T), -np.inf)
            if s.shape[1] == 0:
                continue
            m = s.max(1)
            ok = m > -np.inf
            p = np.where(ok[:, None], np.exp(s - np.where(ok, m, 0)[:, None]), 0.0)
            z = np.where(ok, p.sum(1), 1.0)
            p /= z[:, None]
            O[b, :, h], A[b, :, h] = p @ v, p @ np.abs(v)
            L[b, h] = np.where(ok, m + np.log(z), -np.inf)
            M[b, h] = scale * np.max(np.where(see, np.abs(Q[b, :, h]) @ np.abs(k).T, 0.0), 1)
    return O, L, A, M


def key_weights(Q, K, LSE, lens, scale, causal, queries=None):
    """Per sequence [Hkv, lens[b]]: the sums of exp(s - L), and the sums of their rounding errors' sizes."""
    B, nq, hq, d = Q.shape
    out, err = [], []
    for b in range(B):
        n, hkv = int(lens[b]), K[b].shape[1]
        w, e = np.zeros((hkv, n)), np.zeros((hkv, n))
        for h in range(hq):
            g = h // (hq // hkv)
            k, L = K[b][:n, g], LSE[b, h][:, None]
            see = sees(nq, n, causal) & (L > -np.inf)
            if queries is not None:
                see &= np.arange(nq)[:, None] < queries[b]
            s = scale * (Q[b, :, h] @ k.T)
            p = np.where(see, np.exp(s - np.where(L > -np.inf, L, np.inf)), 0.0)
            size = d * scale * (np.abs(Q[b, :, h]) @ np.abs(k).T) / 2**24 + (np.abs(s) + np.abs(np.where(L > -np.inf, L, 0)) + 1) / 2**21
            w[g] += p.sum(0)
            e[g] += (p * size).sum(0)
        out.append(w)
        err.append(e)
    return out, err


def kept_slots(weights, positions, n, budget, sinks, recent):
    """One head: (slot that each of the first min(n, budget) slots holds afterwards)."""
    if n <= budget:
        return np.arange(n)
    w, pos = weights[:n], positions[:n].astype(np.int64)
    safe = (pos < sinks) | (pos > pos.max() - recent)
    order = sorted(range(n), key=lambda i: (not safe[i], *((0,) if safe[i] else (1, 0.0) if np.isnan(w[i]) else (0, -float(w[i]))), i))
    keep = np.zeros(n, bool)
    keep[order[:budget]] = True
    out = np.arange(budget)
    out[~keep[:budget]] = np.flatnonzero(keep[budget:]) + budget
    return out


def verify(drafts, q, target, uniform, logits=False, inv_temperature=1.0):
    """-> tokens [B,k+1], accepted [B], and the least relative distance of any decision from its border."""
    B, k = drafts.shape
    V = target.shape[2]
    tokens, accepted, margin = np.full((B, k + 1), -1), np.zeros(B, int), np.inf
    for b in range(B):
        for i in range(k + 1):
            p = target[b, i].astype(np.float64)
            if logits:
                x = p * inv_temperature
                m = x.max()
                e = np.exp(x - m) if m > -np.inf else np.zeros(V)
                p = e / e.sum() if e.sum() > 0 else e
            x = int(drafts[b, i]) if i < k else -1
            if not 0 <= x < V:
                r = p
                break
            d = np.zeros(V)
            if q is None:
                d[x] = 1.0
            else:
                d = q[b, i].astype(np.float64)
            u = float(uniform[b, i]) * d[x]
            margin = min(margin, abs(u - p[x]) / max(p[x], u, 1e-300))
            if not u < p[x]:
                r = np.maximum(p - d, 0.0)
                r = r if r.sum() > 0 else p
                break
            tokens[b, i] = x
            accepted[b] += 1
        c = np.cumsum(r)
        if c[-1] > 0:
            want = float(uniform[b, k]) * c[-1]
            past = np.flatnonzero((c > want) & (r > 0))
            tokens[b, accepted[b]] = past[0] if len(past) else np.flatnonzero(r > 0)[-1]
            margin = min(margin, np.min(np.abs(c - want)) / c[-1])
    return tokens, accepted, margin
