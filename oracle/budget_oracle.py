"""Oracle of a KV cache inside a budget and of sampled tokens, in 64 bits: the definitions of include/harli.h written down plainly,
one sequence, layer, head or row at a time.  Nothing here knows of pages, chunks or fixed point."""
from __future__ import annotations

import math

import numpy as np


def attend_weights(q, K, V, weight, decay, newest_position):
    """One sequence and layer.  q [n_q, d]; K, V [n, n_kv, d]; weight [n, n_kv].  Returns out [n_q, d], the new weights [n, n_kv]
    and the probabilities [n_q, n]."""
    q, K, V = (np.asarray(a, np.float64) for a in (q, K, V))
    n, n_kv, d = K.shape
    n_q = q.shape[0]
    out, P = np.zeros((n_q, d)), np.zeros((n_q, n))
    if n == 0:
        return out, np.zeros((0, n_kv)), P
    new = np.zeros((n, n_kv)) if decay == 0 else decay * np.asarray(weight, np.float64)
    new[n - 1] = 0
    for h in range(n_q):
        c = h // (n_q // n_kv)
        s = K[:, c] @ q[h] / math.sqrt(d)
        e = np.exp(s - s.max())
        P[h] = e / e.sum()
        out[h] = P[h] @ V[:, c]
        new[:, c] += P[h]
    return out, new, P


def evict_moves(weight, position, keep, next_position, sink, recent):
    """One head: [(from, to)] of an eviction of n tokens down to `keep`."""
    n = len(weight)
    keep = max(int(keep), 0)
    if n <= keep:
        return []

    def rank(t):
        if position[t] < sink or position[t] >= next_position - recent:
            return (0, 0.0, t)
        w = float(weight[t])
        return (1, -w, t) if not math.isnan(w) else (2, 0.0, t)

    stays = set(sorted(range(n), key=rank)[:keep])
    holes = [t for t in range(keep) if t not in stays]
    movers = [t for t in range(keep, n) if t in stays]
    assert len(holes) == len(movers)
    return list(zip(movers, holes))


def sample_kept(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """One row: (indices that stay, in the order of the row's tokens; their weights, in 64 bits)."""
    z = np.asarray(logits, np.float64)
    z = np.where(np.isnan(z), -np.inf, z)
    if z.max() == -np.inf:
        return [], []
    order = [int(i) for i in np.argsort(-z, kind="stable") if z[i] > -np.inf]
    if not temperature > 0:
        return order[:1], [1.0]
    top = z[order[0]]
    weight = {i: 1.0 if z[i] == top else 0.0 if top == np.inf else math.exp((z[i] - top) / temperature) for i in order}
    kept = order[:top_k] if 0 < top_k < len(z) else order
    if top_p < 1:
        whole, before, cut = math.fsum(weight[i] for i in kept), 0.0, []
        for i in kept:
            if cut and not before < top_p * whole:
                break
            cut.append(i)
            before = math.fsum(weight[j] for j in cut)
        kept = cut
    if min_p > 0:
        kept = [i for i in kept if weight[i] >= min(min_p, 1.0)]
    return kept, [weight[i] for i in kept]


def sample_token(logits, uniform, **settings):
    """One row: (token, log probability among what stays)."""
    kept, weight = sample_kept(logits, **settings)
    if not kept:
        return -1, -math.inf
    by_index = sorted(zip(kept, weight))
    total = math.fsum(w for _, w in by_index)
    u = uniform if uniform > 0 else 0.0
    reach = 0.0
    for i, w in by_index:
        reach += w
        if reach > u * total:
            return i, math.log(w / total)
    i, w = [x for x in by_index if x[1] > 0][-1]
    return i, math.log(w / total)
