"""Accumulated attention weights and eviction by them, in fp64 (the oracle).

TEST INFRASTRUCTURE ONLY: only tests may use this module.

A key's weight in one call is what the softmax of every query that sees it
gives it, summed over the call's queries and over the query heads of its KV
head. An eviction keeps, of a sequence's L positions and per KV head, the last
R, the first S and the highest-scored of the others, up to a budget; R goes
before S where there is no room for both, equal scores go by position (lowest
first), and a NaN is a score of -infinity.
"""

from __future__ import annotations

import numpy as np


def attention_weights(q, k, q_pos, scale) -> np.ndarray:
    """[Hkv, L]: weights of the keys k [L, Hkv, D] under the queries
    q [Tq, Hq, D] at positions q_pos (a negative one sees no key)."""
    q, k = np.asarray(q, dtype=np.float64), np.asarray(k, dtype=np.float64)
    n, hkv, _ = k.shape
    group = q.shape[1] // hkv
    total = np.zeros((hkv, n))
    for t, p in enumerate(q_pos):
        if p < 0:
            continue
        for h in range(q.shape[1]):
            s = scale * (k[: p + 1, h // group] @ q[t, h])
            e = np.exp(s - s.max())
            total[h // group, : p + 1] += e / e.sum()
    return total


def kept_positions(scores, length: int, budget: int, recent: int, sinks: int) -> np.ndarray:
    """Kept positions in increasing order of one KV head's scores [>= length]."""
    keep = max(0, min(int(budget), int(length)))
    last = min(int(recent), keep)
    first = min(int(sinks), keep - last)
    s = np.asarray(scores[:length], dtype=np.float64)
    s = np.where(np.isnan(s), -np.inf, s)
    middle = np.arange(first, length - last)
    best = middle[np.argsort(-s[middle], kind="stable")][: keep - last - first]
    return np.concatenate([np.arange(first), np.sort(best), np.arange(length - last, length)]).astype(np.int64)
