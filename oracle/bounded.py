"""Oracle: accumulated attention weights and eviction of the positions that have the least of it (fp64).

TEST INFRASTRUCTURE ONLY - never imported by the product path.

A trace over its budget keeps its `recent` last positions and, of those before them, the budget - recent with the
largest weights - per layer and KV head.  Slots: with m = budget - recent, a chosen position below m stays, the free slots
below m take the other chosen positions in order, slots m .. budget - 1 take the last positions in order.
"""
from __future__ import annotations

import math

import numpy as np

from . import kv_pool as KP
from .attention import gather_trace_kv, softmax_weights


def decode_weights(q, K, V):
    """q [Hq, d]; K, V [S, Hkv, d] -> out [Hq, d], weight of every position per KV head [Hkv, S], sums with |v| [Hq, d]."""
    Hq, d = q.shape
    S, Hkv, _ = K.shape
    out, mag, w = np.zeros((Hq, d)), np.zeros((Hq, d)), np.zeros((Hkv, S))
    if S == 0:
        return out, w, mag
    for h in range(Hq):
        g = h // (Hq // Hkv)
        p = softmax_weights(K[:, g] @ np.asarray(q[h], np.float64) / math.sqrt(d))
        out[h], mag[h] = p @ V[:, g], p @ np.abs(V[:, g])
        w[g] += p
    return out, w, mag


def slots(weights, S, budget, recent):
    """The position that every slot of a cut head gets, [budget]; weights [>= S]."""
    first, m = S - recent, budget - recent

    def order(j):
        x = float(weights[j])
        return (1, 0.0, j) if math.isnan(x) else (0, -x, j)

    chosen = set(sorted(range(first), key=order)[:m])
    come = iter(sorted(j for j in chosen if j >= m))
    return [j if j in chosen else next(come) for j in range(m)] + list(range(first, S))


def evict(pool, trace_ids, weights, budget, recent):
    """On a KVPoolOracle.  weights [L, n, Hkv, stride].  Returns (weights afterwards, kept [L, n, Hkv, budget] with -1 in
    rows of entries left alone)."""
    L, n, Hkv, stride = weights.shape
    P, nbp = pool.P, -(-budget // pool.P)
    after, kept = np.array(weights), np.full((L, n, Hkv, budget), -1, dtype=np.int64)
    cut, seen = [], set()
    for i, t in enumerate(int(x) for x in trace_ids):       # every entry's own blocks come first
        if t in seen or t < 0 or t >= pool.max_traces or not pool.live[t]:
            pool._flag(KP.ERR_BAD_TRACE)
            continue
        seen.add(t)
        S = int(pool.seq_lens[t])
        if S <= budget:
            continue
        if S > stride:
            pool._flag(KP.ERR_CAPACITY)
            continue
        row = [int(b) for b in pool.block_table[t, :-(-S // P)]]
        cut.append((i, t, S, row))
    ready = []
    for i, t, S, row in cut:
        shared = [p for p in range(nbp) if pool.refcount[row[p]] > 1]
        if len(shared) > pool.free_count:
            pool._flag(KP.ERR_NO_BLOCKS)
            continue
        new = row[:nbp]
        for p in shared:
            new[p] = pool._pop()
        ready.append((i, t, S, row, new))
    for i, t, S, row, new in ready:
        for l in range(L):
            for h in range(Hkv):
                kept[l, i, h] = slots(weights[l, i, h], S, budget, recent)
                after[l, i, h] = 0
                after[l, i, h, :budget] = weights[l, i, h, kept[l, i, h]]
        if pool.store_payload:
            K, V = zip(*(gather_trace_kv(pool.k_pages[l], pool.v_pages[l], np.array(row), S) for l in range(L)))
            for l in range(L):
                for h in range(Hkv):
                    for j, src in enumerate(kept[l, i, h]):
                        pool.k_pages[l, new[j // P], h, j % P] = K[l][src, h]
                        pool.v_pages[l, new[j // P], h, j % P] = V[l][src, h]
    for i, t, S, row, new in ready:
        for p, b in enumerate(row):
            if p < nbp and new[p] == b:
                continue
            pool.refcount[b] -= 1
            if pool.refcount[b] == 0:
                pool.free_list.append(b)
        pool.block_table[t, :] = -1
        pool.block_table[t, :nbp] = new
        for p, b in enumerate(new):
            if b != row[p]:
                pool.refcount[b] = 1
        pool.seq_lens[t] = budget
    return after, kept
