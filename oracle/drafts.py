"""Oracle: attention of drafted-token trees, and storing the accepted part of a draft (fp64).

TEST INFRASTRUCTURE ONLY - never imported by the product path.

A trace's continuation is drafted as a tree: node u continues node parents[u] < u, or the cached text itself if that is
-1.  Node u attends to every cached position, to itself and to its ancestors.
"""
from __future__ import annotations

import math

import numpy as np

from . import kv_pool as KP
from .attention import gather_trace_kv, softmax_weights


def path_to_root(parents, u):
    """u and its ancestors.  A parent that does not come before its node counts as none."""
    seen = []
    while u >= 0:
        seen.append(u)
        p = int(parents[u])
        u = p if -1 <= p < u else -1
    return seen


def tree_attention(q, K, V, k_draft, v_draft, parents, nodes):
    """One trace.  q [T, Hq, d]; K, V [S, Hkv, d] cached; k_draft, v_draft [T, Hkv, d] -> [T, Hq, d]; rows from `nodes`
    on are zeros.  Second result: the same sums with |v| in place of v, for error bounds."""
    T, Hq, d = q.shape
    G = Hq // K.shape[1]
    out, mag = np.zeros((T, Hq, d)), np.zeros((T, Hq, d))
    for u in range(nodes):
        see = path_to_root(parents, u)
        k = np.concatenate([K, np.asarray(k_draft, np.float64)[see]])
        v = np.concatenate([V, np.asarray(v_draft, np.float64)[see]])
        for h in range(Hq):
            p = softmax_weights(k[:, h // G] @ np.asarray(q[u, h], np.float64) / math.sqrt(d))
            out[u, h], mag[u, h] = p @ v[:, h // G], p @ np.abs(v[:, h // G])
    return out, mag


def paged_tree_attention(q, k_pages, v_pages, k_draft, v_draft, parents, n_nodes, block_table, seq_lens):
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    for t in range(q.shape[0]):
        K, V = gather_trace_kv(k_pages, v_pages, block_table[t], int(seq_lens[t]))
        out[t], mag[t] = tree_attention(q[t], K, V, k_draft[t], v_draft[t], parents[t], int(n_nodes[t]))
    return out, mag


def append_path(pool, trace_ids, T, path, path_len, k_draft=None, v_draft=None):
    """append_kv of path_len[i] rows of entry i's draft, in the order path[i] names them; a trace listed twice is served
    at its first place."""
    seen = set()
    for i, t in enumerate(int(x) for x in trace_ids):
        k = int(path_len[i])
        if t in seen:
            pool._flag(KP.ERR_BAD_TRACE)
            continue
        seen.add(t)
        if t < 0 or t >= pool.max_traces or not pool.live[t]:
            pool._flag(KP.ERR_BAD_TRACE)
            continue
        if k < 0 or k > path.shape[1] or np.any(path[i, :k] < 0) or np.any(path[i, :k] >= T):
            pool._flag(KP.ERR_INVALID_ARG)
            continue
        rows = path[i, :k]
        pay = (k_draft[i][None, rows], v_draft[i][None, rows]) if pool.store_payload else (None, None)
        pool.append_kv([t], k, *pay)
