"""Oracle: rotary positions, and a cache that is written layer by layer (extended precision, then fp64).

TEST INFRASTRUCTURE ONLY - never imported by the product path.

A pair (x1, x2) of a head's first D dims, at position p, is turned by the angle p * f_i: as a complex number it is multiplied
by scale * exp(j p f_i).  Angles of far positions lose everything in 32 bits and too much in 64 for a test of fp32
results at 2^31, so they are made in numpy's longdouble.
"""
from __future__ import annotations

import math

import numpy as np

from . import kv_pool as KP

LD = np.longdouble
TWO_PI = LD("6.283185307179586476925286766559005768")


def frequencies(D, base, scaling=None, factor=1.0, original_positions=0, fast=None, slow=1.0, divisors=None):
    """f_i, i < D / 2: t_i = base^(-2i / D), stretched for contexts longer than trained on."""
    i = np.arange(D // 2, dtype=LD)
    b = LD(base)
    if scaling == "base":
        b = b * LD(factor) ** (LD(D) / LD(D - 2))
    t = b ** (-2 * i / LD(D))
    if scaling == "linear":
        t = t / LD(factor)
    elif scaling == "yarn":
        fast = 32.0 if fast is None else fast
        place = [D * math.log(original_positions / (n * 2 * math.pi)) / (2 * math.log(base)) for n in (fast, slow)]
        first, last = max(math.floor(place[0]), 0), min(math.ceil(place[1]), D - 1)
        r = np.clip((i - first) / max(last - first, 1e-3), 0, 1)
        t = t * (1 - r) + t / LD(factor) * r
    elif scaling == "bands":
        fast = 4.0 if fast is None else fast
        turns = original_positions * t / TWO_PI
        r = np.clip((fast - turns) / (fast - slow), 0, 1)
        t = t * (1 - r) + t / LD(factor) * r
    if divisors is not None:
        t = t / np.asarray(divisors, dtype=LD)
    return t


def output_scale(scaling, factor):
    return 0.1 * math.log(factor) + 1.0 if scaling == "yarn" and factor > 1 else 1.0


def rotate(x, positions, f, interleaved, scale=1.0, transpose=False):
    """x [..., heads, d], positions [...] -> fp64; dims behind 2 len(f) as they are."""
    x = np.asarray(x, dtype=np.float64)
    D = 2 * len(f)
    a = np.asarray(positions, dtype=LD)[..., None, None] * f
    c, s = (np.cos(a) * LD(scale)).astype(np.float64), (np.sin(a) * LD(scale)).astype(np.float64)
    if transpose:
        s = -s
    one, two = (slice(0, D, 2), slice(1, D, 2)) if interleaved else (slice(0, D // 2), slice(D // 2, D))
    y = x.copy()
    y[..., one] = x[..., one] * c - x[..., two] * s
    y[..., two] = x[..., two] * c + x[..., one] * s
    return y


def extend(pool, trace_ids, n_tokens):
    """append_kv's allocation without rows: the old lengths, -1 for what was skipped; a trace listed twice is served at its
    first place."""
    start, seen, payload = [], set(), pool.store_payload
    pool.store_payload = False
    for t in (int(x) for x in trace_ids):
        S = int(pool.seq_lens[t]) if 0 <= t < pool.max_traces else -1
        if t in seen:
            pool._flag(KP.ERR_BAD_TRACE)
            start.append(-1)
            continue
        seen.add(t)
        start.append(S if pool.append_kv([t], n_tokens)[0] else -1)
    pool.store_payload = payload
    return np.array(start, dtype=np.int64)


def store(pool, layer0, trace_ids, start, k, v):
    """Rows k (already rotated and rounded), v [n, T, layers, Hkv, d] at positions start[i] + s.  Returns the entries served."""
    n, T, layers = k.shape[:3]
    served = []
    for i in range(n):
        t, st = int(trace_ids[i]), int(start[i])
        if st < 0:
            continue
        if t < 0 or t >= pool.max_traces or not pool.live[t]:
            pool._flag(KP.ERR_BAD_TRACE)
            continue
        if st + T > pool.seq_lens[t]:
            pool._flag(KP.ERR_INVALID_ARG)
            continue
        served.append(i)
        for s in range(T):
            b, slot = int(pool.block_table[t, (st + s) // pool.P]), (st + s) % pool.P
            pool.k_pages[layer0:layer0 + layers, b, :, slot] = k[i, s]
            pool.v_pages[layer0:layer0 + layers, b, :, slot] = v[i, s]
    return served
