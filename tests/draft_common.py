"""Error bounds and pool set-up shared by the tests of tree attention, weight-counting attention and position eviction."""
import math

import numpy as np
import torch

from oracle import attention as OA
from paper_2601_09093_b200 import harness as H
from paper_2601_09093_b200 import workloads as W
from gpu_common import Twin

BF16_HALF_STEP, FP32_HALF_STEP = 2.0 ** -8, 2.0 ** -24


def score_slack(q, k):
    """How far the natural logarithm of a softmax weight can be off when scores are made in fp32: a dot product of d terms
    (each addition may lose a whole step in the tensor cores' accumulators: 2 half steps), the scale and the base-2
    argument (three roundings of a value up to the largest score), the exponential (2 steps); q [.., d], k [S, d]."""
    d = q.shape[-1]
    size = float(np.max(np.abs(q) @ np.abs(k).T)) / math.sqrt(d) if len(k) else 0.0
    return 2 * (d + 3) * FP32_HALF_STEP * size + 8 * FP32_HALF_STEP


def relative_bound(q, k):
    """Bound on the relative error of a softmax weight: numerator and denominator are each off by the slack above, and
    the sums of S terms by S steps at most."""
    return 2 * score_slack(q, k) + 2 * (len(k) + 8) * 2 * FP32_HALF_STEP


def config(heads, dtype, page=16, layers=2, n=6, seed=77):
    Hq, Hkv, d = heads
    return W.scaled(W.C1, n_traces=n, num_layers=layers, num_q_heads=Hq, num_kv_heads=Hkv, head_dim=d, page_size=page,
                    dtype=dtype, seed=seed)


def twin(cfg, lens, prefix=0, spare=64, max_pages=None, num_blocks=None):
    """A CUDA pool and an oracle pool whose traces have the given lengths (at least `prefix`, the shared prompt), blocks
    handed out in shuffled order."""
    P = cfg.page_size
    lens = np.asarray(lens)
    pages = max_pages or int(-(-max(1, lens.max()) // P)) + 8
    blocks = num_blocks or int((-(-lens // P)).sum()) + len(lens) + spare
    tw = Twin(cfg, blocks, pages, len(lens), shuffle=True)
    ids, _ = tw.fork(len(lens), prefix)
    for sel, inc in H.ragged_append_plan(lens - prefix):
        assert all(tw.append([ids[i] for i in sel], inc))
    # whatever a block holds beyond a trace's positions must not matter: NaN patterns in every byte never written
    return tw


def poison_unused(tw):
    """NaN in every stored byte of the CUDA pool, then the same rows again: slots behind a trace's length hold NaN."""
    storage = tw.gpu.kv_storage
    keep = storage.clone()
    used = torch.zeros_like(storage)
    # a row of zeros cannot be told from an unwritten one, and needs not be: normal draws are never all zero
    flat = keep.view(-1, 16)
    used = (flat != 0).any(1)
    flat[~used] = 0xFF
    storage.copy_(flat.view(-1))


def draw(cfg, tid, shape, sub):
    b, x = W.normal(cfg.seed, tid, shape, cfg.dtype, sub=sub)
    return H.to_device(b, cfg.dtype), x.astype(np.float64)


def trace_kv(tw, layer, t):
    o = tw.ora
    return OA.gather_trace_kv(o.k_pages[layer], o.v_pages[layer], o.block_table[t], int(o.seq_lens[t]))
