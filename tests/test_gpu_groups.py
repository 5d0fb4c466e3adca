"""decode_attention_groups against the oracle."""
import os

import numpy as np
import pytest
import torch

from oracle import attention as OA
from oracle import rotary as OR
from paper_2601_09093_b200 import binding as B
from paper_2601_09093_b200 import harness as H
from paper_2601_09093_b200 import workloads as W

from draft_common import BF16_HALF_STEP, config, draw, poison_unused, relative_bound, trace_kv
from gpu_common import Twin, exact_f32

pytestmark = pytest.mark.gpu


def build(cfg, problems, ended=(), spare=16, max_pages=None):
    """problems: [(prompt length, [own lengths])].  Returns the pools and the groups (first rows, shared pages)."""
    P = cfg.page_size
    own = [o for _, os in problems for o in os]
    n = len(own)
    most = max(p + max(os) for p, os in problems)
    blocks = sum(p // P + sum(-(-(p % P + o) // P) + 1 for o in os) for p, os in problems) + spare
    tw = Twin(cfg, blocks, max_pages or -(-most // P) + 2, n, shuffle=True)
    for p, os in problems:
        tw.fork(len(os), p)
    for sel, inc in H.ragged_append_plan(np.asarray(own)):
        assert all(tw.append([int(i) for i in sel], inc))
    if len(ended):
        tw.gpu.release_traces(torch.tensor(list(ended), dtype=torch.int32, device="cuda"))
        for t in sorted(ended):
            tw.ora.release_trace(t)
    rows = np.cumsum([0] + [len(os) for _, os in problems])
    return tw, rows.astype(np.int32), np.array([p // P for p, _ in problems], dtype=np.int32)


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


def check(tw, layer, got, qx, lens=None, tables=None):
    """Bound per element as for decode_attention_tree: probabilities that may be rounded to bf16 on their way into the second
    product (bf16 pools), fp32 errors of the probabilities, one rounding of the output."""
    cfg, o = tw.cfg, tw.ora
    G = cfg.num_q_heads // cfg.num_kv_heads
    half = BF16_HALF_STEP if cfg.dtype == "bf16" else 0.0
    for t in range(len(qx)):
        S = int((o.seq_lens if lens is None else lens)[t])
        if S == 0:
            assert np.all(got[t] == 0), t
            continue
        K, V = OA.gather_trace_kv(o.k_pages[layer], o.v_pages[layer], (o.block_table if tables is None else tables)[t], S)
        for h in range(cfg.num_kv_heads):
            q = qx[t, h * G:(h + 1) * G]
            p = OA.softmax_weights(q @ K[:, h].T / np.sqrt(cfg.head_dim))
            want, mag = p @ V[:, h], p @ np.abs(V[:, h])
            tol = (half + relative_bound(q, K[:, h])) * mag
            tol = tol + half * (np.abs(want) + tol) + 1e-30
            err = np.abs(got[t, h * G:(h + 1) * G] - want)
            assert np.all(err <= tol), (t, h, float((err / tol).max()))


def run(tw, rows, pages, layer=0, sub=5, poison=True, status=(0, 0), **kw):
    cfg, n = tw.cfg, len(tw.ora.seq_lens)
    if poison:
        poison_unused(tw)
    q, qx = draw(cfg, W.TID_Q, (n, cfg.num_q_heads, cfg.head_dim), sub)
    v = tw.gpu.views()
    out = tw.gpu.decode_attention_groups(layer, q, v["block_table"], v["seq_lens"], dev(rows), dev(pages), **kw)
    assert out.dtype == tw.gpu.torch_dtype
    check(tw, layer, exact_f32(out), qx)
    assert tw.gpu.last_error() == status
    return out


HEADS = [((8, 2, 128), "bf16", 16), ((8, 1, 128), "bf16", 16), ((5, 1, 128), "bf16", 16), ((16, 1, 128), "bf16", 16), ((2, 2, 128), "bf16", 16),
         ((4, 1, 64), "fp32", 16), ((8, 2, 64), "bf16", 16), ((4, 2, 12), "fp32", 5)]


@pytest.mark.parametrize("heads,dtype,page", HEADS)
@pytest.mark.parametrize("prompts", [(0, 5), (16, 100), (128, 129), (127, 1000), (1025, 2051)])
def test_forks_of_several_prompts(heads, dtype, page, prompts):
    rng = np.random.default_rng(prompts[1])
    cfg = config(heads, dtype, page=page, n=12)
    tw, rows, pages = build(cfg, [(prompts[0], rng.integers(0, 40, 5)), (prompts[1], [0, 1, 15, 16, 17, 300]), (33, [3])])
    run(tw, rows, pages, layer=1)


@pytest.mark.parametrize("heads", [(8, 2, 128), (5, 1, 128), (16, 1, 128), (8, 1, 128), (4, 4, 128)])
@pytest.mark.parametrize("per", [2, 9, 31, 33, 64, 65, 130])
def test_groups_around_a_tile_of_rows(heads, per):
    """Row blocks of one lane, of two, and several of them; the last of one lane or two."""
    rng = np.random.default_rng(per)
    cfg = config(heads, "bf16", n=per + 3, layers=1)
    tw, rows, pages = build(cfg, [(450, rng.integers(0, 35, per)), (200, [7, 0, 40])])
    run(tw, rows, pages)


def test_ended_and_short_rows():
    """Ended traces in a group's first place and elsewhere, a group with one trace left, one with none."""
    cfg = config((8, 2, 128), "bf16", n=14, layers=1)
    problems = [(300, [5, 0, 70, 31, 2]), (170, [1, 2, 3]), (96, [4, 4]), (64, [0, 0, 18, 1])]
    tw, rows, pages = build(cfg, problems, ended=[0, 3, 5, 7, 8, 9, 13])
    run(tw, rows, pages)
    # lengths of the call's own: rows shorter than what their group shares, down to one position, read their own tables
    v, o = tw.gpu.views(), tw.ora
    q, qx = draw(cfg, W.TID_Q, (14, 8, 128), 6)
    lens = o.seq_lens.copy()
    lens[1], lens[2], lens[4], lens[10] = 1, 287, 288, 63
    out = tw.gpu.decode_attention_groups(0, q, v["block_table"], dev(lens), dev(rows), dev(pages))
    check(tw, 0, exact_f32(out), qx, lens=lens)
    assert tw.gpu.last_error() == (0, 0)


def test_rows_of_no_group_and_empty_groups():
    cfg = config((8, 2, 128), "bf16", n=9, layers=1)
    tw, _, _ = build(cfg, [(100, [3, 50, 7]), (260, [1, 2, 3, 4, 5, 6])])
    same = [run(tw, [3, 3, 9, 9], [4, 16, 2], poison=False), run(tw, [0, 3, 9], [6, 16], poison=False), run(tw, [4, 8], [10], poison=False),
            run(tw, [9, 9], [1], poison=False), run(tw, [0], [], poison=False), run(tw, [0, 3, 9], [0, 0], poison=False)]
    v = tw.gpu.views()
    q, _ = draw(cfg, W.TID_Q, (9, 8, 128), 5)
    none = tw.gpu.decode_attention_groups(0, q, v["block_table"], v["seq_lens"], None, None)
    assert torch.equal(none, same[4]) and torch.equal(none, same[3]) and torch.equal(none, same[5])


@pytest.mark.parametrize("heads,dtype", [((8, 2, 128), "bf16"), ((4, 1, 64), "fp32")])
def test_a_description_out_of_order_is_flagged_and_not_followed(heads, dtype):
    cfg = config(heads, dtype, n=8, layers=1)
    tw, rows, pages = build(cfg, [(100, [3, 50, 7]), (260, [1, 2, 3, 4, 5])])
    plain = run(tw, [0], [], poison=False)
    for r, p in (([0, 3, 9], [6, 16]), ([-1, 3, 8], [6, 16]), ([3, 0, 8], [6, 16]), ([0, 3, 8], [6, -1]), ([0, 3, 8], [6, 1 << 20]),
                 ([0, 8, 4], [6, 6]), ([1 << 30, 1 << 30, 1 << 30], [1, 1])):
        assert torch.equal(run(tw, r, p, poison=False, status=(1, 1 << 1)), plain)


def test_the_shared_pages_are_read_through_the_first_row_that_is_long_enough():
    """Rows whose tables hold something else there (out of range even) get the same result."""
    cfg = config((8, 2, 128), "bf16", n=5, layers=1)
    tw, rows, pages = build(cfg, [(400, [9, 20, 0, 33, 2])], ended=[0])
    want = run(tw, rows, pages)
    v = tw.gpu.views()
    table = v["block_table"].clone()
    table[2:, :25] = 1 << 30
    q, _ = draw(cfg, W.TID_Q, (5, 8, 128), 5)
    assert torch.equal(tw.gpu.decode_attention_groups(0, q, table, v["seq_lens"], dev(rows), dev(pages)), want)
    assert tw.gpu.last_error() == (0, 0)
    table[1, 3] = -1
    tw.gpu.decode_attention_groups(0, q, table, v["seq_lens"], dev(rows), dev(pages))
    assert tw.gpu.last_error() == (7, 1 << 7)
    table[1, 3], table[4, 25] = v["block_table"][1, 3], 1 << 30
    tw.gpu.decode_attention_groups(0, q, table, v["seq_lens"], dev(rows), dev(pages))
    assert tw.gpu.last_error() == (7, 1 << 7)


def test_many_groups_of_few_rows():
    rng = np.random.default_rng(3)
    cfg = config((4, 2, 128), "bf16", n=200, layers=1)
    tw, rows, pages = build(cfg, [(int(rng.integers(0, 70)), rng.integers(0, 30, 2)) for _ in range(100)], ended=[3, 8, 9])
    run(tw, rows, pages)


def test_many_pieces_of_one_tile_one_after_another():
    """Sequences of shared pages that are a tile long: of the two chains of such a piece one has nothing to do, and runs ahead of
    the other or falls behind it by whole pieces."""
    rng = np.random.default_rng(7)
    cfg = config((24, 8, 128), "bf16", n=150, layers=1)
    tw, rows, pages = build(cfg, [(int(rng.integers(16, 260)), rng.integers(0, 120, 2 + k % 2)) for k in range(60)])
    want = run(tw, rows, pages, poison=False)
    q, _ = draw(cfg, W.TID_Q, (150, 24, 128), 5)
    v, r, p = tw.gpu.views(), dev(rows), dev(pages)
    outs = [tw.gpu.decode_attention_groups(0, q, v["block_table"], v["seq_lens"], r, p) for _ in range(3000)]
    assert tw.gpu.last_error() == (0, 0)
    assert all(torch.equal(o, want) for o in outs)


def test_long_prompts_and_long_own_texts_are_cut_in_many_pieces():
    rng = np.random.default_rng(4)
    cfg = config((8, 2, 128), "bf16", n=40, layers=1)
    tw, rows, pages = build(cfg, [(5000, rng.integers(0, 900, 33)), (1500, [4000, 1, 0, 20, 5, 6, 700])])
    run(tw, rows, pages, poison=False)


@pytest.mark.parametrize("n", [2048, 2049])
def test_at_and_beyond_the_tensor_core_kernels_trace_limit(n):
    cfg = config((2, 1, 128), "bf16", n=n, layers=1)
    own = np.random.default_rng(n).integers(0, 20, size=n)
    tw, rows, pages = build(cfg, [(40, own[:1000]), (5, own[1000:1003]), (16, own[1003:])])
    run(tw, rows, pages, poison=False)


def test_what_is_not_finite_in_a_shared_page_reaches_the_rows_that_share_it_and_no_other():
    cfg = config((8, 2, 128), "bf16", n=7, layers=1)
    tw, rows, pages = build(cfg, [(64, [5, 0, 9]), (80, [1, 2, 3, 30])])
    q, qx = draw(cfg, W.TID_Q, (7, 8, 128), 5)
    v = tw.gpu.views()
    args = (v["block_table"], v["seq_lens"], dev(rows), dev(pages))
    clean = tw.gpu.decode_attention_groups(0, q, *args)
    # v of position 20 of the second prompt: infinity in one dim; of the last own position of row 1 (none) and row 2: NaN
    kv = tw.gpu.kv_storage.view(torch.bfloat16).view(1, -1, 2, 2, 16, 128)
    page = int(v["block_table"][4, 1])
    spot = kv[0, page, 1, 1, 4]
    spot[0] = float("inf")
    dims = [int(i) for i in torch.isinf(tw.gpu.read_kv(0, 1, v["block_table"][4], 81)[1][20]).nonzero()[:, 0]]
    assert len(dims) == 1
    got = tw.gpu.decode_attention_groups(0, q, *args)
    hit = torch.zeros_like(got, dtype=torch.bool)
    hit[3:, 4:, dims[0]] = True
    assert torch.isinf(got[hit]).all() and torch.equal(got[~hit], clean[~hit])
    page = int(v["block_table"][2, 4])
    kv[0, page, 0, 1, 8] = float("nan")                                  # the last of row 2's own nine
    kv[0, page, 0, 1, 9:] = float("nan")                                 # and what stands behind it
    again = tw.gpu.decode_attention_groups(0, q, *args)
    assert torch.isnan(again[2, :4]).all()
    again[2, :4] = got[2, :4]
    assert torch.equal(again, got)


def test_same_bits_every_time_and_under_a_graph_on_another_stream():
    rng = np.random.default_rng(5)
    cfg = config((8, 2, 128), "bf16", n=45, layers=2)
    tw, rows, pages = build(cfg, [(3000, rng.integers(0, 200, 40)), (500, [1, 2, 3, 400, 5])])
    first = run(tw, rows, pages, layer=1)
    assert torch.equal(first, run(tw, rows, pages, layer=1, poison=False))
    q, _ = draw(cfg, W.TID_Q, (45, 8, 128), 5)
    v, r, p = tw.gpu.views(), dev(rows), dev(pages)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(first)
    tw.gpu.decode_attention_groups(1, q, v["block_table"], v["seq_lens"], r, p, out=out, stream=s)
    s.synchronize()
    assert torch.equal(out, first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        tw.gpu.decode_attention_groups(1, q, v["block_table"], v["seq_lens"], r, p, out=out)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)


def test_two_pools_at_once_on_streams_of_their_own():
    pairs = []
    for seed in (1, 2):
        cfg = config((8, 2, 128), "bf16", n=20, layers=1, seed=seed)
        tw, rows, pages = build(cfg, [(2000, np.random.default_rng(seed).integers(0, 300, 20))])
        want = run(tw, rows, pages, poison=False)
        q, _ = draw(cfg, W.TID_Q, (20, 8, 128), 5)
        pairs.append((tw, dev(rows), dev(pages), want, q, torch.cuda.Stream()))
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(20):
        for i, (tw, r, p, want, q, s) in enumerate(pairs):
            v = tw.gpu.views()
            outs[i].append(tw.gpu.decode_attention_groups(0, q, v["block_table"], v["seq_lens"], r, p, stream=s))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, pairs[i][3]) for o in outs[i])


@pytest.mark.parametrize("heads", [(3, 1, 128), (6, 1, 128), (14, 2, 128), (12, 1, 128), (8, 8, 128)])
def test_other_numbers_of_heads_for_a_kv_head(heads):
    """Tiles of query rows that the heads of a group do not fill."""
    cfg = config(heads, "bf16", n=47, layers=1)
    tw, rows, pages = build(cfg, [(333, np.random.default_rng(1).integers(0, 40, 44)), (90, [1, 20, 0])])
    run(tw, rows, pages)


def test_two_calls_on_one_pool_at_once():
    """Layers of one pool, each call on a stream and with a workspace of its own."""
    cfg = config((8, 2, 128), "bf16", n=24, layers=2)
    tw, rows, pages = build(cfg, [(1500, np.random.default_rng(2).integers(0, 300, 20)), (64, [5, 6, 7, 200])])
    want = [run(tw, rows, pages, layer=l, poison=False) for l in range(2)]
    q, _ = draw(cfg, W.TID_Q, (24, 8, 128), 5)
    v, r, p = tw.gpu.views(), dev(rows), dev(pages)
    streams = [torch.cuda.Stream() for _ in range(2)]
    spaces = [torch.empty(96 << 20, dtype=torch.uint8, device="cuda") for _ in range(2)]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(20):
        for l in range(2):
            outs[l].append(tw.gpu.decode_attention_groups(l, q, v["block_table"], v["seq_lens"], r, p, workspace=spaces[l], stream=streams[l]))
    torch.cuda.synchronize()
    for l in range(2):
        assert all(torch.equal(o, want[l]) for o in outs[l])


@pytest.mark.parametrize("heads,dtype", [((8, 2, 128), "bf16"), ((4, 1, 64), "fp32")])
def test_a_length_beyond_the_table_is_cut_and_flagged(heads, dtype):
    cfg = config(heads, dtype, n=3, layers=1)
    tw, rows, pages = build(cfg, [(32, [100, 60, 12])], max_pages=9)
    v = tw.gpu.views()
    q, qx = draw(cfg, W.TID_Q, (3, cfg.num_q_heads, cfg.head_dim), 5)
    lens = tw.ora.seq_lens.copy()
    lens[2] = -5
    over = lens.copy()
    over[0] = 1 << 30
    table = v["block_table"].clone()
    table[0, 8:] = table[0, 8].clone()                                    # trace 0 has 132 positions; the table holds 144
    out = tw.gpu.decode_attention_groups(0, q, table, dev(over), dev(rows), dev(pages))
    assert tw.gpu.last_error() == (4, 1 << 4)
    lens[0] = 144
    plain = tw.gpu.decode_attention_groups(0, q, table, dev(lens), None, None)
    assert tw.gpu.last_error() == (0, 0)
    assert torch.isfinite(out).all() and (out[2] == 0).all() and (plain[2] == 0).all()
    # the same positions, summed in pieces of another number: fp32 errors, one rounding each of probabilities and output
    half = BF16_HALF_STEP if dtype == "bf16" else 2.0 ** -24
    assert (out - plain).abs().max().item() <= 4 * half * 6 + 1e-4 * (dtype == "fp32")


def test_a_table_too_wide_for_32_bit_positions():
    Hkv, d, pages = 64, 128, 1 << 25
    pool = B.KVPool(1, Hkv, Hkv, d, 16, num_blocks=12, max_traces=1, max_pages_per_trace=pages)
    gen = torch.Generator(device="cuda").manual_seed(3)
    k, v, q = (torch.randn(s, generator=gen, device="cuda").bfloat16() for s in ((1, 50, 1, Hkv, d), (1, 50, 1, Hkv, d), (1, Hkv, d)))
    pool.fork_prefix(1, 0, None, None)
    pool.append_kv(torch.zeros(1, dtype=torch.int32, device="cuda"), 50, k, v)
    w = pool.views()
    out = pool.decode_attention_groups(0, q, w["block_table"], w["seq_lens"], None, None).double()
    p = (torch.einsum("nhd,nshd->nhs", q.double(), k[:, :, 0].double()) / d ** 0.5).softmax(-1)
    # fp32 arithmetic, one rounding of the output; values below 6
    assert (out - torch.einsum("nhs,nshd->nhd", p, v[:, :, 0].double())).abs().max().item() <= 2 * BF16_HALF_STEP * 6
    assert pool.last_error() == (0, 0)


def test_a_captured_decode_step_replayed_over_growing_traces():
    """extend, store and attend of two layers in one graph: lengths, shares and pieces are another at every replay."""
    outs = []
    for graphed in (False, True):
        cfg = config((8, 2, 128), "bf16", n=10, layers=2)
        tw, rows, pages = build(cfg, [(200, [14, 15, 0, 30, 100]), (48, [0, 1, 2, 15, 31])], spare=64, max_pages=30)
        g, v, r = tw.gpu, tw.gpu.views(), B.Rotary(128)
        kd, _ = draw(cfg, W.TID_KNEW, (10, 1, 2, 2, 128), 9)
        vd, _ = draw(cfg, W.TID_VNEW, (10, 1, 2, 2, 128), 9)
        qd, _ = draw(cfg, W.TID_Q, (2, 10, 1, 8, 128), 9)
        ids, start = torch.arange(10, dtype=torch.int32, device="cuda"), torch.empty(10, dtype=torch.int32, device="cuda")
        qo, out, gr, gp = torch.empty_like(qd), torch.empty((2, 10, 8, 128), dtype=torch.bfloat16, device="cuda"), dev(rows), dev(pages)

        def step():
            g.extend(ids, 1, start_out=start)
            for l in range(2):
                g.store_kv_rotated(l, ids, start, kd[:, :, l:l + 1], vd[:, :, l:l + 1], r, q=qd[l:l + 1], q_out=qo[l:l + 1])
                g.decode_attention_groups(l, qo[l, :, 0], v["block_table"], v["seq_lens"], gr, gp, out=out[l])

        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        got = []
        with torch.cuda.stream(s):
            graph = torch.cuda.CUDAGraph()
            if graphed:
                with torch.cuda.graph(graph, stream=s):
                    step()
            for _ in range(20):
                graph.replay() if graphed else step()
                got.append(out.clone())
        s.synchronize()
        assert g.last_error() == (0, 0)
        assert v["seq_lens"].tolist() == [int(x) + 20 for x in tw.ora.seq_lens]
        outs.append(got)
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("heads", [(8, 2, 128), (16, 2, 128)])
def test_a_wait_that_runs_out_is_flagged_and_leaves_nothing_behind(heads):
    """A limit of zero takes whatever has not landed at the first look for lost (healthy copies, which land a microsecond
    later).  Between such calls, on the same pool and without a reset, results are as ever."""
    cfg = config(heads, "bf16", n=40, layers=1)
    tw, rows, pages = build(cfg, [(3000, np.random.default_rng(6).integers(0, 300, 38)), (500, [9, 1])])
    first = run(tw, rows, pages)
    q, _ = draw(cfg, W.TID_Q, (40, cfg.num_q_heads, 128), 5)
    v, r, p = tw.gpu.views(), dev(rows), dev(pages)

    def call():
        return tw.gpu.decode_attention_groups(0, q, v["block_table"], v["seq_lens"], r, p)

    for limit in (0, 1, 500, 5_000, 0):
        tw.gpu.set_wait_limit_ns(limit)
        for _ in range(8):
            out = call()
        torch.cuda.synchronize()
        code, mask = tw.gpu.last_error()
        assert mask == 1 << 6 if limit == 0 else mask in (0, 1 << 6), (limit, mask)      # STEP_ERR_TIMEOUT
        if mask == 0:
            assert torch.equal(out, first), limit
        tw.gpu.set_wait_limit_ns(2_000_000_000)
        assert torch.equal(call(), first), limit
        assert tw.gpu.last_error() == (0, 0)


def test_the_general_kernel_gives_the_same_within_the_same_bounds():
    cfg = config((8, 2, 128), "bf16", n=9, layers=1)
    tw, rows, pages = build(cfg, [(100, [3, 50, 7]), (260, [1, 2, 3, 4, 5, 6])])
    tw.gpu.set_attention_config(fast_path=-1)
    run(tw, rows, pages)
    tw.gpu.set_attention_config(fast_path=1)
    run(tw, rows, pages, poison=False)


def test_a_pool_beyond_32_bit_offsets():
    Hq, Hkv, d, P, n, prompt = 4, 2, 128, 16, 3, 150
    blocks = 2_500_000_000 // (Hkv * 2 * P * d)
    pool = B.KVPool(1, Hq, Hkv, d, P, num_blocks=blocks, max_traces=n, max_pages_per_trace=16)
    v = pool.views()
    v["free_list"].copy_(torch.arange(blocks, dtype=torch.int32, device="cuda"))        # pops from the end: the highest first
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda").bfloat16()     # noqa: E731
    kp, vp, k, w, q = rand(1, Hkv, prompt, d), rand(1, Hkv, prompt, d), rand(n, 30, 1, Hkv, d), rand(n, 30, 1, Hkv, d), rand(n, Hq, d)
    pool.fork_prefix(n, prompt, kp, vp)
    pool.append_kv(torch.arange(n, dtype=torch.int32, device="cuda"), 30, k, w)
    assert int(v["block_table"][:, 0].min()) > blocks - 32
    out = pool.decode_attention_groups(0, q, v["block_table"], v["seq_lens"], dev([0, 3]), dev([prompt // P])).double()
    kk = torch.cat((kp[0].transpose(0, 1).expand(n, -1, -1, -1), k[:, :, 0]), 1).double().repeat_interleave(2, 2)
    vv = torch.cat((vp[0].transpose(0, 1).expand(n, -1, -1, -1), w[:, :, 0]), 1).double().repeat_interleave(2, 2)
    p = (torch.einsum("nhd,nshd->nhs", q.double(), kk) / d ** 0.5).softmax(-1)
    # probabilities rounded to bf16, one rounding of the output; values below 6
    assert (out - torch.einsum("nhs,nshd->nhd", p, vv)).abs().max().item() <= 2 * BF16_HALF_STEP * 6
    assert pool.last_error() == (0, 0)


def test_a_decode_step_layer_by_layer():
    """What the calls are for: room for a token, then for every layer its rotated key and query and the attention to what the
    layer's cache now holds - against the oracle on rows rotated by the oracle, two steps in a row."""
    cfg = config((8, 2, 128), "bf16", n=9, layers=3)
    tw, rows, pages = build(cfg, [(100, [3, 15, 7]), (260, [1, 2, 3, 4, 5, 12])])
    r, f = B.Rotary(128, 500000.0), OR.frequencies(128, 500000.0)
    n, g = 9, tw.gpu
    ids, v = torch.arange(n, dtype=torch.int32, device="cuda"), tw.gpu.views()
    for step in range(2):
        start = g.extend(ids, 1)
        at = OR.extend(tw.ora, range(n), 1)
        for l in (0, 1, 2):
            sub = 100 + 10 * step + l
            kd, kx = draw(cfg, W.TID_KNEW, (n, 1, 1, 2, 128), sub)
            vd, vx = draw(cfg, W.TID_VNEW, (n, 1, 1, 2, 128), sub)
            qd, qx = draw(cfg, W.TID_Q, (1, n, 1, 8, 128), sub)
            qo = g.store_kv_rotated(l, ids, start, kd, vd, r, q=qd)
            out = g.decode_attention_groups(l, qo[0, :, 0], v["block_table"], v["seq_lens"], dev(rows), dev(pages))
            # the rotation is tested by itself: here the rows that went in, to a step of bf16, then exactly as stored
            want = OR.rotate(kx[:, :, 0], at[:, None], f, False)
            stored = np.stack([np.stack([exact_f32(g.read_kv(l, h, v["block_table"][t], int(at[t]) + 1)[0][-1]) for h in range(2)]) for t in range(n)])[:, None]
            assert np.all(np.abs(stored - want) <= 2 * BF16_HALF_STEP * np.abs(want) + 1e-5)
            OR.store(tw.ora, l, range(n), at, stored[:, :, None], vx)
            check(tw, l, exact_f32(out), exact_f32(qo[0, :, 0]))
    tw.assert_meta_equal()
    assert g.last_error() == (0, 0)


FUZZ = int(os.environ.get("STEP_FUZZ_SEEDS", "40"))


@pytest.mark.parametrize("first", range(0, FUZZ, 20))
def test_random_groups_against_the_plain_call(first):
    """Heads, prompts, own texts, ended traces and declared pages at random, blocks shuffled, NaN wherever nothing is stored: what
    decode_attention makes of the same pool, twice the same bits."""
    for seed in range(first, min(FUZZ, first + 20)):
        rng = np.random.default_rng(9000 + seed)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        Hkv = int(rng.choice([1, 2, 3, 8]))
        Hq = Hkv * int(rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16]))
        d, P, dt = (128, 16, "bf16") if rng.random() < 0.8 else [(64, 16, "bf16"), (64, 8, "fp32"), (128, 32, "bf16")][rng.integers(3)]
        few = rng.random() < 0.8
        problems = [(int(rng.integers(0, 6000 if rng.random() < 0.2 else 400)), rng.choice([0, 1, 15, 16, 17, 90, 700 if rng.random() < 0.1 else 33],
                     int(rng.choice([1, 2, 4, 17, 33, 65]) if few else rng.integers(1, 4)))) for _ in range(int(rng.integers(1, 5)) if few else 60)]
        n, tdt = sum(len(o) for _, o in problems), torch.bfloat16 if dt == "bf16" else torch.float32
        blocks = sum(p // P + sum((p % P + int(x)) // P + 2 for x in o) for p, o in problems) + 8
        pool = B.KVPool(1, Hq, Hkv, d, P, num_blocks=blocks, max_traces=n, max_pages_per_trace=max(p + int(max(o)) for p, o in problems) // P + 1,
                        dtype=B.STEP_BF16 if dt == "bf16" else B.STEP_FP32)
        v = pool.views()
        v["free_list"].copy_(torch.from_numpy(rng.permutation(blocks).astype(np.int32)))
        pool.kv_storage.fill_(255)
        rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(tdt)          # noqa: E731
        for p, o in problems:
            pool.fork_prefix(len(o), p, rand(1, Hkv, p, d), rand(1, Hkv, p, d))
        for sel, inc in H.ragged_append_plan(np.concatenate([o for _, o in problems])):
            pool.append_kv(dev(sel), inc, rand(len(sel), inc, 1, Hkv, d), rand(len(sel), inc, 1, Hkv, d))
        ended = np.nonzero(rng.random(n) < rng.choice([0, 0.1, 0.5]))[0]
        if len(ended):
            pool.release_traces(dev(ended))
        pages = np.array([p // P if rng.random() < 0.8 else rng.integers(0, p // P + 1) for p, _ in problems])
        rows = dev(np.cumsum([0] + [len(o) for _, o in problems]))
        q = rand(n, Hq, d)
        got = [pool.decode_attention_groups(0, q, v["block_table"], v["seq_lens"], rows, dev(pages)) for _ in range(2)]
        plain = pool.decode_attention(0, q, v["block_table"], v["seq_lens"])
        # each side rounds its probabilities (bf16 pools), this one its output; values below 6.  fp32: sums in another order
        tol = 3 * BF16_HALF_STEP * 6 if dt == "bf16" else 2e-4
        assert pool.last_error() == (0, 0) and torch.equal(*got), seed
        assert (got[0].float() - plain).abs().max().item() <= tol, seed


def test_refusals():
    cfg = config((8, 2, 128), "bf16", n=4, layers=1)
    tw, rows, pages = build(cfg, [(40, [1, 2, 3, 4])])
    p, v = tw.gpu, tw.gpu.views()
    q = torch.zeros((4, 8, 128), dtype=torch.bfloat16, device="cuda")
    ok = dict(layer=0, q=q, block_table=v["block_table"], seq_lens=v["seq_lens"], group_rows=dev(rows), group_pages=dev(pages))
    p.decode_attention_groups(**ok)
    off = torch.zeros(q.numel() + 8, dtype=torch.bfloat16, device="cuda")
    for change in (dict(layer=1), dict(q=q.float()), dict(q=q.cpu()), dict(out=off[4:-4].view(q.shape)), dict(q=off[4:-4].view(q.shape)),
                   dict(workspace=torch.empty(1024, dtype=torch.uint8, device="cuda")), dict(group_pages=dev(pages).cpu())):
        with pytest.raises(B.StepError) as e:
            p.decode_attention_groups(**{**ok, **change})
        assert e.value.code == 1, change
    assert p.decode_attention_groups(0, q[:0], v["block_table"][:0], v["seq_lens"][:0], None, None).shape == (0, 8, 128)
    L = B.lib()
    assert L.decode_attention_groups(p.handle, 0, None, None, None, 4, None, None, 1, None, None, 0, None) == 1
    assert p.last_error() == (0, 0)
