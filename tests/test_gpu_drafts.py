"""decode_attention_tree and append_kv_path against the oracle."""
import numpy as np
import pytest
import torch

from oracle import drafts as OD
from paper_2601_09093_b200 import binding as B
from paper_2601_09093_b200 import workloads as W

from draft_common import BF16_HALF_STEP, config, draw, poison_unused, relative_bound, trace_kv, twin
from gpu_common import exact_f32

pytestmark = pytest.mark.gpu


def random_parents(rng, n, T, kind):
    if kind == "chain":
        p = np.arange(T) - 1
        return np.tile(p, (n, 1)).astype(np.int32)
    if kind == "star":
        return np.full((n, T), -1, dtype=np.int32)
    return np.stack([[rng.integers(max(-1, u - 6), u) for u in range(T)] for _ in range(n)]).astype(np.int32)


def check_tree(tw, layer, got, q, kd, vd, parents, nodes):
    """Bound per element: the probabilities may be rounded to bf16 on their way into the second product (bf16 pools),
    fp32 errors of the probabilities, one rounding of the output."""
    cfg = tw.cfg
    half = BF16_HALF_STEP if cfg.dtype == "bf16" else 0.0
    for t in range(q.shape[0]):
        K, V = trace_kv(tw, layer, t)
        want, mag = OD.tree_attention(q[t], K, V, kd[t, :, layer], vd[t, :, layer], parents[t], int(nodes[t]))
        keys = np.concatenate([K, kd[t, :, layer]])
        rel = max(relative_bound(q[t].reshape(-1, cfg.head_dim), keys[:, h]) for h in range(cfg.num_kv_heads))
        err = np.abs(got[t] - want)
        tol = (half + rel) * mag
        tol = tol + half * (np.abs(want) + tol) + 1e-30
        assert np.all(err <= tol), (t, float((err / tol).max()))
        assert np.all(got[t, int(nodes[t]):] == 0)


def run_tree(tw, layer, T, kind="random", nodes=None, seed=5, poison=True, **kw):
    cfg, n = tw.cfg, len(tw.ora.seq_lens)
    rng = np.random.default_rng(seed)
    if poison:
        poison_unused(tw)
    q, qx = draw(cfg, W.TID_Q, (n, T, cfg.num_q_heads, cfg.head_dim), seed)
    shape = (n, T, cfg.num_layers, cfg.num_kv_heads, cfg.head_dim)
    kd, kx = draw(cfg, W.TID_K, shape, seed)
    vd, vx = draw(cfg, W.TID_V, shape, seed)
    parents = random_parents(rng, n, T, kind)
    nodes_dev = None
    if nodes is None:
        nodes = np.full(n, T)
    else:
        nodes_dev = torch.from_numpy(np.asarray(nodes, dtype=np.int32)).cuda()
        for t in range(n):                              # what lies behind a tree's end is not looked at
            kd[t, nodes[t]:] = float("nan")
            vd[t, nodes[t]:] = float("nan")
            q[t, nodes[t]:] = float("nan")
            parents[t, nodes[t]:] = 99
    v = tw.gpu.views()
    out = tw.gpu.decode_attention_tree(layer, q, kd, vd, torch.from_numpy(parents).cuda(), v["block_table"][:n], v["seq_lens"][:n],
                                       n_nodes=nodes_dev, **kw)
    assert out.dtype == tw.gpu.torch_dtype
    check_tree(tw, layer, exact_f32(out), qx, kx, vx, parents, nodes)
    assert tw.gpu.last_error() == (0, 0)
    return out


LENS = [0, 1, 15, 16, 17, 127, 128, 129, 200, 384]


@pytest.mark.parametrize("T", [1, 2, 13, 33, 64])
@pytest.mark.parametrize("heads", [(8, 2, 128), (8, 1, 128), (5, 1, 128), (16, 1, 128), (2, 2, 128)])
def test_tree_bf16(heads, T):
    cfg = config(heads, "bf16", n=len(LENS))
    run_tree(twin(cfg, LENS), 1, T)


@pytest.mark.parametrize("heads,dtype,page", [((4, 1, 64), "fp32", 16), ((8, 2, 64), "bf16", 16), ((6, 2, 128), "bf16", 32),
                                              ((4, 2, 8), "bf16", 3), ((4, 2, 12), "fp32", 5), ((2, 1, 512), "fp32", 16),
                                              ((2, 1, 512), "bf16", 16), ((4, 2, 128), "fp32", 16)])
@pytest.mark.parametrize("T", [1, 7, 64])
def test_tree_other_pools(heads, dtype, page, T):
    cfg = config(heads, dtype, page=page, n=len(LENS))
    run_tree(twin(cfg, LENS), 1, T)


@pytest.mark.parametrize("kind", ["chain", "star"])
@pytest.mark.parametrize("heads,dtype", [((8, 2, 128), "bf16"), ((4, 1, 64), "fp32")])
def test_tree_shapes(kind, heads, dtype):
    run_tree(twin(config(heads, dtype, n=4), [3, 64, 100, 300]), 0, 24, kind)


@pytest.mark.parametrize("heads,dtype", [((8, 2, 128), "bf16"), ((64, 8, 128), "bf16"), ((4, 1, 64), "fp32")])
def test_ragged_trees_with_a_shared_prompt(heads, dtype):
    """Trees of different sizes, empty ones among them, over traces that share their prompt's pages."""
    lens = [70, 81, 128, 300, 257]
    run_tree(twin(config(heads, dtype, n=5, layers=1), lens, prefix=70), 0, 40, nodes=[0, 1, 40, 17, 39])


@pytest.mark.parametrize("heads,dtype", [((8, 2, 128), "bf16"), ((4, 1, 64), "fp32")])
def test_empty_everything(heads, dtype):
    run_tree(twin(config(heads, dtype, n=3), [0, 0, 5]), 0, 6, nodes=[0, 6, 0])


def test_long_cache_split_over_many_ctas():
    cfg = config((8, 1, 128), "bf16", layers=1, n=2)
    run_tree(twin(cfg, [20000, 9001]), 0, 5, poison=False)


def test_tree_of_one_is_decode_attention_after_append():
    """A draft of one token sees what decode_attention sees once that token is stored."""
    cfg = config((8, 2, 128), "bf16", n=5, layers=1)
    tw = twin(cfg, [0, 16, 31, 200, 300])
    q, _ = draw(cfg, W.TID_Q, (5, 1, 8, 128), 1)
    kd, _ = draw(cfg, W.TID_K, (5, 1, 1, 2, 128), 1)
    vd, _ = draw(cfg, W.TID_V, (5, 1, 1, 2, 128), 1)
    v = tw.gpu.views()
    ids = torch.arange(5, dtype=torch.int32, device="cuda")
    tree = tw.gpu.decode_attention_tree(0, q, kd, vd, torch.full((5, 1), -1, dtype=torch.int32, device="cuda"), v["block_table"], v["seq_lens"])
    tw.gpu.append_kv_path(ids, kd, vd, torch.zeros((5, 1), dtype=torch.int32, device="cuda"), torch.ones(5, dtype=torch.int32, device="cuda"))
    plain = tw.gpu.decode_attention(0, q[:, 0].contiguous(), v["block_table"], v["seq_lens"])
    # both round their probabilities to bf16 (one half step of at most max|v| each), the tree its output
    tol = 3 * BF16_HALF_STEP * 5.0
    assert (tree[:, 0].float() - plain).abs().max().item() <= tol
    assert v["seq_lens"].tolist() == [1, 17, 32, 201, 301]


def test_same_bits_every_time_and_under_a_graph_on_another_stream():
    cfg = config((8, 2, 128), "bf16", n=6, layers=1)
    tw = twin(cfg, [100, 2000, 31, 700, 1, 0])
    first = run_tree(tw, 0, 9, seed=3)
    again = run_tree(tw, 0, 9, seed=3, poison=False)
    assert torch.equal(first, again)
    n = 6
    q, _ = draw(cfg, W.TID_Q, (n, 9, 8, 128), 3)
    kd, _ = draw(cfg, W.TID_K, (n, 9, 1, 2, 128), 3)
    vd, _ = draw(cfg, W.TID_V, (n, 9, 1, 2, 128), 3)
    parents = torch.from_numpy(random_parents(np.random.default_rng(3), n, 9, "random")).cuda()
    v = tw.gpu.views()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(first)
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            tw.gpu.decode_attention_tree(0, q, kd, vd, parents, v["block_table"], v["seq_lens"], out=out)
        for _ in range(3):
            out.zero_()
            graph.replay()
    s.synchronize()
    assert torch.equal(out, first)


def test_a_bad_parent_counts_as_none_and_is_flagged():
    for heads, dtype in (((8, 2, 128), "bf16"), ((4, 1, 64), "fp32")):
        cfg = config(heads, dtype, n=2, layers=1)
        tw = twin(cfg, [20, 40])
        T, Hq, Hkv, d = 5, cfg.num_q_heads, cfg.num_kv_heads, cfg.head_dim
        q, qx = draw(cfg, W.TID_Q, (2, T, Hq, d), 1)
        kd, kx = draw(cfg, W.TID_K, (2, T, 1, Hkv, d), 1)
        vd, vx = draw(cfg, W.TID_V, (2, T, 1, Hkv, d), 1)
        parents = np.array([[-1, 0, 2, 1, 70], [-2, 0, 1, -1, 3]], dtype=np.int32)
        v = tw.gpu.views()
        out = tw.gpu.decode_attention_tree(0, q, kd, vd, torch.from_numpy(parents).cuda(), v["block_table"], v["seq_lens"])
        check_tree(tw, 0, exact_f32(out), qx, kx, vx, parents, [T, T])
        assert tw.gpu.last_error() == (1, 1 << 1)
        nodes = torch.tensor([6, -1], dtype=torch.int32, device="cuda")
        good = torch.from_numpy(np.array([[-1, 0, 1, 1, 2]] * 2, dtype=np.int32)).cuda()
        out = tw.gpu.decode_attention_tree(0, q, kd, vd, good, v["block_table"], v["seq_lens"], n_nodes=nodes)
        check_tree(tw, 0, exact_f32(out), qx, kx, vx, good.cpu().numpy(), [T, 0])
        assert tw.gpu.last_error() == (1, 1 << 1)


@pytest.mark.parametrize("heads,dtype,T", [((8, 2, 128), "bf16", 13), ((8, 1, 128), "bf16", 64), ((16, 1, 128), "bf16", 20),
                                           ((4, 1, 64), "fp32", 13), ((4, 2, 256), "bf16", 40)])
@pytest.mark.parametrize("many", [False, True])
def test_infinities_and_nan_reach_only_the_nodes_that_see_them(heads, dtype, T, many):
    """Also the padded batch without n_nodes: what stands in nodes that nobody continues stays there.  `many`: several short
    sequences for every CTA, where a few longer ones are cut in pieces."""
    lens = np.random.default_rng(8).integers(0, 40, 2600 // T) if many else LENS
    cfg = config(heads, dtype, layers=2, n=len(lens))
    tw = twin(cfg, lens)
    poison_unused(tw)
    n, layer = len(lens), 1
    q, qx = draw(cfg, W.TID_Q, (n, T, cfg.num_q_heads, cfg.head_dim), 3)
    shape = (n, T, cfg.num_layers, cfg.num_kv_heads, cfg.head_dim)
    kd, kx = draw(cfg, W.TID_K, shape, 3)
    vd, vx = draw(cfg, W.TID_V, shape, 3)
    parents = random_parents(np.random.default_rng(3), n, T, "random")
    odd = {1: (np.inf, 0), T // 2: (-np.inf, 5), T - 3: (np.nan, cfg.head_dim - 1)}          # node: value and dim of its v
    for u, (x, c) in odd.items():
        vd[:, u, :, :, c], vx[:, u, :, :, c] = x, x
    for x, dev in ((kx, kd), (vx, vd), (qx, q)):                                             # a node of padding
        x[:, T - 2], dev[:, T - 2] = np.nan, float("nan")
    parents[:, T - 1][parents[:, T - 1] == T - 2] = -1
    v = tw.gpu.views()
    got = exact_f32(tw.gpu.decode_attention_tree(layer, q, kd, vd, torch.from_numpy(parents).cuda(), v["block_table"], v["seq_lens"]))
    tame = np.where(np.isfinite(vx), vx, 0.0)
    for t in range(n):
        K, V = trace_kv(tw, layer, t)
        with np.errstate(invalid="ignore"):
            want, _ = OD.tree_attention(qx[t], K, V, kx[t, :, layer], vx[t, :, layer], parents[t], T)
        assert np.array_equal(np.isnan(got[t]), np.isnan(want)), t
        assert np.array_equal(got[t][np.isinf(want)], want[np.isinf(want)]), t
        assert not np.isinf(got[t][np.isfinite(want)]).any()
        # elsewhere the bound of finite values (the node of padding aside: it is NaN throughout)
        live = np.arange(T) != T - 2
        fin, mag = OD.tree_attention(np.nan_to_num(qx[t]), K, V, np.nan_to_num(kx[t, :, layer]), tame[t, :, layer], parents[t], T)
        keys = np.concatenate([K, np.nan_to_num(kx[t, :, layer])])
        rel = max(relative_bound(qx[t][live].reshape(-1, cfg.head_dim), keys[:, h]) for h in range(cfg.num_kv_heads))
        half = BF16_HALF_STEP if dtype == "bf16" else 0.0
        tol = (half + rel) * mag
        tol = tol + half * (np.abs(fin) + tol) + 1e-30
        ok = live[:, None, None] & np.isfinite(want)
        assert np.all(np.abs(got[t] - fin)[ok] <= tol[ok]), t
        assert np.isnan(got[t][~live]).all()
    assert tw.gpu.last_error() == (0, 0)


def test_a_bad_block_is_flagged():
    for heads, dtype in (((8, 2, 128), "bf16"), ((4, 1, 64), "fp32")):
        cfg = config(heads, dtype, n=2, layers=1)
        tw = twin(cfg, [20, 400])
        T, Hq, Hkv, d = 3, cfg.num_q_heads, cfg.num_kv_heads, cfg.head_dim
        q, kd, vd = (torch.ones(s, dtype=tw.gpu.torch_dtype, device="cuda") for s in ((2, T, Hq, d), (2, T, 1, Hkv, d), (2, T, 1, Hkv, d)))
        v = tw.gpu.views()
        table = v["block_table"].clone()
        table[1, 3], table[0, 1] = 1 << 30, -7
        tw.gpu.decode_attention_tree(0, q, kd, vd, torch.full((2, T), -1, dtype=torch.int32, device="cuda"), table, v["seq_lens"])
        assert tw.gpu.last_error() == (7, 1 << 7)


def test_the_general_kernel_gives_the_same_within_the_same_bounds():
    cfg = config((8, 2, 128), "bf16", n=len(LENS))
    tw = twin(cfg, LENS)
    tw.gpu.set_attention_config(fast_path=-1)
    run_tree(tw, 1, 9)
    tw.gpu.set_attention_config(fast_path=1)
    run_tree(tw, 1, 9, poison=False)


@pytest.mark.parametrize("n", [2048, 2049])
def test_at_and_beyond_the_tensor_core_kernels_trace_limit(n):
    lens = np.random.default_rng(n).integers(0, 20, size=n)
    cfg = config((2, 1, 128), "bf16", n=n, layers=1)
    run_tree(twin(cfg, lens, max_pages=3), 0, 2, poison=False)


def test_a_pool_beyond_32_bit_offsets():
    """Blocks at the far end of a pool of 2.5e9 elements: tree attention, path append, counting attention and eviction
    against plain fp64 arithmetic on the rows that went in."""
    Hq, Hkv, d, P, n, S, T = 4, 2, 128, 16, 2, 83, 3
    blocks = 2_500_000_000 // (Hkv * 2 * P * d)
    pool = B.KVPool(1, Hq, Hkv, d, P, num_blocks=blocks, max_traces=n, max_pages_per_trace=8)
    v = pool.views()
    v["free_list"].copy_(torch.arange(blocks, dtype=torch.int32, device="cuda"))        # pops from the end: the highest first
    gen = torch.Generator(device="cuda").manual_seed(1)
    draw_ = lambda *shape: torch.randn(shape, generator=gen, device="cuda").bfloat16()   # noqa: E731
    pool.fork_prefix(n, 0, None, None)
    ids = torch.arange(n, dtype=torch.int32, device="cuda")
    k, w, kd, vd, q = draw_(n, S, 1, Hkv, d), draw_(n, S, 1, Hkv, d), draw_(n, T, 1, Hkv, d), draw_(n, T, 1, Hkv, d), draw_(n, T, Hq, d)
    pool.append_kv(ids, S, k, w)
    assert int(v["block_table"][:, 0].min()) > blocks - 16
    parents = torch.tensor([[-1, 0, 0]] * n, dtype=torch.int32, device="cuda")
    out = pool.decode_attention_tree(0, q, kd, vd, parents, v["block_table"], v["seq_lens"]).double()
    see = torch.tensor([[1, 0, 0], [1, 1, 0], [1, 0, 1]], device="cuda").bool()

    def attend(q, k, v, mask=None):                      # q [n, T, Hq, d]; k, v [n, S, Hkv, d]
        a = torch.einsum("nthd,nshd->nths", q.double(), k.double().repeat_interleave(2, 2)) / d ** 0.5
        if mask is not None:
            a = a.masked_fill(~mask[None, :, None], -torch.inf)
        p = a.softmax(-1)
        return torch.einsum("nths,nshd->nthd", p, v.double().repeat_interleave(2, 2)), p

    kk, vv = torch.cat((k, kd), 1)[:, :, 0], torch.cat((w, vd), 1)[:, :, 0]
    want, p = attend(q, kk, vv, torch.cat((torch.ones((T, S), device="cuda").bool(), see), 1))
    # probabilities rounded to bf16, fp32 sums of scores below 8, one rounding of the output; values below 6
    assert (out - want).abs().max().item() <= 2 * BF16_HALF_STEP * 6
    path = torch.tensor([[0, 2], [1, 0]], dtype=torch.int32, device="cuda")
    pool.append_kv_path(ids, kd, vd, path, torch.tensor([2, 1], dtype=torch.int32, device="cuda"))
    sums = torch.zeros((n, Hkv, S + 2), device="cuda")
    one = q[:, :1]
    out = pool.decode_attention_weights(0, one[:, 0].contiguous(), v["block_table"], v["seq_lens"], sums)
    for t, rows in ((0, [0, 2]), (1, [1])):
        kk, vv = torch.cat((k[t], kd[t, rows]))[None, :, 0], torch.cat((w[t], vd[t, rows]))[None, :, 0]
        want, p = attend(one[t:t + 1], kk, vv)
        rel = max(relative_bound(exact_f32(one[t, 0, 2 * h:2 * h + 2]), exact_f32(kk[0, :, h])) for h in range(Hkv))
        assert (out[t] - want[0, 0]).abs().max().item() <= rel * 6                   # sums of values below 6, weighted by 1 in all
        weights = p[0, 0].view(Hkv, 2, -1).sum(1)
        assert ((sums[t, :, :kk.shape[1]] - weights).abs() <= (rel + 2.0 ** -22) * weights).all()
    kept = pool.evict_positions(ids, sums[None].contiguous(), 40, 7)[0].long()
    for t, rows in ((0, [0, 2]), (1, [1])):
        whole = torch.cat((k[t], kd[t, rows]))[:, 0]
        for h in range(Hkv):
            got, _ = pool.read_kv(0, h, v["block_table"][t], 40)
            assert torch.equal(got, whole[kept[t, h], h])
    assert pool.last_error() == (0, 0)


@pytest.mark.parametrize("heads,T", [((8, 2, 128), 9), ((8, 1, 128), 64), ((2, 2, 128), 1)])
def test_a_wait_that_runs_out_is_flagged_and_leaves_nothing_behind(heads, T):
    """A limit of zero takes whatever has not landed at the first look for lost: query rows are fetched while the softmax warps
    look for them, so every CTA gives up with copies of K, V and q under way.  (Healthy copies, which land a microsecond later.)
    Longer limits run out somewhere or not at all.  Between such calls, on the same pool and without a reset, results are as ever."""
    cfg = config(heads, "bf16", n=7, layers=1)
    tw = twin(cfg, [9000, 130, 0, 2000, 77, 16, 511])
    first = run_tree(tw, 0, T, seed=4)
    v = tw.gpu.views()
    n, d = 7, cfg.head_dim
    q, _ = draw(cfg, W.TID_Q, (n, T, cfg.num_q_heads, d), 4)
    kd, _ = draw(cfg, W.TID_K, (n, T, 1, cfg.num_kv_heads, d), 4)
    vd, _ = draw(cfg, W.TID_V, (n, T, 1, cfg.num_kv_heads, d), 4)
    parents = torch.from_numpy(random_parents(np.random.default_rng(4), n, T, "random")).cuda()

    def call():
        return tw.gpu.decode_attention_tree(0, q, kd, vd, parents, v["block_table"], v["seq_lens"])

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


# ---------------------------------------------------------------- append_kv_path
def same_payload(tw):
    for l in range(tw.cfg.num_layers):
        for t in range(len(tw.ora.seq_lens)):
            if not tw.ora.live[t]:
                continue
            K, V = trace_kv(tw, l, t)
            for h in range(tw.cfg.num_kv_heads):
                k, v = tw.gpu.read_kv(l, h, tw.gpu.views()["block_table"][t], len(K))
                np.testing.assert_array_equal(exact_f32(k), K[:, h])
                np.testing.assert_array_equal(exact_f32(v), V[:, h])


def both_paths(tw, ids, T, path, path_len, sub=9):
    c = tw.cfg
    shape = (len(ids), T, c.num_layers, c.num_kv_heads, c.head_dim)
    kd, kx = draw(c, W.TID_KNEW, shape, sub)
    vd, vx = draw(c, W.TID_VNEW, shape, sub)
    path, path_len = np.asarray(path, dtype=np.int32), np.asarray(path_len, dtype=np.int32)
    tw.gpu.append_kv_path(torch.tensor(ids, dtype=torch.int32, device="cuda"), kd, vd, torch.from_numpy(path).cuda(), torch.from_numpy(path_len).cuda())
    OD.append_path(tw.ora, ids, T, path, path_len, kx, vx)


@pytest.mark.parametrize("heads,dtype,page,layers", [((8, 2, 128), "bf16", 16, 3), ((4, 1, 64), "fp32", 16, 1), ((4, 2, 8), "bf16", 3, 2)])
@pytest.mark.parametrize("T,most", [(1, 1), (9, 5), (70, 70)])
def test_append_path(heads, dtype, page, layers, T, most):
    cfg = config(heads, dtype, page=page, layers=layers, n=6)
    tw = twin(cfg, [33, 40, 33, 48, 64, 33], prefix=33, max_pages=80, num_blocks=300)
    rng = np.random.default_rng(T)
    path = rng.integers(0, T, size=(6, most))
    lens = rng.integers(0, most + 1, size=6)
    lens[0], lens[1] = 0, most
    both_paths(tw, [3, 1, 5, 0, 4, 2], T, path, lens)
    assert tw.status() == (0, 0)
    tw.assert_meta_equal()
    same_payload(tw)


def test_append_path_flags_and_skips():
    cfg = config((8, 2, 128), "bf16", n=6, layers=1)
    tw = twin(cfg, [16, 16, 16, 32, 16, 160], max_pages=10, num_blocks=6 + 10 + 3)
    # entry 1 names a row outside the draft, 2 too many rows, 3 is listed twice, 4 not a trace, 6 has no page left, the
    # rest asks for four blocks where three are left
    path = [[0, 1], [0, 2], [0, 1], [0, 0], [1, 0], [1, 1], [0, 1], [1, 0], [0, 0]]
    lens = [2, 2, 3, 1, 1, 2, 1, 2, 1]
    both_paths(tw, [0, 1, 2, 0, 77, 3], 2, path[:6], lens[:6])             # (a list has max_traces entries at most)
    both_paths(tw, [5, 4, 4], 2, path[6:], lens[6:])
    mask, want = tw.status()
    assert mask == want and mask & (1 << 1) and mask & (1 << 3) and mask & (1 << 4)
    tw.assert_meta_equal()
    same_payload(tw)


def test_append_path_when_the_free_list_is_short():
    cfg = config((4, 1, 64), "fp32", n=4, layers=2)
    tw = twin(cfg, [16, 16, 16, 16], max_pages=10, num_blocks=4 + 3)
    both_paths(tw, [2, 0, 1, 3], 40, np.tile(np.arange(40), (4, 1)), [17, 33, 16, 1])
    mask, want = tw.status()
    assert mask == want == 1 << 2
    tw.assert_meta_equal()
    same_payload(tw)


# ---------------------------------------------------------------- refusals
def test_refusals():
    cfg = config((8, 2, 128), "bf16", n=2, layers=1)
    tw = twin(cfg, [4, 5])
    p, v, dev = tw.gpu, tw.gpu.views(), "cuda"
    q = torch.zeros((2, 3, 8, 128), dtype=torch.bfloat16, device=dev)
    kd = torch.zeros((2, 3, 1, 2, 128), dtype=torch.bfloat16, device=dev)
    par = torch.full((2, 3), -1, dtype=torch.int32, device=dev)
    ok = dict(layer=0, q=q, k_draft=kd, v_draft=kd, parents=par, block_table=v["block_table"], seq_lens=v["seq_lens"])
    p.decode_attention_tree(**ok)
    wide = torch.zeros((2, 65, 8, 128), dtype=torch.bfloat16, device=dev)
    bad = [dict(layer=1), dict(layer=-1), dict(q=q.float()), dict(q=q[:1]), dict(q=q.cpu()), dict(k_draft=kd[:, :2]), dict(q=q[0]),
           dict(v_draft=kd.float()), dict(parents=par.long()), dict(parents=par[:, :2]), dict(block_table=v["block_table"][:1]),
           dict(seq_lens=v["seq_lens"].long()), dict(n_nodes=torch.zeros(3, dtype=torch.int32, device=dev)),
           dict(out=q.float()), dict(q=q.transpose(0, 1).contiguous().transpose(0, 1)),
           dict(q=wide, k_draft=torch.zeros((2, 65, 1, 2, 128), dtype=torch.bfloat16, device=dev),
                v_draft=torch.zeros((2, 65, 1, 2, 128), dtype=torch.bfloat16, device=dev), parents=torch.full((2, 65), -1, dtype=torch.int32, device=dev))]
    off = torch.zeros(q.numel() + 8, dtype=torch.bfloat16, device=dev)
    bad += [dict(out=off[8:].view(q.shape)), dict(q=off[4:-4].view(q.shape))]        # 16 and 8 bytes behind an aligned address
    for change in bad:
        with pytest.raises(B.StepError) as e:
            p.decode_attention_tree(**{**ok, **change})
        assert e.value.code == 1
    ids, path, pl = (torch.zeros(s, dtype=torch.int32, device=dev) for s in ((2,), (2, 3), (2,)))
    ids[1] = 1
    good = dict(trace_ids=ids, k_draft=kd, v_draft=kd, path=path, path_len=pl)
    p.append_kv_path(**good)
    for change in (dict(trace_ids=ids[:1]), dict(trace_ids=ids.long()), dict(path=path[:1]), dict(path=path.float()), dict(path_len=pl[:1]),
                   dict(k_draft=kd.float()), dict(v_draft=kd[:, :1]), dict(path_len=pl.cpu())):
        with pytest.raises(B.StepError) as e:
            p.append_kv_path(**{**good, **change})
        assert e.value.code == 1
    assert p.last_error() == (0, 0)
    # null pointers and a workspace that is too small, at the C boundary
    L = B.lib()
    assert L.append_kv_path(p.handle, None, 2, 3, None, None, None, None, 3, None) == 1
    assert L.decode_attention_tree(p.handle, 0, None, None, None, None, None, 3, None, None, 2, None, None, 0, None) == 1
