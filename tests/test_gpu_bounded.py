"""decode_attention_weights and kv_pool_evict_positions against the oracle, and a bounded-cache run of all four calls."""
import numpy as np
import pytest
import torch

from oracle import bounded as OB
from oracle import drafts as OD
from paper_2601_09093_b200 import binding as B
from paper_2601_09093_b200 import harness as H
from paper_2601_09093_b200 import workloads as W

from draft_common import FP32_HALF_STEP, config, draw, poison_unused, relative_bound, trace_kv, twin
from gpu_common import exact_f32
from test_gpu_drafts import both_paths, check_tree, random_parents, same_payload

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------- decode_attention_weights
def run_weights(tw, layer, stride, seed=5, poison=True, **kw):
    cfg, n = tw.cfg, len(tw.ora.seq_lens)
    if poison:
        poison_unused(tw)
    q, qx = draw(cfg, W.TID_Q, (n, cfg.num_q_heads, cfg.head_dim), seed)
    start = np.random.default_rng(seed).random((n, cfg.num_kv_heads, stride), dtype=np.float32)
    sums = torch.from_numpy(start.copy()).cuda()
    v = tw.gpu.views()
    out = tw.gpu.decode_attention_weights(layer, q, v["block_table"][:n], v["seq_lens"][:n], sums, **kw)
    got, w_got = exact_f32(out), exact_f32(sums)
    G = cfg.num_q_heads // cfg.num_kv_heads
    for t in range(n):
        K, V = trace_kv(tw, layer, t)
        S = len(K)
        want, w, mag = OB.decode_weights(qx[t], K, V)
        rel = max(relative_bound(qx[t][h * G:(h + 1) * G], K[:, h]) for h in range(cfg.num_kv_heads))
        assert np.all(np.abs(got[t] - want) <= rel * mag + 1e-30), t
        k = min(S, stride)
        full = start[t, :, :k] + w[:, :k]
        assert np.all(np.abs(w_got[t, :, :k] - full) <= rel * w[:, :k] + (G + 2) * FP32_HALF_STEP * full + 1e-30), t
        np.testing.assert_array_equal(w_got[t, :, k:], start[t, :, k:])
    return out, sums


LENS = [0, 1, 15, 16, 17, 127, 128, 129, 200, 385]


@pytest.mark.parametrize("heads", [(8, 2, 128), (8, 1, 128), (5, 1, 128), (16, 1, 128), (2, 2, 128), (12, 1, 128)])
def test_weights_bf16(heads):
    tw = twin(config(heads, "bf16", n=len(LENS)), LENS)
    run_weights(tw, 1, 400)
    assert tw.gpu.last_error() == (0, 0)


@pytest.mark.parametrize("heads,dtype,page", [((4, 1, 64), "fp32", 16), ((8, 2, 64), "bf16", 16), ((6, 2, 128), "bf16", 32),
                                              ((4, 2, 8), "bf16", 3), ((4, 2, 12), "fp32", 5), ((2, 1, 512), "fp32", 16)])
def test_weights_other_pools(heads, dtype, page):
    tw = twin(config(heads, dtype, page=page, n=len(LENS)), LENS)
    run_weights(tw, 0, 387)
    assert tw.gpu.last_error() == (0, 0)


@pytest.mark.parametrize("heads,dtype", [((8, 2, 128), "bf16"), ((4, 1, 64), "fp32")])
def test_weights_behind_the_stride_are_flagged_and_not_counted(heads, dtype):
    tw = twin(config(heads, dtype, n=4), [300, 33, 47, 48])
    run_weights(tw, 1, 47)
    assert tw.gpu.last_error() == (4, 1 << 4)


def test_weights_of_long_caches_in_many_pieces():
    tw = twin(config((8, 1, 128), "bf16", layers=1, n=3), [12000, 40, 5003])
    run_weights(tw, 0, 12000, poison=False)
    tw.gpu.set_attention_balance(0)
    run_weights(tw, 0, 12001, poison=False)
    tw.gpu.set_attention_config(grid_ctas=3)
    run_weights(tw, 0, 12002, poison=False)
    assert tw.gpu.last_error() == (0, 0)


def test_weights_of_many_traces():
    n = 150
    lens = np.random.default_rng(4).integers(0, 60, size=n)
    tw = twin(config((4, 2, 128), "bf16", layers=1, n=n), lens)
    run_weights(tw, 0, 64)
    assert tw.gpu.last_error() == (0, 0)


def test_every_query_head_adds_one_to_the_sums_and_calls_repeat_bit_for_bit():
    cfg = config((8, 2, 128), "bf16", layers=1, n=3)
    tw = twin(cfg, [700, 64, 3])
    out, sums = run_weights(tw, 0, 704, seed=6)
    out2, sums2 = run_weights(tw, 0, 704, seed=6, poison=False)
    assert torch.equal(out, out2) and torch.equal(sums, sums2)
    q, _ = draw(cfg, W.TID_Q, (3, 8, 128), 6)
    v = tw.gpu.views()
    fresh = torch.zeros((3, 2, 704), device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            tw.gpu.decode_attention_weights(0, q, v["block_table"], v["seq_lens"], fresh)
        fresh.zero_()
        for _ in range(4):
            graph.replay()
    s.synchronize()
    # four calls, each adding four heads' worth: 16 per KV head, 704 entries each a sum of 16 rounded terms
    total = fresh.double().sum(-1)
    assert (total - 16).abs().max().item() <= 16 * (16 + 704) * 2 * FP32_HALF_STEP + 16 * 2 * 300 * FP32_HALF_STEP


# ---------------------------------------------------------------- eviction
def run_evict(tw, ids, weights, budget, recent, in_place=False):
    dev_w = torch.from_numpy(weights).cuda()
    out = dev_w if in_place else torch.full_like(dev_w, 7.0)
    L, n, Hkv, _ = weights.shape
    kept = torch.full((L, n, Hkv, budget), -1, dtype=torch.int32, device="cuda")
    got = tw.gpu.evict_positions(torch.tensor(ids, dtype=torch.int32, device="cuda"), dev_w, budget, recent,
                                 weights_out=None if in_place else out, kept_out=kept)
    assert got is kept
    after, want = OB.evict(tw.ora, ids, weights, budget, recent)
    np.testing.assert_array_equal(kept.cpu().numpy(), want)
    np.testing.assert_array_equal(out.cpu().numpy(), after)
    if not in_place:
        np.testing.assert_array_equal(dev_w.cpu().numpy(), weights)
    mask, omask = tw.status()
    assert mask == omask
    tw.assert_meta_equal()
    same_payload(tw)
    return mask


def some_weights(rng, shape, kind="random"):
    w = np.exp(1.5 * rng.standard_normal(shape)).astype(np.float32)
    if kind == "ties":
        w = rng.integers(0, 4, size=shape).astype(np.float32)
    if kind == "equal":
        w = np.ones(shape, dtype=np.float32)
    if kind == "odd":
        pick = rng.integers(0, 7, size=shape)
        for k, x in enumerate((np.nan, np.inf, -np.inf, 0.0, -0.0, np.finfo(np.float32).min)):
            w[pick == k] = x
    return w


POOLS = [((8, 2, 128), "bf16", 16, 2), ((4, 1, 64), "fp32", 16, 3), ((4, 2, 8), "bf16", 3, 1), ((2, 1, 512), "fp32", 16, 1),
         ((2, 2, 12), "fp32", 5, 2)]


@pytest.mark.parametrize("heads,dtype,page,layers", POOLS)
@pytest.mark.parametrize("kind", ["random", "ties", "equal", "odd"])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict(heads, dtype, page, layers, kind, in_place):
    lens = [200, 97, 96, 130, 95, 333]
    cfg = config(heads, dtype, page=page, layers=layers, n=6)
    tw = twin(cfg, lens)
    w = some_weights(np.random.default_rng(1), (layers, 6, heads[1], 340), kind)
    assert run_evict(tw, [3, 0, 1, 5, 4, 2], w[:, [3, 0, 1, 5, 4, 2]].copy(), 96, 20, in_place) == 0


@pytest.mark.parametrize("budget,recent", [(1, 0), (1, 1), (17, 17), (16, 0), (64, 1), (63, 62), (299, 150), (300, 7)])
def test_evict_sizes(budget, recent):
    cfg = config((8, 2, 128), "bf16", layers=2, n=3)
    tw = twin(cfg, [300, 301, 64])
    w = some_weights(np.random.default_rng(2), (2, 3, 2, 301))
    run_evict(tw, [0, 1, 2], w, budget, recent)


@pytest.mark.parametrize("heads,dtype", [((8, 2, 128), "bf16"), ((4, 1, 64), "fp32")])
def test_evict_gives_every_trace_pages_of_its_own(heads, dtype):
    """Traces share their prompt; two of three are cut, then the third, then all of them again."""
    cfg = config(heads, dtype, layers=2, n=3)
    tw = twin(cfg, [120, 150, 130], prefix=100)
    rng = np.random.default_rng(3)
    w = some_weights(rng, (2, 3, heads[1], 160))
    run_evict(tw, [2, 0], w[:, [2, 0]].copy(), 60, 8)
    run_evict(tw, [1], w[:, 1:2].copy(), 60, 8, in_place=True)
    tw.append([0, 1, 2], 19)
    run_evict(tw, [0, 1, 2], w, 60, 8)


def test_evict_leaves_alone_what_cannot_be_served():
    cfg = config((8, 2, 128), "bf16", layers=1, n=5)
    # prompt of 6 shared pages; 2 free blocks are not enough for anybody's kept pages
    tw = twin(cfg, [120, 150, 130, 96, 20 + 96], prefix=96, num_blocks=6 + 2 + 4 + 3 + 0 + 2 + 2)
    w = some_weights(np.random.default_rng(4), (1, 7, 2, 145))
    # entry 1 has more positions than weights, 3 is at its budget, 4 is listed twice; then two that are no traces
    mask = run_evict(tw, [0, 1, 2, 3, 0], w[:, :5].copy(), 96, 10)
    assert mask == (1 << 2) | (1 << 3) | (1 << 4)
    assert run_evict(tw, [-1, 5], w[:, :2].copy(), 96, 10) == 1 << 3


@pytest.mark.parametrize("in_place", [False, True])
def test_evict_from_a_long_cache(in_place):
    cfg = config((2, 1, 128), "bf16", layers=1, n=2)
    tw = twin(cfg, [40000, 9000])
    w = some_weights(np.random.default_rng(5), (1, 2, 1, 40000))
    run_evict(tw, [0, 1], w, 8000, 700, in_place)


def test_evict_under_a_graph_on_another_stream():
    cfg = config((8, 2, 128), "bf16", layers=2, n=3)
    tw = twin(cfg, [200, 210, 97])
    w = some_weights(np.random.default_rng(6), (2, 3, 2, 220))
    dev_w, out = torch.from_numpy(w).cuda(), torch.zeros((2, 3, 2, 220), device="cuda")
    kept = torch.full((2, 3, 2, 100), -1, dtype=torch.int32, device="cuda")
    ids = torch.arange(3, dtype=torch.int32, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            tw.gpu.evict_positions(ids, dev_w, 100, 30, weights_out=out, kept_out=kept)
        graph.replay()
    s.synchronize()
    after, want = OB.evict(tw.ora, [0, 1, 2], w, 100, 30)
    np.testing.assert_array_equal(kept.cpu().numpy(), want)
    np.testing.assert_array_equal(out.cpu().numpy(), after)
    tw.assert_meta_equal()
    same_payload(tw)


# ---------------------------------------------------------------- together
@pytest.mark.parametrize("heads,dtype", [((8, 2, 128), "bf16"), ((4, 1, 64), "fp32")])
def test_a_bounded_cache_with_drafts(heads, dtype):
    """A few steps of speculative decoding with a bounded cache: verify a draft tree, store the accepted path, attend and
    count, evict.  Both sides evict by the CUDA side's counts, so that the choice is the same."""
    cfg = config(heads, dtype, layers=2, n=4)
    tw = twin(cfg, [120, 95, 40, 110], prefix=33)
    rng, n, T, budget = np.random.default_rng(8), 4, 11, 100
    stride = 140
    counts = torch.zeros((2, n, cfg.num_kv_heads, stride), device="cuda")
    v = tw.gpu.views()
    for step in range(4):
        shape = (n, T, 2, cfg.num_kv_heads, cfg.head_dim)
        kd, kx = draw(cfg, W.TID_K, shape, 50 + step)
        vd, vx = draw(cfg, W.TID_V, shape, 50 + step)
        q, qx = draw(cfg, W.TID_Q, (n, T, cfg.num_q_heads, cfg.head_dim), 50 + step)
        parents = random_parents(rng, n, T, "random")
        for layer in range(2):
            out = tw.gpu.decode_attention_tree(layer, q, kd, vd, torch.from_numpy(parents).cuda(), v["block_table"], v["seq_lens"])
            check_tree(tw, layer, exact_f32(out), qx, kx, vx, parents, [T] * n)
        leaf = rng.integers(0, T, size=n)
        paths = [OD.path_to_root(p, u)[::-1] for p, u in zip(parents, leaf)]
        path = np.zeros((n, T), dtype=np.int32)
        for i, p in enumerate(paths):
            path[i, :len(p)] = p
        lens = np.array([len(p) for p in paths], dtype=np.int32)
        ids = list(range(n))
        tw.gpu.append_kv_path(torch.tensor(ids, dtype=torch.int32, device="cuda"), kd, vd, torch.from_numpy(path).cuda(), torch.from_numpy(lens).cuda())
        OD.append_path(tw.ora, ids, T, path, lens, kx, vx)
        last, lx = draw(cfg, W.TID_Q, (n, cfg.num_q_heads, cfg.head_dim), 90 + step)
        for layer in range(2):
            out = tw.gpu.decode_attention_weights(layer, last, v["block_table"], v["seq_lens"], counts[layer])
            for t in range(n):
                K, V = trace_kv(tw, layer, t)
                want, _, mag = OB.decode_weights(lx[t], K, V)
                rel = max(relative_bound(lx[t].reshape(cfg.num_kv_heads, -1, cfg.head_dim)[h], K[:, h]) for h in range(cfg.num_kv_heads))
                assert np.all(np.abs(exact_f32(out)[t] - want) <= rel * mag + 1e-30)
        before = counts.cpu().numpy()
        kept = tw.gpu.evict_positions(torch.tensor(ids, dtype=torch.int32, device="cuda"), counts, budget, 16)
        after, want = OB.evict(tw.ora, ids, before, budget, 16)
        np.testing.assert_array_equal(kept.cpu().numpy(), want)
        np.testing.assert_array_equal(counts.cpu().numpy(), after)
        assert tw.status() == (0, 0)
        tw.assert_meta_equal()
        same_payload(tw)
    assert int(tw.ora.seq_lens.max()) == budget


def test_calls_take_a_stream_and_two_pools_may_run_side_by_side():
    """The same steps on two pools: one after the other, and at the same time on two streams that the calls are given."""
    results = []
    for together in (False, True):
        outs = []
        twins = [twin(config((8, 2, 128), "bf16", layers=1, n=3, seed=50 + k), [600, 77, 130]) for k in range(2)]
        inputs = []
        for k, tw in enumerate(twins):
            c = tw.cfg
            q, _ = draw(c, W.TID_Q, (3, 4, 8, 128), 1)
            kd, _ = draw(c, W.TID_K, (3, 4, 1, 2, 128), 2)
            vd, _ = draw(c, W.TID_V, (3, 4, 1, 2, 128), 3)
            parents = torch.tensor([[-1, 0, 1, 0]] * 3, dtype=torch.int32, device="cuda")
            path = torch.tensor([[0, 1, 2]] * 3, dtype=torch.int32, device="cuda")
            inputs.append((q, kd, vd, parents, path, torch.tensor([3, 0, 2], dtype=torch.int32, device="cuda"),
                           torch.zeros((3, 2, 640), device="cuda"), torch.arange(3, dtype=torch.int32, device="cuda")))
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream() for _ in twins] if together else [None, None]
        for _ in range(3):
            for tw, (q, kd, vd, parents, path, lens, sums, ids), s in zip(twins, inputs, streams):
                v = tw.gpu.views()
                tree = tw.gpu.decode_attention_tree(0, q, kd, vd, parents, v["block_table"], v["seq_lens"], stream=s)
                tw.gpu.append_kv_path(ids, kd, vd, path, lens, stream=s)
                with torch.cuda.stream(s):
                    last = q[:, 0].contiguous()
                out = tw.gpu.decode_attention_weights(0, last, v["block_table"], v["seq_lens"], sums, stream=s)
                with torch.cuda.stream(s):
                    w = sums[None].clone()
                kept = tw.gpu.evict_positions(ids, w, 70, 9, stream=s)
                outs += [tree, out, w, kept]
        torch.cuda.synchronize()
        results.append(outs)
        assert all(tw.gpu.last_error() == (0, 0) for tw in twins)
    for x, y in zip(*results):
        assert torch.equal(x, y)


# ---------------------------------------------------------------- refusals
def test_refusals():
    cfg = config((8, 2, 128), "bf16", n=2, layers=1)
    tw = twin(cfg, [40, 50])
    p, v, dev = tw.gpu, tw.gpu.views(), "cuda"
    q, sums = torch.zeros((2, 8, 128), dtype=torch.bfloat16, device=dev), torch.zeros((2, 2, 50), device=dev)
    ok = dict(layer=0, q=q, block_table=v["block_table"], seq_lens=v["seq_lens"], weight_sum=sums)
    p.decode_attention_weights(**ok)
    for change in (dict(layer=1), dict(layer=-1), dict(q=q.float()), dict(q=q[:1]), dict(weight_sum=sums.double()), dict(weight_sum=sums[:, :1]),
                   dict(weight_sum=sums.transpose(1, 2)), dict(out=q), dict(seq_lens=v["seq_lens"][:1]), dict(block_table=v["block_table"].long()),
                   dict(workspace=torch.empty(64, dtype=torch.uint8, device=dev)), dict(weight_sum=sums.cpu()), dict(weight_sum=sums[..., :0])):
        with pytest.raises(B.StepError) as e:
            p.decode_attention_weights(**{**ok, **change})
        assert e.value.code == 1
    ids = torch.arange(2, dtype=torch.int32, device=dev)
    w = torch.zeros((1, 2, 2, 50), device=dev)
    good = dict(trace_ids=ids, weights=w, budget=45, recent=4)
    p.evict_positions(**good)
    for change in (dict(budget=0), dict(budget=51), dict(budget=1 << 20), dict(recent=-1), dict(recent=46), dict(weights=w[0]), dict(weights=w.double()),
                   dict(trace_ids=ids[:1]), dict(trace_ids=ids.long()), dict(weights_out=w[..., :49]), dict(kept_out=torch.zeros((1, 2, 2, 44), dtype=torch.int32, device=dev)),
                   dict(workspace=torch.empty(4, dtype=torch.uint8, device=dev))):
        with pytest.raises(B.StepError) as e:
            p.evict_positions(**{**good, **change})
        assert e.value.code == 1
    assert p.last_error() == (0, 0)
    L = B.lib()
    assert L.decode_attention_weights(p.handle, 0, None, None, None, 2, None, None, 5, None, 0, None) == 1
    assert L.kv_pool_evict_positions(p.handle, None, 2, None, None, 50, 45, 4, None, None, 0, None) == 1


# ---------------------------------------------------------------- values below the smallest normal number
def tiny_weights(rng, shape):
    """Zeros of both signs, subnormals of both signs and the smallest normal numbers, each about as often."""
    bits = rng.integers(1, 0x00800000, size=shape, dtype=np.uint32)              # subnormals
    pick = rng.integers(0, 5, size=shape)
    bits[pick == 0] = 0
    bits[pick == 1] = rng.integers(1, 5, size=int((pick == 1).sum()))            # the smallest ones, with ties
    bits[pick == 2] |= 0x00800000                                                # 2^-126 and just above
    sign = rng.random(shape) < 0.3
    return (bits | (sign.astype(np.uint32) << 31)).view(np.float32)


@pytest.mark.parametrize("heads,dtype,page,layers", POOLS[:2])
@pytest.mark.parametrize("in_place", [False, True])
def test_evict_tells_subnormal_weights_apart(heads, dtype, page, layers, in_place):
    """Only the two zeros are equal: a caller whose sums decay ends up with weights this small."""
    cfg = config(heads, dtype, page=page, layers=layers, n=3)
    tw = twin(cfg, [333, 200, 97])
    w = tiny_weights(np.random.default_rng(9), (layers, 3, heads[1], 340))
    assert run_evict(tw, [0, 1, 2], w, 96, 20, in_place) == 0


@pytest.mark.parametrize("in_place", [False, True])
def test_evict_tells_subnormal_weights_of_a_long_cache_apart(in_place):
    cfg = config((2, 1, 128), "bf16", layers=1, n=1)
    tw = twin(cfg, [14000])
    run_evict(tw, [0], tiny_weights(np.random.default_rng(10), (1, 1, 1, 14000)), 5000, 100, in_place)


@pytest.mark.parametrize("heads,dtype", [((8, 2, 128), "bf16"), ((4, 1, 64), "fp32")])
def test_a_subnormal_sum_survives_a_weight_of_zero(heads, dtype):
    """weight_sum += p leaves the sum as it is where p is nothing, however small the sum."""
    lens = [200, 385]
    cfg = config(heads, dtype, layers=1, n=2)
    tw = twin(cfg, lens)
    shape = (2, cfg.num_q_heads, cfg.head_dim)
    _, qx = draw(cfg, W.TID_Q, shape, 11)
    qx = qx * 256                                                               # (exact in both types)
    q = torch.from_numpy(qx).to(tw.gpu.torch_dtype).cuda()
    start = np.abs(tiny_weights(np.random.default_rng(11), (2, cfg.num_kv_heads, 386)))
    sums = torch.from_numpy(start.copy()).cuda()
    v = tw.gpu.views()
    tw.gpu.decode_attention_weights(0, q, v["block_table"], v["seq_lens"], sums)
    got = sums.cpu().numpy()
    for t in range(2):
        K, V = trace_kv(tw, 0, t)
        _, w, _ = OB.decode_weights(qx[t], K, V)
        # scores spread over hundreds: most weights are far below half of the smallest subnormal, 2^-150
        none = w < 2.0 ** -400
        assert none.sum() > none.size // 3
        k = none.shape[1]
        np.testing.assert_array_equal(got[t, :, :k].view(np.uint32)[none], start[t, :, :k].view(np.uint32)[none])
    assert tw.gpu.last_error() == (0, 0)
