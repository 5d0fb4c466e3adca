"""rotate_positions, kv_pool_extend and store_kv_rotated against the oracle."""
import numpy as np
import pytest
import torch

from oracle import rotary as OR
from paper_2601_09093_b200 import binding as B
from paper_2601_09093_b200 import workloads as W

from draft_common import BF16_HALF_STEP, FP32_HALF_STEP, config, draw, trace_kv, twin
from gpu_common import exact_f32

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}


def bound(x, want, D, interleaved, scale, dtype):
    """A cosine or sine: the angle's rounding (a float of at most pi / 4), sincospif (2 steps of a value up to 1) and the scale;
    two products and their sum: 8 half steps of |x1| + |x2| are more than enough.  Then one rounding to the type.  Dims behind
    D are copied."""
    one, two = (slice(0, D, 2), slice(1, D, 2)) if interleaved else (slice(0, D // 2), slice(D // 2, D))
    tol = np.zeros_like(want)
    both = (np.abs(x[..., one]) + np.abs(x[..., two])) * abs(scale) * 8 * FP32_HALF_STEP
    tol[..., one] = tol[..., two] = both
    if dtype == "bf16":
        tol[..., :D] += BF16_HALF_STEP * (np.abs(want[..., :D]) + tol[..., :D])
    return tol


def check(got, x, positions, rotary, f, dtype, transpose=False):
    """x, got: fp64 [..., heads, d]"""
    scale, inter = rotary.struct.scale, bool(rotary.struct.interleaved)
    want = OR.rotate(x, positions, f, inter, scale, transpose)
    err = np.abs(got - want)
    assert np.all(err <= bound(x, want, 2 * len(f), inter, scale, dtype)), float(err.max())


def both(D, base=10000.0, **kw):
    dev = {k: kw.pop(k) for k in ("interleaved", "output_scale") if k in kw}
    return B.Rotary(D, base, **dev, **kw), OR.frequencies(D, base, **kw)


FAR = [0, 1, -1, 7, 4095, 131071, 999_983, -(1 << 31), (1 << 31) - 1, 123_456_789]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,D", [(128, 128), (128, 64), (64, 16), (128, 96), (64, 20), (128, 2), (12, 12), (7, 4), (512, 512), (256, 240)])
def test_rotate(dtype, interleaved, d, D):
    r, f = both(D, interleaved=interleaved)
    for batch, rows, heads in ((1, 1, 1), (1, 10, 5), (3, 10, 33)):
        pos = np.resize(np.array(FAR), (batch, rows)).astype(np.int32)
        x = torch.randn((batch, rows, heads, d), generator=torch.Generator().manual_seed(D)).to(TYPES[dtype]).cuda()
        for transpose in (False, True):
            y = B.rotate_positions(x, r, torch.from_numpy(pos).cuda(), transpose=transpose)
            assert y.dtype == x.dtype and y.shape == x.shape
            check(exact_f32(y), exact_f32(x), pos, r, f, dtype, transpose)


@pytest.mark.parametrize("kw", [dict(scaling="linear", factor=8.0), dict(scaling="base", factor=4.0), dict(scaling="yarn", factor=4.0, original_positions=32768),
                                dict(scaling="bands", factor=8.0, original_positions=8192), dict(divisors=np.linspace(1, 9, 64)), dict(output_scale=0.25)])
def test_rotate_for_long_contexts(kw):
    r, f = both(128, 500000.0, **kw)
    pos = np.arange(300) * 3001
    x = torch.randn((300, 4, 128), generator=torch.Generator().manual_seed(5)).cuda()
    check(exact_f32(B.rotate_positions(x, r, torch.from_numpy(pos.astype(np.int32)).cuda())), exact_f32(x), pos, r, f, "fp32")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [128, 32])
def test_strides_and_places(dtype, D):
    """Slices of a packed projection, keys laid out head by head, rows that do not start on 16 bytes, broadcast input,
    results into such places, in place."""
    r, f = both(D)
    t, d = TYPES[dtype], 128
    gen = torch.Generator().manual_seed(1)
    pos = np.array([[5, 900, 3], [70000, 0, 12]], dtype=np.int32)
    p = torch.from_numpy(pos).cuda()
    packed = torch.randn((2, 3, 12, d), generator=gen).to(t).cuda()
    by_head = torch.randn((2, 8, 3, d), generator=gen).to(t).cuda()
    loose = torch.randn((2, 3, 8, d + 1), generator=gen).to(t).cuda()
    one = torch.randn((2, 3, 1, d), generator=gen).to(t).cuda()
    inputs = [packed[:, :, 3:11], by_head.transpose(1, 2), loose[..., :d], loose[..., 1:], one.expand(2, 3, 8, d), packed[:1, :, 4:12].expand(2, 3, 8, d)]
    for x in inputs:
        want = exact_f32(x)
        check(exact_f32(B.rotate_positions(x, r, p)), want, pos, r, f, dtype)
        for out in (torch.zeros((2, 3, 12, d), dtype=t, device="cuda")[:, :, 2:10], torch.zeros((2, 3, 8, d + 3), dtype=t, device="cuda")[..., 3:],
                    torch.zeros((2, 8, 3, d), dtype=t, device="cuda").transpose(1, 2)):
            assert B.rotate_positions(x, r, p, out=out) is out
            check(exact_f32(out), want, pos, r, f, dtype)
    around = packed.clone()
    for x in inputs[:4]:
        before = exact_f32(x)
        B.rotate_positions(x, r, p, out=x)
        check(exact_f32(x), before, pos, r, f, dtype)
    assert torch.equal(packed[:, :, :3], around[:, :, :3]) and torch.equal(packed[:, :, 11:], around[:, :, 11:])


def test_positions_by_row_for_all_or_none_given():
    r, f = both(64)
    x = torch.randn((4, 9, 2, 64), generator=torch.Generator().manual_seed(2)).cuda()
    rows = np.array([3, 1, 4, 1, 5, 9, 2, 6, 5], dtype=np.int32)
    check(exact_f32(B.rotate_positions(x, r, torch.from_numpy(rows).cuda())), exact_f32(x), np.tile(rows, (4, 1)), r, f, "fp32")
    check(exact_f32(B.rotate_positions(x, r)), exact_f32(x), np.tile(np.arange(9), (4, 1)), r, f, "fp32")
    wide = torch.arange(80, dtype=torch.int32, device="cuda").view(4, 20)
    check(exact_f32(B.rotate_positions(x, r, wide[:, 3:12])), exact_f32(x), wide[:, 3:12].cpu().numpy(), r, f, "fp32")
    assert B.rotate_positions(x[:, :0], r).shape == (4, 0, 2, 64)


@pytest.mark.parametrize("interleaved", [False, True])
def test_the_transposed_rotation_is_the_gradient(interleaved):
    """Against torch's own derivative of the formula in 64 bits, and against differences of the kernel's results (the rotation is
    linear: a difference over a large step is exact but for rounding)."""
    r, f = both(64, interleaved=interleaved, scaling="yarn", factor=4.0, original_positions=100)
    gen = torch.Generator().manual_seed(3)
    x, w = torch.randn((2, 1, 50, 3, 80), generator=gen).cuda()
    pos = torch.randint(0, 5000, (1, 50), generator=gen, dtype=torch.int32).cuda()
    g = B.rotate_positions(w, r, pos, transpose=True)
    leaf = x.double().requires_grad_()
    a = pos.double()[..., None, None] * torch.from_numpy(f.astype(np.float64)).cuda()
    one, two = (slice(0, 64, 2), slice(1, 64, 2)) if interleaved else (slice(0, 32), slice(32, 64))
    c, s = a.cos() * r.struct.scale, a.sin() * r.struct.scale
    loss = ((leaf[..., one] * c - leaf[..., two] * s) * w[..., one] + (leaf[..., two] * c + leaf[..., one] * s) * w[..., two]).sum() + (leaf[..., 64:] * w[..., 64:]).sum()
    loss.backward()
    wx, want = exact_f32(w), leaf.grad.cpu().numpy()
    assert np.all(np.abs(exact_f32(g) - want) <= bound(wx, want, 64, interleaved, r.struct.scale, "fp32") + 1e-9)   # 1e-9: 64-bit angles
    rng = np.random.default_rng(1)
    for _ in range(6):
        row, h, e = rng.integers(50), rng.integers(3), rng.integers(80)
        step = torch.zeros_like(x)
        step[0, row, h, e] = 64.0
        diff = (B.rotate_positions(x + step, r, pos) - B.rotate_positions(x - step, r, pos)).double() / 128
        # x + step is off by half a step of a value below 128, each result by 8 half steps of one below 2 * 70
        assert abs((diff * w.double()).sum().item() - g[0, row, h, e].item()) <= 2 * 16 * 140 * FP32_HALF_STEP / 128 * 4 * float(w.abs().max())


def test_what_is_not_finite_stays_in_its_pair_and_the_rest_is_copied_bit_by_bit():
    r, f = both(64)
    x = torch.randn((1, 2, 3, 128), generator=torch.Generator().manual_seed(4)).bfloat16().cuda()
    x[0, 1, 2, 5], x[0, 0, 1, 40] = float("nan"), float("inf")
    x[0, 0, 0, 100], x[0, 0, 0, 101] = float("nan"), 1e-40                # behind D: bits, subnormal ones too
    y = B.rotate_positions(x, r, torch.tensor([3, 9], dtype=torch.int32, device="cuda"))
    bad = ~torch.isfinite(y)
    where = {tuple(i) for i in bad.nonzero().tolist()}
    assert where == {(0, 1, 2, 5), (0, 1, 2, 37), (0, 0, 1, 40), (0, 0, 1, 8), (0, 0, 0, 100)}
    assert torch.equal(y[..., 64:].view(torch.int16), x[..., 64:].view(torch.int16))


def test_many_rows_and_offsets_beyond_32_bits():
    r, f = both(64)
    big = torch.empty((3, (1 << 30) + 64), dtype=torch.bfloat16, device="cuda")      # rows 2^31 bytes and more apart
    x = big[:, 32:32 + 4 * 64].unflatten(1, (4, 64))
    x.copy_(torch.randn((3, 4, 64), generator=torch.Generator().manual_seed(5)))
    before, pos = exact_f32(x), np.array([1, 22, 333], dtype=np.int32)
    B.rotate_positions(x, r, torch.from_numpy(pos).cuda(), out=x)
    check(exact_f32(x), before, pos, r, f, "bf16")
    del big, x
    x = torch.randn((70001, 2, 64), device="cuda")
    y = B.rotate_positions(x, r)
    pick = [0, 1, 35000, 65535, 65536, 70000]
    check(exact_f32(y[pick]), exact_f32(x[pick]), np.array(pick), r, f, "fp32")


def test_rotate_on_another_stream_and_captured():
    r, f = both(128)
    x = torch.randn((64, 8, 128), generator=torch.Generator().manual_seed(6)).bfloat16().cuda()
    pos = torch.arange(64, dtype=torch.int32, device="cuda") * 100
    want = B.rotate_positions(x, r, pos)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(x)
    B.rotate_positions(x, r, pos, out=out, stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        B.rotate_positions(x, r, pos, out=out)
    out.zero_()
    pos += 1
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, B.rotate_positions(x, r, pos))               # the positions of the replay, not of the capture


def test_rotate_refusals():
    r, _ = both(64)
    x = torch.zeros((2, 3, 4, 64), device="cuda")
    p = torch.zeros((2, 3), dtype=torch.int32, device="cuda")
    B.rotate_positions(x, r, p)
    for a, kw in (((x[0, 0], r), {}), ((x.half(), r), {}), ((x.cpu(), r), {}), ((x[..., :32], r), {}), ((x.transpose(2, 3), r), {}),
                  ((x, r, p.long()), {}), ((x, r, p[:, :2]), {}), ((x, r, p.cpu()), {}), ((x, r, p.t().contiguous().t()), {}),
                  ((x, r, p), dict(out=x[:1])), ((x, r, p), dict(out=x.bfloat16())), ((x, r, p), dict(out=torch.zeros((2, 3, 64, 4), device="cuda").transpose(2, 3))),
                  ((x, B.Rotary(64, device="cpu"), p), {})):
        with pytest.raises(B.StepError) as e:
            B.rotate_positions(*a, **kw)
        assert e.value.code == 1


# ---------------------------------------------------------------- the cache, layer by layer
def grown(cfg, lens, T, **kw):
    tw = twin(cfg, lens, **kw)
    ids = list(range(len(lens)))
    start = tw.gpu.extend(torch.tensor(ids, dtype=torch.int32, device="cuda"), T)
    want = OR.extend(tw.ora, ids, T)
    assert start.tolist() == want.tolist()
    return tw, start


def same_cache(tw, layers, fresh, rotary, dtype):
    """Everything in the cache is the oracle's bit for bit, but for the keys of `fresh` positions {trace: (first, unrotated
    keys [T, layers, Hkv, d], positions)}, which are within the bound."""
    f = fresh.pop("f")
    for l in layers:
        for t in range(len(tw.ora.seq_lens)):
            if not tw.ora.live[t]:
                continue
            K, V = trace_kv(tw, l, t)
            for h in range(tw.cfg.num_kv_heads):
                k, v = (exact_f32(x) for x in tw.gpu.read_kv(l, h, tw.gpu.views()["block_table"][t], len(K)))
                np.testing.assert_array_equal(v, V[:, h])
                same = np.ones(len(K), dtype=bool)
                if t in fresh:
                    st, x, pos = fresh[t]
                    check(k[st:st + len(x), None], x[:, l, h:h + 1], pos, rotary, f, dtype)
                    same[st:st + len(x)] = False
                np.testing.assert_array_equal(k[same], K[same, h])
    fresh["f"] = f


POOLS = [((8, 2, 128), "bf16", 16, 128, False), ((8, 2, 128), "bf16", 16, 64, True), ((64, 8, 128), "bf16", 16, 128, False), ((5, 1, 128), "bf16", 16, 32, False),
         ((4, 1, 64), "fp32", 16, 64, False), ((4, 2, 64), "bf16", 16, 20, True), ((4, 2, 8), "bf16", 3, 8, False), ((4, 2, 12), "fp32", 5, 10, True),
         ((2, 1, 512), "bf16", 16, 512, False), ((2, 2, 256), "fp32", 16, 200, False)]


@pytest.mark.parametrize("heads,dtype,page,D,interleaved", POOLS)
@pytest.mark.parametrize("T,one_by_one,given", [(1, True, False), (1, False, True), (17, False, False), (5, True, True)])
def test_store(heads, dtype, page, D, interleaved, T, one_by_one, given):
    lens = [0, 1, page - 1, page, 33, 2 * page]
    cfg = config(heads, dtype, page=page, layers=3, n=6)
    tw, start = grown(cfg, lens, T)
    r, f = both(D, 500000.0, interleaved=interleaved, scaling="yarn", factor=4.0, original_positions=4096)
    Hq, Hkv, d = heads
    shape = (6, T, 3, Hkv, d)
    kd, kx = draw(cfg, W.TID_KNEW, shape, 3)
    vd, vx = draw(cfg, W.TID_VNEW, shape, 3)
    qd, qx = draw(cfg, W.TID_Q, (3, 6, T, Hq, d), 3)
    first = np.array([9, 70000, 3, 2, 1 << 30, 5]) if given else np.asarray(lens)
    positions = torch.from_numpy(first.astype(np.int32)).cuda() if given else None
    ids = torch.arange(6, dtype=torch.int32, device="cuda")
    pos = first[:, None] + np.arange(T)
    if one_by_one:
        qo = torch.zeros_like(qd)
        for l in (2, 0, 1):
            assert tw.gpu.store_kv_rotated(l, ids, start, kd[:, :, l:l + 1], vd[:, :, l:l + 1], r, q=qd[l:l + 1], q_out=qo[l:l + 1], positions=positions) is not None
    else:
        qo = tw.gpu.store_kv_rotated(0, ids, start, kd, vd, r, q=qd, positions=positions)
    for l in range(3):
        check(exact_f32(qo[l]), qx[l], pos, r, f, dtype)
    OR.store(tw.ora, 0, range(6), lens, kx, vx)
    tw.assert_meta_equal()
    same_cache(tw, range(3), {**{t: (lens[t], kx[t], pos[t]) for t in range(6)}, "f": f}, r, dtype)
    assert tw.status() == (0, 0)


def test_store_from_slices_in_place_and_without_queries():
    """Rows of a packed projection [n, Hq + 2 Hkv, d], queries turned where they stand."""
    cfg = config((8, 2, 128), "bf16", layers=2, n=4)
    lens = [10, 16, 31, 0]
    tw, start = grown(cfg, lens, 1)
    r, f = both(128)
    packed = torch.randn((4, 1, 12, 128), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    keep = packed.clone()
    q, k, v = packed[:, :, :8], packed[:, :, 8:10], packed[:, :, 10:]
    ids = torch.arange(4, dtype=torch.int32, device="cuda")
    for l in range(2):
        assert tw.gpu.store_kv_rotated(l, ids, start, k[:, :, None], v[:, :, None], r) is None
    assert torch.equal(packed, keep)
    tw.gpu.store_kv_rotated(1, ids, start, k[:, :, None], v[:, :, None], r, q=q[None], q_out=q[None])
    check(exact_f32(q), exact_f32(keep[:, :, :8]), np.asarray(lens)[:, None], r, f, "bf16")
    assert torch.equal(packed[:, :, 8:], keep[:, :, 8:])
    kx, vx = (np.repeat(exact_f32(x)[:, :, None], 2, 2) for x in (k, v))
    OR.store(tw.ora, 0, range(4), lens, kx, vx)
    same_cache(tw, range(2), {**{t: (lens[t], kx[t], np.array([lens[t]])) for t in range(4)}, "f": f}, r, "bf16")


def test_what_cannot_be_stored_is_skipped_and_flagged():
    cfg = config((8, 2, 128), "bf16", layers=2, n=6)
    tw = twin(cfg, [20, 30, 40, 16, 5, 9], max_pages=4)
    tw.gpu.release_traces(torch.tensor([3], dtype=torch.int32, device="cuda"))
    tw.ora.release_trace(3)
    r, f = both(128)
    T = 3
    ids, start = [0, 1, 77, 3, -1, 4], [18, 5, 0, 0, 0, -1]              # beyond the end; fine; no trace; dead; no trace; passed over
    kd, kx = draw(cfg, W.TID_KNEW, (6, T, 2, 2, 128), 1)
    vd, vx = draw(cfg, W.TID_VNEW, (6, T, 2, 2, 128), 1)
    qd, qx = draw(cfg, W.TID_Q, (2, 6, T, 8, 128), 1)
    qo = torch.full_like(qd, 7.0)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")                              # noqa: E731
    tw.gpu.store_kv_rotated(0, dev(ids), dev(start), kd, vd, r, q=qd, q_out=qo)
    assert OR.store(tw.ora, 0, ids, start, kx, vx) == [1]
    mask, want = tw.status()
    assert mask == want == 1 << 1 | 1 << 3
    assert (qo[:, [0, 2, 3, 4, 5]] == 7).all()
    check(exact_f32(qo[:, 1]), qx[:, 1], np.tile(5 + np.arange(T), (2, 1)), r, f, "bf16")
    tw.assert_meta_equal()
    same_cache(tw, range(2), {1: (5, kx[1], 5 + np.arange(T)), "f": f}, r, "bf16")
    # a start for which start + T passes 32 bits
    tw.gpu.store_kv_rotated(0, dev([0] * 6), dev([(1 << 31) - 1] * 6), kd, vd, r)
    assert tw.status()[0] == 1 << 1
    # a table entry out of range
    table = tw.gpu.views()["block_table"]
    keep, table[1, 0] = int(table[1, 0]), 1 << 30
    tw.gpu.store_kv_rotated(0, dev([1]), dev([2]), kd[:1], vd[:1], r)
    assert tw.status()[0] == 1 << 7
    table[1, 0] = keep
    same_cache(tw, range(2), {1: (5, kx[1], 5 + np.arange(T)), "f": f}, r, "bf16")


def test_extend_skips_and_flags_as_append_does():
    cfg = config((4, 1, 64), "fp32", layers=1, n=5)
    tw = twin(cfg, [16, 16, 0, 30, 16], max_pages=4, num_blocks=7 + 3)
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")                              # noqa: E731
    # 0 listed twice, 9 not a trace, 3 past its table, then a free list that serves some
    for ids, T in (([0, 0, 9], 0), ([3, 9], 40), ([4, 1, 2], 17), ([0, 2], 1)):
        assert tw.gpu.extend(dev(ids), T).tolist() == OR.extend(tw.ora, ids, T).tolist()
    mask, want = tw.status()
    assert mask == want and mask
    tw.assert_meta_equal()
    with pytest.raises(B.StepError):
        tw.gpu.extend(dev([0] * 6), 1)                                   # more entries than traces
    assert tw.gpu.extend(dev([]), 1).shape == (0,)


def test_extend_and_store_captured_and_replayed():
    """A decode step of one layer's cache in a graph: every replay stores one token further on."""
    cfg = config((8, 2, 128), "bf16", layers=1, n=3)
    lens = [14, 0, 33]
    tw = twin(cfg, lens)
    r, f = both(128)
    kd, kx = draw(cfg, W.TID_KNEW, (3, 1, 1, 2, 128), 1)
    vd, vx = draw(cfg, W.TID_VNEW, (3, 1, 1, 2, 128), 1)
    qd, qx = draw(cfg, W.TID_Q, (1, 3, 1, 8, 128), 1)
    ids, start, qo = torch.arange(3, dtype=torch.int32, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda"), torch.empty_like(qd)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        tw.gpu.extend(ids, 1, start_out=start)
        tw.gpu.store_kv_rotated(0, ids, start, kd, vd, r, q=qd, q_out=qo)
    for _ in range(4):
        graph.replay()
    torch.cuda.synchronize()
    for step in range(4):
        at = OR.extend(tw.ora, range(3), 1)
        OR.store(tw.ora, 0, range(3), at, kx, vx)
    tw.assert_meta_equal()
    check(exact_f32(qo), qx, (np.asarray(lens) + 3)[None, :, None], r, f, "bf16")
    same_cache(tw, [0], {**{t: (lens[t], np.repeat(kx[t], 4, 0), lens[t] + np.arange(4)) for t in range(3)}, "f": f}, r, "bf16")


def test_a_store_at_the_far_end_of_a_pool_beyond_32_bit_offsets():
    Hq, Hkv, d, P, n, S, T = 4, 2, 128, 16, 2, 30, 5
    blocks = 2_500_000_000 // (Hkv * 2 * P * d)
    pool = B.KVPool(1, Hq, Hkv, d, P, num_blocks=blocks, max_traces=n, max_pages_per_trace=8)
    v = pool.views()
    v["free_list"].copy_(torch.arange(blocks, dtype=torch.int32, device="cuda"))        # pops from the end: the highest first
    pool.fork_prefix(n, 0, None, None)
    ids = torch.arange(n, dtype=torch.int32, device="cuda")
    pool.extend(ids, S)
    start = pool.extend(ids, T)
    k, w = torch.randn((2, n, T, 1, Hkv, d), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
    r, f = both(128)
    pool.store_kv_rotated(0, ids, start, k, w, r)
    assert int(v["block_table"][:, 0].min()) > blocks - 16
    for t in range(n):
        for h in range(Hkv):
            kr, vr = pool.read_kv(0, h, v["block_table"][t], S + T)
            assert torch.equal(vr[S:], w[t, :, 0, h])
            check(exact_f32(kr[S:, None]), exact_f32(k[t, :, 0, h:h + 1]), S + np.arange(T), r, f, "bf16")
    assert pool.last_error() == (0, 0)
