"""rotate_positions and store_kv_rotated where values, sizes or tensors are unusual."""
import numpy as np
import pytest
import torch

from oracle import rotary as OR
from paper_2601_09093_b200 import binding as B

from draft_common import FP32_HALF_STEP

pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
# half of the spacing of subnormal numbers
SMALLEST = {"bf16": 2.0 ** -134, "fp32": 2.0 ** -150}


def subnormals(shape, dtype, seed=1):
    """Numbers around the smallest normal one, 2^-126, most of them below it."""
    x = torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64) * 2.0 ** -127
    x = x.to(TYPES[dtype])
    return torch.where(x == 0, torch.full_like(x, 2.0 ** -128), x).cuda()


def off(y, x, positions, f, D, dtype):
    """Steps of the bound: products and their sum are rounded to the spacing of subnormal numbers (three times), cosine and sine as
    elsewhere; then the type's rounding, relative above 2^-126 and absolute below."""
    x, y = x.double().cpu().numpy(), y.double().cpu().numpy()
    want = OR.rotate(x, positions, f, False)
    big = 2 * np.abs(x).max()
    tol = 8 * FP32_HALF_STEP * big + 3 * SMALLEST["fp32"] + (2.0 ** -8 * big + SMALLEST["bf16"] if dtype == "bf16" else 0.0)
    return float((np.abs(y - want) / tol).max())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("heads,d,D", [(32, 128, 128), (2, 64, 32), (3, 22, 6)])
def test_subnormal_values_are_kept(dtype, heads, d, D):
    """Rows of many heads, of few, and pair by pair.  At position 0 nothing is turned: the bits are those that went in."""
    r, f = B.Rotary(D), OR.frequencies(D, 10000.0)
    x = subnormals((9, heads, d), dtype)
    y = B.rotate_positions(x, r)
    assert torch.equal(y[0], x[0])
    assert off(y, x, np.arange(9), f, D, dtype) <= 1.0


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 12])
def test_subnormal_values_are_stored(dtype, D):
    pool = B.KVPool(1, 4, 2, 64, 16, num_blocks=4, max_traces=1, max_pages_per_trace=2, dtype=B.STEP_BF16 if dtype == "bf16" else B.STEP_FP32)
    pool.fork_prefix(1, 0, None, None)
    ids = torch.zeros(1, dtype=torch.int32, device="cuda")
    start = pool.extend(ids, 5)
    k, v, q = subnormals((1, 5, 1, 2, 64), dtype), subnormals((1, 5, 1, 2, 64), dtype, 2), subnormals((1, 1, 5, 4, 64), dtype, 3)
    r, f = B.Rotary(D), OR.frequencies(D, 10000.0)
    qo = pool.store_kv_rotated(0, ids, start, k, v, r, q=q)
    assert torch.equal(qo[0, 0, 0], q[0, 0, 0]) and off(qo[0, 0], q[0, 0], np.arange(5), f, D, dtype) <= 1.0
    for h in range(2):
        kr, vr = pool.read_kv(0, h, pool.views()["block_table"][0], 5)
        assert torch.equal(kr[0], k[0, 0, 0, h]) and torch.equal(vr, v[0, :, 0, h])
        assert off(kr[:, None], k[0, :, 0, h:h + 1], np.arange(5), f, D, dtype) <= 1.0
    assert pool.last_error() == (0, 0)


def test_a_tensor_that_wants_a_gradient_is_refused_while_torch_records():
    """The result would be cut off from x without a word; turned in place, x would change behind torch's back."""
    r = B.Rotary(64)
    x = torch.randn((3, 2, 64), generator=torch.Generator().manual_seed(7)).cuda()
    want = B.rotate_positions(x, r)
    leaf = x.clone().requires_grad_()
    for a, kw in ((leaf, {}), (leaf * 1.0, {}), (leaf, dict(out=torch.empty_like(x))), (x, dict(out=leaf)), (leaf, dict(out=leaf)),
                  (leaf, dict(stream=torch.cuda.Stream()))):
        with pytest.raises(B.StepError) as e:
            B.rotate_positions(a, r, **kw)
        assert e.value.code == 1
    assert torch.equal(leaf, x)
    assert torch.equal(B.rotate_positions(leaf.detach(), r), want)
    with torch.no_grad():
        assert torch.equal(B.rotate_positions(leaf, r), want)

    class Rotate(torch.autograd.Function):                              # as a training loop has it
        @staticmethod
        def forward(ctx, a):
            return B.rotate_positions(a, r)

        @staticmethod
        def backward(ctx, g):
            return B.rotate_positions(g.contiguous(), r, transpose=True)

    y = Rotate.apply(leaf)
    assert torch.equal(y, want)
    w = torch.randn((3, 2, 64), generator=torch.Generator().manual_seed(8)).cuda()
    (y * w).sum().backward()
    assert torch.equal(leaf.grad, B.rotate_positions(w, r, transpose=True))


@pytest.mark.parametrize("heads,d,D", [(63, 273_000_016, 16), (4, 1 << 20, 64), (64, 600_000, 32)])
def test_dims_that_are_copied_by_the_billion(heads, d, D):
    """63 heads of 34 million chunks of 16 bytes: more of them in one row than 31 bits count.  (One head of x serves as all.)"""
    r = B.Rotary(D)
    x = torch.empty((1, 1, 1, d), dtype=torch.bfloat16, device="cuda")
    x.view(torch.int16).copy_((torch.arange(d, dtype=torch.int32, device="cuda") * 40503 >> 3).to(torch.int16) & 0x3fff)
    out = torch.zeros((1, 1, heads, d), dtype=torch.bfloat16, device="cuda")
    p = torch.full((1,), 77, dtype=torch.int32, device="cuda")
    assert B.rotate_positions(x.expand(1, 1, heads, d), r, p, out=out) is out
    turned = B.rotate_positions(x[..., :D].contiguous(), r, p)
    for h in range(heads):
        assert torch.equal(out[0, 0, h, D:], x[0, 0, 0, D:]) and torch.equal(out[0, 0, h, :D], turned[0, 0, 0]), h


def test_results_that_share_a_place_are_refused():
    r = B.Rotary(64)
    x = torch.randn((2, 3, 4, 64), generator=torch.Generator().manual_seed(9)).cuda()
    keep = x.clone()
    flat = x.view(-1)
    for a, out in ((x, torch.zeros((2, 3, 1, 64), device="cuda").expand_as(x)), (x, torch.zeros((3, 4, 64), device="cuda").expand_as(x)),
                   (x, flat.as_strided((2, 3, 4, 64), (768, 64, 192, 1))), (x[:1].expand_as(x), x[:1].expand_as(x))):
        with pytest.raises(B.StepError) as e:
            B.rotate_positions(a, r, out=out)
        assert e.value.code == 1
    assert torch.equal(x, keep)
    # dims of one: a stride that is not used may be anything
    assert torch.equal(B.rotate_positions(x[:1, :1], r, out=x[:1, :1].clone().as_strided((1, 1, 4, 64), (0, 0, 64, 1))), x[:1, :1])

    pool = B.KVPool(2, 4, 2, 64, 16, num_blocks=4, max_traces=2, max_pages_per_trace=1, dtype=B.STEP_FP32)
    pool.fork_prefix(2, 0, None, None)
    ids = torch.arange(2, dtype=torch.int32, device="cuda")
    with pytest.raises(B.StepError):
        pool.extend(ids, 3, start_out=ids)
    start = pool.extend(ids, 3)
    k = torch.randn((2, 3, 2, 2, 64), generator=torch.Generator().manual_seed(10)).cuda()
    q = torch.randn((2, 2, 3, 4, 64), generator=torch.Generator().manual_seed(11)).cuda()
    before = q.clone()
    for out in (torch.zeros((1, 2, 3, 4, 64), device="cuda").expand_as(q), torch.zeros((2, 1, 1, 4, 64), device="cuda").expand_as(q),
                q.view(-1).as_strided(q.shape, (256, 3 * 512, 512, 64, 1))):
        with pytest.raises(B.StepError) as e:
            pool.store_kv_rotated(0, ids, start, k, k, r, q=q, q_out=out)
        assert e.value.code == 1
    assert torch.equal(q, before) and ids.tolist() == [0, 1]
    pool.store_kv_rotated(0, ids, start, k, k, r, q=q, q_out=q)
    assert pool.last_error() == (0, 0)
