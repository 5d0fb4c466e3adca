"""Calls that are a host thread's first."""
import threading

import numpy as np
import pytest
import torch

from paper_2601_09093_b200 import binding as B

pytestmark = pytest.mark.gpu


def dev(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def calls():
    """name: (call into buffers of its own, what it fills); everything it takes exists already, so that nothing but the call itself
    touches the device in its thread."""
    gen = torch.Generator(device="cuda").manual_seed(1)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda").bfloat16()               # noqa: E731
    pool = B.KVPool(1, 8, 2, 128, 16, num_blocks=64, max_traces=3, max_pages_per_trace=16)
    pool.fork_prefix(3, 100, rand(1, 2, 100, 128), rand(1, 2, 100, 128))
    ids = dev([0, 1, 2])
    pool.append_kv(ids, 9, rand(3, 9, 1, 2, 128), rand(3, 9, 1, 2, 128))
    v = pool.views()
    table, lens, space = v["block_table"], v["seq_lens"], torch.empty(96 << 20, dtype=torch.uint8, device="cuda")
    q, kd, vd, parents = rand(3, 8, 128), rand(3, 1, 1, 2, 128), rand(3, 1, 1, 2, 128), dev([[-1]] * 3)
    rows, pages, start, rotary = dev([0, 3]), dev([6]), dev([100] * 3), B.Rotary(128)
    out, out32, x = torch.zeros_like(q), torch.zeros((3, 8, 128), device="cuda"), rand(5, 8, 128)
    turned, qt = torch.zeros_like(x), torch.zeros((1, 3, 1, 8, 128), dtype=torch.bfloat16, device="cuda")
    out_tree, scores = torch.zeros((3, 1, 8, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros(3, device="cuda")
    w = B.ScorerWeights(rand(128, 256) * 0.1, rand(128), rand(128), 0.1, B.STEP_BF16)
    hidden, mask = rand(3, 256), torch.ones(3, dtype=torch.uint8, device="cuda")
    pool.set_scorer_config(mode=1)
    torch.cuda.synchronize()
    return pool, {
        "decode_attention_groups": (lambda: pool.decode_attention_groups(0, q, table, lens, rows, pages, out=out, workspace=space), out),
        "decode_attention_tree": (lambda: pool.decode_attention_tree(0, q[:, None], kd, vd, parents, table, lens, out=out_tree, workspace=space), out_tree),
        "decode_attention": (lambda: pool.decode_attention(0, q, table, lens, out=out32), out32),
        "rotate_positions": (lambda: B.rotate_positions(x, rotary, out=turned), turned),
        "store_kv_rotated": (lambda: pool.store_kv_rotated(0, ids, start, kd, vd, rotary, q=q[None, :, None], q_out=qt), qt),
        "score_steps": (lambda: pool.score_steps(hidden, mask, None, w, step_scores_out=scores), scores),
    }


def in_a_thread(call):
    wrong = []

    def work():
        try:
            call()
        except B.StepError as e:
            wrong.append(e)

    t = threading.Thread(target=work)
    t.start()
    t.join()
    torch.cuda.synchronize()
    return wrong


NAMES = ["decode_attention_groups", "decode_attention_tree", "decode_attention", "rotate_positions", "store_kv_rotated", "score_steps"]


@pytest.mark.parametrize("name", NAMES)
def test_the_first_call_of_a_host_thread(name):
    """A thread that has made no CUDA call has no context yet; the encoder of tensor maps, the one driver call there is, does not make one."""
    pool, table = calls()
    call, out = table[name]
    for first_in_the_pool in (True, False):
        out.zero_()
        torch.cuda.synchronize()
        assert in_a_thread(call) == [], first_in_the_pool
        got = out.clone()
        out.zero_()
        call()
        assert torch.equal(out, got) and bool((out != 0).any())
    assert pool.last_error() == (0, 0)


def test_a_pool_made_by_a_thread():
    made = []
    storage = {}

    def make():
        storage["pool"] = B.KVPool(1, 4, 2, 128, 16, num_blocks=8, max_traces=2, max_pages_per_trace=4)
        made.append(storage["pool"].last_error())

    assert in_a_thread(make) == [] and made == [(0, 0)]
    pool = storage["pool"]
    gen = torch.Generator(device="cuda").manual_seed(2)
    k, v, q = (torch.randn(s, generator=gen, device="cuda").bfloat16() for s in ((1, 2, 20, 128), (1, 2, 20, 128), (2, 4, 128)))
    pool.fork_prefix(2, 20, k, v)
    w = pool.views()
    out = pool.decode_attention_groups(0, q, w["block_table"], w["seq_lens"], dev([0, 2]), dev([1]))
    p = (torch.einsum("nhgd,hsd->nhgs", q.view(2, 2, 2, 128).double(), k[0].double()) / 128 ** 0.5).softmax(-1)
    want = torch.einsum("nhgs,hsd->nhgd", p, v[0].double()).reshape(2, 4, 128)
    assert np.all((out.double() - want).abs().cpu().numpy() <= 2.0 ** -8 * want.abs().cpu().numpy() + 1e-3)
