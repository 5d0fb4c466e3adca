"""Argument checks of the draft and bounded-cache calls that need no GPU."""
import ctypes as C

import types

import pytest
import torch

from paper_2601_09093_b200 import binding as B


@pytest.fixture(scope="module")
def lib():
    return B.lib()


def test_no_pool_is_refused(lib):
    b = C.c_size_t()
    assert lib.decode_attention_tree_workspace_bytes(None, 1, 1, C.byref(b)) == 1
    assert lib.decode_attention_weights_workspace_bytes(None, 1, 1, C.byref(b)) == 1
    assert lib.kv_pool_evict_workspace_bytes(None, 1, 1, C.byref(b)) == 1
    assert lib.decode_attention_tree(None, 0, None, None, None, None, None, 1, None, None, 1, None, None, 0, None) == 1
    assert lib.append_kv_path(None, None, 1, 1, None, None, None, None, 1, None) == 1
    assert lib.decode_attention_weights(None, 0, None, None, None, 1, None, None, 1, None, 0, None) == 1
    assert lib.kv_pool_evict_positions(None, None, 1, None, None, 1, 1, 0, None, None, 0, None) == 1


def test_a_stream_of_another_device_is_refused():
    """Work on it would not be ordered by it: the call's kernels run on the pool's device."""
    pool = types.SimpleNamespace(_device=lambda: torch.device("cuda", 0))
    with pytest.raises(B.StepError) as e:
        B.KVPool._call(pool, "append_kv_path", (), stream=types.SimpleNamespace(device=torch.device("cuda", 1)))
    assert e.value.code == 1


def bare_pool(device="cpu"):
    """What the binding's own checks look at, without a GPU; a call that gets past them fails."""
    def reached(*args, **kwargs):
        raise AssertionError("the library was called")
    dev = torch.device(device)
    pool = types.SimpleNamespace(_device=lambda: dev, num_layers=2, num_q_heads=4, num_kv_heads=2, head_dim=8, page_size=4,
                                 max_pages_per_trace=5, torch_dtype=torch.float32, _call=reached)
    pool._empty = lambda shape, dtype, stream: torch.empty(shape, dtype=dtype, device=dev)
    return pool


@pytest.mark.parametrize("budget,recent", [(0, 0), (21, 1), (-3, 0), (10, 11), (10, -1), (10, (1 << 32) + 4), ((1 << 32) + 10, 4),
                                           (1 << 40, 0), (1 << 70, 0), (10, 1 << 70)])
def test_a_budget_that_the_pool_cannot_have_is_refused_before_anything_is_made(budget, recent):
    """Also numbers that 32 bits would cut down to good ones, and those for which kept_out would not fit any memory."""
    ids, w = torch.zeros(3, dtype=torch.int32), torch.zeros((2, 3, 2, 20))
    with pytest.raises(B.StepError) as e:
        B.KVPool.evict_positions(bare_pool(), ids, w, budget, recent)
    assert e.value.code == 1


@pytest.mark.parametrize("layer", [-1, 2, 1 << 32, (1 << 32) + 1])
def test_a_layer_that_the_pool_does_not_have_is_refused(layer):
    q, kd = torch.zeros((1, 1, 4, 8)), torch.zeros((1, 1, 2, 2, 8))
    table, lens = torch.zeros((1, 5), dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(B.StepError) as e:
        B.KVPool.decode_attention_tree(bare_pool(), layer, q, kd, kd, torch.zeros((1, 1), dtype=torch.int32), table, lens)
    assert e.value.code == 1
    with pytest.raises(B.StepError) as e:
        B.KVPool.decode_attention_weights(bare_pool(), layer, q[:, 0], table, lens, torch.zeros((1, 2, 20)))
    assert e.value.code == 1


def test_rows_longer_than_32_bits_count_are_refused():
    pool, wide = bare_pool("meta"), (1 << 32) + 20
    ints = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="meta")                   # noqa: E731
    floats = lambda *shape: torch.zeros(shape, device="meta")                                    # noqa: E731
    for call in (lambda: B.KVPool.evict_positions(pool, ints(1), floats(2, 1, 2, wide), 10, 4, kept_out=ints(2, 1, 2, 10)),
                 lambda: B.KVPool.decode_attention_weights(pool, 0, floats(1, 4, 8), ints(1, 5), ints(1), floats(1, 2, wide)),
                 lambda: B.KVPool.append_kv_path(pool, ints(1), floats(1, 3, 2, 2, 8), floats(1, 3, 2, 2, 8), ints(1, wide), ints(1)),
                 lambda: B.KVPool.append_kv_path(pool, ints(1), floats(1, wide, 2, 2, 8), floats(1, wide, 2, 2, 8), ints(1, 2), ints(1))):
        with pytest.raises(B.StepError) as e:
            call()
        assert e.value.code == 1
