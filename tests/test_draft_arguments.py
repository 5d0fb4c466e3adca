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
