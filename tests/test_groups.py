"""Argument checks of decode_attention_groups that need no GPU."""
import ctypes as C
import types

import pytest
import torch

from paper_2601_09093_b200 import binding as B


def test_no_pool_is_refused():
    L, b = B.lib(), C.c_size_t()
    assert L.decode_attention_groups_workspace_bytes(None, 1, 1, C.byref(b)) == 1
    assert L.decode_attention_groups(None, 0, None, None, None, 1, None, None, 0, None, None, 0, None) == 1


def test_the_binding_refuses_what_does_not_fit():
    def reached(*args, **kwargs):
        raise AssertionError("the library was called")
    pool = types.SimpleNamespace(_device=lambda: torch.device("cpu"), num_layers=2, num_q_heads=4, num_kv_heads=2, head_dim=8, page_size=4,
                                 max_pages_per_trace=5, torch_dtype=torch.float32, _call=reached)
    pool._empty = lambda shape, dtype, stream: torch.empty(shape, dtype=dtype)
    ints = lambda *shape: torch.zeros(shape, dtype=torch.int32)                                  # noqa: E731
    ok = dict(layer=1, q=torch.zeros(3, 4, 8), block_table=ints(3, 5), seq_lens=ints(3), group_rows=ints(3), group_pages=ints(2))
    for good in ({}, dict(group_rows=None, group_pages=None), dict(group_rows=ints(1), group_pages=ints(0))):
        with pytest.raises(AssertionError):
            B.KVPool.decode_attention_groups(pool, **{**ok, **good})
    for change in (dict(layer=2), dict(layer=-1), dict(layer=1 << 32), dict(q=torch.zeros(3, 4, 8).bfloat16()), dict(q=torch.zeros(3, 2, 8)), dict(q=torch.zeros(4, 8)),
                   dict(q=torch.zeros(3, 8, 4).transpose(1, 2)), dict(block_table=ints(2, 5)), dict(block_table=ints(3, 6)), dict(seq_lens=ints(2)),
                   dict(seq_lens=ints(3).long()), dict(group_rows=ints(2)), dict(group_rows=None), dict(group_pages=None), dict(group_pages=ints(2).long()),
                   dict(group_rows=ints(6)[::2]), dict(out=torch.zeros(3, 4, 4)), dict(out=torch.zeros(3, 4, 8).double())):
        with pytest.raises(B.StepError) as e:
            B.KVPool.decode_attention_groups(pool, **{**ok, **change})
        assert e.value.code == 1, change
