"""Rotary positions without a GPU: frequencies and scales at the ends of their ranges."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import rotary as OR
from paper_2601_09093_b200 import binding as B


@pytest.mark.parametrize("kw", [dict(divisors=[1e-300, 1.0]), dict(divisors=[1.0, 1e-20]), dict(divisors=[1.0, 1e-8]), dict(scaling="linear", factor=1e-12),
                                dict(scaling="base", factor=1e-30), dict(output_scale=1e39), dict(output_scale=1.7e308)])
def test_what_a_table_cannot_hold_is_refused(kw):
    """Turns per position whose fraction extended precision has lost came out as no rotation at all; a scale that is no float made
    a rotary that every call refused."""
    with pytest.raises(B.StepError) as e:
        B.Rotary(4, device="cpu", **kw)
    assert e.value.code == 1


def test_fast_frequencies_are_as_good_as_said():
    """2^-60 of the turns a position, below the limit of 2^16 of them."""
    for divisors in ([0.01, 3e-4], [2.5e-6, 1.0], [1.0, 2.43e-8]):
        f = OR.frequencies(4, 10000.0, divisors=divisors)
        turns = f / OR.TWO_PI
        assert 1 < turns.max() < 2 ** 16
        got = B.Rotary(4, divisors=divisors, device="cpu").table.numpy().view(np.uint64).astype(OR.LD) / OR.LD(2) ** 64
        gap = np.abs(got - (turns - np.floor(turns)))
        # the oracle's own quotients are off by as much
        assert np.all(np.minimum(gap, 1 - gap) <= 2.0 ** -64 + 2 * turns * 2.0 ** -60)


def test_the_largest_scale_that_is_a_float():
    assert B.Rotary(4, output_scale=3e38, device="cpu").struct.scale == np.float32(3e38)


def test_results_that_share_a_place_are_refused():
    """Before the device is looked at: rows, heads or batch entries of out in one place, x turned in place by other strides."""
    r = B.Rotary(8, device="cpu")
    some, other = torch.zeros(4096), torch.zeros(4096)
    base = dict(x=some.data_ptr(), out=other.data_ptr(), dtype=1, batch=2, rows=3, heads=4, head_dim=8,
                x_batch=96, x_row=32, x_head=8, out_batch=96, out_row=32, out_head=8)
    for change in (dict(out_batch=0), dict(out_row=0), dict(out_head=0),
                   dict(out=some.data_ptr(), out_batch=128), dict(out=some.data_ptr(), out_row=40), dict(x=other.data_ptr(), x_head=0)):
        assert B.lib().rotate_positions(C.byref(B.rotate_args(**{**base, **change})), C.byref(r.struct), None) == 1, change
