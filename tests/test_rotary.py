"""Rotary positions without a GPU: the frequency table, argument checks, and pins of the oracle."""
import ctypes as C
import math
import types

import numpy as np
import pytest
import torch

from oracle import attention as OA
from oracle import rotary as OR
from oracle.kv_pool import KVPoolOracle
from paper_2601_09093_b200 import binding as B

SCALINGS = [dict(), dict(scaling="linear", factor=8.0), dict(scaling="base", factor=4.0),
            dict(scaling="yarn", factor=4.0, original_positions=32768), dict(scaling="yarn", factor=40.0, original_positions=4096, fast=32.0, slow=1.0),
            dict(scaling="bands", factor=8.0, original_positions=8192), dict(scaling="bands", factor=32.0, original_positions=8192, fast=6.0, slow=2.0)]


@pytest.mark.parametrize("D,base", [(128, 1e6), (64, 10000.0), (2, 10000.0), (20, 500000.0), (512, 1e7)])
@pytest.mark.parametrize("kw", SCALINGS)
def test_table(D, base, kw):
    """The table's entries are the frequencies in turns, to a unit of 2^-64 and the rounding of extended precision."""
    if kw.get("scaling") == "base" and D == 2:
        with pytest.raises(B.StepError):
            B.Rotary(D, base, device="cpu", **kw)
        return
    r = B.Rotary(D, base, device="cpu", **kw)
    f = OR.frequencies(D, base, **kw)
    got = r.table.numpy().view(np.uint64).astype(OR.LD) / OR.LD(2) ** 64
    # 1: the unit; the logarithm of the base (up to 19) and the quotient 2i / D lose some half steps of 2^-64 in the exponent;
    # the stretching's borders are computed in 64 bits by the oracle, but are whole numbers
    assert np.all(np.abs(got - f / OR.TWO_PI) <= 2.0 ** -64 + f * 100 * 2.0 ** -64)
    assert r.struct.rotary_dim == D and r.struct.scale == np.float32(OR.output_scale(kw.get("scaling"), kw.get("factor", 1.0)))


def test_table_by_hand():
    r = B.Rotary(4, base=100.0, device="cpu")                          # frequencies 1 and 0.1
    assert [int(x) & (2 ** 64 - 1) for x in r.table] == [int(OR.LD(2) ** 64 / OR.TWO_PI + OR.LD(0.5)), int(OR.LD(2) ** 64 / OR.TWO_PI / 10 + OR.LD(0.5))]
    # a divisor below one can take a frequency beyond a turn per position: whole turns do not matter
    q = B.Rotary(2, divisors=[0.1], device="cpu")
    assert abs(int(q.table[0]) / 2.0 ** 64 % 1 - (10 / (2 * math.pi) - 1)) < 1e-15
    assert B.Rotary(4, divisors=[1.0, 1.0], output_scale=0.5, device="cpu").struct.scale == 0.5


def test_stretching_leaves_fast_pairs_and_slows_slow_ones():
    for kw in SCALINGS[3:]:
        f, t = OR.frequencies(128, 1e6, **kw), OR.frequencies(128, 1e6)
        assert f[0] == t[0] and abs(f[-1] * kw["factor"] / t[-1] - 1) < 1e-15
        assert np.all(np.diff(f) < 0)


def test_only_differences_of_positions_matter():
    rng = np.random.default_rng(0)
    q, k = rng.standard_normal((2, 1, 1, 16))
    for interleaved in (False, True):
        f = OR.frequencies(12, 1e4)
        dots = [np.sum(OR.rotate(q, [p], f, interleaved) * OR.rotate(k, [p - 7], f, interleaved)) for p in (7, 100, 1 << 30)]
        np.testing.assert_allclose(dots, dots[0], rtol=1e-9)


def test_rotation_by_hand_and_transposed():
    x = np.array([[1.0, 0.0, 0.0, 2.0, 9.0]])                          # D = 4: halves pair (0, 2), (1, 3)
    f = np.array([math.pi / 2, math.pi])
    np.testing.assert_allclose(OR.rotate(x, 1, f, False), [[0, 0, 1, -2, 9]], atol=1e-15)
    np.testing.assert_allclose(OR.rotate(x, 1, f, True), [[0, 1, 0, -2, 9]], atol=1e-15)
    y = OR.rotate(np.array([[3.0, 4.0]]), 5, np.array([0.3]), True, scale=2.0)
    assert abs(np.hypot(*y[0]) - 10) < 1e-12
    # the transposed rotation gives the gradient: d(w . y)/dx by central differences
    rng = np.random.default_rng(1)
    x, w = rng.standard_normal((2, 3, 8))
    f = OR.frequencies(6, 100.0)
    g = OR.rotate(w, 11, f, False, 1.5, transpose=True)
    for h in range(3):
        for c in range(8):
            d = np.zeros_like(x)
            d[h, c] = 1e-6
            num = np.sum(w * (OR.rotate(x + d, 11, f, False, 1.5) - OR.rotate(x - d, 11, f, False, 1.5))) / 2e-6
            # dims behind D are copied, whatever the scale
            assert abs(num - g[h, c]) < 1e-8


def test_extend_and_store_is_append():
    rng = np.random.default_rng(3)
    pools = [KVPoolOracle(3, 2, 4, 4, 30, 4, 6) for _ in range(2)]
    k, v = rng.standard_normal((2, 3, 5, 3, 2, 4))
    for p in pools:
        p.fork_prefix(3, 3, *rng.standard_normal((2, 3, 2, 3, 4)))
    pools[1].k_pages[:], pools[1].v_pages[:] = pools[0].k_pages, pools[0].v_pages
    pools[0].append_kv([2, 0, 1], 5, k, v)
    start = OR.extend(pools[1], [2, 0, 1], 5)
    assert start.tolist() == [3, 3, 3]
    for l in range(3):
        assert OR.store(pools[1], l, [2, 0, 1], start, k[:, :, l:l + 1], v[:, :, l:l + 1]) == [0, 1, 2]
    for t in range(3):
        for a, b in zip(OA.gather_trace_kv(pools[0].k_pages[1], pools[0].v_pages[1], pools[0].block_table[t], 8),
                        OA.gather_trace_kv(pools[1].k_pages[1], pools[1].v_pages[1], pools[1].block_table[t], 8)):
            np.testing.assert_array_equal(a, b)
    assert OR.extend(pools[1], [0, 0, 7, 3], 1).tolist() == [8, -1, -1, -1] and pools[1].status == 1 << 3


@pytest.mark.parametrize("kw", [dict(rotary_dim=0), dict(rotary_dim=3), dict(rotary_dim=-2), dict(rotary_dim=(1 << 32) + 8), dict(base=1.0), dict(base=0.0),
                                dict(base=float("nan")), dict(base=float("inf")), dict(scaling="linear", factor=0.0), dict(scaling="linear", factor=float("nan")),
                                dict(scaling="what"), dict(scaling="yarn", factor=4.0), dict(scaling="bands", factor=4.0, original_positions=-1),
                                dict(scaling="yarn", factor=4.0, original_positions=100, fast=1.0, slow=1.0), dict(scaling="bands", factor=2.0, original_positions=100, slow=0.0),
                                dict(divisors=[1.0]), dict(divisors=[1.0, 0.0, 1.0, 1.0]), dict(divisors=[1.0, 1.0, float("nan"), 1.0]),
                                dict(output_scale=-1.0), dict(output_scale=float("inf"))])
def test_a_rotary_that_cannot_be_is_refused(kw):
    with pytest.raises(B.StepError) as e:
        B.Rotary(**{**dict(rotary_dim=8), **kw}, device="cpu")
    assert e.value.code == 1


def test_the_library_refuses_without_looking_at_the_device():
    L = B.lib()
    r = B.Rotary(8, device="cpu")
    a = B.rotate_args(head_dim=8, batch=1, rows=1, heads=1)
    call = lambda args, rot: L.rotate_positions(C.byref(args), C.byref(rot), None)                  # noqa: E731
    assert L.rotate_positions(None, C.byref(r.struct), None) == 1 and L.rotate_positions(C.byref(a), None, None) == 1
    assert call(a, r.struct) == 1                                       # no x
    assert call(B.rotate_args(head_dim=8, batch=0, rows=1, heads=1), r.struct) == 0
    some = torch.zeros(64)
    for change in (dict(batch=-1), dict(rows=-1), dict(heads=-1), dict(head_dim=0), dict(head_dim=6), dict(dtype=2), dict(transpose=2),
                   dict(x=some.data_ptr() + 1), dict(out=some.data_ptr() + 2), dict(positions=some.data_ptr() + 1)):
        args = dict(x=some.data_ptr(), out=some.data_ptr(), dtype=1, batch=1, rows=1, heads=1, head_dim=8)
        assert call(B.rotate_args(**{**args, **change}), r.struct) == 1, change
    for change in (dict(table=None), dict(rotary_dim=7), dict(rotary_dim=0), dict(rotary_dim=10), dict(interleaved=2), dict(scale=float("nan"))):
        rot = B.step_rotary(r.struct.table, 8, 0, 1.0)
        for k, v in change.items():
            setattr(rot, k, v)
        assert call(B.rotate_args(x=some.data_ptr(), out=some.data_ptr(), dtype=1, batch=1, rows=1, heads=1, head_dim=8), rot) == 1, change
    assert L.store_kv_rotated(None, C.byref(B.kv_store_args(n_layers=1)), C.byref(r.struct), None) == 1
    assert L.kv_pool_extend(None, None, 1, 1, None, None) == 1


def test_tensors_that_are_not_on_a_gpu_are_refused():
    with pytest.raises(B.StepError) as e:
        B.rotate_positions(torch.zeros(2, 3, 8), B.Rotary(8, device="cpu"))
    assert e.value.code == 1


def bare_pool():
    def reached(*args, **kwargs):
        raise AssertionError("the library was called")
    pool = types.SimpleNamespace(_device=lambda: torch.device("cpu"), num_layers=3, num_q_heads=4, num_kv_heads=2, head_dim=8,
                                 torch_dtype=torch.float32, _call=reached)
    pool._empty = lambda shape, dtype, stream: torch.empty(shape, dtype=dtype)
    return pool


def test_the_binding_refuses_what_does_not_fit():
    r = B.Rotary(8, device="cpu")
    ints = lambda *shape: torch.zeros(shape, dtype=torch.int32)                                  # noqa: E731
    rows = lambda n=3, T=2, L=2, H=2, d=8: torch.zeros((n, T, L, H, d))                             # noqa: E731
    q = lambda L=2, n=3, T=2, H=4, d=8: torch.zeros((L, n, T, H, d))                              # noqa: E731
    ok = dict(layer0=1, trace_ids=ints(3), start=ints(3), k=rows(), v=rows(), rotary=r, q=q(), q_out=q())
    with pytest.raises(AssertionError):
        B.KVPool.store_kv_rotated(bare_pool(), **ok)
    wide = torch.zeros((3, 3, 2, 2, 8))[:, :2]                          # rows with a gap between entries
    for change in (dict(layer0=2), dict(layer0=-1), dict(layer0=3), dict(layer0=(1 << 32) + 1), dict(trace_ids=ints(2)), dict(start=ints(4)),
                   dict(start=ints(3).long()), dict(positions=ints(2)), dict(k=rows(L=1)), dict(v=rows(T=1)), dict(k=rows().double()), dict(k=rows()[0]),
                   dict(k=wide), dict(v=wide), dict(q=q(L=1)), dict(q=q(H=2)), dict(q=q(n=2)), dict(q_out=q().bfloat16()), dict(q=None),
                   dict(q=torch.zeros((2, 3, 2, 8, 4)).transpose(3, 4)), dict(rotary=B.Rotary(10, device="cpu"))):
        with pytest.raises(B.StepError) as e:
            B.KVPool.store_kv_rotated(bare_pool(), **{**ok, **change})
        assert e.value.code == 1, change
    for args in ((ints(3).long(), 1), (ints(3, 1), 1), (ints(3), -1), (ints(3), 1 << 32), (ints(3), 1, ints(2))):
        with pytest.raises(B.StepError) as e:
            B.KVPool.extend(bare_pool(), *args)
        assert e.value.code == 1


def test_struct_layouts_match_the_binding(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = ["step_rotary_config", "step_rotary", "rotate_args", "kv_store_args"]
    lines = ['#include <stdio.h>', '#include <stddef.h>', '#include "step.h"', "int main(void) {"]
    for s in names:
        lines.append('  printf("%s %%zu\\n", sizeof(%s));' % (s, s))
        lines += ['  printf("%s.%s %%zu\\n", offsetof(%s, %s));' % (s, f, s, f) for f, _ in getattr(B, s)._fields_]
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["  return 0;", "}"]))
    subprocess.run(["gcc", "-std=c99", "-pedantic", "-Wall", "-Werror", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    out = dict(line.split() for line in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.splitlines())
    for s in names:
        cls = getattr(B, s)
        assert int(out[s]) == C.sizeof(cls), s
        for f, _ in cls._fields_:
            assert int(out["%s.%s" % (s, f)]) == getattr(cls, f).offset, (s, f)
