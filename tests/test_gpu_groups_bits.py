"""decode_attention_groups to the last bits of its output: against torch in 64 bits, element by element."""
import math
import os
import threading

import numpy as np
import pytest
import torch

from paper_2601_09093_b200 import binding as B
from paper_2601_09093_b200 import harness as H

from draft_common import BF16_HALF_STEP, FP32_HALF_STEP

pytestmark = pytest.mark.gpu

# What a probability loses on its way into the second product of bf16 pools, relative to itself: it goes in two bf16 parts, of which the
# second, at most 2^-7 + 2^-10 of it, is rounded.
SPLIT = BF16_HALF_STEP * (2.0 ** -7 + 2.0 ** -10)
TYPES = {"bf16": (B.STEP_BF16, torch.bfloat16), "fp32": (B.STEP_FP32, torch.float32)}


def dev(x):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).cuda()


class Forks:
    """A pool of traces forked from several prompts, and every trace's rows in the order they went in."""

    def __init__(self, heads, dtype, page, problems, make, rng, spare=8):
        Hq, Hkv, d = heads
        own = np.concatenate([np.asarray(o) for _, o in problems])
        n, dt = len(own), TYPES[dtype][1]
        blocks = sum(p // page + sum((p % page + int(x)) // page + 2 for x in o) for p, o in problems) + spare
        most = max(p + int(max(o)) for p, o in problems) // page + 1
        self.pool = B.KVPool(1, Hq, Hkv, d, page, num_blocks=blocks, max_traces=n, max_pages_per_trace=most, dtype=TYPES[dtype][0])
        self.views, self.dtype, self.n = self.pool.views(), dtype, n
        self.views["free_list"].copy_(torch.from_numpy(rng.permutation(blocks).astype(np.int32)))
        self.pool.kv_storage.fill_(255)                                # NaN wherever nothing is stored
        kv = [[[], []] for _ in range(n)]
        t = 0
        for p, o in problems:
            k, v = (make(p, Hkv, d).to(dt) for _ in range(2))
            self.pool.fork_prefix(len(o), p, *(x.transpose(0, 1)[None].contiguous() for x in (k, v)))
            for i in range(t, t + len(o)):
                kv[i][0].append(k)
                kv[i][1].append(v)
            t += len(o)
        for sel, inc in H.ragged_append_plan(own):
            k, v = (make(len(sel) * inc, Hkv, d).to(dt).view(len(sel), inc, 1, Hkv, d) for _ in range(2))
            self.pool.append_kv(dev(sel), inc, k, v)
            for j, i in enumerate(sel):
                kv[i][0].append(k[j, :, 0])
                kv[i][1].append(v[j, :, 0])
        self.kv = kv
        self.rows = dev(np.cumsum([0] + [len(o) for _, o in problems]))

    def attend(self, q, pages):
        return self.pool.decode_attention_groups(0, q, self.views["block_table"], self.views["seq_lens"], self.rows, dev(pages))

    def check(self, got, q, ended=(), without=slice(0, 0)):
        """A weight is off by the errors of its score (a product of d terms, each of whose additions may lose a step; three roundings of a
        value up to the largest score; the exponential, 2 steps) in numerator and denominator and by a step per key in the sums, as
        draft_common.relative_bound has it; by SPLIT besides, in bf16 pools.  The output is rounded once.  without: positions that the
        oracle leaves out."""
        half = BF16_HALF_STEP if self.dtype == "bf16" else FP32_HALF_STEP
        worst = 0.0
        for i in range(self.n):
            if i in ended:
                assert (got[i] == 0).all(), i
                continue
            K, V = (torch.cat(x).double() for x in self.kv[i])
            S, Hkv, d = K.shape
            if S == 0:
                assert (got[i] == 0).all(), i
                continue
            keep = torch.ones(S, dtype=torch.bool, device="cuda")
            keep[without] = False
            K, V = K[keep], V[keep]
            x = q[i].double().view(Hkv, -1, d)
            K, V = K.transpose(0, 1), V.transpose(0, 1)
            p = (x @ K.transpose(1, 2) / math.sqrt(d)).softmax(-1)
            size = (x.abs() @ K.abs().transpose(1, 2)).max() / math.sqrt(d)
            slack = 2 * (d + 3) * FP32_HALF_STEP * size + 8 * FP32_HALF_STEP
            off = 2 * slack + 2 * (S + 8) * 2 * FP32_HALF_STEP + (SPLIT if self.dtype == "bf16" else 0.0)
            want, tol = p @ V, off * (p @ V.abs())
            tol = tol + half * (want.abs() + tol) + 1e-30
            worst = max(worst, float(((got[i].double().view(want.shape) - want).abs() / tol).max()))
        assert worst <= 1.0, worst                                     # (in steps of the bound)


def normal(seed, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return lambda *shape: torch.randn(shape, generator=gen, device="cuda") * scale


@pytest.mark.parametrize("G", [1, 4, 5, 8, 12, 16])
@pytest.mark.parametrize("per", [1, 2, 40])
def test_probabilities_are_not_rounded_to_the_values_type(G, per):
    """Scores close to one another: every weight is a little below one of its row, where bf16 has steps of 2^-8, and the bound on
    everything else is small.  Shared pages with row blocks of one chain and of two, own pages, rows beyond the first eight."""
    rng = np.random.default_rng(G)
    make = normal(G)
    f = Forks((2 * G, 2, 128), "bf16", 16, [(160, rng.integers(0, 60, per)), (16, [100, 3])], make, rng)
    q = (make(f.n, 2 * G, 128) * 2.0 ** -5).bfloat16()
    f.check(f.attend(q, [10, 1]), q)
    assert f.pool.last_error() == (0, 0)


def test_one_weight_against_many():
    """One key's weight is 1, that of 111 others 1 - 2^-9, halfway between two bf16 numbers; values that cancel: what is left of the
    output is what the weights' last bits make it."""
    S, d = 112, 128
    score = math.log1p(-2.0 ** -9)
    k, v = torch.zeros((1, 1, S, d), device="cuda"), torch.ones((1, 1, S, d), device="cuda")
    k[0, 0, 1:, 0] = 1.0
    v[0, 0, 0] = -(S - 1)
    k, v = k.bfloat16(), v.bfloat16()
    q = torch.zeros((3, 4, d), device="cuda")
    q[..., 0] = score * math.sqrt(d)
    q = q.bfloat16()
    for shared in (0, 7):
        pool = B.KVPool(1, 4, 1, d, 16, num_blocks=16, max_traces=3, max_pages_per_trace=8)
        pool.fork_prefix(3, S, k, v)
        w = pool.views()
        out = pool.decode_attention_groups(0, q, w["block_table"], w["seq_lens"], dev([0, 3]), dev([shared])).double()
        p = (q.double() @ k[0, 0].double().T / math.sqrt(d)).softmax(-1)
        want, mag = p @ v[0, 0].double(), p @ v[0, 0].double().abs()
        # scores are below 2^-8: fp32 errors of a weight are 8 half steps of its exponential and those of the sums
        tol = mag * (SPLIT + (16 + 4 * (S + 8)) * FP32_HALF_STEP)
        assert ((out - want).abs() <= tol + BF16_HALF_STEP * (want.abs() + tol)).all(), shared


def test_an_infinite_value_keeps_its_sign():
    """Both parts of a probability are positive: an infinity in V times either is that infinity."""
    make = normal(3)
    rng = np.random.default_rng(3)
    for G in (4, 16):
        f = Forks((G, 1, 128), "bf16", 16, [(64, [5, 0, 20])], make, rng)
        kv = f.pool.kv_storage.view(torch.bfloat16).view(1, -1, 1, 2, 16, 128)
        q = make(3, G, 128).bfloat16()
        clean = f.attend(q, [4])
        for page, rows in ((1, [0, 1, 2]), (4, [2])):                  # a shared page, trace 2's first own page
            for sign in (float("inf"), -float("inf")):
                block = int(f.views["block_table"][2, page])
                keep = kv[0, block, 0, 1, 3].clone()
                kv[0, block, 0, 1, 3] = sign
                got = f.attend(q, [4])
                kv[0, block, 0, 1, 3] = keep
                rest = [i for i in range(3) if i not in rows]
                assert (got[rows] == sign).all() and torch.equal(got[rest], clean[rest]), (G, page, sign)
        assert torch.equal(f.attend(q, [4]), clean)


def test_the_bound_would_show_a_page_that_is_left_out():
    """The oracle without 16 of 6000 positions, of the prompt or of an own text: the right results are far outside the bound."""
    rng = np.random.default_rng(1)
    make = normal(1)
    f = Forks((8, 2, 128), "bf16", 16, [(5500, [600, 0, 33])], make, rng)
    q = make(3, 8, 128).bfloat16()
    got = f.attend(q, [343])
    f.check(got, q)
    for first in (0, 2560, 5472, 5600):
        with pytest.raises(AssertionError):
            f.check(got, q, without=slice(first, first + 16))


def test_first_calls_of_several_host_threads_at_once():
    """Threads that meet in a new pool's first call, each with a stream, a workspace and an output of its own; every other one attends with
    a tree of one drafted token first, whose kernel reads the pool through the same description."""
    rng = np.random.default_rng(2)
    make = normal(2)
    n_threads, wrong = 8, []
    for turn in range(12):
        f = Forks((8, 2, 128), "bf16", 16, [(200, [5, 40]), (33, [3])], make, rng)
        q = make(f.n, 8, 128).bfloat16()
        kd = make(f.n, 1, 1, 2, 128).bfloat16()
        parents = torch.full((f.n, 1), -1, dtype=torch.int32, device="cuda")
        pages, spaces = dev([12, 2]), [torch.empty(96 << 20, dtype=torch.uint8, device="cuda") for _ in range(n_threads)]
        outs = [torch.zeros_like(q) for _ in range(n_threads)]
        streams = [torch.cuda.Stream() for _ in range(n_threads)]
        meet = threading.Barrier(n_threads)
        torch.cuda.synchronize()

        def work(i):
            try:
                table, lens = f.views["block_table"], f.views["seq_lens"]
                meet.wait(20)
                if i % 2:
                    f.pool.decode_attention_tree(0, q[:, None], kd, kd, parents, table, lens, workspace=spaces[i], stream=streams[i])
                f.pool.decode_attention_groups(0, q, table, lens, f.rows, pages, out=outs[i], workspace=spaces[i], stream=streams[i])
            except Exception as e:                                     # noqa: BLE001 (told by the test's own thread)
                wrong.append(e)

        threads = [threading.Thread(target=work, args=(i,)) for i in range(n_threads)]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
        torch.cuda.synchronize()
        assert not wrong, wrong
        want = f.attend(q, [12, 2])
        f.check(want, q)
        assert all(torch.equal(o, want) for o in outs), turn
        assert f.pool.last_error() == (0, 0)


FUZZ = int(os.environ.get("STEP_FUZZ_SEEDS", "40"))


@pytest.mark.parametrize("first", range(0, FUZZ, 10))
def test_random_groups_element_by_element(first):
    """Heads, prompts, own texts, ended traces and declared pages at random, blocks shuffled, NaN wherever nothing is stored."""
    for seed in range(first, min(FUZZ, first + 10)):
        rng = np.random.default_rng(41000 + seed)
        Hkv = int(rng.choice([1, 2, 3, 8]))
        Hq = Hkv * int(rng.choice([1, 2, 3, 4, 5, 7, 8, 12, 16]))
        d, P, dt = (128, 16, "bf16") if rng.random() < 0.8 else [(64, 16, "bf16"), (64, 8, "fp32"), (128, 32, "bf16")][rng.integers(3)]
        few = rng.random() < 0.8
        problems = []
        for _ in range(int(rng.integers(1, 5)) if few else 60):
            prompt = int(rng.integers(0, 6000 if rng.random() < 0.3 else 400))
            traces = int(rng.choice([1, 2, 4, 17, 33, 65]) if few else rng.integers(1, 4))
            problems.append((prompt, rng.choice([0, 1, 15, 16, 17, 90, 700 if rng.random() < 0.2 else 33], traces)))
        f = Forks((Hq, Hkv, d), dt, P, problems, normal(seed), rng)
        ended = np.nonzero(rng.random(f.n) < rng.choice([0, 0.1, 0.5]))[0]
        if len(ended):
            f.pool.release_traces(dev(ended))
        q = normal(5000 + seed)(f.n, Hq, d).to(TYPES[dt][1])
        got = f.attend(q, [p // P if rng.random() < 0.8 else rng.integers(0, p // P + 1) for p, _ in problems])
        f.check(got, q, ended=set(ended.tolist()))
        assert f.pool.last_error() == (0, 0), seed
