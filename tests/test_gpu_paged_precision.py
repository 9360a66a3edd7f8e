"""Paged decode over INT8 caches with FP16 outputs: every probability is two FP16 numbers, wherever a chunk ends.

Scores are near zero, so that the bound of their rounding (which grows with their size) hides nothing: what is left is half a
step of the output, u^2 of a probability and the FP32 sums.  One FP16 number a probability would be off by u / 2 on average."""
import copy

import numpy as np
import pytest
import torch

from tests import paged_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def tm():
    from paper_2608_17336_b200 import binding
    return binding


def check(s, q, res, rows):
    """Within the bound of a 16-bit cache, whose probabilities are two numbers (paged_ref.attend), and what FP16's subnormals
    may add: the second number is off by 2^-25 at most, in units of 2^-14 and of a power of two up to twice the largest scale:
    2^-39 of twice the largest value a key."""
    like16 = copy.copy(s)
    like16.int8 = False
    out, _, tol, _ = ref.attend(like16, q, only=rows)
    got = ref.f64(res["out"])
    for b, h in rows:
        v, present = s.context("v", b)
        more = 2.0 ** -38 * len(v) * np.abs(v).max()
        off = np.abs(got[b, h] - out[b, h])
        assert (off <= tol[b, h] + more).all(), (b, h, (off / (tol[b, h] + more)).max())


# enough rows that chunks are cut as large as they are, and rows of one and several whole chunks, which end inside one too
@pytest.mark.parametrize("d,hk,hq", [(128, 8, 8), (128, 8, 32), (64, 8, 24), (128, 4, 64), (64, 4, 40)])
def test_whole_chunks(d, hk, hq):
    lens = [64, 32, 128, 96, 77, 31, 160, 15] * 60
    s = ref.Setup("fp16", True, d, 32, hk, lens, seed=d + hq, stale=float("nan"), device=DEV)
    s.table[2, 1] = -1
    g = torch.Generator().manual_seed(1)
    q = (torch.randn((len(lens), hq, d), generator=g) * 1e-3).half().to(DEV)
    res = tm().tilemix_paged_decode(s.cache(), q)
    check(s, q, res, [(b, h) for b in list(range(10)) + [240, 241, 242, 479] for h in (0, hq // 2, hq - 1)])


@pytest.mark.parametrize("d", [64, 128])
def test_neighbours_leave_the_rounding_alone(d):
    """A sequence by itself (small chunks) and beside many others (whole ones) keeps the same bound."""
    lens = [64, 200] + [64] * 478
    s = ref.Setup("fp16", True, d, 32, 8, lens, seed=3, stale=float("nan"), device=DEV)
    g = torch.Generator().manual_seed(1)
    q = (torch.randn((len(lens), 8, d), generator=g) * 1e-3).half().to(DEV)
    res = tm().tilemix_paged_decode(s.cache(), q)
    check(s, q, res, [(b, h) for b in (0, 1) for h in range(8)])
    few = copy.copy(s)
    few.table, few.cache_len = s.table[:2], s.cache_len[:2]
    check(few, q[:2], tm().tilemix_paged_decode(few.cache(), q[:2]), [(b, h) for b in (0, 1) for h in range(8)])
