"""Paged decode at scores whose FP32 spacing is a whole number or more, and at multipliers of a score near zero.

Keys are +-a times one vector of equal entries, so that the products q . k are sums of equal numbers that FP32 holds exactly in
any order: equal keys have equal scores, and the softmax is the mean over the largest ones, without a tolerance for the scores."""
import math

import numpy as np
import pytest
import torch

from tests import paged_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# act, int8, magnitudes of q and k: scores of 2e3, 1.4e6, 4.2e7, 2.7e9 and 6e10 log2 units; of bfloat16 also 2e37, and -2e38
FP16 = [16.0, 400.0, 1600.0, 16384.0, 61440.0]
CASES = ([("fp16", i, a, d) for i in (False, True) for a in FP16 for d in (64, 128)]
         + [("bf16", i, a, 128) for i in (False, True) for a in (16.0, 1600.0, 2.0 ** 40, 2.0 ** 60)])


def tm():
    from paper_2608_17336_b200 import binding
    return binding


def run(act, int8, a, d, signs, hq=3, q_sign=1.0):
    """signs[b][j]: key j of sequence b is signs[b][j] * a in every entry.  Returns (setup, q, result)."""
    s = ref.Setup(act, int8, d, 16, 1, [len(x) for x in signs], seed=5, device=DEV)
    for b, row in enumerate(signs):
        for j, sign in enumerate(row):
            page, r = int(s.table[b, j // 16]), j % 16
            if int8:
                s.k_pool[page, 0, r] = int(math.copysign(127, sign))
                s.k_scale[page, 0, r] = abs(sign) * a / 128          # (a power of two times a few bits: products stay exact)
            else:
                s.k_pool[page, 0, r] = sign * a
    q = torch.full((len(signs), hq, d), q_sign * a).to(s.act).to(DEV)
    return s, q, tm().tilemix_paged_decode(s.cache(), q, want_lse=True)


def check(s, q, res, best):
    """Each row is the mean of v over best[b]: half a step of the type for the rounding, and what attend() derives for the
    probabilities (all of them equal: one number of 2^-11 at worst) and FP32 sums."""
    u = torch.finfo(s.act).eps / 2
    up = 2.0 ** -11 if s.int8 else u * u
    _, lse, _, tol_lse = ref.attend(s, q)
    got, got_lse = ref.f64(res["out"]), ref.f64(res["lse"])
    for b, keys in enumerate(best):
        v, _ = s.context("v", b)
        want, mass = v[keys, 0].mean(0), np.abs(v[keys, 0]).mean(0)
        tol = u * np.abs(want) + (up + 2 * (2.0 ** -22 + len(keys) * 2.0 ** -24)) * 1.01 * mass + torch.finfo(s.act).tiny * u
        assert np.isfinite(got[b]).all(), (b, got[b])
        assert (np.abs(got[b] - want) <= tol).all(), b
    assert np.isfinite(got_lse).all() and (np.abs(got_lse - lse) <= tol_lse).all()


@pytest.mark.parametrize("act,int8,a,d", CASES)
def test_one_key(act, int8, a, d):
    s, q, res = run(act, int8, a, d, [[1.0], [-1.0]])
    check(s, q, res, [[0], [0]])


@pytest.mark.parametrize("act,int8,a,d", CASES)
def test_equal_keys_weigh_the_same(act, int8, a, d):
    """In one block, across blocks, warps and CTAs; the largest ones first, last and between."""
    n = 700
    signs = [[1.0] * n, [-1.0] * 40, [1.0 if j in (3, 17, 400, 699) else 0.5 for j in range(n)], [-1.0 if j < n - 1 else -0.5 for j in range(n)]]
    s, q, res = run(act, int8, a, d, signs)
    check(s, q, res, [list(range(n)), list(range(40)), [3, 17, 400, 699], [n - 1]])


@pytest.mark.parametrize("act,int8", [("fp16", False), ("bf16", False), ("fp16", True), ("bf16", True)])
@pytest.mark.parametrize("scale", [1e-44, 1e-30])
def test_scales_near_zero(act, int8, scale):
    """All scores are (nearly) 0: the mean of all values, keys past the end and in holes excluded as ever."""
    lens = [1, 13, 50, 700]
    s = ref.Setup(act, int8, 128, 16, 2, lens, seed=7, stale=float("nan"), device=DEV)
    s.table[3, 5] = -1
    g = torch.Generator().manual_seed(2)
    q = torch.randn((4, 6, 128), generator=g).to(s.act).to(DEV)
    res = tm().tilemix_paged_decode(s.cache(), q, want_lse=True, softmax_scale=scale)
    ref.check_decode(s, q, res, scale=scale)


@pytest.mark.parametrize("int8", [False, True])
def test_queries_near_zero_bf16(int8):
    """Queries among bfloat16's smallest numbers: the power of two that brings them into FP16's range is at its limit."""
    s = ref.Setup("bf16", int8, 128, 16, 1, [5, 33, 300], seed=9, stale=float("nan"), device=DEV)
    g = torch.Generator().manual_seed(4)
    q = (torch.randn((3, 4, 128), generator=g) * 2.0 ** -125).bfloat16().to(DEV)
    ref.check_decode(s, q, tm().tilemix_paged_decode(s.cache(), q, want_lse=True))
    ref.check_decode(s, q, tm().tilemix_paged_decode(s.cache(), q, want_lse=True, softmax_scale=1e-8), scale=1e-8)
