"""Bounded waits of the paged decode under limits from nothing to more than a copy takes."""
import pytest
import torch

from tests import paged_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def tm():
    from paper_2608_17336_b200 import binding
    return binding


def query(s, hq, seed=1):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((len(s.lens), hq, s.d), generator=g) * 2).to(s.act).to(DEV)


@pytest.mark.parametrize("act,int8,d,hq", [("fp16", True, 128, 8), ("bf16", False, 128, 8), ("fp16", False, 64, 16), ("bf16", True, 64, 128)])
def test_short_limits(act, int8, d, hq):
    """With every copy in place, and with every warp's second chunk left out: a row is what it always is or, whole, NaN; the
    call returns, and the next one is in order.  (Whether a warp's lanes agree on a copy that lands just then is left to chance:
    that they are asked together shows in the code alone.)"""
    t = tm()
    s = ref.Setup(act, int8, d, 16, 8, [10, 40000, 12, 3000, 0, 700], seed=3, device=DEV)
    q, c = query(s, hq), s.cache()
    good = t.tilemix_paged_decode(c, q, want_lse=True)
    ref.check_decode(s, q, good, only=[(b, h) for b in (0, 2, 3, 5) for h in (0, hq - 1)])
    for which in (1, 2):                                # (1 drops a copy of another kernel: here it sets the limit alone)
        for limit in (1, 1000, 16000, 1000000):
            t.tilemix_test_drop_copy(which, limit)
            try:
                res = [t.tilemix_paged_decode(c, q, want_lse=True) for _ in range(10)]
                torch.cuda.synchronize()
            finally:
                t.tilemix_test_drop_copy(0)
            for r in res:
                gone = torch.isnan(r["lse"])
                assert torch.isnan(r["out"][gone]).all() and (which == 1 or gone[1].all())
                assert torch.equal(r["out"][~gone], good["out"][~gone]) and torch.equal(r["lse"][~gone], good["lse"][~gone])
    again = t.tilemix_paged_decode(c, q, want_lse=True)
    assert torch.equal(again["out"], good["out"]) and torch.equal(again["lse"], good["lse"])
