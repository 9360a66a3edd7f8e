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


@pytest.mark.parametrize("act,int8,d,hq,lens", [
    ("fp16", True, 128, 8, [10, 40000, 12, 3000, 0, 700]), ("bf16", False, 64, 8, [9000] * 30 + [17, 0, 5000]),
    ("fp16", False, 128, 128, [1 + 37 * i % 700 for i in range(150)]), ("bf16", True, 64, 24, [1 + 41 * i % 300 for i in range(400)]),
    ("fp16", True, 64, 8, [50 + i for i in range(64)]), ("bf16", False, 128, 8, [16000] * 40)])
@pytest.mark.parametrize("which", [4, 5, 6, 7])
def test_lengths_that_warps_do_not_agree_on(act, int8, d, hq, lens, which):
    """As if the lengths had changed while the call ran: teams of other sizes, other rows, other numbers of barriers and chunks
    from warp to warp.  The call ends, nothing outside its buffers is touched, and the next call is in order."""
    t = tm()
    s = ref.Setup(act, int8, d, 16, 8, lens, seed=3, room=1, device=DEV)
    q, c = query(s, hq), s.cache()
    good = t.tilemix_paged_decode(c, q, want_lse=True)
    ref.check_decode(s, q, good, only=[(b, h) for b in (0, 2, len(lens) - 1) for h in (0, hq - 1)])
    size = t.tilemix_paged_decode_workspace_size(c, hq)
    ws = torch.full((size + 4096,), 0x37, dtype=torch.uint8, device=DEV)
    big = torch.full((q.numel() + 4096,), 5.0, dtype=s.act, device=DEV)
    out = big[2048:2048 + q.numel()].view(q.shape)
    pools = [x.clone() for x in (s.k_pool, s.v_pool)]
    t.tilemix_test_drop_copy(which, 1_000_000)
    try:
        for _ in range(2):
            t.tilemix_paged_decode(c, q, out=out, workspace=ws[:size], want_lse=True)
        torch.cuda.synchronize()
    finally:
        t.tilemix_test_drop_copy(0)
    assert (ws[size:] == 0x37).all() and (big[:2048] == 5).all() and (big[2048 + q.numel():] == 5).all()
    assert torch.equal(pools[0], s.k_pool) and torch.equal(pools[1], s.v_pool)
    again = t.tilemix_paged_decode(c, q, workspace=ws[:size], want_lse=True)
    assert torch.equal(again["out"], good["out"]) and torch.equal(again["lse"], good["lse"])
