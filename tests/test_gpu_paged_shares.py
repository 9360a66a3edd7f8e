"""Paged decode and read-back: shares that are cut in pieces in every instance that has them, and lengths that the table cannot
hold or that are negative."""
import numpy as np
import pytest
import torch

from tests import paged_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def tm():
    from paper_2608_17336_b200 import binding
    return binding


def query(s, hq, gain=2.0):
    g = torch.Generator().manual_seed(1)
    return (torch.randn((len(s.lens), hq, s.d), generator=g) * gain).to(s.act).to(DEV)


# 16-bit caches; shares of 32 units and more, a unit being 4 chunks of 16 keys (128 features) or 32 (64).  Up to eight query
# heads a KV head: 444 CTAs, hence 14208 units and more; sixteen: 296 CTAs, 9472 units.  Fewer rows than workers, and more.
@pytest.mark.parametrize("act,d,hk,r,lens", [
    ("fp16", 64, 8, 2, [120000, 50, 0, 110000, 3]), ("bf16", 64, 8, 1, [2050] * 113),
    ("bf16", 128, 4, 16, [80000, 5, 76000, 0]), ("fp16", 128, 4, 9, [1040] * 150),
    ("fp16", 64, 8, 12, [100000, 1, 60000]), ("bf16", 64, 8, 16, [2050] * 80)])
def test_shares_in_pieces(act, d, hk, r, lens):
    unit = 4 * (16 if d == 128 else 32)
    assert hk * sum(-(-n // unit) for n in lens) >= 32 * (444 if r <= 8 else 296)
    s = ref.Setup(act, False, d, 64, hk, lens, seed=21, device=DEV)
    q = query(s, r * hk)
    res = tm().tilemix_paged_decode(s.cache(), q, want_lse=True)
    live = torch.tensor(lens) > 0
    assert torch.isfinite(res["out"]).all() and torch.isfinite(res["lse"][live]).all() and torch.isneginf(res["lse"][~live]).all()
    ref.check_decode(s, q, res, only=[(b, h) for b in {0, 1, len(lens) // 2, len(lens) - 1} for h in (0, r, r * hk - 1)])
    # a row that lost a part would differ from what the sequence gives by itself
    for b in sorted({0, len(lens) // 2, len(lens) - 2, len(lens) - 1}):
        one = tm().paged_cache(s.k_pool, s.v_pool, s.table[b:b + 1], s.cache_len[b:b + 1])
        alone = tm().tilemix_paged_decode(one, q[b:b + 1], want_lse=True)
        # (two roundings of the output, and of the FP32 sums' orders)
        u = torch.finfo(s.act).eps
        assert ((alone["out"][0].float() - res["out"][b].float()).abs() <= u * alone["out"][0].float().abs() + 2e-6).all()
        if lens[b]:
            assert (alone["lse"][0] - res["lse"][b]).abs().max() <= 1e-5 * alone["lse"][0].abs().max()


@pytest.mark.parametrize("act,int8", [("fp16", False), ("bf16", False), ("fp16", True), ("bf16", True)])
def test_lengths_outside_the_table(act, int8):
    """Below zero: no token.  Past the table: all that it names.  Decode and read-back, packed and dense."""
    lens = [70, 96, 33, 96, 96, 0]
    s = ref.Setup(act, int8, 128, 16, 2, lens, seed=2, device=DEV)
    s.cache_len = torch.tensor([-1, 97, 33, (1 << 31) - 1, 112, -(1 << 31)], dtype=torch.int32, device=DEV)
    hold = [0, 96, 33, 96, 96, 0]
    q = query(s, 8)
    res = tm().tilemix_paged_decode(s.cache(), q, want_lse=True)
    ref.check_decode(s, q, res)
    assert not res["out"][[0, 5]].any() and torch.isneginf(res["lse"][[0, 5]]).all()
    want = {p: [torch.from_numpy(s.context(p, b)[0].astype(np.float32)).to(s.act) for b in range(6)] for p in "kv"}
    assert [len(x) for x in want["k"]] == hold
    cu = torch.tensor([0] + hold, dtype=torch.int32).cumsum(0).int().to(DEV)
    packed = [torch.full((sum(hold) + 5, 2, 128), 9.0, dtype=s.act, device=DEV) for _ in "kv"]
    tm().tilemix_paged_gather(s.cache(), *packed, cu_out=cu)
    dense = [torch.full((6, 2, 120, 128), 9.0, dtype=s.act, device=DEV) for _ in "kv"]
    tm().tilemix_paged_gather(s.cache(), *dense)
    for i, p in enumerate("kv"):
        assert torch.equal(packed[i][:sum(hold)].cpu(), torch.cat(want[p])) and (packed[i][sum(hold):] == 9).all()
        for b in range(6):
            assert torch.equal(dense[i][b, :, :hold[b]].cpu(), want[p][b].transpose(0, 1)) and (dense[i][b, :, hold[b]:] == 9).all()
