"""Paged key/value cache on the GPU: appended rows bit for bit, read-back bit for bit, attention against float64 within the
bound that paged_ref.attend derives; then the calls together, as a serving program uses them."""
import numpy as np
import pytest
import torch

from tests import paged_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def tm():
    from paper_2608_17336_b200 import binding
    return binding


def bits(t):
    t = t.detach().cpu().contiguous()
    return t.numpy() if t.dtype == torch.int8 else t.view(torch.int32 if t.dtype == torch.float32 else torch.int16).numpy()


def query(s, hq, seed=1, gain=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((len(s.lens), hq, s.d), generator=g) * gain).to(s.act).to(DEV)


# ---------------------------------------------------------------------------------------------------- append

def expected_append(s, k_new, v_new, cu):
    """The pools after the append, from the definition (numpy copies)."""
    want = {n: getattr(s, n).cpu().clone() for n in ("k_pool", "v_pool", "k_scale", "v_scale") if getattr(s, n) is not None}
    table, lens = s.table.cpu(), s.cache_len.cpu()
    for p, x in (("k", k_new), ("v", v_new)):
        code, delta = ref.quantise(x.float().cpu().numpy()) if s.int8 else (x.cpu(), None)
        for b in range(len(lens)):
            n = int(cu[b + 1] - cu[b])
            for i in range(n):
                pos = int(lens[b]) - n + i
                if not 0 <= pos < table.shape[1] * s.page:
                    continue
                page = int(table[b, pos // s.page])
                if not 0 <= page < want["k_pool"].shape[0]:
                    continue
                want[p + "_pool"][page, :, pos % s.page] = torch.as_tensor(code[int(cu[b]) + i])
                if s.int8:
                    want[p + "_scale"][page, :, pos % s.page] = torch.as_tensor(delta[int(cu[b]) + i])
    return want


def same_bits(a, b):
    a, b = bits(a), bits(b)
    if a.dtype == np.int32:       # scales: any NaN is a NaN
        nan = np.isnan(a.view(np.float32)) & np.isnan(b.view(np.float32))
        return np.array_equal(np.where(nan, 0, a), np.where(nan, 0, b))
    return np.array_equal(a, b)


def run_append(s, new, seed=5, hard=False, strided=False, pad=0, cu_none=False):
    g = torch.Generator().manual_seed(seed)
    cu = np.concatenate([[0], np.cumsum(new)])
    n = int(cu[-1]) + pad
    x = torch.randn((2, n, s.hk, s.d), generator=g)
    if hard:        # magnitudes from subnormal to large, zero rows, infinities, NaN, exact half-integers
        x *= 2.0 ** torch.randint(-24 if s.act == torch.float16 else -126, 10, (2, n, s.hk, 1), generator=g)
        x[0, ::7] = 0
        x[1, 3::11, 0, 5] = float("inf")
        x[0, 5::13, -1, 0] = float("nan")
        x[1, ::5, :, 1] = 1.0
        x[1, ::5, :, 2:] = 0.5
        x[1, ::5, :, 0] = -0.25
    x = x.to(s.act)
    if strided:     # the K and V parts of a fused projection
        fused = torch.zeros((n, 3, s.hk, s.d), dtype=s.act)
        fused[:, 1], fused[:, 2] = x[0], x[1]
        fused = fused.to(DEV)
        k, v = fused[:, 1], fused[:, 2]
    else:
        k, v = x[0].to(DEV), x[1].to(DEV)
    want = expected_append(s, x[0], x[1], cu)
    tm().tilemix_paged_append(s.cache(), k, v, cu_new=None if cu_none else torch.tensor(cu, dtype=torch.int32, device=DEV))
    torch.cuda.synchronize()
    for name, w in want.items():
        assert same_bits(getattr(s, name), w), name


@pytest.mark.parametrize("act", ["fp16", "bf16"])
@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("d,page,hk,nhd", [(128, 16, 1, False), (64, 32, 3, False), (128, 64, 8, True), (64, 256, 2, True)])
def test_append_rows(act, int8, d, page, hk, nhd):
    lens = [1, 0, 37, page, page + 1, 300, 5]
    s = ref.Setup(act, int8, d, page, hk, lens, seed=d + page, nhd=nhd, device=DEV)
    run_append(s, [1, 0, 20, page, 1, 300, 0], hard=True, strided=hk == 3, pad=9)


@pytest.mark.parametrize("int8", [False, True])
def test_append_one_token_each(int8):
    s = ref.Setup("fp16", int8, 128, 16, 2, [1, 16, 17, 0, 400], device=DEV)      # (the empty place of the batch: dropped)
    run_append(s, [1] * 5, cu_none=True)


def test_append_many_sequences():
    """More sequences than a warp looks at together; several without a new token one behind the other."""
    lens = [(7 * i) % 41 + 3 for i in range(300)]
    new = [0 if i % 3 or 90 < i < 170 else min(lens[i], i % 5) for i in range(300)]
    run_append(ref.Setup("fp16", True, 64, 16, 1, lens, device=DEV), new)


def test_append_drops_rows_without_a_place():
    """More new rows than the length counts, lengths at and past the table's end, negative ones, holes."""
    s = ref.Setup("fp16", True, 128, 16, 2, [5, 40, 64, 30, 60, 64], device=DEV)
    s.cache_len = torch.tensor([5, 1 << 30, -3, 30, 66, 64], dtype=torch.int32, device=DEV)       # the table has 64 places
    s.table[3, 0], s.table[3, 1] = -1, 1 << 30
    g = torch.Generator().manual_seed(2)
    x = torch.randn((2, 43, 2, 128), generator=g).half()
    cu = np.array([0, 9, 16, 20, 33, 38, 43])
    want = expected_append(s, x[0], x[1], cu)
    tm().tilemix_paged_append(s.cache(), x[0].to(DEV), x[1].to(DEV), torch.tensor(cu, dtype=torch.int32, device=DEV))
    for name, w in want.items():
        assert same_bits(getattr(s, name), w), name


# ---------------------------------------------------------------------------------------------------- gather

def expected_rows(s, p, b):
    """[len, Hk, d] in act_type: FP32 product, rounded."""
    n = int(s.cache_len[b])
    pool, scale, table = getattr(s, p + "_pool").cpu(), getattr(s, p + "_scale"), s.table.cpu()
    out = torch.zeros((n, s.hk, s.d), dtype=s.act)
    for j in range(n):
        page = int(table[b, j // s.page])
        if 0 <= page < pool.shape[0]:
            x = pool[page, :, j % s.page].float()
            out[j] = (x * scale.cpu()[page, :, j % s.page, None] if scale is not None else x).to(s.act)
    return out


@pytest.mark.parametrize("act", ["fp16", "bf16"])
@pytest.mark.parametrize("int8", [False, True])
@pytest.mark.parametrize("d,page,hk,nhd", [(128, 16, 1, False), (64, 64, 3, False), (128, 32, 4, True)])
def test_gather(act, int8, d, page, hk, nhd):
    lens = [33, 0, 1, page, 3 * page + 1, 200]
    s = ref.Setup(act, int8, d, page, hk, lens, seed=3, nhd=nhd, device=DEV)
    s.table[5, 1] = -7                                    # a hole
    c = s.cache()
    want = {p: [expected_rows(s, p, b) for b in range(len(lens))] for p in "kv"}
    # packed, some padding behind, from a start
    start = [0, 0, 0, 5, page, 250]
    n = [max(0, x - y) for x, y in zip(lens, start)]
    cu = np.concatenate([[0], np.cumsum(n)])
    out = [torch.full((int(cu[-1]) + 7, hk, d), 9.0, dtype=s.act, device=DEV) for _ in "kv"]
    tm().tilemix_paged_gather(c, *out, start=torch.tensor(start, dtype=torch.int32, device=DEV),
                              cu_out=torch.tensor(cu, dtype=torch.int32, device=DEV))
    for o, p in zip(out, "kv"):
        flat = torch.cat([want[p][b][start[b]:] for b in range(len(lens))] + [torch.full((7, hk, d), 9.0, dtype=s.act)])
        assert same_bits(o, flat), p
    # dense, fewer rows than the longest, token-major outputs
    rows = 3 * page
    out = [torch.full((len(lens), rows, hk, d), 9.0, dtype=s.act, device=DEV).transpose(1, 2) for _ in "kv"]
    tm().tilemix_paged_gather(c, *out)
    for o, p in zip(out, "kv"):
        dense = torch.full((len(lens), hk, rows, d), 9.0, dtype=s.act)
        for b in range(len(lens)):
            x = want[p][b][:rows].transpose(0, 1)
            dense[b, :, :x.shape[1]] = x
        assert same_bits(o, dense), p


# ---------------------------------------------------------------------------------------------------- decode

KINDS = [("fp16", False), ("bf16", False), ("fp16", True), ("bf16", True)]


@pytest.mark.parametrize("act,int8", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("page,hq,hk", [(16, 1, 1), (32, 6, 2), (64, 16, 2), (128, 9, 1), (256, 64, 2), (16, 17, 1)])
def test_decode_lengths(act, int8, d, page, hq, hk):
    """Lengths around every tile size, empty ones among them, every group size of query heads."""
    lens = [0, 1, 15, 16, 17, 31, 33, 63, 64, 65, 127, 128, 129, 255, 256, 257, 400, 0, 700, 1025]
    s = ref.Setup(act, int8, d, page, hk, lens, seed=page + hq, stale=float("nan"), device=DEV)
    q = query(s, hq, gain=2.0)
    res = tm().tilemix_paged_decode(s.cache(), q, want_lse=True)
    ref.check_decode(s, q, res)
    assert not res["out"][[0, 17]].any()


@pytest.mark.parametrize("act,int8", KINDS)
@pytest.mark.parametrize("d,nhd", [(64, True), (128, False)])
def test_decode_long(act, int8, d, nhd):
    """Rows shared by many CTAs beside short ones."""
    s = ref.Setup(act, int8, d, 64, 2, [20000, 3, 9001], seed=8, nhd=nhd, device=DEV)
    q = query(s, 8, gain=3.0)
    ref.check_decode(s, q, tm().tilemix_paged_decode(s.cache(), q, want_lse=True))


@pytest.mark.parametrize("act,int8", KINDS)
def test_decode_many_rows(act, int8):
    """More rows than the GPU has places for CTAs; a batch above a warp's and a CTA's width."""
    lens = [(37 * i) % 211 for i in range(333)]
    s = ref.Setup(act, int8, 64, 16, 2, lens, seed=9, device=DEV)
    q = query(s, 4)
    ref.check_decode(s, q, tm().tilemix_paged_decode(s.cache(), q, want_lse=True))


@pytest.mark.parametrize("act,int8,d", [("bf16", False, 128), ("fp16", False, 64), ("fp16", True, 128), ("bf16", True, 64)])
def test_decode_many_short_rows(act, int8, d):
    """Runs of several short rows a worker, of very different lengths, which begin and end anywhere in and between rows; empty
    sequences between them and at the end."""
    lens = [0 if i % 7 == 3 else 1 + (i * i * 131 + 77 * i) % 800 for i in range(140)] + [1, 1, 0]
    s = ref.Setup(act, int8, d, 16, 8, lens, seed=31, stale=float("nan"), device=DEV)
    q = query(s, 8, gain=2.0)
    ref.check_decode(s, q, tm().tilemix_paged_decode(s.cache(), q, want_lse=True))


@pytest.mark.parametrize("act,int8,hk,lens", [("bf16", False, 8, [60000, 100, 0, 57100, 3]), ("fp16", False, 8, [1101] * 113), ("fp16", True, 4, [50000, 7, 41000])])
def test_decode_large(act, int8, hk, lens):
    """Shares long enough to be cut in pieces (16-bit caches), rows of many CTAs, more rows than there are workers; every row
    finite, some of them against float64."""
    s = ref.Setup(act, int8, 128, 64, hk, lens, seed=21, device=DEV)
    q = query(s, 2 * hk, gain=2.0)
    res = tm().tilemix_paged_decode(s.cache(), q, want_lse=True)
    assert torch.isfinite(res["out"]).all() and torch.isfinite(res["lse"][torch.tensor(lens) > 0]).all()
    ref.check_decode(s, q, res, only=[(b, h) for b in {0, 1, len(lens) // 2, len(lens) - 2, len(lens) - 1} for h in (0, hk, 2 * hk - 1)])
    # any row that lost a part would differ from what the sequence gives by itself
    for b in (0, len(lens) - 2):
        one = tm().paged_cache(s.k_pool, s.v_pool, s.table[b:b + 1], s.cache_len[b:b + 1], s.k_scale, s.v_scale, dtype=s.act)
        alone = tm().tilemix_paged_decode(one, q[b:b + 1], want_lse=True)
        u = torch.finfo(s.act).eps
        assert ((alone["out"][0].float() - res["out"][b].float()).abs() <= u * alone["out"][0].float().abs() + 2e-6).all()
        assert (alone["lse"][0] - res["lse"][b]).abs().max() <= 1e-5 * alone["lse"][0].abs().max()


@pytest.mark.parametrize("act,int8", KINDS)
def test_decode_strides_and_scale(act, int8):
    s = ref.Setup(act, int8, 128, 32, 2, [100, 77], seed=4, nhd=True, device=DEV)
    q = torch.zeros((2, 3, 8, 128), dtype=s.act, device=DEV)
    q[:, 1] = query(s, 8)
    big = torch.full((8, 2, 256), 7.0, dtype=s.act, device=DEV)
    out = big[:, :, 128:].transpose(0, 1)
    res = tm().tilemix_paged_decode(s.cache(), q[:, 1], out=out, want_lse=True, softmax_scale=0.3)
    ref.check_decode(s, q[:, 1], res, scale=0.3)
    assert (big[:, :, :128] == 7).all()


@pytest.mark.parametrize("act,int8", KINDS)
@pytest.mark.parametrize("d", [64, 128])
def test_decode_holes(act, int8, d):
    """Pages that are not resident have no part; a sequence of holes alone is empty."""
    s = ref.Setup(act, int8, d, 16, 2, [150, 64, 900, 33], seed=6, stale=float("nan"), device=DEV)
    s.table[0, 0] = -1
    s.table[0, 5] = s.k_pool.shape[0]
    s.table[1, :] = -(1 << 31)
    s.table[2, 3:40] = 1 << 30
    s.table[3, 2] = -1
    q = query(s, 8, gain=2.0)
    res = tm().tilemix_paged_decode(s.cache(), q, want_lse=True)
    ref.check_decode(s, q, res)
    assert not res["out"][1].any() and torch.isneginf(res["lse"][1]).all()


@pytest.mark.parametrize("act,int8", KINDS)
def test_decode_values_that_are_not_finite(act, int8):
    """A NaN in a value, a NaN or an infinity in a key reach their own KV head's rows of their own sequence, and nothing else."""
    s = ref.Setup(act, int8, 128, 16, 2, [50, 50, 50, 50], seed=6, device=DEV)
    clean = ref.Setup(act, int8, 128, 16, 2, [50, 50, 50, 50], seed=6, device=DEV)
    q = query(s, 8)
    at = lambda b, j: (int(s.table[b, j // 16]), j % 16)      # noqa: E731
    for b, pool in ((0, "v"), (1, "k")):
        page, row = at(b, 20)
        if int8:
            getattr(s, pool + "_scale")[page, 1, row] = float("nan")
        else:
            getattr(s, pool + "_pool")[page, 1, row, 3] = float("nan")
    res = tm().tilemix_paged_decode(s.cache(), q, want_lse=True)
    base = tm().tilemix_paged_decode(clean.cache(), q, want_lse=True)
    out = res["out"].float()
    if int8:
        assert torch.isnan(out[0, 4:]).all()
    else:
        assert torch.isnan(out[0, 4:, 3]).all()
        keep = [i for i in range(128) if i != 3]
        assert torch.equal(out[0, 4:][:, keep], base["out"].float()[0, 4:][:, keep])
    assert torch.isnan(out[1, 4:]).all() and torch.isnan(res["lse"][1, 4:]).all()
    assert torch.equal(res["out"][:, :4], base["out"][:, :4]) and torch.equal(res["out"][2:], base["out"][2:])


@pytest.mark.parametrize("act", ["fp16", "bf16"])
def test_decode_scales_of_very_different_size(act):
    """INT8 values whose scales span the type's range: the rounding of a scaled probability stays relative to the largest."""
    s = ref.Setup(act, True, 128, 16, 1, [300, 300, 300], seed=2, device=DEV)
    lo = 1e-7 if act == "fp16" else 1e-30
    s.v_scale[:] = lo
    for b in (1, 2):
        page = int(s.table[b, 7])
        s.v_scale[page, 0, 3] = 1.0
    s.v_scale[int(s.table[2, 0])] = 0.0
    s.v_pool[int(s.table[2, 0])] = 0
    q = query(s, 4)
    out, _, tol, _ = ref.attend(s, q)
    if act == "fp16":
        tol = tol + 2.0 ** -25          # outputs of 1e-6 are subnormal FP16
    # scaled probabilities below 2^-28 of the largest scaled one are subnormal: 2^-39 of the largest scale each
    tol = tol + 300 * 127 * 2.0 ** -39 * np.array([lo, 1.0, 1.0])[:, None, None]
    got = ref.f64(tm().tilemix_paged_decode(s.cache(), q)["out"])
    assert (np.abs(got - out) <= tol).all()


def test_decode_large_queries_bf16():
    """Queries beyond FP16's range over an INT8 cache (scores stay moderate: small keys)."""
    s = ref.Setup("bf16", True, 128, 16, 1, [200], seed=2, device=DEV, gain=1.0)
    s.k_scale *= 1e-30
    q = query(s, 4, gain=1e30)
    ref.check_decode(s, q, tm().tilemix_paged_decode(s.cache(), q, want_lse=True))
    s.k_scale *= 1e30      # (in two steps: 1e50 is not an FP32 number)
    s.k_scale *= 1e20
    q = query(s, 4, gain=1e-20)
    ref.check_decode(s, q, tm().tilemix_paged_decode(s.cache(), q, want_lse=True))


def test_decode_offsets_past_32_bits():
    """A pool of more than 2^32 bytes, pages at both ends of it."""
    n_pages, hk, page, d = 131500, 2, 128, 128          # 4.3e9 codes
    pool = torch.empty((n_pages, hk, page, d), dtype=torch.int8, device=DEV)
    scale = torch.ones((n_pages, hk, page), device=DEV)
    table = torch.tensor([[n_pages - 1, 0, n_pages - 2, 77]], dtype=torch.int32, device=DEV)
    g = torch.Generator().manual_seed(1)
    small = torch.randint(-127, 128, (4, hk, page, d), generator=g).to(torch.int8)
    pool[table[0].long()] = small.to(DEV)
    scale[:] = 0.01
    s = ref.Setup("fp16", True, d, page, hk, [page * 4 - 5])
    s.k_pool = s.v_pool = pool
    s.k_scale = s.v_scale = scale
    s.table, s.cache_len = table, s.cache_len.to(DEV)
    q = query(s, 4)
    ref.check_decode(s, q, tm().tilemix_paged_decode(s.cache(), q, want_lse=True))
    k, v = torch.zeros((2, 1, hk, page * 4, d), dtype=torch.float16, device=DEV)
    tm().tilemix_paged_gather(s.cache(), k, v)
    assert same_bits(k[0, :, :page], (small[0].float() * scale[0, 0, 0].cpu()).half())
    new = torch.randn((1, hk, d), generator=g).half()
    tm().tilemix_paged_append(s.cache(), new.to(DEV), new.to(DEV))
    assert np.array_equal(bits(pool[77, :, page - 6]), ref.quantise(new[0].float().numpy())[0])


def test_decode_repeats_bit_for_bit():
    s = ref.Setup("fp16", True, 128, 16, 4, [5000, 100, 3000], seed=8, device=DEV)
    q = query(s, 16)
    c = s.cache()
    a = tm().tilemix_paged_decode(c, q, want_lse=True)
    for _ in range(5):
        x = tm().tilemix_paged_decode(c, q, want_lse=True)
        assert torch.equal(a["out"], x["out"]) and torch.equal(a["lse"], x["lse"])


def test_decode_workspace_may_hold_anything():
    s = ref.Setup("bf16", False, 128, 16, 4, [5000, 0, 3000], seed=8, device=DEV)
    q, c = query(s, 16), s.cache()
    size = tm().tilemix_paged_decode_workspace_size(c, 16)
    a = tm().tilemix_paged_decode(c, q, want_lse=True)
    for fill in (0, 255):
        guard = torch.full((size + 512,), fill, dtype=torch.uint8, device=DEV)
        guard[size:] = 77
        x = tm().tilemix_paged_decode(c, q, want_lse=True, workspace=guard[:size])
        assert torch.equal(a["out"], x["out"]) and torch.equal(a["lse"], x["lse"])
        assert (guard[size:] == 77).all()


@pytest.mark.parametrize("act,int8,hq", [("fp16", True, 8), ("bf16", False, 8), ("bf16", True, 128)])
def test_bounded_waits(act, int8, hq):
    """A copy that never lands: the wait runs out, the call returns, the rows that a warp had still to work on are NaN, the
    others as ever, and the context and the next call are in order."""
    t = tm()
    s = ref.Setup(act, int8, 64, 16, 8, [10, 40000, 12], seed=3, device=DEV)
    q = query(s, hq)
    c = s.cache()
    good = t.tilemix_paged_decode(c, q, want_lse=True)
    torch.cuda.synchronize()
    t.tilemix_test_drop_copy(2, 20_000_000)
    try:
        res = t.tilemix_paged_decode(c, q, want_lse=True)
        torch.cuda.synchronize()
    finally:
        t.tilemix_test_drop_copy(0)
    assert torch.isnan(res["out"][1]).all() and torch.isnan(res["lse"][1]).all()
    whole = ~torch.isnan(res["lse"])
    assert whole[0, 0] and torch.equal(res["out"][whole], good["out"][whole]) and torch.isnan(res["out"][~whole]).all()
    again = t.tilemix_paged_decode(c, q, want_lse=True)
    assert torch.equal(again["out"], good["out"]) and torch.equal(again["lse"], good["lse"])
    ref.check_decode(s, q, again)


def test_decode_calls_share_a_workspace_in_turn():
    """Calls of other shapes, and two captured graphs, one after the other on one workspace: what one leaves there says nothing
    to the next."""
    t = tm()
    cases = []
    for i, (d, hk, hq, lens) in enumerate([(128, 2, 8, [3000, 5]), (64, 4, 16, [100] * 40), (128, 8, 64, [700, 900]), (64, 1, 16, [9000])]):
        s = ref.Setup("fp16", True, d, 16, hk, lens, seed=i, device=DEV)
        cases.append((s.cache(), query(s, hq, seed=i), s))
    ws = torch.full((max(t.tilemix_paged_decode_workspace_size(c, q.shape[1]) for c, q, _ in cases),), 173, dtype=torch.uint8, device=DEV)
    want = [t.tilemix_paged_decode(c, q)["out"] for c, q, _ in cases]
    graphs, outs = [], []
    for c, q, _ in cases:
        out = torch.empty_like(q)
        g = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(g):
            t.tilemix_paged_decode(c, q, out=out, workspace=ws)
        graphs.append(g)
        outs.append(out)
    for _ in range(3):
        for (c, q, s), w in zip(cases, want):
            assert torch.equal(t.tilemix_paged_decode(c, q, workspace=ws)["out"], w)
        for g, o, w in zip(graphs, outs, want):
            o.zero_()
            g.replay()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(o, w)
    for (c, q, s), w in zip(cases, want):
        ref.check_decode(s, q, {"out": w, "lse": None})


def test_decode_on_two_streams_at_once():
    """Two calls that overlap, each with its own workspace."""
    t = tm()
    cases = []
    for i in range(2):
        s = ref.Setup("bf16", i == 0, 128, 16, 4, [4000, 100, 2500], seed=i, device=DEV)
        cases.append((s.cache(), query(s, 16, seed=i)))
    want = [t.tilemix_paged_decode(c, q)["out"] for c, q in cases]
    ws = [torch.empty(t.tilemix_paged_decode_workspace_size(c, 16), dtype=torch.uint8, device=DEV) for c, _ in cases]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(30):
        for i, (c, q) in enumerate(cases):
            with torch.cuda.stream(streams[i]):
                got[i].append(t.tilemix_paged_decode(c, q, workspace=ws[i])["out"])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])


def test_binding_refusals():
    t = tm()
    s = ref.Setup("fp16", True, 64, 16, 2, [20, 3], device=DEV)
    c, q = s.cache(), query(s, 4)
    x = torch.zeros((2, 2, 64), dtype=torch.float16, device=DEV)
    bad = [lambda: t.tilemix_paged_decode(c, q.float()), lambda: t.tilemix_paged_decode(c, q[:1]), lambda: t.tilemix_paged_decode(c, q[..., :32]),
           lambda: t.tilemix_paged_decode(c, q.cpu()), lambda: t.tilemix_paged_decode(c, q, out=q[:, :2]),
           lambda: t.tilemix_paged_append(c, x, x.bfloat16()), lambda: t.tilemix_paged_append(c, x, x[:, :1]),
           lambda: t.tilemix_paged_append(c, x, x, cu_new=torch.zeros(3, device=DEV)),
           lambda: t.tilemix_paged_append(c, x, x, cu_new=torch.zeros(2, dtype=torch.int32, device=DEV)),
           lambda: t.tilemix_paged_gather(c, x, x), lambda: t.tilemix_paged_gather(c, x, x, start=torch.zeros(2, device=DEV), cu_out=s.cache_len)]
    for f in bad:
        with pytest.raises((AssertionError, ValueError)):
            f()
    with pytest.raises(t.TilemixError):
        t.tilemix_paged_append(c, x[:1], x[:1])                         # one token for two sequences, and no cu_new
    with pytest.raises(t.TilemixError):
        t.tilemix_paged_decode(c, torch.cat([q, q[:, :1]], 1))          # five query heads over two
    with pytest.raises(t.TilemixError):
        t.tilemix_paged_decode(c, q, workspace=torch.empty(64, dtype=torch.uint8, device=DEV))


# ---------------------------------------------------------------------------------------------------- together

@pytest.mark.parametrize("act,int8", KINDS)
def test_serving_run(act, int8):
    """Two prompts are appended in chunks, then tokens one by one; every step's attention is checked against float64 over the
    cache as it is, and the cache against what was written."""
    t = tm()
    s = ref.Setup(act, int8, 128, 16, 2, [0, 0], seed=1, room=20, device=DEV)
    c = s.cache()
    g = torch.Generator().manual_seed(3)
    written = [[torch.empty((0, 2, 128), dtype=s.act)] * 2 for _ in range(2)]

    def step(new):
        k, v = torch.randn((2, sum(new), 2, 128), generator=g).to(s.act)
        cu = np.concatenate([[0], np.cumsum(new)])
        s.cache_len += torch.tensor(new, dtype=torch.int32, device=DEV)
        one = max(new) == 1 and min(new) == 1
        t.tilemix_paged_append(c, k.to(DEV), v.to(DEV), None if one else torch.tensor(cu, dtype=torch.int32, device=DEV))
        for b in range(2):
            for i, x in enumerate((k, v)):
                written[b][i] = torch.cat([written[b][i], x[cu[b]:cu[b + 1]]])
        q = query(s, 8, seed=sum(new), gain=2.0)
        ref.check_decode(s, q, t.tilemix_paged_decode(c, q, want_lse=True))

    for new in ([100, 3], [28, 0], [1, 1], [1, 1], [0, 77], [1, 1]):
        step(new)
    for b in range(2):
        for i, p in enumerate("kv"):
            x = written[b][i].double().numpy()
            got, _ = s.context(p, b)
            # a code is off by at most half a step of max|x| / 127, a little more where the FP32 quotient is rounded
            assert (np.abs(got - x) <= (np.abs(x).max(-1, keepdims=True) / 127 * 0.5001 if int8 else 0)).all()


def test_chunked_prefill_over_the_cache():
    """A prompt's chunk attends, through the chunked prefill, to the context read back from the INT8 cache: its last query
    row equals the decode step of the same query over the same cache."""
    t = tm()
    L, chunk, hq, hk, d = 384, 128, 4, 2, 128
    s = ref.Setup("fp16", True, d, 32, hk, [L], seed=11, device=DEV)
    c = s.cache()
    k, v = (torch.zeros((1, hk, L, d), dtype=torch.float16, device=DEV) for _ in "kv")
    t.tilemix_paged_gather(c, k, v)
    g = torch.Generator().manual_seed(1)
    q = torch.randn((1, hq, chunk, d), generator=g).half().to(DEV)
    p = t.problem(1, hq, hk, chunk, d, 128, 128, flags=t.FORCE_FP16)
    pre = t.tilemix_attention_fwd_chunk(p, L, q, k, v, None, None, None, None, None, want_lse=True)
    last = t.tilemix_paged_decode(c, q[:, :, -1], want_lse=True)
    out, lse, tol, tol_lse = ref.attend(s, q[:, :, -1])
    # the prefill sees keys and values rounded to FP16: half a step of each moves a score by 2^-11 S, a value by 2^-11 |v|
    worst = (np.abs(ref.f64(q[:, :, -1])).sum(-1).max() * np.abs(ref.f64(k)).max()) / d ** 0.5
    moved = tol + 2.0 ** -11 * (2 * worst + 1) * np.abs(ref.f64(v)).max()
    assert (np.abs(ref.f64(pre["out"][:, :, -1]) - out) <= moved).all()
    assert (np.abs(ref.f64(last["out"]) - out) <= tol).all()
    assert (np.abs(ref.f64(pre["lse"][:, :, -1]) - lse) <= tol_lse + 2.0 ** -11 * worst).all()


@pytest.mark.parametrize("act,int8", KINDS)
def test_graph_replayed_while_the_sequences_grow(act, int8):
    """One captured step (append, decode) replayed with lengths, tokens and queries changed in place; two graphs, one workspace
    each, and an eager call between."""
    t = tm()
    s = ref.Setup(act, int8, 64, 16, 2, [40, 700], seed=1, room=4, device=DEV)
    c = s.cache()
    new = torch.zeros((2, 2, 2, 64), dtype=s.act, device=DEV)
    q = query(s, 4)
    ws = torch.empty(t.tilemix_paged_decode_workspace_size(c, 4), dtype=torch.uint8, device=DEV)
    out = torch.empty_like(q)

    def call():
        t.tilemix_paged_append(c, new[0], new[1])
        return t.tilemix_paged_decode(c, q, out=out, want_lse=True, workspace=ws)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        res = call()
    g = torch.Generator().manual_seed(9)
    for i in range(20):
        s.cache_len += 1
        new.copy_(torch.randn(new.shape, generator=g))
        q.copy_(torch.randn(q.shape, generator=g))
        graph.replay()
        torch.cuda.synchronize()
        ref.check_decode(s, q, res)
        if i == 10:
            eager = t.tilemix_paged_decode(c, q)
            assert torch.equal(eager["out"], out)


def test_back_to_back_steps_on_one_stream():
    """Steps that follow each other without a wait: each step's append is in place before its decode reads, and a decode has
    read the cache before the next append changes it."""
    t = tm()
    s = ref.Setup("fp16", True, 128, 16, 8, [2000] * 4, seed=1, room=20, device=DEV)
    c = s.cache()
    g = torch.Generator().manual_seed(2)
    new = torch.randn((50, 2, 4, 8, 128), generator=g).half().to(DEV)
    q = torch.randn((50, 4, 32, 128), generator=g).half().to(DEV)
    base = s.cache_len.clone()

    def steps(wait):
        s.cache_len.copy_(base)
        outs = []
        for i in range(50):
            if i % 3 == 0:
                s.cache_len += 1
            t.tilemix_paged_append(c, new[i, 0], new[i, 1])      # two of three steps write the same place again
            outs.append(t.tilemix_paged_decode(c, q[i])["out"])
            if wait:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        return torch.stack(outs)

    assert torch.equal(steps(True), steps(False))
