"""What a program that serves with a paged key/value cache has this library do: write new tokens, read contexts back, attend.

The cache of a layer is a pool of pages of ``page`` tokens, ``[n_pages, Hk, page, d]`` for K and for V, and a table that
gives each sequence its pages.  The pool holds the type of the activations (``act``), or INT8 codes with one FP32 scale a
(token, head) in ``[n_pages, Hk, page]`` (``int8``); ``nhd``: the tokens of a page lie outside its heads.

  append    the keys and values of ``new_lo`` to ``new_hi`` new tokens a sequence, packed, are written behind a context; from an
            INT8 cache they are then read back, as a prefill does that attends to what later steps will see.
  gather    the context of every sequence is read back, packed, or dense for the chunked prefill (``dense``).
  decode    one new token a sequence attends to its context (``peak``: the queries' scale, large ones attend to few keys);
            ``append`` too: the token's own key and value are written first, as in a whole step (16-bit caches: the pools are
            outputs).

Lengths lie between ``shortest`` and ``longest``, drawn from ``lens``.
"""
import math
import random

import torch

own = False

TYPES = {"fp16": torch.float16, "bf16": torch.bfloat16}
MOST_BYTES = 2.1e9      # of a drawn case: the largest listed one needs 2.2e9


def _case(name, kind, B, Hq, Hk, d, page, act, int8, shortest, longest, lens=0, nhd=False, new_lo=0, new_hi=0, dense=False,
          peak=1.0, append=False, lse=False):
    return dict(name=name, kind=kind, B=B, Hq=Hq, Hk=Hk, d=d, page=page, act=act, int8=int8, shortest=shortest, longest=longest,
                lens=lens, nhd=nhd, new_lo=new_lo, new_hi=new_hi, dense=dense, peak=peak, append=append, lse=lse)


def listed():
    return [
        # the smallest call: the new token of one sequence; the launch counts
        _case("append_1_token", "append", 1, 8, 8, 128, 16, "fp16", False, 700, 700, new_lo=1, new_hi=1),
        # prompts of a batch into a 16-bit cache whose tokens lie outside the heads
        _case("append_8_prompts_bf16", "append", 8, 32, 8, 128, 16, "bf16", False, 40, 5000, lens=7, nhd=True, new_lo=37, new_hi=5000),
        # the new tokens of a decode batch, quantised as they are written
        _case("append_64_tokens_int8", "append", 64, 32, 8, 128, 64, "fp16", True, 100, 4000, lens=3, new_lo=1, new_hi=1),
        # one chunk of a long prompt, quantised
        _case("append_8k_chunk_int8", "append", 1, 32, 8, 128, 128, "fp16", True, 24576, 24576, new_lo=8192, new_hi=8192),
        # the context that a chunked prefill attends to, dense
        _case("gather_24k_int8_dense", "gather", 1, 32, 8, 128, 128, "fp16", True, 24576, 24576, dense=True),
        # contexts of a batch, packed, heads of 64
        _case("gather_16_ragged_bf16_d64", "gather", 16, 32, 8, 64, 32, "bf16", False, 1, 12288, lens=5),
        # one short conversation
        _case("decode_1x500_int8", "decode", 1, 32, 8, 128, 16, "fp16", True, 500, 500, peak=2.0),
        # a batch of eight long sequences
        _case("decode_8x32k_int8", "decode", 8, 32, 8, 128, 128, "fp16", True, 32768, 32768),
        # the same, more of them, in a 16-bit cache: the largest
        _case("decode_16x32k_bf16", "decode", 16, 32, 4, 128, 64, "bf16", False, 30000, 32768, lens=2, peak=2.0, lse=True),
        # a whole step of a batch in mixed stages, small pages, heads of 64
        _case("step_64_ragged_fp16_d64", "decode", 64, 32, 8, 64, 16, "fp16", False, 1, 8192, lens=4, peak=4.0, append=True),
        # many short sequences and empty places of the batch, seven query heads of 64 a KV head
        _case("decode_256_short_int8_d64", "decode", 256, 28, 4, 64, 16, "fp16", True, 0, 700, lens=6, lse=True, peak=2.0),
        # one very long sequence of a model with two KV heads
        _case("decode_1x128k_int8", "decode", 1, 32, 2, 128, 64, "bf16", True, 131000, 131000, peak=4.0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        kind = rng.choice(["append", "append", "gather", "gather", "decode", "decode", "decode", "decode"])
        Hq, Hk = rng.choice([(8, 8), (32, 32), (32, 8), (16, 4), (28, 4), (64, 8), (32, 2), (12, 1), (6, 2)])
        longest = _log(rng, 1, 131072)
        shortest = rng.choice([longest, rng.randint(1, longest), 0])
        c = _case("", kind, _log(rng, 1, 256), Hq, Hk, rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128]),
                  rng.choice(["fp16", "bf16"]), rng.random() < 0.5, shortest, longest, lens=rng.randrange(1 << 20),
                  nhd=rng.random() < 0.25, dense=rng.random() < 0.5, peak=rng.choice([1.0, 2.0, 4.0]),
                  append=rng.random() < 0.3, lse=rng.random() < 0.5)
        if kind == "append":
            c["new_hi"] = _log(rng, 1, 16384)
            c["new_lo"] = rng.choice([c["new_hi"], 1, rng.randint(1, c["new_hi"])])
        if c["append"] and (kind != "decode" or c["int8"] or c["shortest"] < 1):
            c["append"] = False
        del c["name"]
        w = work(c)
        if w["bytes"] <= MOST_BYTES and sum(_lengths(c)[0]) * c["Hk"] * c["d"] <= 6e8:
            return c


def _lengths(case):
    """Tokens of each sequence's context, new ones included, and how many of them are new."""
    r = random.Random(case["lens"])
    ctx = [r.randint(case["shortest"], case["longest"]) for _ in range(case["B"])]
    new = [r.randint(case["new_lo"], case["new_hi"]) for _ in range(case["B"])] if case["kind"] == "append" else [0] * case["B"]
    return [c + n for c, n in zip(ctx, new)], new


def _quantise(x):
    """Codes (as FP32) and scales of rows of ``x``: delta = max|x| / 127, code = x / delta to the nearest, ties to even."""
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    delta = top / torch.full_like(top, 127.0)       # (by a tensor: a number would be multiplied by its reciprocal)
    return torch.where(delta > 0, x / delta, 0.0).round().clamp(-127, 127), delta


def _pool(case, n_pages, gen):
    """One pool with values in every row (rows that no sequence reaches hold what was there before), and its scales."""
    Hk, P, d = case["Hk"], case["page"], case["d"]
    shape = (n_pages, P, Hk, d) if case["nhd"] else (n_pages, Hk, P, d)
    pool = torch.empty(shape, dtype=torch.int8 if case["int8"] else TYPES[case["act"]], device="cuda")
    scale = torch.empty(shape[:-1], dtype=torch.float32, device="cuda") if case["int8"] else None
    step = max(1, (1 << 26) // (P * Hk * d))
    for a in range(0, n_pages, step):
        x = torch.randn((min(step, n_pages - a),) + shape[1:], generator=gen, device="cuda")
        if case["int8"]:
            codes, delta = _quantise(x.to(TYPES[case["act"]]))
            pool[a:a + step] = codes.to(torch.int8)
            scale[a:a + step] = delta[..., 0]
        else:
            pool[a:a + step] = x.to(pool.dtype)
    if case["nhd"]:     # the views that the calls take are [n_pages, Hk, page, d]; scales are dense in that order
        pool = pool.transpose(1, 2)
        scale = scale.transpose(1, 2).contiguous() if case["int8"] else None
    return pool, scale


def prepare(case, seed):
    B, Hq, Hk, d, P = (case[k] for k in ("B", "Hq", "Hk", "d", "page"))
    gen = torch.Generator(device="cuda").manual_seed(seed)
    act = TYPES[case["act"]]
    lens, new = _lengths(case)
    need = torch.tensor([-(-n // P) for n in lens])
    n_pages = int(need.sum()) + 3
    width = max(1, int(need.max()))
    order = torch.randperm(n_pages, generator=torch.Generator().manual_seed(seed + 1))
    at = (need.cumsum(0) - need)[:, None] + torch.arange(width)[None]
    table = torch.where(torch.arange(width)[None] < need[:, None], order[at.clamp(max=n_pages - 1)], 0)
    s = dict(case=case, table=table.int().cuda(), lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
    s["k_pool"], s["k_scale"] = _pool(case, n_pages, gen)
    s["v_pool"], s["v_scale"] = _pool(case, n_pages, gen)
    fresh = new if case["kind"] == "append" else [1] * B if case["append"] else None
    if fresh is not None:
        s["total"] = sum(fresh)
        s["cu"] = torch.tensor([0] + fresh, dtype=torch.int32).cumsum(0).int().cuda()
        s["k_new"] = torch.randn((s["total"], Hk, d), generator=gen, device="cuda").to(act)
        s["v_new"] = torch.randn((s["total"], Hk, d), generator=gen, device="cuda").to(act)
        s["start"] = s["lens"] - torch.tensor(fresh, dtype=torch.int32, device="cuda")
        s["single"] = max(fresh) == 1 and min(fresh) == 1
    if case["kind"] == "gather":
        s["total"], s["longest"] = sum(lens), max(lens)
        s["cu"] = torch.tensor([0] + lens, dtype=torch.int32).cumsum(0).int().cuda()
        s["start"] = None
    if case["kind"] == "gather" or (case["kind"] == "append" and case["int8"]):
        shape = (B, Hk, s["longest"], d) if case["kind"] == "gather" and case["dense"] else (s["total"], Hk, d)
        s["k_out"] = torch.zeros(shape, dtype=act, device="cuda")
        s["v_out"] = torch.zeros(shape, dtype=act, device="cuda")
    if case["kind"] == "decode":
        s["q"] = (torch.randn((B, Hq, d), generator=gen, device="cuda") * case["peak"]).to(act)
    return s


# ---------------------------------------------------------------------------------------------------- the plain forms

def _places(s):
    """Of the packed tokens [start, cache_len) of the sequences: page and row."""
    t = torch.arange(s["total"], device="cuda")
    b = torch.searchsorted(s["cu"][1:].contiguous(), t.int(), right=True)
    pos = t - s["cu"].long()[b] + (s["start"].long()[b] if s["start"] is not None else 0)
    return s["table"].long()[b, pos // s["case"]["page"]], pos % s["case"]["page"]


def _values(pool, scale, *at):
    x = pool[at].float()
    return x if scale is None else x * scale[at][..., None]


def _plain_append(s):
    page, row = _places(s)
    for x, pool, scale in ((s["k_new"], s["k_pool"], s["k_scale"]), (s["v_new"], s["v_pool"], s["v_scale"])):
        if scale is None:
            pool[page, :, row] = x
        else:
            codes, delta = _quantise(x)
            pool[page, :, row] = codes.to(torch.int8)
            scale[page, :, row] = delta[..., 0]


def _plain_gather(s, dense):
    act = TYPES[s["case"]["act"]]
    if not dense:
        page, row = _places(s)
        return tuple(_values(s[p + "_pool"], s[p + "_scale"], page, slice(None), row).to(act) for p in "kv")
    n = s["longest"]
    live = (torch.arange(n, device="cuda")[None] < s["lens"][:, None])[:, None, :, None]
    return tuple(torch.where(live, _contexts(s, p, n), 0.0).to(act) for p in "kv")


def _contexts(s, p, n):
    """[B, Hk, n, d] in FP32: the pages of each sequence one behind the other."""
    c = s["case"]
    x = _values(s[p + "_pool"], s[p + "_scale"], s["table"].long())
    return x.transpose(1, 2).reshape(c["B"], c["Hk"], -1, c["d"])[:, :, :n]


def _plain_decode(s):
    c, q = s["case"], s["q"]
    B, Hk, d = c["B"], c["Hk"], c["d"]
    n = s["table"].shape[1] * c["page"]
    live = (torch.arange(n, device="cuda")[None] < s["lens"][:, None])[:, None, None]
    scores = q.float().view(B, Hk, -1, d) @ _contexts(s, "k", n).transpose(2, 3) / math.sqrt(d)
    scores = torch.where(live, scores, -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top > -math.inf, top, 0.0)
    p = torch.exp(scores - top)
    z = p.sum(-1, keepdim=True)                     # 0 where there is no key: the row is 0, its log-sum-exp -inf
    v = torch.where(live.transpose(2, 3), _contexts(s, "v", n), 0.0)
    out = ((p / torch.where(z > 0, z, 1.0)) @ v).reshape(B, -1, d).to(q.dtype)
    return out, (top + torch.log(z)).reshape(B, -1)


# ---------------------------------------------------------------------------------------------------- one pass

def _cache(s):
    """The description of the cache that a program keeps beside its pools, and the workspace of its stream."""
    if "cache" not in s:
        from paper_2608_17336_b200 import binding as tm
        s["tm"] = tm
        s["cache"] = tm.paged_cache(s["k_pool"], s["v_pool"], s["table"], s["lens"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                                    dtype=TYPES[s["case"]["act"]])
        s["ws"] = torch.empty(tm.tilemix_paged_decode_workspace_size(s["cache"], s["case"]["Hq"]), dtype=torch.uint8, device="cuda")
    return s["tm"], s["cache"]


def run(s):
    c = s["case"]
    if own:
        tm, cache = _cache(s)
        if c["kind"] == "append" or c["append"] and c["kind"] == "decode":
            tm.tilemix_paged_append(cache, s["k_new"], s["v_new"], cu_new=None if s["single"] else s["cu"])
        if c["kind"] == "decode":
            r = tm.tilemix_paged_decode(cache, s["q"], want_lse=c["lse"], workspace=s["ws"])
            out, lse = r["out"], r["lse"]
        elif c["kind"] == "gather" and c["dense"]:
            tm.tilemix_paged_gather(cache, s["k_out"], s["v_out"])
        elif c["kind"] == "gather" or c["int8"]:
            tm.tilemix_paged_gather(cache, s["k_out"], s["v_out"], start=s["start"], cu_out=s["cu"])
        if c["kind"] == "append" and not c["int8"]:
            return {"k": s["k_pool"], "v": s["v_pool"]}
        if c["kind"] != "decode":
            return {"k": s["k_out"], "v": s["v_out"]}
    else:
        if c["kind"] == "append" or c["append"] and c["kind"] == "decode":
            _plain_append(s)
        if c["kind"] == "append" and not c["int8"]:
            return {"k": s["k_pool"], "v": s["v_pool"]}
        if c["kind"] != "decode":
            return dict(zip("kv", _plain_gather(s, c["kind"] == "gather" and c["dense"])))
        out, lse = _plain_decode(s)
    r = {"out": out, "lse": lse} if c["lse"] else {"out": out}
    return r | {"k": s["k_pool"], "v": s["v_pool"]} if c["append"] else r


def work(case):
    lens, new = _lengths(case)
    rows = case["Hk"] * (sum(new) if case["kind"] == "append" else sum(lens))      # (token, head) pairs that the pass is about
    d = case["d"]
    held = 2 * (d + 4 if case["int8"] else 2 * d)                                  # bytes of a pair in the cache, K and V
    dense = 2 * 2 * d
    small = 4 * case["B"] + 4 * sum(-(-n // case["page"]) for n in (new if case["kind"] == "append" else lens))
    if case["kind"] == "append":
        # the new rows in; the cache's rows out; for the INT8 cache the values that they stand for, out
        return {"bytes": rows * (dense + held + (dense if case["int8"] else 0)) + small, "flops": rows * 2 * d * (4 if case["int8"] else 0)}
    if case["kind"] == "gather":
        return {"bytes": rows * (held + dense) + small, "flops": rows * 2 * d if case["int8"] else 0}
    n = case["B"] * case["Hq"]
    step = case["B"] * case["Hk"] * (dense + held) if case["append"] else 0
    return {"bytes": rows * held + n * d * 4 + (4 * n if case["lse"] else 0) + small + step,
            "flops": 4 * d * sum(lens) * case["Hq"]}


# ---------------------------------------------------------------------------------------------------- in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    lens, new = _lengths(case)
    B, Hk, d, P = (case[k] for k in ("B", "Hk", "d", "page"))
    if sum(lens) * Hk * d > 6e8:
        return None
    table = s["table"].long()

    def requantised(x):
        x = x.double()
        delta = x.abs().amax(-1, keepdim=True) / 127
        return torch.where(delta > 0, torch.round(x / delta) * delta, x)

    def context(p, b):
        """[len, Hk, d]: the values of sequence b as the cache holds them after the pass's writes."""
        n = lens[b]
        at = table[b, :-(-n // P)]
        x = s[p + "_pool"][at].double()
        if case["int8"]:
            x = x * s[p + "_scale"][at].double()[..., None]
        x = x.permute(0, 2, 1, 3).reshape(-1, Hk, d)[:n]
        if case["kind"] == "append" or case["append"]:
            fresh = s[p + "_new"][int(s["cu"][b]):int(s["cu"][b + 1])]
            x = torch.cat([x[:n - fresh.shape[0]], requantised(fresh) if case["int8"] else fresh.double()])
        return x

    if case["kind"] == "append" and not case["int8"]:
        return None         # a copy
    if case["kind"] == "append":
        return {p: requantised(s[p + "_new"]) for p in "kv"}
    if case["kind"] == "gather":
        if not case["dense"]:
            return {p: torch.cat([context(p, b) for b in range(B)]) for p in "kv"}
        found = {p: torch.zeros((B, Hk, max(lens), d), dtype=torch.float64, device="cuda") for p in "kv"}
        for p in "kv":
            for b in range(B):
                found[p][b, :, :lens[b]] = context(p, b).transpose(0, 1)
        return found
    out, lse = [], []
    for b in range(B):
        q = s["q"][b].double().view(Hk, -1, d)
        scores = torch.einsum("hrd,nhd->hrn", q, context("k", b)) * d ** -0.5
        weight = torch.softmax(scores, -1)          # (of no key: the sum below is empty)
        out.append(torch.einsum("hrn,nhd->hrd", weight, context("v", b)).reshape(-1, d))
        lse.append(torch.logsumexp(scores, -1).reshape(-1))
    r = {"out": torch.stack(out)} | ({"lse": torch.stack(lse)} if case["lse"] else {})
    return r | {"k": None, "v": None} if case["append"] else r      # (the pools: a copy)
