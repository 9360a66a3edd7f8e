"""Paged key/value cache in 64 bits, from its definition: test infrastructure of the paged calls."""
import math

import numpy as np
import torch

ACT = {"fp16": torch.float16, "bf16": torch.bfloat16}


def f64(t):
    return t.detach().cpu().double().numpy()


def quantise(x):
    """Rows of float32 values -> codes, scales: delta = RN(max|x| / 127), code = RN(RN(x / delta)) in IEEE binary32, zero rows
    delta 0 and codes 0, rows with a value that is not finite delta NaN and codes 0."""
    x = np.asarray(x, np.float32)
    with np.errstate(all="ignore"):
        delta = np.abs(x).max(-1) / np.float32(127)
        code = np.rint(x / delta[..., None])
    bad = ~np.isfinite(x).all(-1)
    delta = np.where(bad, np.float32(np.nan), delta).astype(np.float32)
    code = np.where((bad | (delta == 0))[..., None], 0, np.clip(code, -127, 127))
    return code.astype(np.int8), delta


class Setup:
    """A cache with random contents in every row of its pools (rows that no sequence reaches included), pages dealt out at
    random.  ``stale``: what the pools hold in rows that no sequence reaches (NaN: reading them shows)."""

    def __init__(self, act, int8, d, page, hk, lens, seed=0, nhd=False, spare=2, room=0, stale=None, device="cpu", gain=1.0):
        g = torch.Generator().manual_seed(seed)
        self.act, self.int8, self.d, self.page, self.hk, self.lens = ACT[act], int8, d, page, hk, list(lens)
        B = len(lens)
        need = [-(-n // page) for n in lens]
        width = max(1, max(need)) + room
        n_pages = B * room + sum(need) + spare
        order = torch.randperm(n_pages, generator=g)
        table = torch.full((B, width), 1 << 29, dtype=torch.int32)      # entries past a sequence's end are not looked at
        used = 0
        live = torch.zeros((n_pages, page), dtype=torch.bool)
        for b in range(B):
            k = need[b] + room
            table[b, :k] = order[used:used + k].int()
            used += k
            for j in range(need[b]):
                live[table[b, j], :min(page, lens[b] - j * page)] = True
        shape = (n_pages, page, hk, d) if nhd else (n_pages, hk, page, d)
        self.table = table
        self.cache_len = torch.tensor(lens, dtype=torch.int32)
        for p in "kv":
            x = (torch.randn(shape, generator=g) * gain).to(self.act)
            scale = None
            if nhd:
                x = x.transpose(1, 2)
            if int8:
                code, delta = quantise(x.float().numpy())
                scale = torch.from_numpy(np.ascontiguousarray(delta))
                pool = torch.from_numpy(code)
                x = torch.empty(shape, dtype=torch.int8)
                x = x.transpose(1, 2) if nhd else x
                x.copy_(pool)
                if stale is not None:
                    scale.transpose(1, 2)[~live] = stale
            elif stale is not None:
                x.transpose(1, 2)[~live] = stale
            setattr(self, p + "_pool", x)
            setattr(self, p + "_scale", scale)
        if device != "cpu":
            self.to(device)

    def to(self, device):
        for name in ("table", "cache_len", "k_pool", "v_pool", "k_scale", "v_scale"):
            t = getattr(self, name)
            if t is not None:       # (keeps the strides of a view)
                u = torch.empty_strided(t.shape, t.stride(), dtype=t.dtype, device=device)
                setattr(self, name, u.copy_(t))
        return self

    def cache(self):
        from paper_2608_17336_b200 import binding as tm
        return tm.paged_cache(self.k_pool, self.v_pool, self.table, self.cache_len, self.k_scale, self.v_scale, dtype=self.act)

    def context(self, p, b):
        """(values [len, Hk, d] in float64, present [len]) of sequence b; holes are zeros and not present."""
        n = int(self.cache_len[b])
        n = min(max(n, 0), self.table.shape[1] * self.page)
        pool, scale, table = getattr(self, p + "_pool"), getattr(self, p + "_scale"), self.table[b].cpu()
        out, present = np.zeros((n, self.hk, self.d)), np.zeros(n, bool)
        for j in range(-(-n // self.page)):
            page, rows = int(table[j]), min(self.page, n - j * self.page)
            if not 0 <= page < pool.shape[0]:
                continue
            x = f64(pool[page])
            if scale is not None:
                x = x * f64(scale[page])[..., None]
            out[j * self.page:j * self.page + rows] = x.transpose(1, 0, 2)[:rows]
            present[j * self.page:j * self.page + rows] = True
        return out, present


def attend(s, q, scale=0.0, only=None):
    """float64 (out [B,Hq,d], lse [B,Hq]) and bounds of what the kernel may be off by, from the arithmetic it states.

    ``only``: (sequence, head) pairs; the rest stays empty.
    u = half a step of the 16-bit type: outputs are rounded (u |o|).  A probability is a sum of two 16-bit numbers, the second
    the first's rounding error, rounded (u^2 of it; in all u^2 A, A = sum p |v|), over INT8 caches one FP16 number (2^-11;
    of the last keys two); those below 2^-28 of the largest are subnormal FP16 (at most 2^-39 of the
    largest each).  A score of magnitude S (sum of |q_i k_i|,
    log2 units) is off by at most (d + 8) 2^-23 S (FP32 products summed in any order, each sum rounded to nearest or
    towards zero; scales), the exponential by 2^-22, FP32 sums over n keys by n 2^-24: relative errors of p of at most e,
    hence 2 e A (numerator and denominator)."""
    B, hq, d = q.shape
    scale = scale or 1 / math.sqrt(d)
    u = torch.finfo(s.act).eps / 2
    up = 2.0 ** -11 if s.int8 else u * u
    out, lse = np.zeros((B, hq, d)), np.full((B, hq), -np.inf)
    tol, tol_lse = np.zeros((B, hq, d)), np.zeros((B, hq))
    qd = f64(q)
    for b in range(B):
        if only is not None and not any(x == b for x, _ in only):
            continue
        k, present = s.context("k", b)
        v, _ = s.context("v", b)
        k, v = k[present], v[present]
        n = len(k)
        if n == 0:
            continue
        for h in range(hq):
            if only is not None and (b, h) not in only:
                continue
            kk, vv = k[:, h * s.hk // hq], v[:, h * s.hk // hq]
            sc = (kk @ qd[b, h]) * scale
            top = sc.max()
            p = np.exp(sc - top)
            z = p.sum()
            out[b, h], lse[b, h] = (p / z) @ vv, top + np.log(z)
            big = (np.abs(kk) @ np.abs(qd[b, h])).max() * scale * math.log2(math.e)
            e = (d + 8) * 2.0 ** -23 * big + 2.0 ** -22 + n * 2.0 ** -24
            mass = (p / z) @ np.abs(vv)
            tol[b, h] = u * np.abs(out[b, h]) + (up + 2 * e) * 1.01 * mass + n * 2.0 ** -39 * np.abs(vv).max() / z
            tol_lse[b, h] = e + 2.0 ** -22 * (abs(lse[b, h]) + big)
    return out, lse, tol + torch.finfo(s.act).tiny * u, tol_lse


def check_decode(s, q, res, scale=0.0, only=None):
    out, lse, tol, tol_lse = attend(s, q, scale, only)
    got, lse_got = f64(res["out"]), res["lse"]
    if only is not None:
        b, h = (list(x) for x in zip(*only))
        out, lse, tol, tol_lse, got = out[b, h], lse[b, h], tol[b, h], tol_lse[b, h], got[b, h]
        lse_got = None if lse_got is None else lse_got[b, h]
    off = np.abs(got - out)
    assert (off <= tol).all(), f"out: {(off / tol).max():.2f} of the bound at {np.unravel_index((off / tol).argmax(), off.shape)}"
    if lse_got is not None:
        got = f64(lse_got)
        empty = np.isneginf(lse)
        assert (np.isneginf(got) == empty).all()
        assert (np.abs(got[~empty] - lse[~empty]) <= tol_lse[~empty]).all()
    return float((off / np.maximum(tol, 1e-300)).max())
