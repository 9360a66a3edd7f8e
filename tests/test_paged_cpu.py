"""Paged key/value cache, on the CPU: layouts of the C struct, refusals before anything is launched, sizes, the reference."""
import ctypes

import numpy as np
import pytest
import torch

from paper_2608_17336_b200 import binding as b
from tests import paged_ref as ref

ONE = ctypes.c_void_p(4096)
I64 = ctypes.c_int64


@pytest.fixture(scope="module")
def lib():
    from paper_2608_17336_b200 import build
    build.build()
    return b.lib()


def struct(**kw):
    p = b.PagedStruct(2, 2, 128, 16, 10, 4, b.TYPE_FP16, b.CACHE_INT8)
    for n in ("k_pool", "v_pool", "k_scale", "v_scale", "block_table", "cache_len"):
        setattr(p, n, 4096)
    for n, v in kw.items():
        if isinstance(v, tuple):
            getattr(p, n)[:] = v
        else:
            setattr(p, n, v)
    return p


def append(lib, p, n=2, k=ONE, ks=None, v=ONE, vs=None, cu=None):
    return lib.tilemix_paged_append(p and ctypes.byref(p), n, k, ks, v, vs, cu, None)


def gather(lib, p, start=None, cu=None, n=64, k=ONE, ks=None, v=ONE, vs=None):
    return lib.tilemix_paged_gather(p and ctypes.byref(p), start, cu, n, k, ks, v, vs, None)


def decode(lib, p, hq=8, q=ONE, qs=None, out=ONE, os=None, ws=ONE, nbytes=1 << 40):
    return lib.tilemix_paged_decode(p and ctypes.byref(p), hq, 0.0, q, qs, out, os, None, ws, nbytes, None)


def test_struct_layout():
    assert ctypes.sizeof(b.PagedStruct) == 8 * 4 + 7 * 8 + 6 * 8
    assert b.PagedStruct.k_stride.offset == 32 and b.PagedStruct.table_stride.offset == 80 and b.PagedStruct.k_pool.offset == 88


@pytest.mark.parametrize("call", [append, gather, decode])
@pytest.mark.parametrize("want,change", [
    (b.ERR_SHAPE, dict(batch=0)), (b.ERR_SHAPE, dict(heads_kv=-1)), (b.ERR_SHAPE, dict(head_dim=0)), (b.ERR_SHAPE, dict(page_size=0)),
    (b.ERR_SHAPE, dict(n_pages=0)), (b.ERR_SHAPE, dict(max_pages=0)), (b.ERR_SHAPE, dict(max_pages=1 << 27)),
    (b.ERR_SHAPE, dict(table_stride=3)), (b.ERR_UNSUPPORTED, dict(head_dim=96)), (b.ERR_UNSUPPORTED, dict(page_size=8)),
    (b.ERR_UNSUPPORTED, dict(page_size=48)), (b.ERR_UNSUPPORTED, dict(page_size=512)), (b.ERR_UNSUPPORTED, dict(act_type=2)),
    (b.ERR_UNSUPPORTED, dict(cache_type=-1)), (b.ERR_NULL, dict(k_pool=None)), (b.ERR_NULL, dict(v_pool=None)),
    (b.ERR_NULL, dict(k_scale=None)), (b.ERR_NULL, dict(block_table=None)), (b.ERR_NULL, dict(cache_len=None)),
    (b.ERR_ALIGN, dict(k_pool=4104)), (b.ERR_ALIGN, dict(v_scale=4097)), (b.ERR_ALIGN, dict(cache_len=4098)),
    (b.ERR_ALIGN, dict(k_stride=(2 * 16 * 136, 16 * 136, 136))),
    (b.ERR_SHAPE, dict(v_stride=(2 * 16 * 128, 16 * 128, 64))),        # rows that overlap
    (b.ERR_SHAPE, dict(v_stride=(2 * 16 * 128, 0, 128))),              # heads that share their rows
    (b.ERR_SHAPE, dict(k_stride=(16 * 128, 16 * 128, 128))),           # pages on top of heads
    (b.ERR_SHAPE, dict(k_stride=(1 << 42, 16 * 128, 128))),
])
def test_refusals_of_the_description(lib, call, want, change):
    assert call(lib, struct(**change)) == want
    assert lib.tilemix_paged_decode_workspace_size(ctypes.byref(struct(**change)), 8) == 0


def test_refusals_of_the_calls(lib):
    ok = struct()
    for call in (append, gather, decode):
        assert call(lib, None) == b.ERR_NULL
        # the 16-byte multiple is one of the elements' size: 136 halves are, 136 codes are not
    assert append(lib, ok, n=3) == b.ERR_SHAPE and append(lib, ok, n=-1, cu=ONE) == b.ERR_SHAPE
    assert append(lib, ok, n=0, cu=ONE, k=None, v=None) == b.OK                  # nothing to do
    assert append(lib, ok, k=None) == b.ERR_NULL and append(lib, ok, v=None) == b.ERR_NULL
    assert append(lib, ok, k=ctypes.c_void_p(4104)) == b.ERR_ALIGN and append(lib, ok, n=9, cu=ctypes.c_void_p(4098)) == b.ERR_ALIGN
    assert append(lib, ok, ks=(I64 * 2)(260, 128)) == b.ERR_ALIGN and append(lib, ok, vs=(I64 * 2)(-256, 128)) == b.ERR_SHAPE
    assert append(lib, ok, n=1 << 30, cu=ONE) == b.ERR_SHAPE
    assert gather(lib, ok, n=-1) == b.ERR_SHAPE and gather(lib, ok, n=0, k=None, v=None) == b.OK
    assert gather(lib, ok, k=None) == b.ERR_NULL and gather(lib, ok, v=ctypes.c_void_p(4098)) == b.ERR_ALIGN
    assert gather(lib, ok, start=ctypes.c_void_p(4097)) == b.ERR_ALIGN
    assert gather(lib, ok, ks=(I64 * 3)(2 * 64 * 128, 64 * 128, 64)) == b.ERR_SHAPE      # output rows that overlap
    assert gather(lib, ok, vs=(I64 * 3)(2 * 64 * 128, 64 * 132, 132)) == b.ERR_ALIGN
    assert gather(lib, ok, n=1 << 30) == b.ERR_SHAPE
    size = lib.tilemix_paged_decode_workspace_size(ctypes.byref(ok), 8)
    assert size > 0
    for hq in (0, -2, 3):
        assert decode(lib, ok, hq=hq) == b.ERR_SHAPE
        assert lib.tilemix_paged_decode_workspace_size(ctypes.byref(ok), hq) == 0
    assert decode(lib, ok, q=None) == b.ERR_NULL and decode(lib, ok, out=None) == b.ERR_NULL and decode(lib, ok, ws=None) == b.ERR_NULL
    assert decode(lib, ok, q=ctypes.c_void_p(4104)) == b.ERR_ALIGN and decode(lib, ok, out=ctypes.c_void_p(4100)) == b.ERR_ALIGN
    assert decode(lib, ok, qs=(I64 * 2)(8 * 128, 132)) == b.ERR_ALIGN and decode(lib, ok, os=(I64 * 2)(8 * 128, 64)) == b.ERR_SHAPE
    assert decode(lib, ok, nbytes=size - 1) == b.ERR_WORKSPACE
    assert lib.tilemix_paged_decode(ctypes.byref(ok), 8, 0.0, ONE, None, ONE, None, ctypes.c_void_p(4098), ONE, size, None) == b.ERR_ALIGN
    # more places than the counts have bits for
    assert decode(lib, struct(max_pages=1 << 26, heads_kv=1024)) == b.ERR_SHAPE


def test_binding_refuses_before_the_call():
    s = ref.Setup("fp16", True, 64, 16, 2, [20, 3])
    with pytest.raises(AssertionError):
        s.cache()                                         # not on a GPU
    k = s.k_pool
    for kw in (dict(v_pool=s.v_pool[:-1]), dict(block_table=s.table.long()), dict(cache_len=s.cache_len[:1]), dict(dtype=torch.float32),
               dict(k_scale=None), dict(v_scale=s.v_scale.double()), dict(k_pool=k[..., ::2], v_pool=s.v_pool[..., ::2])):
        a = dict(k_pool=k, v_pool=s.v_pool, block_table=s.table, cache_len=s.cache_len, k_scale=s.k_scale, v_scale=s.v_scale)
        with pytest.raises(AssertionError):
            b.paged_cache(**(a | kw))


def test_reference_quantiser_is_the_oracles():
    import oracle
    g = torch.Generator().manual_seed(3)
    x = (torch.randn((1, 2, 50, 64), generator=g) * torch.logspace(-6, 3, 50)[:, None]).half()
    x[0, 1, 7] = 0
    code, delta = ref.quantise(x.float().numpy())
    want, scale = oracle.quantize(x.view(torch.int16).numpy().view(np.uint16), 1)
    assert np.array_equal(code, want) and np.array_equal(delta.view(np.uint32), scale.view(np.uint32))


def test_one_fma_codes_hold_for_bfloat16():
    """The quantiser's rounded quotient from one FMA (csrc/quant8.cuh) equals the definition for every bfloat16 maximum and
    magnitude of one binade set: the arithmetic in float64, whose products of 24-bit factors are exact, rounded as the
    instructions round."""
    f = np.float32
    mant = np.arange(128, 256, dtype=np.float64)
    for e in (-100, -3, 0, 90):
        for a in mant:
            amax = f(a * 2.0 ** e)
            delta = f(amax / f(127))
            r = f(1.0 / np.float64(delta))
            half = f(0.5) * amax
            fma = lambda x, y, z: f(np.float64(x) * np.float64(y) + np.float64(z))      # noqa: E731  (exact here: see below)
            up = fma(-63.5, delta, half) >= f(-1.9073486328125e-6) * delta
            side = fma(half, r, -63.5)
            if up and side < 0:
                r = np.nextafter(r, f(np.inf))
            if not up and side >= 0:
                r = np.nextafter(r, f(0))
            refine = fma(127.0, delta, -amax) == 0 or (fma(half, r, -63.5) >= 0) != up
            x = np.concatenate([mant * 2.0 ** (e - s) for s in range(0, 10)])
            x = x[x <= amax].astype(f)
            want = np.rint(x / delta)
            if refine:
                q = x * r
                res = (x.astype(np.float64) - np.float64(delta) * q).astype(f)          # < 53 bits: exact before the rounding
                q = (q + res.astype(np.float64) * np.float64(r)).astype(f)
                got = np.rint(q)
            else:
                # x r + 1.5 2^23, rounded once to the nearest integer, ties to even: x (8 bits) r (24 bits) is exact
                got = np.rint(x.astype(np.float64) * np.float64(r))
            assert np.array_equal(got, want), (e, a)


def test_expanded_views_are_refused():
    """Strides of zero would mean dense ones: an expanded table or pool must not be read past its end."""
    pool, n = torch.zeros((4, 2, 16, 64), dtype=torch.float16), torch.zeros(3, dtype=torch.int32)
    table = torch.zeros((3, 2), dtype=torch.int32)
    with pytest.raises(AssertionError, match="overlap"):
        b.paged_cache(pool, pool, table[:1].expand(3, 2), n)
    with pytest.raises(AssertionError, match="expanded"):
        b.paged_cache(pool, torch.zeros(64, dtype=torch.float16).expand(4, 2, 16, 64), table, n)
    with pytest.raises(AssertionError, match="one CUDA device"):        # (the others pass the checks of shapes and strides)
        b.paged_cache(pool, pool, table, n)
    with pytest.raises(AssertionError, match="one CUDA device"):
        b.paged_cache(pool, pool, table[:1], n[:1])
