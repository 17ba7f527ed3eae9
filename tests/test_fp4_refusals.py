"""Refusals of the 4-bit operators at the C boundary (CPU: every check comes before any
device work, so the pointers are never followed)."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2609_34608_amd import _lib as L

P = 0x10000  # an aligned address that nothing reads


def _i64(*v):
    return (C.c_int64 * len(v))(*v)


def _set(a, kw):
    for n, v in kw.items():
        at, *names = n.split("__")
        o = a
        for name in names:
            o, at = getattr(o, at), name
        setattr(o, at, v)
    return a


def _refused(fn, a, code, text):
    lib = L.lib()
    assert getattr(lib, fn)(C.byref(a) if a is not None else None, None) == code
    assert text in lib.wam_noalloc_last_error().decode()
    assert fn in lib.wam_noalloc_last_error().decode()


@pytest.mark.parametrize("fn", ["wam_quantize_fp4", "wam_dequantize_fp4", "wam_matmul_fp4", "wam_cache_append",
                                "wam_cache_attention"])
def test_null(fn):
    _refused(fn, None, L.WAM_E_ARG, "null argument")


def _quant(**kw):
    return _set(L.WamQuantizeFp4Args(4, 256, L.WAM_BF16, P, 256, P + 4096, 128, P + 8192, 8), kw)


@pytest.mark.parametrize("kw,code,text", [
    (dict(M=-1), L.WAM_E_ARG, "sizes"), (dict(dtype=L.WAM_FP8), L.WAM_E_ARG, "WAM_FP32"), (dict(x=None), L.WAM_E_ARG, "null"),
    (dict(q=None), L.WAM_E_ARG, "null"), (dict(scale=None), L.WAM_E_ARG, "null"), (dict(x=P + 1), L.WAM_E_ARG, "aligned"),
    (dict(q=P), L.WAM_E_ARG, "different"), (dict(scale=P + 4096), L.WAM_E_ARG, "different"),
    (dict(x_stride=-1), L.WAM_E_ARG, "strides"), (dict(q_stride=127), L.WAM_E_ARG, "distinct"),
    (dict(scale_stride=7), L.WAM_E_ARG, "distinct"), (dict(x_stride=2**41), L.WAM_E_ARG, "strides"),
    (dict(M=2**26, K=512, q_stride=256, scale_stride=16), L.WAM_E_SHAPE, "too many"),
    (dict(M=1, K=2**31 - 1, q_stride=2**30, scale_stride=2**27), L.WAM_E_SHAPE, "too many")])
def test_quantize_refuses(kw, code, text):
    _refused("wam_quantize_fp4", _quant(**kw), code, text)


def _dequant(**kw):
    return _set(L.WamDequantizeFp4Args(4, 256, L.WAM_BF16, P, 128, P + 4096, 8, P + 8192, 256), kw)


@pytest.mark.parametrize("kw,code,text", [
    (dict(K=-1), L.WAM_E_ARG, "sizes"), (dict(dtype=7), L.WAM_E_ARG, "WAM_FP32"), (dict(x=None), L.WAM_E_ARG, "null"),
    (dict(x=P + 8193), L.WAM_E_ARG, "aligned"), (dict(x=P), L.WAM_E_ARG, "must not"), (dict(x_stride=255), L.WAM_E_ARG, "distinct"),
    (dict(q_stride=-1), L.WAM_E_ARG, "strides"), (dict(M=2**26, K=512, x_stride=512), L.WAM_E_SHAPE, "too many")])
def test_dequantize_refuses(kw, code, text):
    _refused("wam_dequantize_fp4", _dequant(**kw), code, text)


def _matmul(**kw):
    return _set(L.WamMatmulFp4Args(4, 64, 256, L.WAM_BF16, L.WAM_ACT_NONE, P, 128, P + 4096, 8, P + 8192, 128, P + 32768, 8,
                                   None, P + 65536, 64), kw)


@pytest.mark.parametrize("kw,code,text", [
    (dict(N=-1), L.WAM_E_ARG, "sizes"), (dict(out_dtype=L.WAM_FP8), L.WAM_E_ARG, "WAM_FP4"), (dict(act=2), L.WAM_E_ARG, "activation"),
    (dict(K=0), L.WAM_E_SHAPE, "K must"), (dict(K=255), L.WAM_E_SHAPE, "even"), (dict(M=2**31 - 1), L.WAM_E_SHAPE, "too large"),
    (dict(a=None), L.WAM_E_ARG, "null"), (dict(w_scale=None), L.WAM_E_ARG, "null"), (dict(out=None), L.WAM_E_ARG, "null"),
    (dict(a=P + 8), L.WAM_E_ARG, "16 bytes"), (dict(w_stride=136), L.WAM_E_ARG, "16 bytes"), (dict(a_stride=112), L.WAM_E_ARG, "16 bytes"),
    (dict(a_scale=P + 4098), L.WAM_E_ARG, "4 bytes"), (dict(w_scale_stride=10), L.WAM_E_ARG, "4 bytes"),
    (dict(a_scale_stride=4), L.WAM_E_ARG, "4 bytes"), (dict(bias=P + 2), L.WAM_E_ARG, "bias"), (dict(out=P + 65537), L.WAM_E_ARG, "aligned"),
    (dict(out_stride=63), L.WAM_E_ARG, "distinct"), (dict(out=P), L.WAM_E_ARG, "operand"), (dict(out_dtype=L.WAM_FP4), L.WAM_E_ARG, "out_scale"),
    (dict(out_dtype=L.WAM_FP4, out_scale=P + 131072, out_scale_stride=1), L.WAM_E_ARG, "out_scale"),
    (dict(out_dtype=L.WAM_FP4, out_scale=P + 131072, out_scale_stride=2, out_stride=31), L.WAM_E_ARG, "distinct"),
    (dict(M=2**30, N=2**20, a_stride=128, out_stride=2**20), L.WAM_E_SHAPE, "too many tiles")])
def test_matmul_refuses(kw, code, text):
    _refused("wam_matmul_fp4", _matmul(**kw), code, text)


@pytest.mark.parametrize("at", [P, P + 4096, P + 8192, P + 32768, P + 65536])
def test_matmul_refuses_scales_in_another_buffer(at):
    _refused("wam_matmul_fp4", _matmul(out_dtype=L.WAM_FP4, out_scale=at, out_scale_stride=2), L.WAM_E_ARG, "out_scale must be")


def _cache():
    c = L.WamCache(8, 16, 2, 64, P, P + 16384, P + 32768, P + 49152)
    c.k_stride = c.v_stride = _i64(1024, 32, 512)
    c.k_scale_stride = c.v_scale_stride = _i64(64, 2, 32)
    return c


_TABLE = L.WamPageTable(P, 4, 4)

CACHE = [
    (dict(cache__pages=-1), L.WAM_E_ARG, "pages"), (dict(cache__H=0), L.WAM_E_ARG, "heads"), (dict(table__width=-1), L.WAM_E_ARG, "table"),
    (dict(cache__dh=48), L.WAM_E_SHAPE, "head size"), (dict(cache__dh=160), L.WAM_E_SHAPE, "head size"),
    (dict(cache__page=8), L.WAM_E_SHAPE, "power of two"), (dict(cache__page=48), L.WAM_E_SHAPE, "power of two"),
    (dict(cache__page=8192), L.WAM_E_SHAPE, "power of two"), (dict(table__width=2**27), L.WAM_E_SHAPE, "2^31"),
    (dict(cache__H=2**24), L.WAM_E_SHAPE, "heads"),
    (dict(cache__k=None), L.WAM_E_ARG, "null"), (dict(cache__v_scale=None), L.WAM_E_ARG, "null"), (dict(table__entry=None), L.WAM_E_ARG, "null"),
    (dict(cache__v=P + 2), L.WAM_E_ARG, "4 bytes"), (dict(table__entry=P + 2), L.WAM_E_ARG, "4 bytes"),
    (dict(cache__k_stride=_i64(1026, 32, 512)), L.WAM_E_ARG, "multiples of 4"), (dict(cache__v_scale_stride=_i64(64, -2, 32)), L.WAM_E_ARG, ">= 0"),
    (dict(table__stride=-4), L.WAM_E_ARG, ">= 0"),
]


def _append(**kw):
    freq = np.ones(32)
    a = L.WamCacheAppendArgs(1, 4, L.WAM_BF16, L.WAM_ROPE_HALVES, (C.c_int32 * 3)(8, 12, 12), _cache(), _TABLE, P, P + 4096,
                             _i64(512, 128, 64), _i64(512, 128, 64), P, None, P, 0, freq.ctypes.data, None, 1e-6)
    return _set(a, kw), freq


@pytest.mark.parametrize("kw,code,text", CACHE + [
    (dict(T=-1), L.WAM_E_ARG, "sizes"), (dict(dtype=L.WAM_FP8), L.WAM_E_ARG, "WAM_FP32"), (dict(layout=3), L.WAM_E_ARG, "layout"),
    (dict(sections=(C.c_int32 * 3)(8, -1, 2)), L.WAM_E_ARG, "sections"),
    (dict(sections=(C.c_int32 * 3)(2**31 - 1, 2**31 - 1, 2)), L.WAM_E_SHAPE, "2 P <= dh"), (dict(freq=None), L.WAM_E_ARG, "freq"),
    (dict(pos=None), L.WAM_E_ARG, "pos"), (dict(pos_stride=-1), L.WAM_E_ARG, "pos"), (dict(k_gain=P, eps=-1.0), L.WAM_E_ARG, "eps"),
    (dict(k_gain=P, eps=math.nan), L.WAM_E_ARG, "eps"), (dict(B=2**20, T=2**10), L.WAM_E_SHAPE, "rows"), (dict(k=None), L.WAM_E_ARG, "null"),
    (dict(start=None), L.WAM_E_ARG, "null"), (dict(v=P + 1), L.WAM_E_ARG, "aligned"), (dict(rows=P + 2), L.WAM_E_ARG, "aligned"),
    (dict(v_stride=_i64(512, -128, 64)), L.WAM_E_ARG, "strides"), (dict(cache__k_stride=_i64(1024, 32, 0)), L.WAM_E_ARG, "distinct"),
    (dict(cache__v_scale_stride=_i64(64, 1, 32)), L.WAM_E_ARG, "distinct")])
def test_append_refuses(kw, code, text):
    a, _ = _append(**kw)
    _refused("wam_cache_append", a, code, text)


def _attend(**kw):
    a = L.WamCacheAttentionArgs(1, 4, 4, L.WAM_BF16, 0, _cache(), _TABLE, P, _i64(1024, 256, 64), P + 65536, _i64(1024, 256, 64), None,
                                _i64(0, 0, 0), P, None, 0.125, None, 0)
    return _set(a, kw)


@pytest.mark.parametrize("kw,code,text", CACHE + [
    (dict(B=-1), L.WAM_E_ARG, "sizes"), (dict(dtype=L.WAM_FP8), L.WAM_E_ARG, "WAM_FP32"), (dict(Hq=3), L.WAM_E_SHAPE, "multiple"),
    (dict(Hq=0), L.WAM_E_SHAPE, "multiple"), (dict(scale=0.0), L.WAM_E_ARG, "scale"), (dict(scale=math.nan), L.WAM_E_ARG, "scale"),
    (dict(scale=math.inf), L.WAM_E_ARG, "scale"), (dict(B=2**20, T=2**10), L.WAM_E_SHAPE, "rows"), (dict(T=2**20, Hq=2**12), L.WAM_E_SHAPE, "rows"),
    (dict(q=None), L.WAM_E_ARG, "null"), (dict(lengths=None), L.WAM_E_ARG, "null"), (dict(out=P + 65537), L.WAM_E_ARG, "aligned"),
    (dict(q_stride=_i64(-1, 256, 64)), L.WAM_E_ARG, "strides"), (dict(out_stride=_i64(1024, 256, 0)), L.WAM_E_ARG, "distinct"),
    (dict(lse=P, lse_stride=_i64(16, 4, 0)), L.WAM_E_ARG, "distinct"), (dict(out=P), L.WAM_E_ARG, "must not")])
def test_attention_refuses(kw, code, text):
    _refused("wam_cache_attention", _attend(**kw), code, text)


def test_attention_asks_for_its_workspace():
    lib = L.lib()
    a = _attend(table__width=4096)
    need = lib.wam_cache_attention_workspace(C.byref(a))
    assert need > 0
    for at, size in ((None, need), (P, need - 1), (P + 8, need)):
        a.workspace, a.workspace_bytes = at, size
        _refused("wam_cache_attention", a, L.WAM_E_WORKSPACE, "workspace")
    assert lib.wam_cache_attention_workspace(None) == 0
    for kw in (dict(T=0), dict(B=0), dict(Hq=3)):
        assert lib.wam_cache_attention_workspace(C.byref(_attend(table__width=4096, **kw))) == 0


def test_which_calls_take_a_workspace():
    """Parts of long sequences do; short ones, and rows enough to fill the chip, do not."""
    lib = L.lib()
    for kw, parts in ((dict(T=2, table__width=188), True), (dict(T=1, Hq=2, table__width=1250), True),
                      (dict(T=2, table__width=4), False), (dict(T=2, table__width=30), False),
                      (dict(T=100000, table__width=188), False), (dict(T=2, table__width=188, dtype=L.WAM_FP32), True)):
        assert (lib.wam_cache_attention_workspace(C.byref(_attend(**kw))) > 0) == parts


def test_nothing_to_do():
    """Calls without rows or pages end before any device work."""
    lib = L.lib()
    for a in (_quant(M=0), _quant(K=0, x=None)):
        assert lib.wam_quantize_fp4(C.byref(a), None) == 0
    assert lib.wam_dequantize_fp4(C.byref(_dequant(M=0)), None) == 0
    assert lib.wam_matmul_fp4(C.byref(_matmul(M=0)), None) == 0
    for kw in (dict(T=0, k=None, pos=None), dict(B=0), dict(cache__pages=0, cache__k=None), dict(table__width=0)):
        a, _ = _append(**kw)
        assert lib.wam_cache_append(C.byref(a), None) == 0
    for kw in (dict(T=0, q=None), dict(B=0)):
        assert lib.wam_cache_attention(C.byref(_attend(**kw)), None) == 0


def test_struct_forms_of_the_binding():
    """The packed arguments have the size of the C structs' twins."""
    from paper_2609_34608_amd import runtime as R
    for form, twin in ((R._FP4_ARGS, L.WamQuantizeFp4Args), (R._FP4_ARGS, L.WamDequantizeFp4Args), (R._MATMUL_ARGS, L.WamMatmulFp4Args),
                       (R._APPEND_ARGS, L.WamCacheAppendArgs), (R._ATTENTION_ARGS, L.WamCacheAttentionArgs)):
        assert form.size == C.sizeof(twin)
