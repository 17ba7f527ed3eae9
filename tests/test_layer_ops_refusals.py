"""Refusals of the layer operators at the C boundary and in the binding (CPU:
every check comes before any device work, so the pointers are never followed)."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2609_34608_amd import _lib as L
from paper_2609_34608_amd import runtime as R

P = 0x10000  # an aligned address that nothing reads


def _i64(*v):
    return (C.c_int64 * len(v))(*v)


def _rope(**kw):
    freq = np.ones(32)
    a = L.WamRopeArgs(1, 4, 2, 2, 64, L.WAM_BF16, L.WAM_ROPE_HALVES, (C.c_int32 * 3)(8, 12, 12), P, P + 4096, P + 8192,
                      P + 12288, _i64(512, 128, 64), _i64(512, 128, 64), _i64(512, 128, 64), _i64(512, 128, 64), P, 0,
                      freq.ctypes.data, None, None, 1e-6)
    for n, v in kw.items():
        setattr(a, n, v)
    return a, freq


def _norm(**kw):
    a = L.WamNormArgs()
    a.B, a.T, a.D, a.post, a.pre, a.res_scale, a.eps = 1, 4, 64, L.WAM_NORM_RMS, L.WAM_NORM_LAYER, 1.0, 1e-6
    a.h_dtype, a.y_dtype, a.u_dtype = L.WAM_FP32, L.WAM_BF16, L.WAM_BF16
    a.h, a.y, a.h_out, a.u = P, P + 4096, P + 8192, P + 12288
    for n in ("h_stride", "y_stride", "h_out_stride", "u_stride"):
        setattr(a, n, _i64(256, 64))
    a.u_scale_stride = _i64(4, 1)
    for n, v in kw.items():
        setattr(a, n, v)
    return a


def _quant(**kw):
    a = L.WamQuantizeArgs(4, 256, L.WAM_BF16, 1, P, 256, P + 4096, 256, P + 8192, 2)
    for n, v in kw.items():
        setattr(a, n, v)
    return a


def _matmul(**kw):
    a = L.WamMatmulArgs(4, 64, 256, L.WAM_BF16, L.WAM_ACT_NONE, P, 256, P + 4096, 2, P + 8192, 256, P + 32768, 2, None,
                        P + 65536, 64)
    for n, v in kw.items():
        setattr(a, n, v)
    return a


def _refused(fn, a, code, text):
    lib = L.lib()
    assert getattr(lib, fn)(C.byref(a) if a is not None else None, None) == code
    assert text in lib.wam_noalloc_last_error().decode()


@pytest.mark.parametrize("kw,code,text", [
    (dict(B=-1), L.WAM_E_ARG, "sizes"), (dict(dh=0), L.WAM_E_SHAPE, "head size"),
    (dict(dh=257), L.WAM_E_SHAPE, "head size"), (dict(dtype=L.WAM_FP8), L.WAM_E_ARG, "dtype"),
    (dict(dtype=9), L.WAM_E_ARG, "dtype"), (dict(layout=2), L.WAM_E_ARG, "layout"),
    (dict(sections=(C.c_int32 * 3)(8, -1, 12)), L.WAM_E_ARG, "sections"),
    (dict(sections=(C.c_int32 * 3)(11, 11, 11)), L.WAM_E_SHAPE, "2 P <= dh"),
    (dict(sections=(C.c_int32 * 3)(2**31 - 1, 2**31 - 1, 2)), L.WAM_E_SHAPE, "2 P <= dh"),
    (dict(freq=None), L.WAM_E_ARG, "freq"), (dict(pos=None), L.WAM_E_ARG, "pos"), (dict(q=None), L.WAM_E_ARG, "null"),
    (dict(k_out=None), L.WAM_E_ARG, "null"), (dict(q=P + 1), L.WAM_E_ARG, "aligned"),
    (dict(k_stride=_i64(512, -128, 64)), L.WAM_E_ARG, "strides"),
    (dict(pos_stride=-1), L.WAM_E_ARG, "strides"),
    (dict(q_out_stride=_i64(512, 128, 0)), L.WAM_E_ARG, "distinct"),
    (dict(q_out_stride=_i64(512, 64, 64)), L.WAM_E_ARG, "distinct"),
    (dict(q_out=P, q_out_stride=_i64(512, 64, 256)), L.WAM_E_ARG, "in place"),
    (dict(q_gain=P, eps=-1.0), L.WAM_E_ARG, "eps"), (dict(q_gain=P, eps=float("nan")), L.WAM_E_ARG, "eps"),
    (dict(B=2**20, T=2**14, q_out_stride=_i64(2**21, 128, 64), k_out_stride=_i64(2**21, 128, 64)), L.WAM_E_SHAPE,
     "too many")])
def test_rope_refuses(kw, code, text):
    a, _keep = _rope(**kw)
    _refused("wam_rope", a, code, text)


def test_null_arguments_are_refused():
    for fn in ("wam_rope", "wam_norm_residual", "wam_quantize_fp8", "wam_matmul_fp8"):
        _refused(fn, None, L.WAM_E_ARG, "null argument")


@pytest.mark.parametrize("kw,code,text", [
    (dict(T=-1), L.WAM_E_ARG, "sizes"), (dict(D=0), L.WAM_E_SHAPE, "D must"), (dict(D=8193), L.WAM_E_SHAPE, "D must"),
    (dict(h_dtype=L.WAM_FP8), L.WAM_E_ARG, "h must"), (dict(y_dtype=L.WAM_FP8), L.WAM_E_ARG, "y must"),
    (dict(u_dtype=3), L.WAM_E_ARG, "u must"), (dict(post=3), L.WAM_E_ARG, "norm"), (dict(pre=-1), L.WAM_E_ARG, "norm"),
    (dict(eps=-1e-6), L.WAM_E_ARG, "eps"), (dict(h=None), L.WAM_E_ARG, "null h"),
    (dict(h_out=None, u=None), L.WAM_E_ARG, "no result"), (dict(h=P + 2), L.WAM_E_ARG, "aligned"),
    (dict(y_stride=_i64(-1, 64)), L.WAM_E_ARG, "strides"), (dict(u_stride=_i64(256, 32)), L.WAM_E_ARG, "distinct"),
    (dict(h_out_stride=_i64(0, 0)), L.WAM_E_ARG, "distinct"), (dict(u_dtype=L.WAM_FP8), L.WAM_E_ARG, "u_scale"),
    (dict(u_dtype=L.WAM_FP8, u_scale=P, u_scale_stride=_i64(4, 0)), L.WAM_E_ARG, "u_scale"),
    (dict(h_out=P, h_out_stride=_i64(1024, 128)), L.WAM_E_ARG, "in place"),
    (dict(u=P, u_dtype=L.WAM_FP32), L.WAM_E_ARG, "must not be h"), (dict(h_out=P + 4096), L.WAM_E_ARG, "must not be y"),
    (dict(u=P + 4096, u_dtype=L.WAM_FP32), L.WAM_E_ARG, "its type and strides"),
    (dict(gate=P + 2), L.WAM_E_ARG, "aligned"), (dict(B=2**20, T=2**12), L.WAM_E_SHAPE, "too many")])
def test_norm_refuses(kw, code, text):
    _refused("wam_norm_residual", _norm(**kw), code, text)


@pytest.mark.parametrize("kw,code,text", [
    (dict(M=-1), L.WAM_E_ARG, "sizes"), (dict(dtype=L.WAM_FP8), L.WAM_E_ARG, "x must"),
    (dict(block_rows=64), L.WAM_E_ARG, "block_rows"), (dict(x=None), L.WAM_E_ARG, "null"),
    (dict(scale=None), L.WAM_E_ARG, "null"), (dict(x=P + 1), L.WAM_E_ARG, "aligned"), (dict(q=P), L.WAM_E_ARG, "q must"),
    (dict(q_stride=255), L.WAM_E_ARG, "distinct"), (dict(scale_stride=1), L.WAM_E_ARG, "distinct"),
    (dict(x_stride=-256), L.WAM_E_ARG, "x_stride")])
def test_quantize_refuses(kw, code, text):
    _refused("wam_quantize_fp8", _quant(**kw), code, text)


@pytest.mark.parametrize("kw,code,text", [
    (dict(N=-1), L.WAM_E_ARG, "sizes"), (dict(K=0), L.WAM_E_SHAPE, "K must"), (dict(K=2**31 - 1), L.WAM_E_SHAPE, "large"),
    (dict(out_dtype=3), L.WAM_E_ARG, "out must"), (dict(out_dtype=L.WAM_FP8), L.WAM_E_ARG, "out_scale"),
    (dict(out_dtype=L.WAM_FP8, out_scale=P, out_scale_stride=0), L.WAM_E_ARG, "out_scale"),
    (dict(out_dtype=L.WAM_FP8, out_scale=P, out_scale_stride=1, a_stride=2**24), L.WAM_E_UNSUPPORTED, "2^23"), (dict(act=2), L.WAM_E_ARG, "activation"),
    (dict(a=None), L.WAM_E_ARG, "null"), (dict(w_scale=None), L.WAM_E_ARG, "null"), (dict(a=P + 8), L.WAM_E_ARG, "16"),
    (dict(w_stride=264), L.WAM_E_ARG, "16"), (dict(a_stride=240), L.WAM_E_ARG, "overlap"),
    (dict(w_stride=0), L.WAM_E_ARG, "overlap"), (dict(a_scale_stride=-2), L.WAM_E_ARG, "scales"),
    (dict(bias=P + 2), L.WAM_E_ARG, "scales"), (dict(out_stride=63), L.WAM_E_ARG, "distinct"),
    (dict(out=P + 65537), L.WAM_E_ARG, "distinct"), (dict(out=P), L.WAM_E_ARG, "must not be a")])
def test_matmul_refuses(kw, code, text):
    _refused("wam_matmul_fp8", _matmul(**kw), code, text)


@pytest.mark.parametrize("fn,a", [("wam_rope", _rope(B=0)[0]), ("wam_rope", _rope(T=0)[0]),
                                  ("wam_rope", _rope(Hq=0, Hk=0)[0]), ("wam_norm_residual", _norm(T=0)),
                                  ("wam_quantize_fp8", _quant(M=0)), ("wam_quantize_fp8", _quant(K=0)),
                                  ("wam_matmul_fp8", _matmul(M=0)), ("wam_matmul_fp8", _matmul(N=0))])
def test_empty_calls_do_nothing(fn, a):
    assert getattr(L.lib(), fn)(C.byref(a), None) == L.WAM_OK


def test_frequencies():
    sec = (8, 12, 12)
    own = R.rope_frequencies(sec, 500.0)
    np.testing.assert_allclose(own, [500.0 ** (-j / n) for n in sec for j in range(n)], rtol=1e-15)
    shared = R.rope_frequencies(sec, shared=True)
    np.testing.assert_allclose(shared, [10000.0 ** (-i / 32) for i in range(32)], rtol=1e-15)
    assert R.rope_frequencies((0, 0, 0)).size == 0
    for bad in ((8, -1, 12), (100, 28, 1)):
        with pytest.raises(R.WamError):
            R.rope_frequencies(bad)
    for theta in (0.0, -1.0, float("inf"), float("nan")):
        with pytest.raises(R.WamError, match="theta"):
            R.rope_frequencies(sec, theta)


@pytest.mark.parametrize("fn,a,code,text", [
    ("wam_rope", _rope(T=L.WAM_MAX_ROWS + 1, q_out_stride=_i64(0, 128, 64), k_out_stride=_i64(0, 128, 64))[0],
     L.WAM_E_SHAPE, "too many rows"),
    ("wam_rope", _rope(Hq=2**24, q_out_stride=_i64(2**40, 2**30, 64))[0], L.WAM_E_SHAPE, "too many heads"),
    ("wam_rope", _rope(k_out=P + 8192)[0], L.WAM_E_ARG, "the other one"),
    ("wam_rope", _rope(q_out=P + 4096)[0], L.WAM_E_ARG, "the other one"),
    ("wam_rope", _rope(k_out=P)[0], L.WAM_E_ARG, "the other one"),
    ("wam_rope", _rope(k=P, q_out=P, q_out_stride=_i64(512, 128, 64))[0], L.WAM_E_ARG, "the other one"),
    ("wam_norm_residual", _norm(T=L.WAM_MAX_ROWS + 1), L.WAM_E_SHAPE, "too many rows"),
    ("wam_quantize_fp8", _quant(M=2**29, K=1), L.WAM_E_SHAPE, "too many blocks"),
    ("wam_quantize_fp8", _quant(M=2**31 - 1, K=1, block_rows=128), L.WAM_E_SHAPE, "too many blocks"),
    ("wam_quantize_fp8", _quant(M=1, K=2**31 - 1), L.WAM_E_SHAPE, "too many blocks"),
    ("wam_matmul_fp8", _matmul(M=2**30, N=1, K=16), L.WAM_E_SHAPE, "too many tiles"),
    ("wam_matmul_fp8", _matmul(M=2**30, N=1, K=16, out_dtype=L.WAM_FP32), L.WAM_E_SHAPE, "too many tiles"),
    ("wam_matmul_fp8", _matmul(M=2**30, N=2**11, K=16, out_stride=2**11, out_dtype=L.WAM_FP8, out_scale=P,
                               out_scale_stride=16), L.WAM_E_SHAPE, "too many tiles")])
def test_sizes_past_a_grid_and_shared_results(fn, a, code, text):
    _refused(fn, a, code, text)


def test_binding_refuses_a_stream_of_another_gpu():
    class Stream:
        device_index, cuda_stream = 1, 0
    with pytest.raises(R.WamError, match="stream of GPU 1"):
        R._call(L.lib().wam_quantize_fp8, None, 0, Stream(), "wam_quantize_fp8")


def test_binding_refuses_host_tensors():
    x = torch.zeros(1, 4, 2, 64)
    with pytest.raises(R.WamError, match="device tensors only"):
        R.rope(x, None, torch.zeros(4, 3), (8, 12, 12), R.rope_frequencies((8, 12, 12)))
    with pytest.raises(R.WamError, match="device tensors only"):
        R.norm_residual(torch.zeros(1, 4, 64))
    with pytest.raises(R.WamError, match="device tensors only"):
        R.quantize_fp8(torch.zeros(4, 64))
    f8 = torch.zeros(4, 64).to(R.FP8)
    with pytest.raises(R.WamError, match="device tensors only"):
        R.matmul_fp8(f8, torch.ones(4, 1), f8, torch.ones(1, 1))


@pytest.mark.parametrize("packed,twin", [("_ROPE_ARGS", L.WamRopeArgs), ("_NORM_ARGS", L.WamNormArgs),
                                         ("_QUANTIZE_ARGS", L.WamQuantizeArgs), ("_MATMUL_ARGS", L.WamMatmulArgs)])
def test_packed_arguments_match_the_struct(packed, twin):
    """The binding's packed bytes have every field where the C struct has it."""
    form = getattr(R, packed)
    flat = [n + 1 for n in range(len(form.unpack(bytes(form.size))))]
    data = form.pack(*flat)
    assert form.size <= C.sizeof(twin) <= form.size + 7
    a = twin.from_buffer_copy(data + bytes(C.sizeof(twin) - form.size))
    got = []
    for name, _ in twin._fields_:
        v = getattr(a, name)
        got += list(v) if isinstance(v, C.Array) else [v]
    assert got == flat
