"""Microscaled 4-bit operands and their products (include/asgd_fp4.h), the narrower form of experts.py's 8-bit ones.

    xq, xs = asgd_quantize4(x, source=source, per_token=8)                # tokens in the experts' order, 4 bits
    h = asgd_product4(xq, xs, wq, ws, offsets=offsets)                    # every expert's rows by its own matrix

Two numbers share a byte (torch.float4_e2m1fn_x2, so a matrix of K columns has ceil(K / 2) of them), 32 neighbours of a row a
power of two (torch.float8_e8m0fnu).  The functions marshal arguments as those of experts.py do, with its rules on devices, streams and autograd.
"""
from __future__ import annotations

import ctypes as C

import torch

from . import binding
from .experts import _FLOAT, _chk, _first, _flat, _handle, _ld, _matrix, _need, _new, _on

BLOCK4 = 32
FP4_EXPORTS = ("asgd_quantize4", "asgd_dequantize4", "asgd_product4")

_FOUR = {torch.float4_e2m1fn_x2: 0}
_POWER = {torch.float8_e8m0fnu: 0}


class Quantize4Args(C.Structure):
    """Mirror of `asgd_quantize4_args`."""
    _fields_ = [("M", C.c_int64), ("K", C.c_int64), ("x", C.c_void_p), ("ldx", C.c_int64), ("rows_x", C.c_int64), ("x_type", C.c_int32),
                ("per_token", C.c_int32), ("source", C.c_void_p), ("weights", C.c_void_p), ("q", C.c_void_p), ("ldq", C.c_int64),
                ("scale", C.c_void_p), ("scale_row", C.c_int64)]


class Product4Args(C.Structure):
    """Mirror of `asgd_product4_args`."""
    _fields_ = [("M", C.c_int64), ("N", C.c_int64), ("K", C.c_int64), ("a", C.c_void_p), ("lda", C.c_int64), ("a_scale", C.c_void_p),
                ("a_scale_row", C.c_int64), ("b", C.c_void_p), ("ldb", C.c_int64), ("b_group", C.c_int64), ("b_scale", C.c_void_p),
                ("b_scale_row", C.c_int64), ("b_scale_group", C.c_int64), ("c", C.c_void_p), ("ldc", C.c_int64), ("offsets", C.c_void_p),
                ("groups", C.c_int32), ("c_type", C.c_int32)]


_lib = None


def _load():
    global _lib
    if _lib is None:
        L = binding.load()
        vp, i64 = C.c_void_p, C.c_int64
        L.asgd_quantize4.argtypes = [C.POINTER(Quantize4Args), vp]
        L.asgd_dequantize4.argtypes = [i64, i64, vp, i64, vp, i64, vp, C.c_int32, i64, vp]
        L.asgd_product4.argtypes = [C.POINTER(Product4Args), vp]
        _lib = L
    return _lib


def _rows16(rows, cols, dtype, dev):
    """A matrix of bytes whose rows start at multiples of 16."""
    return _new((rows, cols), (-(-cols // 16) * 16, 1), dtype=dtype, device=dev)


def asgd_quantize4(x, *, source=None, per_token=1, weights=None, stream=None):
    """x [T, K] in 4 bits: q [M, ceil(K / 2)] and its scales [M, ceil(K / 32)], M = T.  With `source` (see asgd_route) the rows are
    gathered: row r is x[source[r] // per_token], times weights.flatten()[source[r]] if there are any, and zeros where source[r] < 0."""
    if stream is not None:
        return _on(stream, asgd_quantize4, x, source=source, per_token=per_token, weights=weights)
    on, x_type, (T, K), strides = _first(x, _FLOAT, "x")
    M, source_ptr, weights_ptr = T, None, None
    if source is not None:
        M = source.numel()
        source_ptr = _flat(source, on, torch.int32, (M,), "source")
    if weights is not None:
        _need(source is not None, "weights need a source")
        _need(weights.get_device() == on and weights.dtype == torch.float32 and weights.is_contiguous() and weights.numel() == T * per_token,
              "weights must be contiguous fp32 on the device of x, T * per_token of them")
        weights_ptr = weights.data_ptr()
    n, blocks = -(-K // 2), -(-K // BLOCK4)
    q, scale = _rows16(M, n, torch.float4_e2m1fn_x2, x.device), _rows16(M, blocks, torch.float8_e8m0fnu, x.device)
    _chk(_load().asgd_quantize4(C.byref(Quantize4Args(M, K, x.data_ptr(), _ld((T, K), strides), T, x_type, int(per_token), source_ptr, weights_ptr,
                                                      q.data_ptr(), -(-n // 16) * 16, scale.data_ptr(), -(-blocks // 16) * 16)), _handle(on)),
         "asgd_quantize4")
    return q, scale


def _scale_of(s, on, name, shape):
    """The strides of a matrix's scales."""
    strides = s.stride()
    if not (s.shape == shape and s.dtype == torch.float8_e8m0fnu and s.get_device() == on and (strides[-1] == 1 or shape[-1] <= 1)):
        raise ValueError("%s must be float8_e8m0fnu on cuda:%d with shape %s and neighbouring blocks, not %s of shape %s" % (name, on, tuple(shape), s.dtype, tuple(s.shape)))
    return strides


def asgd_dequantize4(q, scale, K=None, *, dtype=torch.bfloat16, stream=None):
    """What 4-bit rows q [M, n] with scales [M, ceil(2 n / 32)] stand for: [M, K] of dtype; K is 2 n (the default) or 2 n - 1."""
    if stream is not None:
        return _on(stream, asgd_dequantize4, q, scale, K, dtype=dtype)
    on, _, (M, n), strides = _first(q, _FOUR, "q")
    K = 2 * n if K is None else int(K)
    _need(-(-K // 2) == n, "K must be %d or one less", 2 * n)
    type_ = _FLOAT.get(dtype)
    _need(type_ is not None, "dtype %s is not supported", dtype)
    blocks = -(-K // BLOCK4)
    s = _scale_of(scale, on, "scale", (M, blocks))
    out = _new((M, K), (K, 1), dtype=dtype, device=q.device)
    _chk(_load().asgd_dequantize4(M, K, q.data_ptr(), _ld((M, n), strides), scale.data_ptr(), _ld((M, blocks), s), out.data_ptr(), type_, K, _handle(on)),
         "asgd_dequantize4")
    return out


def asgd_product4(a, a_scale, b, b_scale, *, offsets=None, out_dtype=torch.bfloat16, out=None, stream=None):
    """C[m, n] = sum_k A[m, k] B[n, k] of 4-bit matrices with their scales: a [M, K / 2], a_scale [M, ceil(K / 32)]; b [N, K / 2], b_scale
    [N, ceil(K / 32)].  With offsets [G + 1] (int32 on the GPU) b is [G, N, K / 2], its scales have G in front, and the rows
    offsets[g] .. offsets[g + 1] of A meet b[g]; rows of no group are left as they are in `out` (undefined without one).  Rows, of
    numbers as of scales, start at multiples of 16 bytes, as asgd_quantize4 lays them out."""
    if stream is not None:
        return _on(stream, asgd_product4, a, a_scale, b, b_scale, offsets=offsets, out_dtype=out_dtype, out=out)
    grouped = offsets is not None
    on, _, a_shape, a_strides = _first(a, _FOUR, "a")
    _, b_shape, b_strides = _matrix(b, on, _FOUR, "b", 3 if grouped else 2)
    (M, n), N = a_shape, b_shape[-2]
    kb = -(-n // (BLOCK4 // 2))
    _need(b_shape[-1] == n, "a and b differ in their last dimension")
    G, offsets_ptr = 0, None
    if grouped:
        G = b_shape[0]
        _need(G > 0, "b holds no group")
        offsets_ptr = _flat(offsets, on, torch.int32, (G + 1,), "offsets")
    sa = _scale_of(a_scale, on, "a_scale", (M, kb))
    s_shape = (G, N, kb) if grouped else (N, kb)
    sb = _scale_of(b_scale, on, "b_scale", s_shape)
    if out is None:
        out, c_type, ldc = _new((M, N), (N, 1), dtype=out_dtype, device=a.device), _FLOAT.get(out_dtype), N
        _need(c_type is not None, "out_dtype %s is not supported", out_dtype)
    else:
        c_type, c_shape, c_strides = _matrix(out, on, _FLOAT, "out")
        _need(c_shape == (M, N), "out must have shape (%d, %d)", M, N)
        ldc = _ld(c_shape, c_strides)
    many = G > 1
    args = Product4Args(M, N, 2 * n, a.data_ptr(), _ld(a_shape, a_strides, 16), a_scale.data_ptr(), _ld((M, kb), sa, 16),
                        b.data_ptr(), _ld(b_shape, b_strides, 16), b_strides[0] if many else 0,
                        b_scale.data_ptr(), _ld(s_shape, sb, 16), sb[0] if many else 0, out.data_ptr(), ldc, offsets_ptr, G, c_type)
    _chk(_load().asgd_product4(C.byref(args), _handle(on)), "asgd_product4")
    return out
