"""The operators of a layer of experts (include/asgd_experts.h): routing, 8-bit operands and products, combination.

The functions carry the C names and marshal arguments: they check shapes and types, take outputs from torch's
allocator and pass strides on.  Every number is computed in the library's kernels, on the current CUDA stream or the
one given.

    ids, weights, offsets, rows, source = asgd_route(logits, 8, score="sigmoid", bias=balance, align=128)
    xq, xs = asgd_quantize(x, source=source, per_token=8)                 # tokens in the experts' order, 8 bits
    h = asgd_product(xq, xs, wq, ws, offsets=offsets)                     # every expert's rows by its own matrix
    y = asgd_combine(h, rows, weights)                                    # back into token order
"""
from __future__ import annotations

import ctypes as C
import functools

import torch

from . import binding
from .binding import ASGD_OK, AsgdError

F32, BF16, F16, E4M3, E5M2 = 0, 1, 2, 3, 4
SCORES = {"softmax": 0, "sigmoid": 1}
BLOCK = 128

_FLOAT = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
_EIGHT = {torch.float8_e4m3fn: E4M3, torch.float8_e5m2: E5M2}

EXPERT_EXPORTS = (
    "asgd_route_workspace_bytes", "asgd_route", "asgd_route_grad", "asgd_quantize", "asgd_product", "asgd_combine",
    "asgd_combine_grad", "asgd_experts_sync", "asgd_product_set_wait_drill",
)


class RouteConfig(C.Structure):
    """Mirror of `asgd_route_config`."""
    _fields_ = [("experts", C.c_int32), ("top_k", C.c_int32), ("score", C.c_int32), ("groups", C.c_int32),
                ("groups_kept", C.c_int32), ("group_top", C.c_int32), ("renormalise", C.c_int32), ("align", C.c_int32),
                ("scale", C.c_float)]


class QuantizeArgs(C.Structure):
    """Mirror of `asgd_quantize_args`."""
    _fields_ = [("M", C.c_int64), ("K", C.c_int64), ("x", C.c_void_p), ("ldx", C.c_int64), ("rows_x", C.c_int64),
                ("x_type", C.c_int32), ("q_type", C.c_int32), ("square", C.c_int32), ("per_token", C.c_int32),
                ("source", C.c_void_p), ("weights", C.c_void_p),
                ("q", C.c_void_p), ("ldq", C.c_int64), ("scale", C.c_void_p), ("scale_row", C.c_int64), ("scale_block", C.c_int64),
                ("qt", C.c_void_p), ("ldqt", C.c_int64), ("scale_t", C.c_void_p), ("scale_t_row", C.c_int64), ("scale_t_block", C.c_int64)]


class ProductArgs(C.Structure):
    """Mirror of `asgd_product_args`."""
    _fields_ = [("M", C.c_int64), ("N", C.c_int64), ("K", C.c_int64),
                ("a", C.c_void_p), ("lda", C.c_int64), ("a_scale", C.c_void_p), ("a_scale_row", C.c_int64), ("a_scale_block", C.c_int64),
                ("b", C.c_void_p), ("ldb", C.c_int64), ("b_group", C.c_int64),
                ("b_scale", C.c_void_p), ("b_scale_row", C.c_int64), ("b_scale_block", C.c_int64), ("b_scale_group", C.c_int64),
                ("c", C.c_void_p), ("ldc", C.c_int64), ("c_group", C.c_int64),
                ("offsets", C.c_void_p), ("groups", C.c_int32), ("inner", C.c_int32),
                ("a_type", C.c_int32), ("b_type", C.c_int32), ("c_type", C.c_int32), ("b_square", C.c_int32)]


_lib = None


def _load():
    global _lib
    if _lib is None:
        L = binding.load()
        vp, i64, i32, f32 = C.c_void_p, C.c_int64, C.c_int32, C.c_float
        L.asgd_route_workspace_bytes.argtypes = [C.POINTER(RouteConfig), i64, C.POINTER(C.c_size_t)]
        L.asgd_route.argtypes = [C.POINTER(RouteConfig), i64, vp, i32, i64, vp, vp, vp, vp, vp, vp, i64, vp, C.c_size_t, vp]
        L.asgd_route_grad.argtypes = [C.POINTER(RouteConfig), i64, vp, i32, i64, vp, vp, vp, i64, vp]
        L.asgd_quantize.argtypes = [C.POINTER(QuantizeArgs), vp]
        L.asgd_product.argtypes = [C.POINTER(ProductArgs), vp]
        L.asgd_combine.argtypes = [i64, i64, i32, vp, i32, i64, i64, vp, vp, vp, i64, vp]
        L.asgd_combine_grad.argtypes = [i64, i64, i32, vp, i32, i64, vp, i64, i64, vp, vp, vp, vp, i64, vp, vp]
        L.asgd_experts_sync.argtypes = [vp]
        L.asgd_product_set_wait_drill.argtypes = [C.c_uint32, i32]
        _lib = L
    return _lib


def _chk(rc, where):
    if rc != ASGD_OK:
        raise AsgdError(rc, where)


def _need(ok, what, *values):
    if not ok:
        raise ValueError(what % values if values else what)


def _matrix(t, types, name, dims=2):
    """A CUDA tensor of one of the types whose last dimension is contiguous; returns its type's number."""
    number = types.get(t.dtype)
    if not (t.is_cuda and number is not None and t.dim() == dims and (t.stride(-1) == 1 or t.shape[-1] <= 1)):
        _need(t.is_cuda, "%s must be a CUDA tensor: the library has no host path", name)
        _need(t.dim() == dims, "%s must have %d dimensions", name, dims)
        _need(number is not None, "%s: dtype %s is not supported", name, t.dtype)
        _need(False, "%s: the last dimension must be contiguous", name)
    return number


def _flat(t, dtype, shape, name):
    _need(t.is_cuda and t.dtype == dtype and t.shape == shape and t.is_contiguous(),
          "%s must be a contiguous CUDA tensor of %s with shape %s", name, dtype, shape)


def _ld(t, unit=1):
    """Elements from one row to the next; for a single row, which has no say, a multiple of `unit`."""
    return t.stride(-2) if t.shape[-2] > 1 else -(-t.shape[-1] // unit) * unit


def _new(shape, strides, dtype, dev):
    return torch.empty_strided(shape, strides, dtype=dtype, device=dev)


def _handle(t):
    """The current stream of the tensor's device, as the C functions take it."""
    return torch._C._cuda_getCurrentRawStream(t.get_device())


def _on(stream, call, *args, **kw):
    """The call with `stream` as the current one: its work, and its allocator's pool for the outputs."""
    with torch.cuda.stream(stream):
        return call(*args, **kw)


@functools.lru_cache(maxsize=256)
def _route_config(E, top_k, score, groups, groups_kept, group_top, renormalise, scale, align, T):
    """The configuration and the workspace's bytes for T tokens."""
    _need(score in SCORES, "score must be one of %s", tuple(SCORES))
    cfg = RouteConfig(E, int(top_k), SCORES[score], int(groups), int(groups if groups_kept is None else groups_kept), int(group_top),
                      1 if renormalise else 0, int(align), float(scale))
    n = C.c_size_t(0)
    _chk(_load().asgd_route_workspace_bytes(C.byref(cfg), T, C.byref(n)), "asgd_route_workspace_bytes")
    return C.pointer(cfg), n.value


def asgd_route(logits, top_k, *, score="softmax", bias=None, groups=1, groups_kept=None, group_top=1, renormalise=True,
               scale=1.0, align=1, plan=True, stream=None):
    """Choice of top_k experts per token (logits [T, E]).  Returns ids [T, top_k] int32 and weights [T, top_k] fp32 and,
    with `plan`, offsets [E + 1], rows [T, top_k] and source [T * top_k + E * (align - 1)] (int32): the grouped order in
    which expert e owns rows offsets[e] .. offsets[e + 1], starting at multiples of `align`."""
    if stream is not None:
        return _on(stream, asgd_route, logits, top_k, score=score, bias=bias, groups=groups, groups_kept=groups_kept, group_top=group_top,
                   renormalise=renormalise, scale=scale, align=align, plan=plan)
    type_ = _matrix(logits, _FLOAT, "logits")
    T, E = logits.shape
    if bias is not None:
        _flat(bias, torch.float32, (E,), "bias")
    cfg, need = _route_config(E, top_k, score, groups, groups_kept, group_top, renormalise, scale, align, T)
    dev = logits.device
    ids = _new((T, top_k), (top_k, 1), torch.int32, dev)
    weights = _new((T, top_k), (top_k, 1), torch.float32, dev)
    bias_ptr = bias.data_ptr() if bias is not None else None
    if not plan:
        _chk(_load().asgd_route(cfg, T, logits.data_ptr(), type_, _ld(logits), bias_ptr, ids.data_ptr(), weights.data_ptr(), None, None, None, 0,
                                None, 0, _handle(logits)), "asgd_route")
        return ids, weights
    n = T * top_k + E * (align - 1)
    offsets = _new((E + 1,), (1,), torch.int32, dev)
    rows = _new((T, top_k), (top_k, 1), torch.int32, dev)
    source = _new((n,), (1,), torch.int32, dev)
    work = _new((need,), (1,), torch.uint8, dev) if need else None
    _chk(_load().asgd_route(cfg, T, logits.data_ptr(), type_, _ld(logits), bias_ptr, ids.data_ptr(), weights.data_ptr(), offsets.data_ptr(),
                            rows.data_ptr(), source.data_ptr(), n, work.data_ptr() if need else None, need, _handle(logits)), "asgd_route")
    return ids, weights, offsets, rows, source


def asgd_route_grad(logits, ids, dweights, *, score="softmax", renormalise=True, scale=1.0, stream=None):
    """Gradient [T, E] (of the logits' type) of the weights that asgd_route gave for `ids`, from dweights [T, top_k]."""
    if stream is not None:
        return _on(stream, asgd_route_grad, logits, ids, dweights, score=score, renormalise=renormalise, scale=scale)
    type_ = _matrix(logits, _FLOAT, "logits")
    T, E = logits.shape
    _need(ids.dim() == 2 and ids.shape[0] == T, "ids must have shape [T, top_k]")
    top_k = ids.shape[1]
    _flat(ids, torch.int32, (T, top_k), "ids")
    _flat(dweights, torch.float32, (T, top_k), "dweights")
    cfg, _ = _route_config(E, top_k, score, 1, 1, 1, renormalise, scale, 1, T)
    out = _new((T, E), (E, 1), logits.dtype, logits.device)
    _chk(_load().asgd_route_grad(cfg, T, logits.data_ptr(), type_, _ld(logits), ids.data_ptr(), dweights.data_ptr(), out.data_ptr(), E,
                                 _handle(logits)), "asgd_route_grad")
    return out


def _eight(rows, cols, dtype, dev):
    """An 8-bit matrix whose rows start at multiples of 16 bytes."""
    return _new((rows, cols), (-(-cols // 16) * 16, 1), dtype, dev)


def _scales(rows, cols, dev):
    """Scales [rows, blocks of cols], block after block in memory."""
    return _new((rows, -(-cols // BLOCK)), (1, rows), torch.float32, dev)


def asgd_quantize(x, *, form="rows", dtype=torch.float8_e4m3fn, source=None, per_token=1, weights=None, stream=None):
    """x [T, K] in 8 bits with a scale for each block of 128.  Forms:
      "rows"         q [M, K], scale [M, ceil(K / 128)]                    blocks along a row
      "columns"      qt [K, M], scale_t [K, ceil(M / 128)]                 the transpose, in its own blocks
      "both"         q, scale, qt, scale_t
      "blocks"       q [M, K], scale [ceil(M / 128), ceil(K / 128)]        blocks of 128 x 128 (weights)
      "blocks both"  q, scale, qt, with scale.t() the scales of qt
    With `source` (see asgd_route) the rows are gathered: row r is x[source[r] // per_token], times weights.flatten()[source[r]]
    if there are any, and zeros where source[r] < 0."""
    if stream is not None:
        return _on(stream, asgd_quantize, x, form=form, dtype=dtype, source=source, per_token=per_token, weights=weights)
    x_type = _matrix(x, _FLOAT, "x")
    _need(form in ("rows", "columns", "both", "blocks", "blocks both"), "form %r is not known", form)
    _need(dtype in _EIGHT, "dtype %s is not supported", dtype)
    T, K = x.shape
    M = T
    square = form.startswith("blocks")
    if source is not None:
        _need(not square, "blocks of 128 x 128 are not gathered")
        M = source.numel()
        _flat(source, torch.int32, (M,), "source")
    if weights is not None:
        _need(source is not None, "weights need a source")
        _need(weights.is_cuda and weights.dtype == torch.float32 and weights.is_contiguous() and weights.numel() == T * per_token,
              "weights must be contiguous fp32 on the GPU, T * per_token of them")
    dev = x.device
    q = scale = qt = scale_t = None
    if form != "columns":
        q = _eight(M, K, dtype, dev)
        blocks = -(-K // BLOCK)
        scale = _new((-(-M // BLOCK), blocks), (blocks, 1), torch.float32, dev) if square else _scales(M, K, dev)
    if form in ("columns", "both", "blocks both"):
        qt = _eight(K, M, dtype, dev)
        scale_t = None if square else _scales(K, M, dev)
    a = QuantizeArgs(M, K, x.data_ptr(), _ld(x), T, x_type, _EIGHT[dtype], 1 if square else 0, int(per_token),
                     source.data_ptr() if source is not None else None, weights.data_ptr() if weights is not None else None,
                     *((q.data_ptr(), q.stride(0), scale.data_ptr(), scale.stride(0), scale.stride(1)) if q is not None else (None, 0, None, 0, 0)),
                     *((qt.data_ptr(), qt.stride(0)) if qt is not None else (None, 0)),
                     *((scale_t.data_ptr(), scale_t.stride(0), scale_t.stride(1)) if scale_t is not None else (None, 0, 0)))
    _chk(_load().asgd_quantize(C.byref(a), _handle(x)), "asgd_quantize")
    return tuple(t for t in (q, scale, qt, scale_t) if t is not None)


def _scale_of(s, name, shape, other=None):
    _need(s.is_cuda and s.dtype == torch.float32, "%s must be fp32 on the GPU", name)
    _need(s.shape == shape or s.shape == other, "%s has shape %s, not %s", name, tuple(s.shape), shape)


def asgd_product(a, a_scale, b, b_scale, *, offsets=None, out_dtype=torch.bfloat16, out=None, stream=None):
    """C[m, n] = sum_k A[m, k] B[n, k] of 8-bit matrices with their scales: a [M, K], a_scale [M, ceil(K / 128)];
    b [N, K], b_scale [N or ceil(N / 128), ceil(K / 128)].  With offsets [G + 1] (int32 on the GPU) b is [G, N, K], its
    scales have G in front, and the rows offsets[g] .. offsets[g + 1] of A meet b[g]; rows of no group are left as
    they are in `out` (undefined without one)."""
    if stream is not None:
        return _on(stream, asgd_product, a, a_scale, b, b_scale, offsets=offsets, out_dtype=out_dtype, out=out)
    a_type, b_type = _matrix(a, _EIGHT, "a"), _matrix(b, _EIGHT, "b", 2 if offsets is None else 3)
    M, K = a.shape
    N, kb = b.shape[-2], -(-K // BLOCK)
    _need(b.shape[-1] == K, "a and b differ in their last dimension")
    G = 0
    lead = ()
    if offsets is not None:
        G = b.shape[0]
        lead = (G,)
        _need(G > 0, "b holds no group")
        _flat(offsets, torch.int32, (G + 1,), "offsets")
    _scale_of(a_scale, "a_scale", (M, kb))
    _scale_of(b_scale, "b_scale", lead + (-(-N // BLOCK), kb), lead + (N, kb))
    c = _new((M, N), (N, 1), out_dtype, a.device) if out is None else out
    c_type = _matrix(c, _FLOAT, "out")
    _need(c.shape == (M, N), "out must have shape (%d, %d)", M, N)
    args = ProductArgs(M, N, K, a.data_ptr(), _ld(a, 16), a_scale.data_ptr(), a_scale.stride(0), a_scale.stride(1),
                       b.data_ptr(), _ld(b, 16), b.stride(0) if G > 1 else 0,
                       b_scale.data_ptr(), b_scale.stride(-2), b_scale.stride(-1), b_scale.stride(0) if G > 1 else 0,
                       c.data_ptr(), _ld(c), 0, offsets.data_ptr() if G else None, G, 0, a_type, b_type, c_type, 1 if b_scale.shape[-2] != N else 0)
    _chk(_load().asgd_product(C.byref(args), _handle(a)), "asgd_product")
    return c


def asgd_product_inner(a, a_scale, b, b_scale, offsets, *, out_dtype=torch.float32, out=None, stream=None):
    """C[g, m, n] = sum of A[m, k] B[n, k] over offsets[g] <= k < offsets[g + 1] (multiples of 128): the groups' weight
    gradients.  a [M, K], a_scale [M, ceil(K / 128)], b [N, K], b_scale [N, ceil(K / 128)]."""
    if stream is not None:
        return _on(stream, asgd_product_inner, a, a_scale, b, b_scale, offsets, out_dtype=out_dtype, out=out)
    a_type, b_type = _matrix(a, _EIGHT, "a"), _matrix(b, _EIGHT, "b")
    M, K = a.shape
    N, kb = b.shape[0], -(-K // BLOCK)
    _need(b.shape[1] == K, "a and b differ in their last dimension")
    G = offsets.numel() - 1
    _need(G > 0, "offsets hold no group")
    _flat(offsets, torch.int32, (G + 1,), "offsets")
    _scale_of(a_scale, "a_scale", (M, kb))
    _scale_of(b_scale, "b_scale", (N, kb))
    c = _new((G, M, N), (M * N, N, 1), out_dtype, a.device) if out is None else out
    c_type = _matrix(c, _FLOAT, "out", 3)
    _need(c.shape == (G, M, N), "out must have shape (%d, %d, %d)", G, M, N)
    args = ProductArgs(M, N, K, a.data_ptr(), _ld(a, 16), a_scale.data_ptr(), a_scale.stride(0), a_scale.stride(1),
                       b.data_ptr(), _ld(b, 16), 0, b_scale.data_ptr(), b_scale.stride(0), b_scale.stride(1), 0,
                       c.data_ptr(), _ld(c), c.stride(0), offsets.data_ptr(), G, 1, a_type, b_type, c_type, 0)
    _chk(_load().asgd_product(C.byref(args), _handle(a)), "asgd_product")
    return c


def asgd_combine(z, rows, weights=None, *, stream=None):
    """y[t] = sum_j weights[t, j] * z[rows[t, j]] of z's type; rows [T, top_k] int32 (negative: no part)."""
    if stream is not None:
        return _on(stream, asgd_combine, z, rows, weights)
    type_ = _matrix(z, _FLOAT, "z")
    _need(rows.dim() == 2, "rows must have shape [T, top_k]")
    T, top_k = rows.shape
    _flat(rows, torch.int32, (T, top_k), "rows")
    if weights is not None:
        _flat(weights, torch.float32, (T, top_k), "weights")
    R, D = z.shape
    y = _new((T, D), (D, 1), z.dtype, z.device)
    _chk(_load().asgd_combine(T, D, top_k, z.data_ptr(), type_, R, _ld(z), rows.data_ptr(), weights.data_ptr() if weights is not None else None,
                              y.data_ptr(), D, _handle(z)), "asgd_combine")
    return y


def asgd_combine_grad(dy, z, rows, weights=None, source=None, *, need_dz=True, need_dweights=True, stream=None):
    """Gradients of asgd_combine: dz [R, D] (zeros in rows whose source is negative; without `source` rows that no token
    takes are undefined) and dweights [T, top_k]; None for what is not needed."""
    if stream is not None:
        return _on(stream, asgd_combine_grad, dy, z, rows, weights, source, need_dz=need_dz, need_dweights=need_dweights)
    type_ = _matrix(dy, _FLOAT, "dy")
    _matrix(z, _FLOAT, "z")
    _need(z.dtype == dy.dtype, "dy and z differ in type")
    T, D = dy.shape
    R = z.shape[0]
    _need(z.shape[1] == D, "dy and z differ in their last dimension")
    _need(rows.dim() == 2 and rows.shape[0] == T, "rows must have shape [T, top_k]")
    top_k = rows.shape[1]
    _flat(rows, torch.int32, (T, top_k), "rows")
    if weights is not None:
        _flat(weights, torch.float32, (T, top_k), "weights")
    if source is not None:
        _flat(source, torch.int32, (R,), "source")
    dz = _new((R, D), (D, 1), dy.dtype, dy.device) if need_dz else None
    dw = _new((T, top_k), (top_k, 1), torch.float32, dy.device) if need_dweights else None
    _chk(_load().asgd_combine_grad(T, D, top_k, dy.data_ptr(), type_, _ld(dy), z.data_ptr(), R, _ld(z), rows.data_ptr(),
                                   weights.data_ptr() if weights is not None else None, source.data_ptr() if source is not None else None,
                                   dz.data_ptr() if need_dz else None, D, dw.data_ptr() if need_dweights else None, _handle(dy)), "asgd_combine_grad")
    return dz, dw


def asgd_experts_sync(stream=None):
    """Wait for the stream; raise what asgd_product calls on this device have reported since the last call."""
    s = stream if stream is not None else torch.cuda.current_stream()
    _chk(_load().asgd_experts_sync(C.c_void_p(s.cuda_stream)), "asgd_experts_sync")


def asgd_product_set_wait_drill(wait_limit: int = 1 << 22, withhold: bool = False):
    _chk(_load().asgd_product_set_wait_drill(int(wait_limit), 1 if withhold else 0), "asgd_product_set_wait_drill")
