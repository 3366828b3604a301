"""The operators of a layer of experts (include/asgd_experts.h): routing, 8-bit operands and products, combination.

The functions carry the C names and marshal arguments: they check shapes and types, take outputs from torch's
allocator and pass strides on.  Every number is computed in the library's kernels, on the current CUDA stream or the
one given; a call's tensors are on the current device (that of the stream, where one is given).
These are calls of a library: outputs carry no gradient, whatever the inputs ask for, and no autograd function joins a
forward call with its gradient's.  A caller keeps what the gradient needs and calls it (expert_layer.Layer.gradients).

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
_FORMS = {"rows": (True, False, 0), "columns": (False, True, 0), "both": (True, True, 0), "blocks": (True, False, 1), "blocks both": (True, True, 1)}

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


_current_device = getattr(torch._C, "_cuda_getDevice", None)               # (none where torch knows no CUDA)


def _wrong(t, on, types, name, dims):
    _need(t.get_device() >= 0, "%s must be a CUDA tensor: the library has no host path", name)
    _need(t.get_device() == on, "%s is on cuda:%d, where cuda:%d is wanted", name, t.get_device(), on)
    _need(t.dim() == dims, "%s must have %d dimensions", name, dims)
    _need(t.dtype in types, "%s: dtype %s is not supported", name, t.dtype)
    _need(False, "%s: the last dimension must be contiguous", name)


# A call takes as long on the host as on the device when the tensors are small, so every attribute of a tensor is read once.
def _first(t, types, name):
    """A call's first matrix: the number of its device, where all of the call's tensors have to be, and what _matrix gives.
    The device has to be the current one, for that is where the library launches."""
    on, number, shape, strides = t.get_device(), types.get(t.dtype), t.shape, t.stride()
    if not (on >= 0 and on == _current_device() and number is not None and len(shape) == 2 and (strides[-1] == 1 or shape[-1] <= 1)):
        _wrong(t, _current_device() if on >= 0 else on, types, name, 2)
    return on, number, shape, strides


def _matrix(t, on, types, name, dims=2):
    """A tensor on device `on` of one of the types whose last dimension is contiguous: its type's number, shape and strides."""
    number, shape, strides = types.get(t.dtype), t.shape, t.stride()
    if not (number is not None and t.get_device() == on and len(shape) == dims and (strides[-1] == 1 or shape[-1] <= 1)):
        _wrong(t, on, types, name, dims)
    return number, shape, strides


def _flat(t, on, dtype, shape, name):
    """Its address."""
    if not (t.get_device() == on and t.dtype == dtype and t.shape == shape and t.is_contiguous()):
        raise ValueError("%s must be a contiguous tensor of %s with shape %s on cuda:%d" % (name, dtype, tuple(shape), on))
    return t.data_ptr()


def _ld(shape, strides, unit=1):
    """Elements from one row to the next; for a single row, which has no say, a multiple of `unit`."""
    return strides[-2] if shape[-2] > 1 else -(-shape[-1] // unit) * unit


_new = torch.empty_strided


def _handle(on):
    """The current stream of the device, as the C functions take it."""
    return torch._C._cuda_getCurrentRawStream(on)


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
    on, type_, (T, E), strides = _first(logits, _FLOAT, "logits")
    bias_ptr = None if bias is None else _flat(bias, on, torch.float32, (E,), "bias")
    cfg, need = _route_config(E, top_k, score, groups, groups_kept, group_top, renormalise, scale, align, T)
    dev, ints, ld = logits.device, torch.int32, _ld((T, E), strides)
    ids = _new((T, top_k), (top_k, 1), dtype=ints, device=dev)
    weights = _new((T, top_k), (top_k, 1), dtype=torch.float32, device=dev)
    if not plan:
        _chk(_load().asgd_route(cfg, T, logits.data_ptr(), type_, ld, bias_ptr, ids.data_ptr(), weights.data_ptr(), None, None, None, 0,
                                None, 0, _handle(on)), "asgd_route")
        return ids, weights
    n = T * top_k + E * (align - 1)
    offsets = _new((E + 1,), (1,), dtype=ints, device=dev)
    rows = _new((T, top_k), (top_k, 1), dtype=ints, device=dev)
    source = _new((n,), (1,), dtype=ints, device=dev)
    work = _new((need,), (1,), dtype=torch.uint8, device=dev) if need else None
    _chk(_load().asgd_route(cfg, T, logits.data_ptr(), type_, ld, bias_ptr, ids.data_ptr(), weights.data_ptr(), offsets.data_ptr(),
                            rows.data_ptr(), source.data_ptr(), n, work.data_ptr() if need else None, need, _handle(on)), "asgd_route")
    return ids, weights, offsets, rows, source


def asgd_route_grad(logits, ids, dweights, *, score="softmax", renormalise=True, scale=1.0, stream=None):
    """Gradient [T, E] (of the logits' type) of the weights that asgd_route gave for `ids`, from dweights [T, top_k]."""
    if stream is not None:
        return _on(stream, asgd_route_grad, logits, ids, dweights, score=score, renormalise=renormalise, scale=scale)
    on, type_, (T, E), strides = _first(logits, _FLOAT, "logits")
    _need(ids.dim() == 2 and ids.shape[0] == T, "ids must have shape [T, top_k]")
    top_k = ids.shape[1]
    ids_ptr = _flat(ids, on, torch.int32, (T, top_k), "ids")
    dw_ptr = _flat(dweights, on, torch.float32, (T, top_k), "dweights")
    cfg, _ = _route_config(E, top_k, score, 1, 1, 1, renormalise, scale, 1, T)
    out = _new((T, E), (E, 1), dtype=logits.dtype, device=logits.device)
    _chk(_load().asgd_route_grad(cfg, T, logits.data_ptr(), type_, _ld((T, E), strides), ids_ptr, dw_ptr, out.data_ptr(), E, _handle(on)),
         "asgd_route_grad")
    return out


def _eight(rows, cols, dtype, dev):
    """An 8-bit matrix whose rows start at multiples of 16 bytes."""
    return _new((rows, cols), (-(-cols // 16) * 16, 1), dtype=dtype, device=dev)


def _scales(rows, cols, dev):
    """Scales [rows, blocks of cols], block after block in memory."""
    return _new((rows, -(-cols // BLOCK)), (1, rows), dtype=torch.float32, device=dev)


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
    on, x_type, (T, K), strides = _first(x, _FLOAT, "x")
    q_type = _EIGHT.get(dtype)
    _need(form in _FORMS, "form %r is not known", form)
    _need(q_type is not None, "dtype %s is not supported", dtype)
    by_rows, by_columns, square = _FORMS[form]
    M, source_ptr, weights_ptr = T, None, None
    if source is not None:
        _need(not square, "blocks of 128 x 128 are not gathered")
        M = source.numel()
        source_ptr = _flat(source, on, torch.int32, (M,), "source")
    if weights is not None:
        _need(source is not None, "weights need a source")
        _need(weights.get_device() == on and weights.dtype == torch.float32 and weights.is_contiguous() and weights.numel() == T * per_token,
              "weights must be contiguous fp32 on the device of x, T * per_token of them")
        weights_ptr = weights.data_ptr()
    dev, blocks = x.device, -(-K // BLOCK)
    args = [M, K, x.data_ptr(), _ld((T, K), strides), T, x_type, q_type, square, int(per_token), source_ptr, weights_ptr]
    out = ()
    if by_rows:
        q = _eight(M, K, dtype, dev)
        scale = _new((-(-M // BLOCK), blocks), (blocks, 1), dtype=torch.float32, device=dev) if square else _scales(M, K, dev)
        args += [q.data_ptr(), -(-K // 16) * 16, scale.data_ptr(), blocks if square else 1, 1 if square else M]
        out = (q, scale)
    else:
        args += [None, 0, None, 0, 0]
    if by_columns:
        qt = _eight(K, M, dtype, dev)
        out += (qt,)
        args += [qt.data_ptr(), -(-M // 16) * 16]
        if not square:
            scale_t = _scales(K, M, dev)
            args += [scale_t.data_ptr(), 1, K]
            out += (scale_t,)
    _chk(_load().asgd_quantize(C.byref(QuantizeArgs(*args)), _handle(on)), "asgd_quantize")
    return out


def _scale_of(s, on, name, shape, other=None):
    """Scales of one of two shapes: the shape and the strides."""
    found = s.shape
    if not ((found == shape or found == other) and s.dtype == torch.float32 and s.get_device() == on):
        raise ValueError("%s must be fp32 on cuda:%d with shape %s, not %s of shape %s" % (name, on, tuple(shape), s.dtype, tuple(found)))
    return found, s.stride()


def asgd_product(a, a_scale, b, b_scale, *, offsets=None, out_dtype=torch.bfloat16, out=None, stream=None):
    """C[m, n] = sum_k A[m, k] B[n, k] of 8-bit matrices with their scales: a [M, K], a_scale [M, ceil(K / 128)];
    b [N, K], b_scale [N or ceil(N / 128), ceil(K / 128)].  With offsets [G + 1] (int32 on the GPU) b is [G, N, K], its
    scales have G in front, and the rows offsets[g] .. offsets[g + 1] of A meet b[g]; rows of no group are left as
    they are in `out` (undefined without one)."""
    if stream is not None:
        return _on(stream, asgd_product, a, a_scale, b, b_scale, offsets=offsets, out_dtype=out_dtype, out=out)
    grouped = offsets is not None
    on, a_type, a_shape, a_strides = _first(a, _EIGHT, "a")
    b_type, b_shape, b_strides = _matrix(b, on, _EIGHT, "b", 3 if grouped else 2)
    (M, K), N, kb = a_shape, b_shape[-2], -(-a_shape[1] // BLOCK)
    _need(b_shape[-1] == K, "a and b differ in their last dimension")
    G, offsets_ptr = 0, None
    if grouped:
        G = b_shape[0]
        _need(G > 0, "b holds no group")
        offsets_ptr = _flat(offsets, on, torch.int32, (G + 1,), "offsets")
    _, sa = _scale_of(a_scale, on, "a_scale", (M, kb))
    square = -(-N // BLOCK)
    s_shape, sb = _scale_of(b_scale, on, "b_scale", (G, square, kb), (G, N, kb)) if grouped else _scale_of(b_scale, on, "b_scale", (square, kb), (N, kb))
    if out is None:
        out, c_type, ldc = _new((M, N), (N, 1), dtype=out_dtype, device=a.device), _FLOAT.get(out_dtype), N
        _need(c_type is not None, "out_dtype %s is not supported", out_dtype)
    else:
        c_type, c_shape, c_strides = _matrix(out, on, _FLOAT, "out")
        _need(c_shape == (M, N), "out must have shape (%d, %d)", M, N)
        ldc = _ld(c_shape, c_strides)
    many = G > 1
    args = ProductArgs(M, N, K, a.data_ptr(), _ld(a_shape, a_strides, 16), a_scale.data_ptr(), sa[0], sa[1],
                       b.data_ptr(), _ld(b_shape, b_strides, 16), b_strides[0] if many else 0,
                       b_scale.data_ptr(), sb[-2], sb[-1], sb[0] if many else 0,
                       out.data_ptr(), ldc, 0, offsets_ptr, G, 0, a_type, b_type, c_type, 1 if s_shape[-2] != N else 0)
    _chk(_load().asgd_product(C.byref(args), _handle(on)), "asgd_product")
    return out


def asgd_product_inner(a, a_scale, b, b_scale, offsets, *, out_dtype=torch.float32, out=None, stream=None):
    """C[g, m, n] = sum of A[m, k] B[n, k] over offsets[g] <= k < offsets[g + 1] (multiples of 128): the groups' weight
    gradients.  a [M, K], a_scale [M, ceil(K / 128)], b [N, K], b_scale [N, ceil(K / 128)]."""
    if stream is not None:
        return _on(stream, asgd_product_inner, a, a_scale, b, b_scale, offsets, out_dtype=out_dtype, out=out)
    on, a_type, a_shape, a_strides = _first(a, _EIGHT, "a")
    b_type, b_shape, b_strides = _matrix(b, on, _EIGHT, "b")
    (M, K), N, kb = a_shape, b_shape[0], -(-a_shape[1] // BLOCK)
    _need(b_shape[1] == K, "a and b differ in their last dimension")
    G = offsets.numel() - 1
    _need(G > 0, "offsets hold no group")
    offsets_ptr = _flat(offsets, on, torch.int32, (G + 1,), "offsets")
    _, sa = _scale_of(a_scale, on, "a_scale", (M, kb))
    _, sb = _scale_of(b_scale, on, "b_scale", (N, kb))
    if out is None:
        out, c_type, ldc, c_group = _new((G, M, N), (M * N, N, 1), dtype=out_dtype, device=a.device), _FLOAT.get(out_dtype), N, M * N
        _need(c_type is not None, "out_dtype %s is not supported", out_dtype)
    else:
        c_type, c_shape, c_strides = _matrix(out, on, _FLOAT, "out", 3)
        _need(c_shape == (G, M, N), "out must have shape (%d, %d, %d)", G, M, N)
        ldc, c_group = _ld(c_shape, c_strides), c_strides[0]
    args = ProductArgs(M, N, K, a.data_ptr(), _ld(a_shape, a_strides, 16), a_scale.data_ptr(), sa[0], sa[1],
                       b.data_ptr(), _ld(b_shape, b_strides, 16), 0, b_scale.data_ptr(), sb[0], sb[1], 0,
                       out.data_ptr(), ldc, c_group, offsets_ptr, G, 1, a_type, b_type, c_type, 0)
    _chk(_load().asgd_product(C.byref(args), _handle(on)), "asgd_product")
    return out


def asgd_combine(z, rows, weights=None, *, stream=None):
    """y[t] = sum_j weights[t, j] * z[rows[t, j]] of z's type; rows [T, top_k] int32 (negative: no part)."""
    if stream is not None:
        return _on(stream, asgd_combine, z, rows, weights)
    on, type_, (R, D), strides = _first(z, _FLOAT, "z")
    shape = rows.shape
    _need(len(shape) == 2, "rows must have shape [T, top_k]")
    T, top_k = shape
    rows_ptr = _flat(rows, on, torch.int32, shape, "rows")
    weights_ptr = None if weights is None else _flat(weights, on, torch.float32, shape, "weights")
    y = _new((T, D), (D, 1), dtype=z.dtype, device=z.device)
    _chk(_load().asgd_combine(T, D, top_k, z.data_ptr(), type_, R, _ld((R, D), strides), rows_ptr, weights_ptr, y.data_ptr(), D, _handle(on)),
         "asgd_combine")
    return y


def asgd_combine_grad(dy, z, rows, weights=None, source=None, *, need_dz=True, need_dweights=True, stream=None):
    """Gradients of asgd_combine: dz [R, D] (zeros in rows whose source is negative; without `source` rows that no token
    takes are undefined) and dweights [T, top_k]; None for what is not needed."""
    if stream is not None:
        return _on(stream, asgd_combine_grad, dy, z, rows, weights, source, need_dz=need_dz, need_dweights=need_dweights)
    on, type_, (T, D), strides = _first(dy, _FLOAT, "dy")
    z_type, (R, z_D), z_strides = _matrix(z, on, _FLOAT, "z")
    _need(z_type == type_, "dy and z differ in type")
    _need(z_D == D, "dy and z differ in their last dimension")
    shape = rows.shape
    _need(len(shape) == 2 and shape[0] == T, "rows must have shape [T, top_k]")
    top_k = shape[1]
    rows_ptr = _flat(rows, on, torch.int32, shape, "rows")
    weights_ptr = None if weights is None else _flat(weights, on, torch.float32, shape, "weights")
    source_ptr = None if source is None else _flat(source, on, torch.int32, (R,), "source")
    dz = _new((R, D), (D, 1), dtype=dy.dtype, device=dy.device) if need_dz else None
    dw = _new((T, top_k), (top_k, 1), dtype=torch.float32, device=dy.device) if need_dweights else None
    _chk(_load().asgd_combine_grad(T, D, top_k, dy.data_ptr(), type_, _ld((T, D), strides), z.data_ptr(), R, _ld((R, D), z_strides), rows_ptr,
                                   weights_ptr, source_ptr, dz.data_ptr() if need_dz else None, D, dw.data_ptr() if need_dweights else None,
                                   _handle(on)), "asgd_combine_grad")
    return dz, dw


def asgd_experts_sync(stream=None):
    """Wait for the stream; raise what asgd_product calls on this device have reported since the last call (one report per
    device, whatever the streams: where there are several, wait for all of them first)."""
    s = stream if stream is not None else torch.cuda.current_stream()
    with torch.cuda.device(s.device):
        _chk(_load().asgd_experts_sync(C.c_void_p(s.cuda_stream)), "asgd_experts_sync")


def asgd_product_set_wait_drill(wait_limit: int = 1 << 22, withhold: bool = False):
    _chk(_load().asgd_product_set_wait_drill(int(wait_limit), 1 if withhold else 0), "asgd_product_set_wait_drill")
