"""A whole layer of experts for the few tokens of a serving step (include/asgd_expert_layer.h), in one call and one kernel.

    y = asgd_expert_layer(x, w1q, w1s, w2q, w2s, 8, router=centres, shift=half_norms, activation="silu")

The matrices are those that asgd_quantize(form="blocks") makes, stacked; the numbers are those of the separate operators of experts.py but for
the roundings between them.  The rules on devices, streams and autograd are those of experts.py.
"""
from __future__ import annotations

import ctypes as C
import functools

import torch

from . import binding
from .experts import (_EIGHT, _FLOAT, BLOCK, RouteConfig, SCORES, _chk, _first, _flat, _handle, _ld, _matrix, _need, _new, _on, _scale_of)

LAYER_EXPORTS = ("asgd_expert_layer_workspace_bytes", "asgd_expert_layer")
ACTIVATIONS = {"relu2": 0, "silu": 1}


class ExpertLayerArgs(C.Structure):
    """Mirror of `asgd_expert_layer_args`."""
    _fields_ = [("T", C.c_int64), ("d", C.c_int64), ("h", C.c_int64), ("x", C.c_void_p), ("ldx", C.c_int64), ("y", C.c_void_p), ("ldy", C.c_int64),
                ("logits", C.c_void_p), ("ld_logits", C.c_int64), ("router", C.c_void_p), ("ld_router", C.c_int64), ("shift", C.c_void_p),
                ("bias", C.c_void_p), ("w1", C.c_void_p), ("ldw1", C.c_int64), ("w1_group", C.c_int64), ("w1_scale", C.c_void_p),
                ("w1_scale_row", C.c_int64), ("w1_scale_block", C.c_int64), ("w1_scale_group", C.c_int64), ("w2", C.c_void_p),
                ("ldw2", C.c_int64), ("w2_group", C.c_int64), ("w2_scale", C.c_void_p), ("w2_scale_row", C.c_int64),
                ("w2_scale_block", C.c_int64), ("w2_scale_group", C.c_int64), ("ids", C.c_void_p), ("weights", C.c_void_p),
                ("type", C.c_int32), ("logits_type", C.c_int32), ("router_type", C.c_int32), ("w1_type", C.c_int32), ("w2_type", C.c_int32),
                ("gated", C.c_int32), ("activation", C.c_int32), ("temperature", C.c_float)]


_lib = None


def _load():
    global _lib
    if _lib is None:
        L = binding.load()
        L.asgd_expert_layer_workspace_bytes.argtypes = [C.POINTER(RouteConfig), C.POINTER(ExpertLayerArgs), C.POINTER(C.c_size_t)]
        L.asgd_expert_layer.argtypes = [C.POINTER(RouteConfig), C.POINTER(ExpertLayerArgs), C.c_void_p, C.c_size_t, C.c_void_p]
        _lib = L
    return _lib


def _config(E, top_k, score, groups, groups_kept, group_top, renormalise, scale, T, d, h, gated, routed):
    """The configuration and the workspace's bytes."""
    return _config_of(E, int(top_k), score, int(groups), None if groups_kept is None else int(groups_kept), int(group_top), bool(renormalise), float(scale),
                      T, d, h, gated, routed)                              # (by plain values, see _route_config)


@functools.lru_cache(maxsize=256)
def _config_of(E, top_k, score, groups, groups_kept, group_top, renormalise, scale, T, d, h, gated, routed):
    _need(score in SCORES, "score must be one of %s", tuple(SCORES))
    cfg = RouteConfig(E, top_k, SCORES[score], groups, groups if groups_kept is None else groups_kept, group_top, 1 if renormalise else 0, 1, scale)
    sizes = ExpertLayerArgs(T=T, d=d, h=h, gated=gated, router=1 if routed else None)          # sizes, and which pointers there are
    n = C.c_size_t(0)
    _chk(_load().asgd_expert_layer_workspace_bytes(C.byref(cfg), C.byref(sizes), C.byref(n)), "asgd_expert_layer_workspace_bytes")
    return C.pointer(cfg), n.value


def asgd_expert_layer(x, w1, w1_scale, w2, w2_scale, top_k, *, logits=None, router=None, shift=None, temperature=1.0, activation="relu2",
                      score="softmax", bias=None, groups=1, groups_kept=None, group_top=1, renormalise=True, scale=1.0, choice=False, stream=None):
    """y [T, d] of x's type from x [T, d] (T up to 128, T * top_k up to 1024): every token's best top_k experts of
      w1 [E, h, d], or [E, 2 h, d] (gated: act(u[:h]) * u[h:]), and w2 [E, d, h], 8 bits, with w1_scale [E, ceil(rows / 128),
      ceil(d / 128)] and w2_scale [E, ceil(d / 128), ceil(h / 128)],
    summed with the weights of asgd_route.  The logits are given ([T, E]), or made here: (x @ router.T - shift) * temperature with
    router [E, d] and shift [E].  A token that no expert takes has zeros, but NaNs where a router made its logits and it is not finite.
    `activation` is "relu2" (max(u, 0)^2) or "silu"; score, bias, groups, groups_kept, group_top, renormalise and scale are those of
    asgd_route.  With `choice` returns y, ids [T, top_k] and weights [T, top_k]."""
    if stream is not None:
        return _on(stream, asgd_expert_layer, x, w1, w1_scale, w2, w2_scale, top_k, logits=logits, router=router, shift=shift, temperature=temperature,
                   activation=activation, score=score, bias=bias, groups=groups, groups_kept=groups_kept, group_top=group_top,
                   renormalise=renormalise, scale=scale, choice=choice)
    on, type_, (T, d), strides = _first(x, _FLOAT, "x")
    w1_type, (E, rows, w1_d), w1_strides = _matrix(w1, on, _EIGHT, "w1", 3)
    w2_type, (w2_E, w2_d, h), w2_strides = _matrix(w2, on, _EIGHT, "w2", 3)
    _need(w1_d == d and w2_d == d and w2_E == E, "w1 must have shape [E, h or 2 h, d], and w2 [E, d, h]")
    _need(rows == h or rows == 2 * h, "w1 must have the hidden numbers' rows, %d, or twice as many, not %d", h, rows)
    _need(E > 0 and d > 0 and h > 0, "there are no experts")
    _need(activation in ACTIVATIONS, "activation must be one of %s", tuple(ACTIVATIONS))
    db, hb = -(-d // BLOCK), -(-h // BLOCK)
    _, s1 = _scale_of(w1_scale, on, "w1_scale", (E, -(-rows // BLOCK), db))
    _, s2 = _scale_of(w2_scale, on, "w2_scale", (E, db, hb))
    _need((logits is None) != (router is None), "either logits or a router is needed")
    args = ExpertLayerArgs(T, d, h, x.data_ptr(), _ld((T, d), strides))
    if router is None:
        _need(shift is None, "shift needs a router")
        args.logits_type, shape, st = _matrix(logits, on, _FLOAT, "logits")
        _need(shape == (T, E), "logits must have shape (%d, %d)", T, E)
        args.logits, args.ld_logits = logits.data_ptr(), _ld(shape, st)
    else:
        args.router_type, shape, st = _matrix(router, on, _FLOAT, "router")
        _need(shape == (E, d), "router must have shape (%d, %d)", E, d)
        args.router, args.ld_router, args.temperature = router.data_ptr(), _ld(shape, st), float(temperature)
        if shift is not None:
            args.shift = _flat(shift, on, torch.float32, (E,), "shift")
    if bias is not None:
        args.bias = _flat(bias, on, torch.float32, (E,), "bias")
    gated = 0 if rows == h else 1
    cfg, need = _config(E, top_k, score, groups, groups_kept, group_top, renormalise, scale, T, d, h, gated, router is not None)
    dev = x.device
    y = _new((T, d), (d, 1), dtype=x.dtype, device=dev)
    args.y, args.ldy = y.data_ptr(), d
    args.w1, args.ldw1, args.w1_group = w1.data_ptr(), _ld((rows, d), w1_strides, 16), w1_strides[0]
    args.w1_scale, args.w1_scale_row, args.w1_scale_block, args.w1_scale_group = w1_scale.data_ptr(), s1[1], s1[2], s1[0]
    args.w2, args.ldw2, args.w2_group = w2.data_ptr(), _ld((d, h), w2_strides, 16), w2_strides[0]
    args.w2_scale, args.w2_scale_row, args.w2_scale_block, args.w2_scale_group = w2_scale.data_ptr(), s2[1], s2[2], s2[0]
    if choice:
        ids = _new((T, top_k), (top_k, 1), dtype=torch.int32, device=dev)
        weights = _new((T, top_k), (top_k, 1), dtype=torch.float32, device=dev)
        args.ids, args.weights = ids.data_ptr(), weights.data_ptr()
    args.type, args.w1_type, args.w2_type, args.gated, args.activation = type_, w1_type, w2_type, gated, ACTIVATIONS[activation]
    work = _new((need,), (1,), dtype=torch.uint8, device=dev)
    _chk(_load().asgd_expert_layer(cfg, C.byref(args), work.data_ptr(), need, _handle(on)), "asgd_expert_layer")
    return (y, ids, weights) if choice else y
