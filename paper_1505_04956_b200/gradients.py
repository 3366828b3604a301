"""The global norm of many gradients, and clipping by it (include/asgd_gradients.h).

    norm = asgd_clip_grads([drouter, dw1, dw2], 1.0)          # in place; the norm from before, on the device

As in experts.py the functions carry the C names and marshal arguments; the numbers are computed in the library's kernels on the
current CUDA stream or the one given, and nothing is known to autograd.
"""
from __future__ import annotations

import ctypes as C
import functools
import operator
import struct

import torch

from . import binding
from .experts import _FLOAT, _chk, _current_device, _handle, _need, _new, _on

GRADIENT_EXPORTS = ("asgd_gradients_workspace_bytes", "asgd_grad_norm", "asgd_clip_grads")


class Gradient(C.Structure):
    """Mirror of `asgd_gradient`."""
    _fields_ = [("x", C.c_void_p), ("out", C.c_void_p), ("n", C.c_int64), ("type", C.c_int32), ("reserved", C.c_int32)]


_lib = None


def _load():
    global _lib
    if _lib is None:
        L = binding.load()
        L.asgd_gradients_workspace_bytes.argtypes = [C.c_int64, C.POINTER(C.c_size_t)]
        L.asgd_grad_norm.argtypes = [C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.asgd_clip_grads.argtypes = [C.c_void_p, C.c_int64, C.c_float, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        _lib = L
    return _lib


# Attribute by attribute over the whole list, without a Python step per tensor where nothing is wrong: a call of hundreds of tensors
# takes longer on the host than on the device.
_dtype = operator.attrgetter("dtype")
_tensor_types = {torch.Tensor, torch.nn.Parameter}


def _checked(tensors, on, what):
    """The types' numbers of contiguous tensors on device `on`."""
    _need(set(map(type, tensors)) <= _tensor_types or all(isinstance(t, torch.Tensor) for t in tensors), "%s must be tensors", what)
    devices = set(map(torch.Tensor.get_device, tensors))
    _need(min(devices, default=0) >= 0, "%s must be CUDA tensors: the library has no host path", what)
    _need(devices <= {on}, "%s must be on cuda:%d, the current device", what, on)
    _need(all(map(torch.Tensor.is_contiguous, tensors)), "%s must be contiguous", what)
    types = list(map(_FLOAT.get, map(_dtype, tensors)))
    _need(None not in types, "%s must be of fp32, bf16 or fp16", what)
    return types


@functools.lru_cache(maxsize=256)
def _workspace(n):
    need = C.c_size_t(0)
    _chk(_load().asgd_gradients_workspace_bytes(n, C.byref(need)), "asgd_gradients_workspace_bytes")
    return need.value


def _call(tensors, out, max_norm):
    if type(tensors) is not list:
        tensors = list(tensors)
    on = _current_device() if _current_device is not None else -1
    _need(on >= 0, "there is no CUDA device: the library has no host path")
    types, n = _checked(tensors, on, "the tensors"), len(tensors)
    at, sizes = list(map(torch.Tensor.data_ptr, tensors)), list(map(torch.Tensor.numel, tensors))
    to = at
    if max_norm is not None:
        if out is not None:
            out = list(out)
            _need(len(out) == n, "out must have a tensor for each of the %d", n)
            _need(_checked(out, on, "out") == types and list(map(torch.Tensor.numel, out)) == sizes, "out must have the tensors' types and sizes")
            to = list(map(torch.Tensor.data_ptr, out))
        there = [p for p, k in zip(to, sizes) if k] if 0 in sizes else to
        _need(len(set(there)) == len(there), "the same memory is given twice")
    flat = [0] * (4 * n)                                  # asgd_gradient by words; a type's upper half is `reserved`
    flat[0::4], flat[1::4], flat[2::4], flat[3::4] = at, to, sizes, types
    table, need, dev = struct.pack("%dq" % (4 * n), *flat), _workspace(n), torch.device("cuda", on)
    work = _new((need,), (1,), dtype=torch.uint8, device=dev)
    norm = _new((), (), dtype=torch.float32, device=dev)
    if max_norm is None:
        _chk(_load().asgd_grad_norm(table or None, n, norm.data_ptr(), work.data_ptr(), need, _handle(on)), "asgd_grad_norm")
    else:
        _chk(_load().asgd_clip_grads(table or None, n, max_norm, norm.data_ptr(), work.data_ptr(), need, _handle(on)), "asgd_clip_grads")
    return norm


def asgd_grad_norm(tensors, *, stream=None):
    """The 2-norm of all numbers of all tensors (contiguous fp32, bf16 or fp16, on the current device) together: a tensor [] fp32."""
    if stream is not None:
        return _on(stream, asgd_grad_norm, tensors)
    return _call(tensors, None, None)


def asgd_clip_grads(tensors, max_norm, *, out=None, stream=None):
    """Scales the tensors by min(1, max_norm / (norm + 1e-6)), in place or into the tensors `out` of the same types and sizes (memory of
    their own, or the tensors themselves), and returns the norm from before, a tensor [] fp32 on the device.  Nothing waits for it: a norm
    that is infinite or NaN shows in the numbers (zeros and NaNs, see the header)."""
    if stream is not None:
        return _on(stream, asgd_clip_grads, tensors, max_norm, out=out)
    max_norm = float(max_norm)
    _need(max_norm > 0, "max_norm must be above zero")
    return _call(tensors, out, max_norm)
