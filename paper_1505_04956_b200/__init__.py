"""K-Means ASGD (Keuper & Pfreundt, arXiv 1505.04956) worker loop as CUDA kernels for B200.

`binding` wraps the C ABI of libasgd.so one to one; `inputs` draws seeded synthetic workloads;
`build` compiles the library in-tree.  `experts` holds the operators of a layer of experts behind learnt
centres: routing, 8-bit operands and products, combination; `serving` is the whole layer for a few tokens, `fp4` has 4-bit
operands and products, `gradients` the norm of many gradients and clipping.  Nothing here computes on the CPU.
"""
import importlib

from .binding import (Asgd, AsgdConfig, AsgdError, make_config, asgd_workspace_bytes, asgd_fit_host,
                      asgd_fit_host_bytes, asgd_eval_noalloc, load, LIB_PATH, EXPORTS, PATH_AUTO, PATH_FP32, PATH_TC_FP16,
                      PATH_TC_BF16, PATH_FP32_GENERAL)

# Looked up when first asked for: the K-Means calls, the build and the binding do without torch.
_EXPERTS = ("EXPERT_EXPORTS", "asgd_combine", "asgd_combine_grad", "asgd_experts_sync", "asgd_product", "asgd_product_inner",
            "asgd_product_set_wait_drill", "asgd_quantize", "asgd_route", "asgd_route_grad")
_GRADIENTS = ("GRADIENT_EXPORTS", "asgd_clip_grads", "asgd_grad_norm")
_FP4 = ("FP4_EXPORTS", "asgd_dequantize4", "asgd_product4", "asgd_quantize4")
_SERVING = ("LAYER_EXPORTS", "asgd_expert_layer")
_MODULE_OF = {name: module for module, names in (("experts", _EXPERTS), ("fp4", _FP4), ("gradients", _GRADIENTS), ("serving", _SERVING)) for name in names}

__all__ = ["Asgd", "AsgdConfig", "AsgdError", "make_config", "asgd_workspace_bytes", "asgd_fit_host",
           "asgd_fit_host_bytes", "asgd_eval_noalloc", "load", "LIB_PATH", "EXPORTS", "PATH_AUTO", "PATH_FP32", "PATH_TC_FP16",
           "PATH_TC_BF16", "PATH_FP32_GENERAL", *_MODULE_OF]


def __getattr__(name):
    if name not in _MODULE_OF and name not in _MODULE_OF.values():
        raise AttributeError("module %r has no attribute %r" % (__name__, name))
    module = importlib.import_module("." + _MODULE_OF.get(name, name), __name__)
    globals()[name] = value = module if name in _MODULE_OF.values() else getattr(module, name)
    return value
