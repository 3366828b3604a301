"""K-Means ASGD (Keuper & Pfreundt, arXiv 1505.04956) worker loop as CUDA kernels for B200.

`binding` wraps the C ABI of libasgd.so one to one; `inputs` draws seeded synthetic workloads;
`build` compiles the library in-tree.  `experts` holds the operators of a layer of experts behind learnt
centres: routing, 8-bit operands and products, combination.  Nothing here computes on the CPU.
"""
import importlib

from .binding import (Asgd, AsgdConfig, AsgdError, make_config, asgd_workspace_bytes, asgd_fit_host,
                      asgd_fit_host_bytes, asgd_eval_noalloc, load, LIB_PATH, EXPORTS, PATH_AUTO, PATH_FP32, PATH_TC_FP16,
                      PATH_TC_BF16, PATH_FP32_GENERAL)

# Looked up when first asked for: the K-Means calls, the build and the binding do without torch.
_EXPERTS = ("EXPERT_EXPORTS", "asgd_combine", "asgd_combine_grad", "asgd_experts_sync", "asgd_product", "asgd_product_inner",
            "asgd_product_set_wait_drill", "asgd_quantize", "asgd_route", "asgd_route_grad")

__all__ = ["Asgd", "AsgdConfig", "AsgdError", "make_config", "asgd_workspace_bytes", "asgd_fit_host",
           "asgd_fit_host_bytes", "asgd_eval_noalloc", "load", "LIB_PATH", "EXPORTS", "PATH_AUTO", "PATH_FP32", "PATH_TC_FP16",
           "PATH_TC_BF16", "PATH_FP32_GENERAL", *_EXPERTS]


def __getattr__(name):
    if name not in _EXPERTS and name != "experts":
        raise AttributeError("module %r has no attribute %r" % (__name__, name))
    module = importlib.import_module(".experts", __name__)
    globals()[name] = value = module if name == "experts" else getattr(module, name)
    return value
