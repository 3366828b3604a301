"""Builds libasgd.so (the CUDA library behind the C ABI) in-tree with nvcc for sm_100a."""
from __future__ import annotations

import os
import subprocess
import sys

PKG = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(PKG, "csrc")
LIB = os.path.join(PKG, "libasgd.so")
SOURCES = ["asgd_api.cu", "asgd_noalloc.cu", "asgd_route.cu", "asgd_quantize.cu", "asgd_product.cu", "asgd_combine.cu",
           "asgd_gradients.cu", "asgd_fp4.cu", "asgd_product4.cu", "asgd_expert_layer.cu"]
OBJ = os.path.join(PKG, "_build")
NVCC_FLAGS = [
    "-gencode", "arch=compute_100a,code=sm_100a", "-lineinfo", "-O3", "-std=c++17",
    "-shared", "-Xcompiler", "-fPIC", "-cudart", "static",
]


def _newest_source_mtime() -> float:
    m = 0.0
    for root in (CSRC, os.path.join(os.path.dirname(PKG), "include")):
        for name in os.listdir(root):
            if name.endswith((".cu", ".cuh", ".h")):
                m = max(m, os.path.getmtime(os.path.join(root, name)))
    return m


def _stale(obj: str, dep: str) -> bool:
    """Whether an object is missing or older than a file that the compiler read for it."""
    if not (os.path.exists(obj) and os.path.exists(dep)):
        return True
    with open(dep) as f:
        read = f.read().replace("\\\n", " ").split(":", 1)[1].split()
    built = os.path.getmtime(obj)
    return any(not os.path.exists(p) or os.path.getmtime(p) > built for p in read)


def build(force: bool = False, verbose: bool = False) -> str:
    """Compile when the library is missing or older than a source; return the library's path.  Each source has an
    object of its own, and those that nothing changed for are kept."""
    if not force and os.path.exists(LIB) and os.path.getmtime(LIB) >= _newest_source_mtime():
        return LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    os.makedirs(OBJ, exist_ok=True)
    compile_flags = [f for f in NVCC_FLAGS if f != "-shared"]
    tag = ".%d.tmp" % os.getpid()
    running, objects = [], []
    for src in SOURCES:
        obj, dep = os.path.join(OBJ, src + ".o"), os.path.join(OBJ, src + ".d")
        objects.append(obj)
        if force or _stale(obj, dep):
            cmd = [nvcc] + compile_flags + (["-Xptxas", "-v"] if verbose else []) + \
                ["-MD", "-MF", dep + tag, "-c", os.path.join(CSRC, src), "-o", obj + tag]
            running.append((obj, dep, subprocess.Popen(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    failed = False
    for obj, dep, proc in running:
        out, _ = proc.communicate()
        if proc.returncode != 0:
            sys.stderr.write(out)
            failed = True
            continue
        if verbose:
            print(out)
        os.replace(dep + tag, dep)
        os.replace(obj + tag, obj)
    if failed:
        raise RuntimeError("nvcc failed building libasgd.so")
    tmp = LIB + tag
    res = subprocess.run([nvcc] + NVCC_FLAGS + objects + ["-o", tmp, "-lcuda"], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout)
        raise RuntimeError("nvcc failed building libasgd.so")
    os.replace(tmp, LIB)
    return LIB


PROBE_LIB = os.path.join(PKG, "libasgd_probe.so")


def build_probe(force: bool = False) -> str:
    """Compile the issue-rate probes (csrc/asgd_probe.cu) into their own library; return its path."""
    src = os.path.join(CSRC, "asgd_probe.cu")
    if not force and os.path.exists(PROBE_LIB) and os.path.getmtime(PROBE_LIB) >= _newest_source_mtime():   # it includes the kernels' headers
        return PROBE_LIB
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    tmp = PROBE_LIB + ".%d.tmp" % os.getpid()
    res = subprocess.run([nvcc] + NVCC_FLAGS + [src, "-o", tmp], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    if res.returncode != 0:
        sys.stderr.write(res.stdout)
        raise RuntimeError("nvcc failed building libasgd_probe.so")
    os.replace(tmp, PROBE_LIB)
    return PROBE_LIB


if __name__ == "__main__":
    print(build(force="--force" in sys.argv, verbose="-v" in sys.argv))
    print(build_probe(force="--force" in sys.argv))
