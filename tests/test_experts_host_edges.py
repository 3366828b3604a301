"""Refusals of the operators of a layer of experts at the edges of what they take, without a GPU."""
import ctypes as C
import os
import subprocess
import sys

import pytest
import torch

from paper_1505_04956_b200 import binding, experts

from .test_experts_host import _cfg, _p, _q

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EUNSUPPORTED, ECUDA, OK = binding.ASGD_EINVAL, binding.ASGD_EUNSUPPORTED, binding.ASGD_ECUDA, binding.ASGD_OK


@pytest.mark.parametrize("bad", [dict(M=(1 << 31) - 255), dict(M=(1 << 31) - 1), dict(N=(1 << 31) - 255, ldc=1 << 31), dict(N=(1 << 31) - 1, ldc=1 << 31),
                                 dict(K=(1 << 31) - 255, lda=1 << 31, ldb=1 << 31)])
@pytest.mark.parametrize("grouped", [dict(), dict(groups=3, offsets=1 << 20)])
def test_product_refuses_sizes_whose_tiles_pass_32_bits(bad, grouped):
    assert experts._load().asgd_product(C.byref(_p(**bad, **grouped)), None) == EUNSUPPORTED


def test_quantize_refuses_rows_whose_blocks_pass_32_bits():
    wide = 1 << 31
    assert experts._load().asgd_quantize(C.byref(_q(M=1, rows_x=1, K=wide - 65535, ldx=wide, ldq=wide, square=1)), None) == EUNSUPPORTED


# ---------------------------------------------------------------------------------------------------------------
# devices
# ---------------------------------------------------------------------------------------------------------------

class _On:
    """Stands for a CUDA tensor of a device."""
    is_cuda = True

    def __init__(self, device, dtype, *shape):
        self.index, self.dtype, self.shape, self.device = device, dtype, torch.Size(shape), torch.device("cuda", device)

    def get_device(self):
        return self.index

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def stride(self):
        out = [1]
        for n in self.shape[:0:-1]:
            out.insert(0, out[0] * n)
        return tuple(out)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


F32, I32, E4 = torch.float32, torch.int32, torch.float8_e4m3fn
_CALLS = [
    ("asgd_route", [(F32, 4, 8), None], dict(top_k=2, bias=(F32, 8))),
    ("asgd_route_grad", [(F32, 4, 8), (I32, 4, 2), (F32, 4, 2)], {}),
    ("asgd_quantize", [(F32, 4, 8)], dict(source=(I32, 8), per_token=2, weights=(F32, 4, 2))),
    ("asgd_product", [(E4, 4, 128), (F32, 4, 1), (E4, 3, 32, 128), (F32, 3, 1, 1)], dict(offsets=(I32, 4), out=(F32, 4, 32))),
    ("asgd_product_inner", [(E4, 4, 256), (F32, 4, 2), (E4, 32, 256), (F32, 32, 2), (I32, 4)], dict(out=(F32, 3, 4, 32))),
    ("asgd_combine", [(F32, 8, 16), (I32, 4, 2), (F32, 4, 2)], {}),
    ("asgd_combine_grad", [(F32, 4, 16), (F32, 8, 16), (I32, 4, 2), (F32, 4, 2), (I32, 8)], {}),
]


@pytest.mark.parametrize("name, args, kw", _CALLS)
def test_tensors_of_another_device_are_refused(name, args, kw, monkeypatch):
    class Reached(Exception):
        pass

    def library():
        raise Reached
    monkeypatch.setattr(experts, "_load", library)
    monkeypatch.setattr(experts, "_route_config", lambda *a: (None, 0))
    monkeypatch.setattr(experts, "_new", lambda shape, strides, dtype, device: _On(device.index, dtype, *shape))
    monkeypatch.setattr(experts, "_handle", lambda where: 0, raising=False)
    monkeypatch.setattr(experts, "_current_device", lambda: 0, raising=False)
    tensors = [i for i, a in enumerate(args) if a] + [k for k, a in kw.items() if isinstance(a, tuple)]

    def call(devices):
        make = lambda key, a: _On(devices.get(key, 0), *a) if isinstance(a, tuple) else a          # noqa: E731
        fn = getattr(experts, name)
        given = {k: make(k, a) for k, a in kw.items()}
        return fn(*[make(i, a) for i, a in enumerate(args) if a], **given)
    with pytest.raises(Reached):                         # all on the current device: the library is called
        call({})
    with pytest.raises(ValueError):                      # all on another one
        call({t: 1 for t in tensors})
    for t in tensors:                                    # one of them elsewhere
        with pytest.raises(ValueError):
            call({t: 1})


# ---------------------------------------------------------------------------------------------------------------
# alignment of 32-bit arrays
# ---------------------------------------------------------------------------------------------------------------

P, ODD = C.c_void_p(1 << 20), C.c_void_p((1 << 20) + 2)


@pytest.mark.parametrize("at", [5, 6, 7, 8, 9, 10])
def test_route_refuses_arrays_that_are_not_aligned(at):
    args = [C.byref(_cfg()), 10, P, 0, 64, P, P, P, P, P, P, 40, None, 0, None]
    args[at] = ODD                                       # bias, ids, weights, offsets, rows, source
    assert experts._load().asgd_route(*args) == EINVAL


@pytest.mark.parametrize("at", [5, 6])
def test_route_grad_refuses_arrays_that_are_not_aligned(at):
    args = [C.byref(_cfg()), 10, P, 0, 64, P, P, P, 64, None]
    args[at] = ODD
    assert experts._load().asgd_route_grad(*args) == EINVAL


@pytest.mark.parametrize("bad", [dict(source=ODD.value), dict(source=P.value, weights=ODD.value), dict(scale=ODD.value),
                                 dict(qt=P.value, ldqt=256, scale_t=ODD.value)])
def test_quantize_refuses_arrays_that_are_not_aligned(bad):
    assert experts._load().asgd_quantize(C.byref(_q(**bad)), None) == EINVAL


@pytest.mark.parametrize("bad", [dict(offsets=ODD.value, groups=2), dict(a_scale=ODD.value), dict(b_scale=ODD.value)])
def test_product_refuses_arrays_that_are_not_aligned(bad):
    assert experts._load().asgd_product(C.byref(_p(**bad)), None) == EINVAL


def test_combine_refuses_arrays_that_are_not_aligned():
    L = experts._load()
    for rows, weights in ((ODD, P), (P, ODD)):
        assert L.asgd_combine(4, 64, 2, P, 1, 8, 64, rows, weights, P, 64, None) == EINVAL
    for i in range(4):
        rows, weights, source, dweights = (ODD if i == j else P for j in range(4))
        assert L.asgd_combine_grad(4, 64, 2, P, 1, 64, P, 8, 64, rows, weights, source, P, 64, dweights, None) == EINVAL


def test_an_error_is_not_reported_again_by_a_later_call():
    # without a GPU the first call fails with a CUDA error; a call that launches nothing has none of its own
    if torch.cuda.is_available():
        pytest.skip("needs a machine without a GPU")
    L = experts._load()
    assert L.asgd_experts_sync(None) == ECUDA
    assert L.asgd_route(C.byref(_cfg()), 0, None, 0, 64, None, None, None, None, None, None, 0, None, 0, None) == OK


# ---------------------------------------------------------------------------------------------------------------
# the package
# ---------------------------------------------------------------------------------------------------------------

def test_the_package_comes_up_without_torch():
    # what needs torch is loaded when it is asked for: building and the K-Means binding are not to wait for it
    code = ("import sys; import paper_1505_04956_b200 as pkg; from paper_1505_04956_b200 import build, binding; pkg.load(); "
            "assert 'torch' not in sys.modules; assert pkg.experts.BLOCK == 128; from paper_1505_04956_b200 import asgd_route; assert pkg.asgd_route is asgd_route; "
            "assert 'torch' in sys.modules; ns = {}; exec('from paper_1505_04956_b200 import *', ns); "
            "assert all(n in ns for n in pkg.__all__) and 'asgd_product' in pkg.__all__; "
            "assert not hasattr(pkg, 'asgd_nothing')")
    subprocess.run([sys.executable, "-c", code], check=True, cwd=ROOT)


def test_kernels_that_come_up_early_take_nothing_for_constant():
    # read-only loads (and const __restrict__, which allows them) promise that nothing writes the memory while the kernel
    # runs; a kernel that waits for the one before it inside the stream cannot promise that
    csrc = os.path.join(ROOT, "paper_1505_04956_b200", "csrc")
    files = [f for f in os.listdir(csrc) if f.startswith(("asgd_route", "asgd_quantize", "asgd_product", "asgd_combine", "asgd_experts"))]
    assert len(files) >= 8
    for f in files:
        text = open(os.path.join(csrc, f)).read()
        for word in ("__ldg", "__restrict__", "ld.global.nc"):
            assert word not in text, (f, word)
