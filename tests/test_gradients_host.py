"""The norm of many gradients and clipping without a GPU: exports, the list's structure, refusals before any launch."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

import paper_1505_04956_b200 as pkg
from paper_1505_04956_b200 import binding, gradients

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EUNSUPPORTED, ENOMEM, OK = binding.ASGD_EINVAL, binding.ASGD_EUNSUPPORTED, binding.ASGD_ENOMEM, binding.ASGD_OK
P = 1 << 20                       # stands for device memory: only calls that are refused get it


def test_header_and_binding_name_the_same_functions():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "asgd_gradients.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(asgd_[a-z0-9_]+)\s*\(", text))
    assert names == set(pkg.GRADIENT_EXPORTS)
    L = C.CDLL(binding.LIB_PATH)
    for n in names:
        assert hasattr(L, n), n
        assert n.endswith("_workspace_bytes") or callable(getattr(pkg, n)), n


def test_the_list_has_the_layout_of_the_header(tmp_path):
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "asgd_gradients.h"\nint main(void) { asgd_gradient g; printf("%zu %zu %zu %zu\\n", sizeof g, '
                   '(size_t)((char*)&g.out - (char*)&g), (size_t)((char*)&g.n - (char*)&g), (size_t)((char*)&g.type - (char*)&g)); return 0; }\n')
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, stdout=subprocess.PIPE, text=True).stdout.split()
    g = gradients.Gradient
    assert [int(v) for v in out] == [C.sizeof(g), g.out.offset, g.n.offset, g.type.offset] == [32, 8, 16, 24]


def _list(*items):
    return (gradients.Gradient * max(1, len(items)))(*(gradients.Gradient(**{**dict(x=P, out=P, n=10, type=0, reserved=0), **i}) for i in items))


def _both(list_, count, norm=P, work=P, bytes_=1 << 20, max_norm=1.0):
    L = gradients._load()
    ptr = None if list_ is None else C.addressof(list_)
    return (L.asgd_grad_norm(ptr, count, norm, work, bytes_, None), L.asgd_clip_grads(ptr, count, max_norm, norm, work, bytes_, None))


@pytest.mark.parametrize("item, want", [
    (dict(x=None), (EINVAL, EINVAL)), (dict(n=-1), (EINVAL, EINVAL)), (dict(type=3), (EINVAL, EINVAL)), (dict(type=-1), (EINVAL, EINVAL)),
    (dict(x=P + 2), (EINVAL, EINVAL)), (dict(x=P + 1, type=1), (EINVAL, EINVAL)), (dict(reserved=1), (EINVAL, EINVAL)),
    (dict(n=(1 << 40) + 1), (EUNSUPPORTED, EUNSUPPORTED))])
def test_refuses_tensors(item, want):
    assert _both(_list(item), 1) == want
    assert _both(_list({}, item), 2) == want


def test_refuses_outputs_that_are_not_there():
    L, bad = gradients._load(), [_list(dict(out=None)), _list(dict(out=P + 2)), _list(dict(out=P + 1, type=2))]
    assert [L.asgd_clip_grads(C.addressof(b), 1, 1.0, P, P, 1 << 20, None) for b in bad] == [EINVAL] * 3


@pytest.mark.parametrize("items", [
    (dict(), dict()), (dict(), dict(x=P + 36, out=P + 36)), (dict(), dict(x=P + 4096, out=P + 16, n=1)), (dict(n=1000), dict(x=P + 80, out=P + 8192), dict(x=P + 400, out=P + 400)),
    (dict(out=P + 4),), (dict(out=P - 4, type=1),), (dict(x=P + 4096, out=P + 8192), dict(x=P + 8200, out=P + 12288)),
    (dict(out=P + 4096), dict(out=P + 4132)), (dict(n=0), dict(n=4, type=1), dict(x=P + 6, out=P + 6, n=1, type=1))])
def test_refuses_to_clip_what_meets(items):
    """Numbers that are written twice, or written while they are another tensor's input."""
    for order in (items, items[::-1]):
        list_ = _list(*order)
        assert gradients._load().asgd_clip_grads(C.addressof(list_), len(items), 1.0, P, P, 1 << 20, None) == EINVAL


def test_refuses_arguments():
    assert _both(None, 1) == (EINVAL, EINVAL)
    assert _both(_list({}), -1) == (EINVAL, EINVAL)
    assert _both(_list({}), 1, norm=None) == (EINVAL, EINVAL)
    assert _both(_list({}), 1, norm=P + 2) == (EINVAL, EINVAL)
    assert _both(_list({}), 1, work=None) == (ENOMEM, ENOMEM)
    n = C.c_size_t(0)
    L = gradients._load()
    assert L.asgd_gradients_workspace_bytes(1, C.byref(n)) == OK and n.value > 0
    assert _both(_list({}), 1, bytes_=n.value - 1) == (ENOMEM, ENOMEM)
    assert _both(_list({}), 1, work=P + 8) == (EINVAL, EINVAL)
    assert _both(_list({}), (1 << 20) + 1) == (EUNSUPPORTED, EUNSUPPORTED)
    for m in (0.0, -1.0, float("nan")):
        assert _both(_list({}), 1, max_norm=m)[1] == EINVAL
    assert L.asgd_gradients_workspace_bytes(-1, C.byref(n)) == EINVAL
    assert L.asgd_gradients_workspace_bytes(0, None) == EINVAL
    one = C.c_size_t(0)
    assert L.asgd_gradients_workspace_bytes(0, C.byref(one)) == OK and one.value > 0
    assert L.asgd_gradients_workspace_bytes(5000, C.byref(n)) == OK and n.value > one.value


def test_python_refuses_host_tensors_and_lists_that_do_not_fit(monkeypatch):
    x = torch.zeros(4)
    monkeypatch.setattr(gradients, "_current_device", lambda: 0)
    monkeypatch.setattr(gradients, "_load", lambda: pytest.fail("the library was reached"))
    for call in (lambda: pkg.asgd_grad_norm([x]), lambda: pkg.asgd_clip_grads([x], 1.0), lambda: pkg.asgd_grad_norm([3.0]),
                 lambda: pkg.asgd_clip_grads([x], 0.0), lambda: pkg.asgd_clip_grads([x], float("nan")), lambda: pkg.asgd_clip_grads([], 1.0, out=[x])):
        with pytest.raises(ValueError):
            call()
