"""The operators of a layer of experts without a GPU: exports, argument structures, refusals before any launch."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

import paper_1505_04956_b200 as pkg
from paper_1505_04956_b200 import binding, experts

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EUNSUPPORTED, ENOMEM, OK = binding.ASGD_EINVAL, binding.ASGD_EUNSUPPORTED, binding.ASGD_ENOMEM, binding.ASGD_OK
P = C.c_void_p(1 << 20)          # stands for device memory: only calls that are refused get it


def test_header_and_binding_name_the_same_functions():
    text = open(os.path.join(ROOT, "include", "asgd_experts.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    names = set(re.findall(r"\b(asgd_[a-z0-9_]+)\s*\(", text))
    assert names == set(pkg.EXPERT_EXPORTS)
    L = C.CDLL(binding.LIB_PATH)
    for n in names:
        assert hasattr(L, n), n
        # asgd_route_workspace_bytes is part of asgd_route in Python
        assert n == "asgd_route_workspace_bytes" or callable(getattr(pkg, n)), n


def test_structures_have_the_sizes_of_the_header(tmp_path):
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include "asgd_experts.h"\nint main(void) { printf("%zu %zu %zu\\n", sizeof(asgd_route_config), '
                   'sizeof(asgd_quantize_args), sizeof(asgd_product_args)); return 0; }\n')
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, stdout=subprocess.PIPE, text=True).stdout.split()
    assert [int(v) for v in out] == [C.sizeof(experts.RouteConfig), C.sizeof(experts.QuantizeArgs), C.sizeof(experts.ProductArgs)]


def _cfg(**kw):
    v = dict(experts=64, top_k=4, score=0, groups=8, groups_kept=4, group_top=2, renormalise=1, align=1, scale=1.0)
    v.update(kw)
    return experts.RouteConfig(*(v[n] for n, _ in experts.RouteConfig._fields_))


@pytest.mark.parametrize("bad, want", [
    (dict(experts=0), EINVAL), (dict(top_k=0), EINVAL), (dict(top_k=33), EINVAL), (dict(score=2), EINVAL), (dict(groups=7), EINVAL),
    (dict(groups_kept=0), EINVAL), (dict(groups_kept=9), EINVAL), (dict(group_top=3), EINVAL), (dict(align=0), EINVAL),
    (dict(renormalise=2), EINVAL), (dict(experts=2048, groups=1, groups_kept=1), EUNSUPPORTED),
    (dict(experts=64, groups=64, groups_kept=40), EUNSUPPORTED), (dict(experts=128, top_k=40), EUNSUPPORTED)])
def test_route_refuses_configurations(bad, want):
    L, n = experts._load(), C.c_size_t(0)
    assert L.asgd_route_workspace_bytes(C.byref(_cfg(**bad)), 10, C.byref(n)) == want
    assert L.asgd_route(C.byref(_cfg(**bad)), 10, P, 0, 4096, None, P, P, P, P, P, 1 << 20, P, 1 << 20, None) == want


def test_route_refuses_arguments():
    L, n = experts._load(), C.c_size_t(0)
    c = C.byref(_cfg())
    assert L.asgd_route_workspace_bytes(c, -1, C.byref(n)) == EINVAL
    assert L.asgd_route_workspace_bytes(c, 64, C.byref(n)) == OK and n.value == 0
    assert L.asgd_route_workspace_bytes(c, 1000, C.byref(n)) == OK and n.value > 0
    good = [c, 1000, P, 0, 64, None, P, P, P, P, P, 4000, P, n.value, None]

    def with_(**kw):
        a = list(good)
        for i, v in kw.items():
            a[int(i[1:])] = v
        return L.asgd_route(*a)
    assert with_(_0=None) == EINVAL
    assert with_(_1=-1) == EINVAL
    assert with_(_2=None) == EINVAL
    assert with_(_2=C.c_void_p((1 << 20) + 2)) == EINVAL                  # not aligned to its type
    assert with_(_3=3) == EINVAL                                          # 8-bit logits
    assert with_(_4=63) == EINVAL                                         # rows shorter than E
    assert with_(_6=None) == EINVAL and with_(_7=None) == EINVAL
    assert with_(_8=None) == EINVAL and with_(_9=None) == EINVAL and with_(_10=None) == EINVAL   # a plan in part
    assert with_(_11=3999) == EINVAL
    assert with_(_11=1 << 31) == EUNSUPPORTED
    assert with_(_12=None) == ENOMEM and with_(_13=n.value - 1) == ENOMEM
    assert with_(_12=C.c_void_p((1 << 20) + 4)) == EINVAL
    assert L.asgd_route_grad(c, 10, P, 0, 64, P, P, P, 63, None) == EINVAL
    assert L.asgd_route_grad(c, 10, P, 0, 64, None, P, P, 64, None) == EINVAL
    assert L.asgd_route_grad(c, 0, None, 0, 64, None, None, None, 64, None) == OK


def _q(**kw):
    v = dict(M=256, K=256, x=1 << 20, ldx=256, rows_x=256, x_type=1, q_type=3, square=0, per_token=1, source=None, weights=None,
             q=1 << 20, ldq=256, scale=1 << 20, scale_row=1, scale_block=256, qt=None, ldqt=0, scale_t=None, scale_t_row=0, scale_t_block=0)
    v.update(kw)
    return experts.QuantizeArgs(*(v[n] for n, _ in experts.QuantizeArgs._fields_))


@pytest.mark.parametrize("bad, want", [
    (dict(M=-1), EINVAL), (dict(x=None), EINVAL), (dict(x=(1 << 20) + 1), EINVAL), (dict(ldx=255), EINVAL), (dict(x_type=3), EINVAL),
    (dict(q_type=1), EINVAL), (dict(q=None), EINVAL), (dict(ldq=255), EINVAL), (dict(scale=None), EINVAL), (dict(square=2), EINVAL),
    (dict(square=1, source=1 << 20), EINVAL), (dict(weights=1 << 20), EINVAL), (dict(rows_x=255), EINVAL), (dict(per_token=0), EINVAL),
    (dict(qt=1 << 20, ldqt=255, scale_t=1 << 20), EINVAL), (dict(qt=1 << 20, ldqt=256), EINVAL), (dict(M=1 << 31, rows_x=1 << 31), EUNSUPPORTED),
    (dict(qt=1 << 20, ldqt=1 << 24, scale_t=1 << 20, M=1 << 24, rows_x=1 << 24), EUNSUPPORTED)])
def test_quantize_refuses(bad, want):
    assert experts._load().asgd_quantize(C.byref(_q(**bad)), None) == want


def test_quantize_of_nothing_is_fine():
    assert experts._load().asgd_quantize(C.byref(_q(M=0, rows_x=0)), None) == OK
    assert experts._load().asgd_quantize(None, None) == EINVAL


def _p(**kw):
    v = dict(M=256, N=256, K=256, a=1 << 20, lda=256, a_scale=1 << 20, a_scale_row=1, a_scale_block=256, b=1 << 20, ldb=256, b_group=0,
             b_scale=1 << 20, b_scale_row=2, b_scale_block=1, b_scale_group=0, c=1 << 20, ldc=256, c_group=0, offsets=None, groups=0,
             inner=0, a_type=3, b_type=4, c_type=1, b_square=1)
    v.update(kw)
    return experts.ProductArgs(*(v[n] for n, _ in experts.ProductArgs._fields_))


@pytest.mark.parametrize("bad, want", [
    (dict(M=-1), EINVAL), (dict(a=None), EINVAL), (dict(a=(1 << 20) + 8), EINVAL), (dict(lda=264), EINVAL), (dict(lda=240), EINVAL),
    (dict(ldb=260), EINVAL), (dict(b=(1 << 20) + 1), EINVAL), (dict(c=None), EINVAL), (dict(c=(1 << 20) + 1), EINVAL), (dict(ldc=255), EINVAL),
    (dict(a_type=1), EINVAL), (dict(c_type=3), EINVAL), (dict(groups=2), EINVAL), (dict(offsets=1 << 20), EINVAL), (dict(inner=1), EINVAL),
    (dict(groups=2, offsets=1 << 20, b_group=8), EINVAL), (dict(a_scale=None), EINVAL), (dict(b_scale=(1 << 20) + 2), EINVAL),
    (dict(groups=1025, offsets=1 << 20), EUNSUPPORTED), (dict(M=1 << 31), EUNSUPPORTED)])
def test_product_refuses(bad, want):
    assert experts._load().asgd_product(C.byref(_p(**bad)), None) == want


def test_product_of_nothing_is_fine():
    assert experts._load().asgd_product(C.byref(_p(M=0)), None) == OK
    assert experts._load().asgd_product(C.byref(_p(N=0, ldc=0)), None) == OK
    assert experts._load().asgd_product(None, None) == EINVAL


def test_combine_refuses():
    L = experts._load()
    assert L.asgd_combine(4, 64, 2, P, 1, 8, 63, P, P, P, 64, None) == EINVAL
    assert L.asgd_combine(4, 64, 2, P, 1, 8, 64, None, P, P, 64, None) == EINVAL
    assert L.asgd_combine(4, 64, 2, P, 4, 8, 64, P, P, P, 64, None) == EINVAL
    assert L.asgd_combine(4, 64, 0, P, 1, 8, 64, P, P, P, 64, None) == EINVAL
    assert L.asgd_combine(4, 64, 33, P, 1, 8, 64, P, P, P, 64, None) == EUNSUPPORTED
    assert L.asgd_combine(4, 64, 2, C.c_void_p((1 << 20) + 1), 1, 8, 64, P, P, P, 64, None) == EINVAL
    assert L.asgd_combine(0, 64, 2, None, 1, 0, 64, None, None, None, 64, None) == OK
    assert L.asgd_combine_grad(4, 64, 2, P, 1, 63, P, 8, 64, P, P, P, P, 64, P, None) == EINVAL
    assert L.asgd_combine_grad(4, 64, 2, P, 1, 64, None, 8, 64, P, P, P, P, 64, P, None) == EINVAL
    assert L.asgd_combine_grad(4, 64, 2, P, 1, 64, P, 8, 64, P, P, P, None, 64, None, None) == OK     # nothing asked for
    assert L.asgd_product_set_wait_drill(0, 0) == EINVAL


def test_python_refuses_host_tensors_and_wrong_shapes():
    x = torch.zeros(4, 64)
    with pytest.raises(ValueError):
        pkg.asgd_route(x, 2)
    with pytest.raises(ValueError):
        pkg.asgd_quantize(x)
    with pytest.raises(ValueError):
        pkg.asgd_combine(x, torch.zeros(2, 2, dtype=torch.int32))
    q = x.to(torch.float8_e4m3fn)
    with pytest.raises(ValueError):
        pkg.asgd_product(q, x, q, x)
