"""4-bit operands and products without a GPU: exports, argument structures, refusals before any launch."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

import paper_1505_04956_b200 as pkg
from paper_1505_04956_b200 import binding, fp4

from .test_experts_host_edges import _On

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EUNSUPPORTED, OK = binding.ASGD_EINVAL, binding.ASGD_EUNSUPPORTED, binding.ASGD_OK
P = 1 << 20                       # stands for device memory: only calls that are refused get it


def test_header_and_binding_name_the_same_functions():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "asgd_fp4.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(asgd_[a-z0-9_]+)\s*\(", text))
    assert names == set(pkg.FP4_EXPORTS)
    L = C.CDLL(binding.LIB_PATH)
    for n in names:
        assert hasattr(L, n) and callable(getattr(pkg, n)), n


def test_structures_have_the_layout_of_the_header(tmp_path):
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "asgd_fp4.h"\nint main(void) { printf("%zu %zu %zu %zu %zu\\n", sizeof(asgd_quantize4_args), '
                   'offsetof(asgd_quantize4_args, scale_row), sizeof(asgd_product4_args), offsetof(asgd_product4_args, c), offsetof(asgd_product4_args, c_type)); return 0; }\n')
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, stdout=subprocess.PIPE, text=True).stdout.split()
    q, p = fp4.Quantize4Args, fp4.Product4Args
    assert [int(v) for v in out] == [C.sizeof(q), q.scale_row.offset, C.sizeof(p), p.c.offset, p.c_type.offset]


def _args(kind, **kw):
    return kind(*(kw[n] for n, _ in kind._fields_))


def _q(**kw):
    return _args(fp4.Quantize4Args, **{**dict(M=256, K=256, x=P, ldx=256, rows_x=256, x_type=1, per_token=1, source=None, weights=None, q=P, ldq=128,
                                              scale=P, scale_row=16), **kw})


@pytest.mark.parametrize("bad, want", [
    (dict(M=-1), EINVAL), (dict(K=-1), EINVAL), (dict(x=None), EINVAL), (dict(x=P + 1), EINVAL), (dict(ldx=255), EINVAL), (dict(x_type=3), EINVAL),
    (dict(q=None), EINVAL), (dict(ldq=127), EINVAL), (dict(K=255, ldq=127), EINVAL), (dict(scale=None), EINVAL), (dict(scale_row=7), EINVAL),
    (dict(weights=P), EINVAL), (dict(rows_x=255), EINVAL), (dict(per_token=0), EINVAL), (dict(source=P + 2), EINVAL),
    (dict(source=P, weights=P + 1), EINVAL), (dict(M=1 << 31, rows_x=1 << 31), EUNSUPPORTED),
    (dict(M=1, rows_x=1, K=(1 << 25) - 511, ldx=1 << 25, ldq=1 << 24, scale_row=1 << 20), EUNSUPPORTED)])
def test_quantize4_refuses(bad, want):
    assert fp4._load().asgd_quantize4(C.byref(_q(**bad)), None) == want


def test_of_nothing_is_fine():
    L = fp4._load()
    assert L.asgd_quantize4(C.byref(_q(M=0, rows_x=0)), None) == OK and L.asgd_quantize4(C.byref(_q(K=0)), None) == OK
    assert L.asgd_dequantize4(0, 64, None, 32, None, 2, None, 0, 64, None) == OK
    assert L.asgd_product4(C.byref(_p(M=0)), None) == OK and L.asgd_product4(C.byref(_p(N=0, ldc=0)), None) == OK
    assert L.asgd_quantize4(None, None) == EINVAL and L.asgd_product4(None, None) == EINVAL


@pytest.mark.parametrize("bad, want", [
    ((-1, 64, P, 32, P, 2, P, 0, 64), EINVAL), ((4, 64, P, 31, P, 2, P, 0, 64), EINVAL), ((4, 64, P, 32, P, 1, P, 0, 64), EINVAL),
    ((4, 64, P, 32, P, 2, P, 0, 63), EINVAL), ((4, 64, P, 32, P, 2, P, 3, 64), EINVAL), ((4, 64, None, 32, P, 2, P, 0, 64), EINVAL),
    ((4, 64, P, 32, None, 2, P, 0, 64), EINVAL), ((4, 64, P, 32, P, 2, None, 0, 64), EINVAL), ((4, 64, P, 32, P, 2, P + 2, 0, 64), EINVAL),
    ((1 << 31, 64, P, 32, P, 2, P, 0, 64), EUNSUPPORTED), ((4, 1 << 25, P, 1 << 24, P, 1 << 20, P, 0, 1 << 25), EUNSUPPORTED)])
def test_dequantize4_refuses(bad, want):
    assert fp4._load().asgd_dequantize4(*bad, None) == want


def _p(**kw):
    return _args(fp4.Product4Args, **{**dict(M=256, N=256, K=256, a=P, lda=128, a_scale=P, a_scale_row=16, b=P, ldb=128, b_group=0, b_scale=P, b_scale_row=16,
                                             b_scale_group=0, c=P, ldc=256, offsets=None, groups=0, c_type=1), **kw})


BIG = 1 << 31


@pytest.mark.parametrize("bad, want", [
    (dict(M=-1), EINVAL), (dict(a=None), EINVAL), (dict(a=P + 8), EINVAL), (dict(lda=136), EINVAL), (dict(lda=112), EINVAL), (dict(ldb=130), EINVAL),
    (dict(b=P + 1), EINVAL), (dict(c=None), EINVAL), (dict(c=P + 1), EINVAL), (dict(ldc=255), EINVAL), (dict(c_type=3), EINVAL), (dict(groups=2), EINVAL),
    (dict(groups=-1), EINVAL), (dict(offsets=P), EINVAL), (dict(groups=2, offsets=P + 2), EINVAL), (dict(groups=2, offsets=P, b_group=8), EINVAL),
    (dict(groups=2, offsets=P, b_group=-16), EINVAL), (dict(groups=2, offsets=P, b_scale_group=8), EINVAL), (dict(a_scale=None), EINVAL),
    (dict(a_scale=P + 8), EINVAL), (dict(b_scale=P + 4), EINVAL), (dict(a_scale_row=24), EINVAL), (dict(b_scale_row=8), EINVAL), (dict(b_scale_row=0), EINVAL),
    (dict(groups=1025, offsets=P), EUNSUPPORTED), (dict(M=BIG), EUNSUPPORTED), (dict(M=BIG - 255), EUNSUPPORTED), (dict(N=BIG - 255, ldc=BIG), EUNSUPPORTED),
    (dict(K=BIG - 255, lda=BIG, ldb=BIG, a_scale_row=BIG, b_scale_row=BIG), EUNSUPPORTED), (dict(N=BIG - 256, M=BIG - 256, ldc=BIG), EUNSUPPORTED)])
def test_product4_refuses(bad, want, monkeypatch):
    got = fp4._load().asgd_product4(C.byref(_p(**bad)), None)
    # (tiles beyond 32 bits are refused behind the device's status word, which a machine without a device does not have)
    assert got == want or (bad.get("M") == BIG - 256 and got == binding.ASGD_ECUDA)


F32, I32, Q, S = torch.float32, torch.int32, torch.float4_e2m1fn_x2, torch.float8_e8m0fnu
_CALLS = [
    ("asgd_quantize4", [(F32, 4, 8)], dict(source=(I32, 8), per_token=2, weights=(F32, 4, 2))),
    ("asgd_dequantize4", [(Q, 4, 16), (S, 4, 1)], {}),
    ("asgd_product4", [(Q, 4, 64), (S, 4, 4), (Q, 3, 32, 64), (S, 3, 32, 4)], dict(offsets=(I32, 4), out=(F32, 4, 32))),
]


@pytest.mark.parametrize("name, args, kw", _CALLS)
def test_tensors_of_another_device_are_refused(name, args, kw, monkeypatch):
    from paper_1505_04956_b200 import experts

    class Reached(Exception):
        pass

    def library():
        raise Reached
    monkeypatch.setattr(experts, "_current_device", lambda: 1)
    monkeypatch.setattr(fp4, "_load", library)
    monkeypatch.setattr(fp4, "_new", lambda *a, **k: _On(1, k["dtype"], *a[0]))
    is_tensor = lambda v: isinstance(v, tuple)                                                # noqa: E731
    tensors = [i for i, v in enumerate(args) if is_tensor(v)] + [k for k, v in kw.items() if is_tensor(v)]

    def call(elsewhere=None):
        made = [_On(0 if i == elsewhere else 1, v[0], *v[1:]) if is_tensor(v) else v for i, v in enumerate(args)]
        return getattr(fp4, name)(*made, **{k: _On(0 if k == elsewhere else 1, v[0], *v[1:]) if is_tensor(v) else v for k, v in kw.items()})
    with pytest.raises(Reached):
        call()
    for one in tensors:
        with pytest.raises(ValueError):
            call(one)


def test_python_refuses_host_tensors_and_wrong_types():
    x = torch.zeros(4, 64)
    q, s = torch.zeros(4, 32, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8)
    for call in (lambda: pkg.asgd_quantize4(x), lambda: pkg.asgd_dequantize4(q.view(Q), s.view(S)), lambda: pkg.asgd_product4(q, s, q, s)):
        with pytest.raises(ValueError):
            call()
