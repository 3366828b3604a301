"""The whole layer for a few tokens without a GPU: exports, argument structure, workspace, refusals before any launch."""
import ctypes as C
import os
import re
import subprocess

import pytest
import torch

import paper_1505_04956_b200 as pkg
from paper_1505_04956_b200 import binding, experts, serving

from .test_experts_host_edges import _On

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
EINVAL, EUNSUPPORTED, ENOMEM, OK = binding.ASGD_EINVAL, binding.ASGD_EUNSUPPORTED, binding.ASGD_ENOMEM, binding.ASGD_OK
P = 1 << 20                       # stands for device memory: only calls that are refused get it


def test_header_and_binding_name_the_same_functions():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "asgd_expert_layer.h")).read(), flags=re.S)
    names = set(re.findall(r"\b(asgd_[a-z0-9_]+)\s*\(", text))
    assert names == set(pkg.LAYER_EXPORTS)
    L = C.CDLL(binding.LIB_PATH)
    for n in names:
        assert hasattr(L, n), n
        assert n.endswith("_workspace_bytes") or callable(getattr(pkg, n)), n


def test_structure_has_the_layout_of_the_header(tmp_path):
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "asgd_expert_layer.h"\nint main(void) { printf("%zu %zu %zu %zu\\n", sizeof(asgd_expert_layer_args), '
                   'offsetof(asgd_expert_layer_args, w2_scale_group), offsetof(asgd_expert_layer_args, type), offsetof(asgd_expert_layer_args, temperature)); return 0; }\n')
    exe = tmp_path / "sizes"
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, stdout=subprocess.PIPE, text=True).stdout.split()
    a = serving.ExpertLayerArgs
    assert [int(v) for v in out] == [C.sizeof(a), a.w2_scale_group.offset, a.type.offset, a.temperature.offset]


def _cfg(**kw):
    v = {**dict(experts=16, top_k=2, score=0, groups=1, groups_kept=1, group_top=1, renormalise=1, align=1, scale=1.0), **kw}
    return experts.RouteConfig(*(v[n] for n, _ in experts.RouteConfig._fields_))


def _args(**kw):
    v = {**dict(T=4, d=256, h=128, x=P, ldx=256, y=P, ldy=256, logits=P, ld_logits=16, w1=P, ldw1=256, w1_group=256 * 256, w1_scale=P, w1_scale_row=2,
                w1_scale_block=1, w1_scale_group=4, w2=P, ldw2=128, w2_group=256 * 128, w2_scale=P, w2_scale_row=1, w2_scale_block=1, w2_scale_group=2,
                type=1, logits_type=0, router_type=0, w1_type=3, w2_type=4, gated=1, activation=1, temperature=1.0), **kw}
    return serving.ExpertLayerArgs(**v)


def _call(cfg, args, work=P, bytes_=1 << 30):
    return serving._load().asgd_expert_layer(C.byref(cfg), C.byref(args), work, bytes_, None)


def _bytes(cfg, args):
    n = C.c_size_t(0)
    return serving._load().asgd_expert_layer_workspace_bytes(C.byref(cfg), C.byref(args), C.byref(n)), n.value


@pytest.mark.parametrize("bad, want", [
    (dict(T=-1), EINVAL), (dict(d=0), EINVAL), (dict(h=0), EINVAL), (dict(gated=2), EINVAL), (dict(T=129), EUNSUPPORTED),
    (dict(d=65537, ldx=65537, ldy=65537), EUNSUPPORTED), (dict(h=32769), EUNSUPPORTED), (dict(h=65537, gated=0), EUNSUPPORTED)])
def test_refuses_sizes(bad, want):
    assert _call(_cfg(), _args(**bad)) == want and _bytes(_cfg(), _args(**bad))[0] == want


@pytest.mark.parametrize("bad, want", [(dict(top_k=0), EINVAL), (dict(experts=0), EINVAL), (dict(groups=3), EINVAL), (dict(experts=2048), EUNSUPPORTED),
                                       (dict(experts=128, top_k=33), EUNSUPPORTED)])
def test_refuses_configurations(bad, want):
    assert _call(_cfg(**bad), _args()) == want and _bytes(_cfg(**bad), _args())[0] == want


def test_refuses_too_many_assignments_and_too_wide_layers():
    assert _call(_cfg(top_k=9), _args(T=114)) == EUNSUPPORTED and _bytes(_cfg(top_k=8), _args(T=128))[0] == OK
    wide = dict(T=128, d=65536, h=32768, ldx=65536, ldy=65536, ldw1=65536, ldw2=32768, w1_group=1 << 32, w2_group=1 << 31)
    assert _call(_cfg(top_k=8), _args(**wide)) == EUNSUPPORTED


@pytest.mark.parametrize("bad", [
    dict(type=3), dict(w1_type=1), dict(w2_type=0), dict(activation=2), dict(activation=-1), dict(logits=None), dict(router=P, ld_router=256), dict(shift=P),
    dict(logits_type=4), dict(ld_logits=15), dict(logits=P + 2), dict(logits=None, router=P, ld_router=255), dict(logits=None, router=P + 1, ld_router=256, router_type=1),
    dict(logits=None, router=P, ld_router=256, router_type=3), dict(logits=None, router=P, ld_router=256, shift=P + 2), dict(ldx=255), dict(ldy=255),
    dict(ldw1=240), dict(ldw1=264), dict(ldw2=112), dict(ldw2=136), dict(w1_group=8), dict(w2_group=-16), dict(w1_scale=P + 2), dict(w2_scale=None),
    dict(w1_scale=None), dict(bias=P + 2), dict(ids=P + 2), dict(weights=P + 1), dict(x=None), dict(y=None), dict(x=P + 1), dict(y=P + 1), dict(w1=None),
    dict(w2=None), dict(w1=P + 8), dict(w2=P + 1)])
def test_refuses_arguments(bad):
    assert _call(_cfg(), _args(**bad)) == EINVAL


def test_workspace():
    rc, n = _bytes(_cfg(), _args())
    assert rc == OK and n > 0 and n % 256 == 0
    assert _call(_cfg(), _args(), bytes_=n - 1) == ENOMEM and _call(_cfg(), _args(), work=None) == ENOMEM and _call(_cfg(), _args(), work=P + 128) == EINVAL
    assert _bytes(_cfg(), _args(T=100))[1] > n and _bytes(_cfg(), _args(logits=None, router=P, ld_router=256))[1] > n
    assert _call(_cfg(), _args(T=0), work=None, bytes_=0) == OK
    assert serving._load().asgd_expert_layer_workspace_bytes(C.byref(_cfg()), C.byref(_args()), None) == EINVAL
    assert serving._load().asgd_expert_layer(None, None, None, 0, None) == EINVAL


F32, E4 = torch.float32, torch.float8_e4m3fn
ARGS = [(F32, 4, 256), (E4, 16, 256, 256), (F32, 16, 2, 2), (E4, 16, 256, 128), (F32, 16, 2, 1)]
KW = dict(router=(F32, 16, 256), shift=(F32, 16), bias=(F32, 16))


def test_tensors_of_another_device_are_refused(monkeypatch):
    class Reached(Exception):
        pass

    def library():
        raise Reached
    monkeypatch.setattr(experts, "_current_device", lambda: 1)
    monkeypatch.setattr(serving, "_load", library)
    monkeypatch.setattr(serving, "_config", lambda *a: (None, 0))
    monkeypatch.setattr(serving, "_new", lambda *a, **k: _On(1, k["dtype"], *a[0]))

    def call(elsewhere=None, logits=False):
        make = lambda key, v: _On(0 if key == elsewhere else 1, *v)                            # noqa: E731
        kw = dict(logits=(F32, 4, 16)) if logits else KW
        return serving.asgd_expert_layer(*[make(i, v) for i, v in enumerate(ARGS)], 2, **{k: make(k, v) for k, v in kw.items()})
    for logits in (False, True):
        with pytest.raises(Reached):
            call(None, logits)
        for one in [*range(5), *(["logits"] if logits else KW)]:
            with pytest.raises(ValueError):
                call(one, logits)


def test_python_refuses_what_does_not_fit(monkeypatch):
    monkeypatch.setattr(experts, "_current_device", lambda: 0)
    monkeypatch.setattr(serving, "_load", lambda: pytest.fail("the library was reached"))

    def refused(change=None, **kw):
        shapes = list(ARGS)
        if change:
            shapes[change[0]] = change[1]
        given = {**dict(logits=_On(0, F32, 4, 16)), **kw}
        with pytest.raises(ValueError):
            serving.asgd_expert_layer(*[_On(0, *v) for v in shapes], 2, **given)
    refused((1, (E4, 16, 200, 256)))              # neither h nor 2 h rows
    refused((1, (E4, 16, 256, 128)))
    refused((2, (F32, 16, 256, 2)))               # scales by rows
    refused((3, (E4, 15, 256, 128)))
    refused((4, (F32, 16, 1, 2)))
    refused((0, (E4, 4, 256)))
    refused(logits=None)
    refused(router=_On(0, F32, 16, 256))          # both
    refused(logits=_On(0, F32, 4, 15))
    refused(shift=_On(0, F32, 16))
    refused(activation="gelu")
    refused(bias=_On(0, F32, 15))
    refused(score="tanh")
    refused(logits=None, router=_On(0, F32, 16, 255))
    with pytest.raises(ValueError):
        pkg.asgd_expert_layer(torch.zeros(4, 256), *[torch.zeros(1)] * 4, 2)
