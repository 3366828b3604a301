"""Settings of a choice are taken as they are at the call, without a GPU."""
import pytest
import torch

from paper_1505_04956_b200 import experts, serving


def _route(**kw):
    v = {**dict(top_k=2, groups=4, groups_kept=2, group_top=1, renormalise=True, scale=1.0), **kw}
    return experts._route_config(16, v["top_k"], "softmax", v["groups"], v["groups_kept"], v["group_top"], v["renormalise"], v["scale"], 1, 8)[0].contents


def _layer(**kw):
    v = {**dict(top_k=2, groups=4, groups_kept=2, group_top=1, renormalise=True, scale=1.0), **kw}
    return serving._config(16, v["top_k"], "softmax", v["groups"], v["groups_kept"], v["group_top"], v["renormalise"], v["scale"], 8, 256, 128, 1, True)[0].contents


@pytest.mark.parametrize("config", [_route, _layer])
@pytest.mark.parametrize("name, first, then", [("scale", 1.0, 2.5), ("top_k", 2, 4), ("groups_kept", 1, 3), ("group_top", 1, 2), ("renormalise", 1, 0)])
def test_a_setting_that_changes_in_place(config, name, first, then):
    held = torch.tensor(first)
    for value in (first, then, first):
        held.fill_(value)
        assert getattr(config(**{name: held}), name) == value == getattr(config(**{name: value}), name)
