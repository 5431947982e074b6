"""What the calls with several rotary axes take for a plan: nothing but one of their own, since its address is read on the host."""
import types

import pytest
import torch


@pytest.fixture(scope="module")
def a2sf():
    from paper_2407_20485_b200 import build

    build.build()
    from paper_2407_20485_b200 import binding

    return binding


@pytest.mark.parametrize("kind", ["none", "number", "other plan", "has an address", "its address"])
def test_what_is_no_plan_of_several_axes_is_refused_before_it_is_read(a2sf, kind):
    plan = a2sf.a2sf_rotary_axes_plan_init([16, 16], a2sf.a2sf_rotary_plan_init(64))
    bad = {"none": None, "number": 7, "other plan": a2sf.a2sf_rotary_plan_init(64), "has an address": types.SimpleNamespace(at=8, axes=2),
           "its address": plan.at}[kind]
    x, pos = torch.zeros((1, 2, 3, 64)), torch.zeros((2, 1, 3), dtype=torch.int32)
    cache = a2sf.PagedCache(1, 2, 64, torch.float32, 16, 4, 2, device="cpu")
    with pytest.raises(ValueError, match="expected a plan of a2sf_rotary_axes_plan_init"):
        a2sf.a2sf_rotary_axes(bad, x, pos)
    with pytest.raises(ValueError, match="expected a plan of a2sf_rotary_axes_plan_init"):
        cache.a2sf_paged_append_axes(x, x, pos, bad)
