"""Corners of the calls that stand between the layers of a block with routed experts, without a GPU."""
import copy
import pickle

import pytest

from paper_2312_03415_amd import binding as rl


@pytest.mark.parametrize("name,value", [("top", 1), ("top", 3), ("experts", 4), ("score", "sigmoid"), ("renormalise", False), ("groups", 2), ("groups_kept", 1),
                                        ("group_top", 2), ("scale", 2.0), ("how", (8, 1, 0, 1, 1, 1, 1)), ("bias", None)])
def test_a_plan_is_not_changed(name, value):
    """Tables are checked against the plan's attributes and written by the numbers handed to the library: with `top` changed in one of the two the kernels
    would write past them."""
    route = rl.Route(8, 2)
    with pytest.raises(AttributeError, match="make another"):
        setattr(route, name, value)
    with pytest.raises(AttributeError):
        delattr(route, name)
    assert (route.experts, route.top, route.score, route.renormalise, route.groups, route.groups_kept, route.group_top, route.scale) == (
        8, 2, "softmax", True, 1, 1, 1, 1.0)
    assert route.how == (8, 2, 0, 1, 1, 1, 1)


def test_a_plans_numbers_are_one():
    route = rl.Route(24, 4, "sigmoid", False, 8, 3, 2, 2.5)
    for r in (route, copy.copy(route), copy.deepcopy(route), pickle.loads(pickle.dumps(route))):
        assert r.how == (24, 4, 1, 0, 8, 3, 2) and (r.experts, r.top, r.score, r.renormalise) == (24, 4, "sigmoid", False)
        d = r.desc()
        assert tuple(getattr(d, f) for f, _ in d._fields_[:7]) == r.how and d.scale == r.scale == 2.5 and d.bias is None


@pytest.mark.parametrize("name,value", [("rows", 41), ("cols", 256), ("data", None), ("scales", None), ("more", 1)])
def test_8bit_rows_are_not_changed(name, value):
    """With `rows` set behind the bytes' back a norm of as many rows would write past them."""
    torch = pytest.importorskip("torch")
    q = rl.Fp8Rows.empty(40, 120, "cpu")
    with pytest.raises(AttributeError, match="make another"):
        setattr(q, name, value)
    with pytest.raises(AttributeError):
        delattr(q, name)
    q.data.fill_(0x38)  # (the bytes themselves are room to write into)
    for r in (q, copy.copy(q), copy.deepcopy(q)):
        assert r.shape == (40, 120) and tuple(r.data.shape) == (40, 128) and tuple(r.scales.shape) == (1, 48)
        assert torch.equal(r.data, q.data)
