"""rope of a tensor that requires a gradient: what it hands over and refuses (no GPU; the
launches are recorded)."""
import pytest
import torch

import paper_2606_00535_gb300 as dreams
from test_kv8_streams import world  # noqa: F401

TRANSPOSE = 17  # its place among the arguments


def launches(w):
    return [(name, a[TRANSPOSE]) for name, _, a in w.calls]


def test_the_backward_pass_is_the_transposed_turn(world):  # noqa: F811
    for transpose in (False, True):
        x = world.z(2, 3, 4, 64).requires_grad_()
        world.calls.clear()
        y = dreams.rope(x, world.rotary, transpose=transpose)
        assert y.requires_grad and launches(world) == [("dreams_rope", int(transpose))]
        g, = torch.autograd.grad(y, x, world.z(2, 3, 4, 64))
        assert launches(world) == [("dreams_rope", int(transpose)), ("dreams_rope", int(not transpose))] and not g.requires_grad


def test_out_is_refused_where_a_gradient_is_asked_for(world):  # noqa: F811
    x, out = world.z(2, 3, 4, 64).requires_grad_(), world.z(2, 3, 4, 64)
    for o in (out, x):
        with pytest.raises(ValueError):
            dreams.rope(x, world.rotary, out=o)
    assert not world.calls
    with torch.no_grad():
        assert dreams.rope(x, world.rotary, out=out) is out and not dreams.rope(x, world.rotary).requires_grad
    assert dreams.rope(x.detach(), world.rotary, out=out) is out
