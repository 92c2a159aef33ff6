"""Sizes beyond 32 bits, which the entry points' structs cannot hold, are refused by the binding and not cut off."""
import pytest
import torch

from paper_2608_03676_b200 import layer

HUGE = 1 << 32
META = torch.device("meta")


@pytest.fixture(autouse=True)
def nothing_is_called(monkeypatch):
    """Tensors without memory; a call that gets as far as the library fails the test."""
    def called(device, what, params, *args):
        raise AssertionError("%s was called" % what)

    monkeypatch.setattr(layer, "_start", lambda t, name, dims: t.device)
    monkeypatch.setattr(layer, "_call", called)


def rows(*shape, dtype=torch.bfloat16):
    return torch.empty(shape, dtype=dtype, device=META)


def indices(*shape):
    return rows(*shape, dtype=torch.int32)


def floats(*shape):
    return rows(*shape, dtype=torch.float32)


CALLS = {
    "columns of a norm": lambda: layer.rms_norm(rows(1, HUGE + 8), rows(HUGE + 8)),
    "columns of a norm's gradient": lambda: layer.rms_norm_backward(rows(1, HUGE + 8), rows(1, HUGE + 8), rows(HUGE + 8), floats(1), want_dweight=False),
    "a group": lambda: layer.rms_norm(rows(4, 256), rows(256), group=HUGE + 32),
    "a group below": lambda: layer.rms_norm(rows(4, 256), rows(256), group=32 - HUGE, out=dict(scales=floats(4, 0))),
    "experts": lambda: layer.route(rows(1, HUGE + 8), 4),
    "places": lambda: layer.route(rows(1, 64), HUGE + 4),
    "groups": lambda: layer.route(rows(4, 64), 4, groups=HUGE + 1),
    "groups that stay": lambda: layer.route(rows(4, 64), 4, groups=8, groups_kept=HUGE + 4),
    "a group's keys": lambda: layer.route(rows(4, 64), 4, groups=8, groups_kept=4, group_top=HUGE + 1),
    "experts of the gradient": lambda: layer.route_backward(rows(1, HUGE + 8), indices(1, 4), floats(1, 4)),
    "places of the gradient": lambda: layer.route_backward(rows(1, 8), indices(1, HUGE + 4), floats(1, HUGE + 4)),
    "columns of send": lambda: layer.send(rows(1, 1, HUGE + 8), indices(1, 1, 1)),
    "scales of send": lambda: layer.send(rows(1, 1, 8), indices(1, 1, 1), scales=floats(1, 1, HUGE + 8)),
    "entries of a token": lambda: layer.send(rows(1, 1, 8), indices(1, 1, HUGE + 1)),
    "counts": lambda: layer.send(rows(1, 1, 8), indices(1, 1, 1), counts=indices(1, HUGE + 1)),
    "columns of combine": lambda: layer.combine(rows(1, 1, HUGE + 8), indices(1, 1, 1)),
    "columns of combine's gradient": lambda: layer.combine_backward(rows(1, 1, HUGE + 8), indices(1, 1, 1)),
}


@pytest.mark.parametrize("what", CALLS)
def test_it_is_refused(what):
    with pytest.raises(layer.TaotError, match="out of range"):
        CALLS[what]()


def test_what_fits_is_called():
    for f in (lambda: layer.rms_norm(rows(4, 256), rows(256), group=32), lambda: layer.route(rows(4, 64), 4, groups=8, groups_kept=4, group_top=2),
              lambda: layer.route_backward(rows(4, 64), indices(4, 4), floats(4, 4)), lambda: layer.combine(rows(1, 4, 8), indices(1, 2, 2)),
              lambda: layer.send(rows(1, 2, 8), indices(1, 2, 2), counts=indices(1, 3), scales=floats(1, 2, 5)),
              lambda: layer.combine_backward(rows(1, 2, 8), indices(1, 2, 2)),
              lambda: layer.rms_norm_backward(rows(4, 256), rows(4, 256), rows(256), floats(4), want_dweight=False)):
        with pytest.raises(AssertionError, match="was called"):
            f()


def test_places_below_one_and_a_bias_without_experts_are_refused():
    for f in (lambda: layer.route(rows(4, 64), -1), lambda: layer.route(rows(4, 64), 0), lambda: layer.route(rows(4, 1), 1, bias=floats())):
        with pytest.raises(layer.TaotError):
            f()
