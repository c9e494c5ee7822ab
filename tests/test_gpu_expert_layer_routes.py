"""expert_layer.py with routers of a caller's own: parts of a route on the host, of other types and shapes, groups filled up and choices dropped, against the layer's own
route."""
from types import SimpleNamespace

import pytest
import torch

from test_expert_layer_routes_host import everything, filled_up, halves, near, replaced
from test_gpu_expert_layer_forms import setup

pytestmark = pytest.mark.gpu
FORMS = pytest.mark.parametrize("norm,form", [("rms", "e4m3"), ("layer", "i8")])
NAMES = (("h", "out"), ("h", "y", "out"), ("x", "gamma", "up", "down", "shared_up", "shared_down", "weight"))
TOKENS, EXPERTS, TOP = 300, 6, 2


@pytest.fixture
def made():
    def make(norm, form):
        layer, given, _ = setup(TOKENS, 264, 136, EXPERTS, TOP, torch.bfloat16, norm)
        layer.prepare(form)
        return layer, [t.cuda() for t in given]
    return make


def equal(got, want):
    for g, w, names in zip(got, want, NAMES):
        for n in names:
            assert torch.equal(getattr(g, n), getattr(w, n)), n


def on_the_host(*names):
    def change(route):
        for n in names:
            setattr(route, n, getattr(route, n).cpu())
    return change


@FORMS
@pytest.mark.parametrize("names", [("place",), ("source",), ("weight",), ("offsets",), ("place", "source", "weight", "offsets")], ids=" ".join)
def test_parts_of_a_route_on_the_host(made, norm, form, names):
    layer, given = made(norm, form)
    want = everything(layer, given)
    equal(everything(replaced(layer, on_the_host(*names)), given), want)


@FORMS
@pytest.mark.parametrize("make", [lambda w: w[:, :1].clone(), lambda w: w[0].clone(), lambda w: w[0, 0].clone(), lambda w: w.double()], ids=["tokens", "row", "one", "f64"])
def test_weights_of_a_route_are_broadcast(made, norm, form, make):
    layer, given = made(norm, form)
    want = everything(replaced(layer, halves), given)

    def change(route):
        halves(route)
        route.weight = make(route.weight)
    equal(everything(replaced(layer, change), given), want)


def with_lists_on_the_host(change):
    """`change`, which goes through lists, and its results back on the GPU."""
    def f(route):
        on_the_host("place", "source", "offsets", "weight")(route)
        change(route)
        for n in ("place", "source", "offsets", "weight"):
            setattr(route, n, getattr(route, n).cuda())
    return f


@FORMS
def test_groups_that_a_router_fills_up(made, norm, form):
    layer, given = made(norm, form)
    want = everything(layer, given)
    got = everything(replaced(layer, with_lists_on_the_host(filled_up)), given)
    assert got[0].route.source.numel() > TOKENS * TOP
    for g, w, names in zip(got, want, NAMES):
        near(g, w, *names)


@FORMS
@pytest.mark.parametrize("fill", [False, True])
def test_choices_that_a_router_drops(made, norm, form, fill):
    layer, given = made(norm, form)

    def zeros(route):
        if fill:
            filled_up(route)
        route.weight = route.weight.clone()
        route.weight[::2, 1] = 0

    def drop(route):
        zeros(route)
        flat = route.place.view(-1, TOP).clone()
        flat[::2, 1] = -1
        route.place = flat.flatten()
    want = everything(replaced(layer, with_lists_on_the_host(zeros)), given)
    want[2].weight[::2, 1] = 0
    # (what memory holds that is allocated and not written)
    torch.full((64, 1 << 20), float("nan"), device="cuda")
    equal(everything(replaced(layer, with_lists_on_the_host(drop)), given), want)
