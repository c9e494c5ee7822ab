"""What expert_layer.py hands to the entry points that move tokens' rows, of its own routes and of a caller's, on the host: each operand is read from an address, as the
kernels read it, so that one with fewer elements, of another type or place is an error here."""
from types import SimpleNamespace

import pytest
import torch

import layer_emulation
import ops_emulation
from paper_2108_13191_amd import binding, expert_layer
from test_expert_layer_host import E, F, H, T, TOP, inputs, same

FORMS = [("rms", "e4m3"), ("rms", "i8"), ("layer", "i8"), ("layer", "e4m3")]


@pytest.fixture(params=FORMS, ids=["-".join(f) for f in FORMS])
def layer(request, monkeypatch):
    for f in ops_emulation.ENTRY_POINTS + layer_emulation.ENTRY_POINTS + layer_emulation.ROW_ENTRY_POINTS:
        monkeypatch.setattr(binding, f.__name__, f)
    monkeypatch.setattr(expert_layer, "_stream", lambda *t: 0)
    monkeypatch.setattr(expert_layer, "_on_gpu", lambda t: True)
    made = expert_layer.ExpertLayer(H, F, E, TOP, seed=1, device="cpu", norm=request.param[0])
    made.prepare(request.param[1])
    return made


def everything(layer, given):
    x, r, dout, dh = given
    served, s = layer.serve(x, r), layer.train_forward(x, r)
    return served, s, layer.backward(s, dout, dh)


def replaced(layer, change):
    """The layer with a router of the caller's own, whose route is the layer's with `change` made to it."""
    own = type(layer).route

    def route(y):
        given = SimpleNamespace(**vars(own(layer, y)))
        change(given)
        return given
    layer.route = route
    return layer


def equal(got, want):
    """(Not the routes, which the caller made.)"""
    for g, w, names in zip(got, want, (("h", "out"), ("h", "y", "out"), ("x", "gamma", "up", "down", "shared_up", "shared_down", "weight"))):
        for n in names:
            assert torch.equal(getattr(g, n), getattr(w, n)), n


@pytest.mark.parametrize("tokens", [0, 1, T])
def test_rows_moved_by_the_entry_points_give_what_torch_gives(layer, tokens, monkeypatch):
    given = inputs(tokens)
    got = everything(layer, given)
    monkeypatch.setattr(expert_layer, "_on_gpu", lambda t: False)
    equal(got, everything(layer, given))


def halves(route):
    route.weight = torch.full_like(route.weight, 0.5)


# weights of tokens x top_k by broadcasting: one for each token, for each choice, for all, and in other types and layouts
@pytest.mark.parametrize("make", [lambda w: w[:, :1].clone(), lambda w: w[:1].clone(), lambda w: w[0].clone(), lambda w: w[0, 0].clone(), lambda w: w[:, :1].expand(-1, TOP), lambda w: w.double(),
                                  lambda w: w.t().contiguous().t()], ids=["tokens", "choices", "row", "one", "expanded", "f64", "transposed"])
def test_weights_of_a_route_are_broadcast(layer, make):
    given = inputs()
    want = everything(replaced(layer, halves), given)

    def change(route):
        halves(route)
        route.weight = make(route.weight)
    equal(everything(replaced(layer, change), given), want)


@pytest.mark.parametrize("make", [lambda w: w[1:], lambda w: w[:, :, None], lambda w: w.flatten(), lambda w: torch.cat([w, w], 1), lambda w: w.to(torch.complex64)],
                         ids=["fewer", "three", "flat", "more", "complex"])
def test_weights_of_no_such_shape_are_refused(layer, make):
    x, r, dout, dh = inputs()
    s = layer.train_forward(x, r)

    def change(route):
        route.weight = make(route.weight)
    replaced(layer, change)
    change(s.route)
    for call in (lambda: layer.serve(x, r), lambda: layer.train_forward(x, r), lambda: layer.backward(s, dout, dh)):
        with pytest.raises(ValueError):
            call()
