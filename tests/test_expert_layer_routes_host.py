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


def near(got, want, *names):
    """Products of another number of rows may add in another order: a unit of bf16 (2 half ones of 2^-8) at each of the four roundings behind one another."""
    for n in names:
        g, w = getattr(got, n).double(), getattr(want, n).double()
        assert (g - w).norm() <= 8 * 2.0 ** -8 * w.norm(), n


def filled_up(route, to=4):
    """Each expert's rows filled up to a multiple of `to` with rows of token 0, as kernels of whole tiles want them."""
    bounds = route.offsets.tolist()
    source, place, offsets = [], torch.zeros(route.place.numel(), dtype=torch.int64), [0]
    by = torch.empty_like(place)
    by[route.place.long()] = torch.arange(place.numel())
    for lo, hi in zip(bounds, bounds[1:]):
        place[by[lo:hi]] = len(source) + torch.arange(hi - lo)
        source += route.source[lo:hi].tolist() + [0] * (-(hi - lo) % to)
        offsets.append(len(source))
    route.source, route.place, route.offsets = torch.tensor(source), place, torch.tensor(offsets, dtype=torch.int32)


@pytest.mark.parametrize("tokens", [1, T])
def test_groups_that_a_router_fills_up(layer, tokens):
    """More rows than choices: all of them are in the result, and those of no choice in no gradient."""
    given = inputs(tokens)
    want = everything(layer, given)
    got = everything(replaced(layer, filled_up), given)
    assert got[0].route.source.numel() > tokens * TOP
    for g, w, names in zip(got, want, (("h", "out"), ("h", "y", "out"), ("x", "gamma", "up", "down", "shared_up", "shared_down", "weight"))):
        near(g, w, *names)


def dropped(route, rows):
    """The second choice of every other token has no row: its place is none of `rows` any more."""
    flat = route.place.view(-1, TOP).clone()
    flat[::2, 1] = torch.tensor([-1, rows, -2 ** 31, 2 ** 31 - 1]).repeat(T)[:flat[::2].shape[0]].to(flat.dtype)
    route.place = flat.flatten()


@pytest.mark.parametrize("index", [torch.int32, torch.int64])
@pytest.mark.parametrize("fill", [False, True])
def test_choices_that_a_router_drops(layer, index, fill, monkeypatch):
    """Their rows stay in the groups: the result and the gradients are those of weights of 0."""
    given = inputs()
    real = torch.empty_like
    monkeypatch.setattr(torch, "empty_like", lambda t, **k: real(t, **k).fill_(float("nan")) if t.is_floating_point() else real(t, **k))

    def zeros(route):
        if fill:
            filled_up(route)
        route.weight = route.weight.clone()
        route.weight[::2, 1] = 0

    def drop(route):
        zeros(route)
        dropped(route, route.source.numel())
        route.place = route.place.to(index)
    want = everything(replaced(layer, zeros), given)
    want[2].weight[::2, 1] = 0
    equal(everything(replaced(layer, drop), given), want)


def test_a_place_that_32_bits_do_not_hold_is_no_row(layer):
    given = inputs()

    def drop(route):
        dropped(route, T * TOP)
        route.place = route.place.long()

    def far(route):
        drop(route)
        route.place = torch.where(route.place < 0, route.place + 2 ** 32 * 5 + 3, route.place)
    equal(everything(replaced(layer, far), given), everything(replaced(layer, drop), given))


def test_fewer_rows_than_choices(layer):
    """A router that takes each token's first choice only, T rows: the other places are none."""
    given = inputs()

    def first(route):
        bounds = torch.bucketize(torch.arange(T * TOP), route.offsets[1:].long(), right=True)          # the expert of each row
        own = route.place.view(-1, TOP)[:, 0].long()
        order = own.sort().indices
        place = torch.full((T, TOP), -1)
        place[order, 0] = torch.arange(T)
        route.source, route.place = order, place.flatten()
        route.offsets = torch.searchsorted(bounds[own[order]], torch.arange(E + 1)).int()

    def zeros(route):
        route.weight = route.weight.clone()
        route.weight[:, 1] = 0
    want = everything(replaced(layer, zeros), given)
    want[2].weight[:, 1] = 0
    got = everything(replaced(layer, first), given)
    for g, w, names in zip(got, want, (("h", "out"), ("h", "y", "out"), ("x", "gamma", "up", "down", "shared_up", "shared_down", "weight"))):
        near(g, w, *names)


@pytest.mark.parametrize("make", [lambda p: p[1:], lambda p: torch.cat([p, p]), lambda p: p.float(), lambda p: p > 3], ids=["fewer", "more", "f32", "bool"])
def test_places_that_are_none_are_refused(layer, make):
    x, r, dout, dh = inputs()
    s = layer.train_forward(x, r)

    def change(route):
        route.place = make(route.place)
    replaced(layer, change)
    change(s.route)
    for call in (lambda: layer.serve(x, r), lambda: layer.train_forward(x, r), lambda: layer.backward(s, dout, dh)):
        with pytest.raises(ValueError):
            call()


def test_parts_of_a_route_go_to_the_rows_device():
    """The kernels get addresses: what lies elsewhere is copied there first."""
    route = SimpleNamespace(place=torch.arange(T * TOP))
    place, weight = expert_layer._places(route, T, TOP, torch.device("meta")), expert_layer._weight(torch.ones(T, 1), T, TOP, torch.device("meta"))
    assert place.device.type == weight.device.type == expert_layer._places32(place).device.type == "meta"
    assert place.shape == weight.shape == (T, TOP) and weight.is_contiguous()


@pytest.mark.parametrize("make", [lambda o: o.long(), lambda o: torch.stack([o, o], 1)[:, 0]], ids=["64 bits", "apart"])
def test_offsets_of_a_route_in_other_forms(layer, make):
    given = inputs()
    want = everything(layer, given)

    def change(route):
        route.offsets = make(route.offsets)
    equal(everything(replaced(layer, change), given), want)


@pytest.mark.parametrize("make", [lambda o: o[1:], lambda o: torch.cat([o, o[-1:]]), lambda o: o[None], lambda o: o.float(), lambda o: o.short()], ids=["fewer", "more", "two", "f32", "16 bits"])
def test_offsets_that_are_none_are_refused(layer, make):
    x, r, dout, dh = inputs()
    s = layer.train_forward(x, r)

    def change(route):
        route.offsets = make(route.offsets)
    replaced(layer, change)
    change(s.route)
    for call in (lambda: layer.serve(x, r), lambda: layer.train_forward(x, r), lambda: layer.backward(s, dout, dh)):
        with pytest.raises(ValueError):
            call()


def test_offsets_go_to_the_rows_device():
    assert expert_layer._offsets(SimpleNamespace(offsets=torch.arange(E + 1)), E, torch.device("meta")).device.type == "meta"
