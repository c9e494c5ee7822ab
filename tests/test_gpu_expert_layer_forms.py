"""expert_layer.py with a layer norm and with 8-bit integers, and its rows moved by the library, against the block's definition in 64 bits on the host and against the same rows
moved by torch."""
from types import SimpleNamespace

import pytest
import torch

from paper_2108_13191_amd import expert_layer
from paper_2108_13191_amd.expert_layer import ExpertLayer
from test_gpu_expert_layer import off

pytestmark = pytest.mark.gpu
SIZES = [(1, 256, 136, 4, 2), (37, 264, 200, 8, 3), (300, 128, 384, 16, 2), (64, 1024, 256, 1, 1), (1500, 256, 128, 6, 2)]
DTYPES = pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])


def definition(layer, x, r, route, p):
    """h and out in 64 bits with the layer's own choice of experts."""
    h = x + r
    h = h + (h.detach().to(layer.dtype).double() - h.detach())          # h is rounded as it is stored
    if layer.norm == "layer":
        y = torch.nn.functional.layer_norm(h, (layer.hidden,), p["gamma"], p["beta"], layer.eps)
    else:
        y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + layer.eps) * p["gamma"]

    def expert(rows, up, down):
        g, v = (rows @ up).chunk(2, dim=-1)
        return (torch.nn.functional.silu(g) * v) @ down
    out = expert(y, p["shared_up"][0], p["shared_down"][0])
    for e in range(layer.experts):
        weight = torch.where(route.expert == e, route.weight, torch.zeros_like(route.weight)).sum(1)
        t = (route.expert == e).any(1).nonzero().flatten()
        if t.numel():
            out = out.index_add(0, t, weight[t, None] * expert(y[t], p["up"][e], p["down"][e]))
    return h, out


def setup(tokens, hidden, ffn, experts, top_k, dtype, norm, grad=False):
    layer = ExpertLayer(hidden, ffn, experts, top_k, dtype=dtype, seed=3, norm=norm)
    gen = torch.Generator().manual_seed(5)
    given = [torch.randn(tokens, hidden, generator=gen).to(dtype) for _ in range(4)]
    names = ("gamma", "up", "down", "shared_up", "shared_down") + (("beta",) if norm == "layer" else ())
    return layer, given, {n: getattr(layer, n).cpu().double().requires_grad_(grad) for n in names}


@pytest.mark.parametrize("tokens,hidden,ffn,experts,top_k", SIZES)
@DTYPES
@pytest.mark.parametrize("norm,form", [("rms", "i8"), ("layer", "i8"), ("layer", "e4m3")])
def test_serve(tokens, hidden, ffn, experts, top_k, dtype, norm, form):
    layer, (x, r, _, _), params = setup(tokens, hidden, ffn, experts, top_k, dtype, norm)
    layer.prepare(form)
    got = layer.serve(x.cuda(), r.cuda())
    route = got.route
    route.expert, route.weight = route.expert.cpu(), route.weight.cpu().double()
    h, out = definition(layer, x.double(), r.double(), route, params)
    assert torch.equal(got.h.cpu().double(), h)
    # Four matrices in 8 bits reach the result, those of the first product (y, W_up) by up to twice.  Integers: the rounding's norm is (largest / rms) / 127 / sqrt(12)
    # of the matrix', the largest at most 4.5 times the rms of a normal row and 12 times a SwiGLU's: sqrt(8 * 0.0102^2 + 0.0273^2 + 0.0102^2) = 0.041.  e4m3: 0.036
    # each, sqrt(10) * 0.036 = 0.11.  And at most ten roundings to 16 bits of half a unit
    assert off(got.out, out) <= (0.041 if form == "i8" else 0.11) + 10 * (2.0 ** -9 if dtype == torch.bfloat16 else 2.0 ** -12)


@pytest.mark.parametrize("tokens,hidden,ffn,experts,top_k", SIZES)
@DTYPES
def test_training_with_a_layer_norm(tokens, hidden, ffn, experts, top_k, dtype):
    layer, (x, r, dout, dh), params = setup(tokens, hidden, ffn, experts, top_k, dtype, "layer", grad=True)
    s = layer.train_forward(x.cuda(), r.cuda())
    d = layer.backward(s, dout.cuda(), dh.cuda())
    route = s.route
    route.expert, route.weight = route.expert.cpu(), route.weight.cpu().double().requires_grad_()
    x64, r64 = x.double().requires_grad_(), r.double().requires_grad_()
    h, out = definition(layer, x64, r64, route, params)
    (h * dh.double()).sum().add((out * dout.double()).sum()).backward()
    bound = 10 * (2.0 ** -9 if dtype == torch.bfloat16 else 2.0 ** -12)          # at most ten roundings of half a unit, as above
    assert torch.equal(s.h.cpu().double(), h.detach())
    assert off(s.out, out) <= bound and off(d.x, x64.grad) <= bound and off(d.weight, route.weight.grad) <= bound
    for name, p in params.items():
        assert off(getattr(d, name), p.grad) <= bound, name


@pytest.mark.parametrize("tokens,experts,top_k", [(1, 4, 2), (37, 8, 2), (700, 16, 2), (3000, 8, 1)])
@pytest.mark.parametrize("norm,form", [("rms", "e4m3"), ("layer", "i8")])
def test_rows_moved_by_torch_give_the_same_bits(tokens, experts, top_k, norm, form, monkeypatch):
    """Orders are equal, and up to two rows a token have one order of addition; dots of rows (the routing weights' gradients) have another."""
    layer, given, _ = setup(tokens, 264, 136, experts, top_k, torch.bfloat16, norm)
    layer.prepare(form)
    x, r, dout, dh = (t.cuda() for t in given)

    def run():
        served, s = layer.serve(x, r), layer.train_forward(x, r)
        return served, s, layer.backward(s, dout, dh)
    got = run()
    monkeypatch.setattr(expert_layer, "_on_gpu", lambda t: False)
    want = run()
    for n in ("expert", "weight", "source", "place", "offsets"):
        assert torch.equal(getattr(got[0].route, n).long() if n != "weight" else got[0].route.weight, getattr(want[0].route, n).long() if n != "weight" else want[0].route.weight), n
    for g, w, names in ((got[0], want[0], ("h", "out")), (got[1], want[1], ("h", "y", "a", "d", "out")), (got[2], want[2], ("x", "gamma", "up", "down", "shared_up", "shared_down"))):
        for n in names:
            assert torch.equal(getattr(g, n), getattr(w, n)), n
    # sums of 264 products in f32, in any order
    magnitude = (got[1].d[got[1].route.place.long()].view(tokens, top_k, -1).float().abs() * dout[:, None].float().abs()).sum(-1)
    assert bool(((got[2].weight - want[2].weight).abs() <= 2 * 264 * 2.0 ** -24 * magnitude).all())


@pytest.mark.parametrize("form", ["e4m3", "i8"])
def test_a_router_of_the_callers_own(form):
    """One that sends every token to its first choice's expert and the next one, with 64-bit orders."""
    layer, given, params = setup(50, 264, 136, 5, 2, torch.bfloat16, "rms")
    layer.prepare(form)
    x, r, dout, dh = (t.cuda() for t in given)
    own = layer.route

    def route(y):
        first = own(y).expert[:, :1]
        expert = torch.cat([first, (first + 1) % 5], 1)
        by = expert.flatten().argsort(stable=True)
        place = torch.empty_like(by)
        place[by] = torch.arange(by.numel(), device=by.device)
        offsets = torch.searchsorted(expert.flatten()[by], torch.arange(6, device=by.device)).to(torch.int32)
        return SimpleNamespace(weight=torch.full((50, 2), 0.5, dtype=torch.float64, device="cuda"), expert=expert, source=by // 2, place=place, offsets=offsets)
    layer.route = route
    got, s = layer.serve(x, r), layer.train_forward(x, r)
    d = layer.backward(s, dout, dh)
    given_route = SimpleNamespace(expert=got.route.expert.cpu(), weight=got.route.weight.cpu().double())
    h, out = definition(layer, given[0].double(), given[1].double(), given_route, params)
    assert off(got.out, out) <= (0.041 if form == "i8" else 0.11) + 10 * 2.0 ** -9 and off(s.out, out) <= 10 * 2.0 ** -9
    assert d.weight.shape == (50, 2)


@pytest.mark.parametrize("norm,form", [("rms", "e4m3"), ("rms", "i8"), ("layer", "i8"), ("layer", "e4m3")])
def test_no_token(norm, form):
    layer, _, _ = setup(1, 264, 136, 4, 2, torch.bfloat16, norm)
    layer.prepare(form)
    none = torch.empty(0, 264, dtype=torch.bfloat16, device="cuda")
    assert layer.serve(none, none).out.shape == (0, 264)
    s = layer.train_forward(none, none)
    d = layer.train_backward(s, none, none)
    assert d.x.shape == (0, 264) and not d.up.any() and not d.gamma.any() and not s.route.offsets.any()


@pytest.mark.parametrize("norm,form", [("layer", "i8"), ("layer", "e4m3")])
def test_on_a_stream_of_its_own(norm, form):
    """Nothing is launched on another stream than the current one: work queued there in front of the layer is waited for."""
    layer, given, _ = setup(200, 256, 128, 8, 2, torch.bfloat16, norm)
    layer.prepare(form)
    args = [t.cuda() for t in given]
    want, s = layer.serve(args[0], args[1]), layer.train_forward(args[0], args[1])
    grads = vars(layer.train_backward(s, args[2], args[3]))
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        late = [torch.zeros_like(t) for t in args]
        busy = torch.randn(4096, 4096, device="cuda")
        for _ in range(8):
            busy = busy @ busy * 1e-2
        for t, a in zip(late, args):
            t.copy_(a)
        got, s2 = layer.serve(late[0], late[1]), layer.train_forward(late[0], late[1])
        again = vars(layer.train_backward(s2, late[2], late[3]))
    stream.synchronize()
    assert torch.equal(got.out, want.out) and torch.equal(s2.out, s.out)
    for name in grads:
        assert torch.equal(grads[name], again[name]), name
