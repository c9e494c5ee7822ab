"""expert_layer.py with a layer norm and with weights of 8-bit integers, on the host: what it hands to the entry points, which read each operand by its
address, pitch and type."""
from types import SimpleNamespace

import pytest
import torch

import layer_emulation
import ops_emulation
from paper_2108_13191_amd import binding, expert_layer
from test_expert_layer_host import E, F, H, T, TOP, columns, inputs, same, transposed

FORMS = [("rms", "i8"), ("layer", "i8"), ("layer", "e4m3")]


@pytest.fixture(params=FORMS, ids=["-".join(f) for f in FORMS])
def layer(request, monkeypatch):
    for f in ops_emulation.ENTRY_POINTS + layer_emulation.ENTRY_POINTS:
        monkeypatch.setattr(binding, f.__name__, f)
    monkeypatch.setattr(expert_layer, "_stream", lambda *t: 0)
    made = expert_layer.ExpertLayer(H, F, E, TOP, seed=1, device="cpu", norm=request.param[0])
    made.prepare(request.param[1])
    return made


@pytest.mark.parametrize("lay", [columns, transposed])
@pytest.mark.parametrize("tokens", [1, T])
def test_matrices_of_any_layout(layer, lay, tokens):
    x, r, dout, dh = inputs(tokens)
    served, s = layer.serve(x, r), layer.train_forward(x, r)
    grads = layer.train_backward(s, dout, dh)
    x, r, dout, dh = map(lay, (x, r, dout, dh))
    assert same(layer.serve(x, r), served)
    s2 = layer.train_forward(x, r)
    assert same(s2, s) and same(layer.train_backward(s2, dout, dh), grads)


def test_serving_is_near_training(layer):
    """Four matrices in 8 bits reach the result, those of the first product twice.  Integers: the rounding's norm is (largest / rms) / 127 / sqrt(12) of the matrix',
    the largest at most 4.5 times the rms of a normal row and 12 times that of a SwiGLU's: sqrt(8 * 0.0102^2 + 0.0273^2 + 0.0102^2) = 0.041.  e4m3: 0.11.  And at
    most ten roundings to bf16 of half a unit in either."""
    x, r, _, _ = inputs()
    got, want = layer.serve(x, r).out.double(), layer.train_forward(x, r).out.double()
    assert (got - want).norm() <= ((0.041 if layer.format == "i8" else 0.11) + 10 * 2.0 ** -9) * want.norm()


def test_gradients_of_the_norm(layer):
    """Those of gamma, beta and x against the norm's derivative in 64 bits, from the gradient of its result."""
    x, r, dout, dh = inputs()
    s = layer.train_forward(x, r)
    seen = {}
    name = "layer_norm_grad" if layer.norm == "layer" else "rms_norm_grad"
    real = getattr(binding, name)

    def spy(M, N, type, dY, *rest):
        seen["dy"] = dY.clone()
        return real(M, N, type, dY, *rest)
    setattr(binding, name, spy)
    try:
        d = layer.train_backward(s, dout, dh)
    finally:
        setattr(binding, name, real)
    h, gamma = s.h.double().requires_grad_(), layer.gamma.double().requires_grad_()
    beta = layer.beta.double().requires_grad_() if layer.norm == "layer" else torch.zeros(H, dtype=torch.float64)
    y = (torch.nn.functional.layer_norm(h, (H,), gamma, beta, layer.eps) if layer.norm == "layer" else h * torch.rsqrt((h * h).mean(-1, keepdim=True) + layer.eps) * gamma)
    y.backward(seen["dy"].double())
    want = {"x": h.grad + dh.double(), "gamma": gamma.grad}
    if layer.norm == "layer":
        want["beta"] = beta.grad
        assert d.beta.dtype == torch.float32
    else:
        assert not hasattr(d, "beta")
    for n, w in want.items():
        assert (getattr(d, n).double() - w).norm() <= 2.0 ** -8 * w.norm(), n


def test_a_router_of_the_callers_own(layer):
    """route() replaced on the layer: rows move by its order, and the result is that of the layer's own where both choose alike."""
    x, r, dout, dh = inputs()
    want, s = layer.serve(x, r), layer.train_forward(x, r)
    grads = layer.train_backward(s, dout, dh)
    own, calls = layer.route, []

    def route(y):
        calls.append(1)
        given = own(y)
        return SimpleNamespace(**vars(given))
    layer.route = route
    assert same(layer.serve(x, r), want) and len(calls) == 1
    s2 = layer.train_forward(x, r)
    assert same(s2, s) and len(calls) == 2 and same(layer.train_backward(s2, dout, dh), grads)


def test_weights_of_any_layout_are_quantised(layer):
    w = torch.randn(3, 136, 264, generator=torch.Generator().manual_seed(4)).bfloat16()
    want = expert_layer.quantize_weights_i8(w)
    assert want.q.dtype == torch.int8 and want.scale.shape == (3, 136) and want.q.stride(1) % 16 == 0
    got = expert_layer.quantize_weights_i8(w.transpose(1, 2).contiguous().transpose(1, 2))
    assert torch.equal(got.q, want.q) and torch.equal(got.scale, want.scale)
    assert torch.equal(expert_layer.quantize_weights_i8(w[1]).q, want.q[1])


def test_refusals(layer):
    for bad in ("", "batch", None):
        with pytest.raises(ValueError):
            expert_layer.ExpertLayer(H, F, E, TOP, device="cpu", norm=bad)
        with pytest.raises(ValueError):
            layer.prepare(bad)
    if layer.norm == "layer":
        x, r, _, _ = inputs()
        layer.beta = layer.beta.float()
        for call in (layer.serve, layer.train_forward):
            with pytest.raises(ValueError):
                call(x, r)
