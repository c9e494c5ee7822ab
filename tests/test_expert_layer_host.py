"""What paper_2108_13191_amd/expert_layer.py hands to the kernels, on the host, where each operand is read by its address, pitch and type: callers' matrices
of other layouts give what contiguous copies of them give, and other types, shapes and places are refused."""
import pytest
import torch

import ops_emulation
from paper_2108_13191_amd import binding, expert_layer

T, H, F, E, TOP = 13, 264, 136, 4, 2


@pytest.fixture
def layer(monkeypatch):
    for f in ops_emulation.ENTRY_POINTS:
        monkeypatch.setattr(binding, f.__name__, f)
    monkeypatch.setattr(expert_layer, "_stream", lambda *t: 0)
    made = expert_layer.ExpertLayer(H, F, E, TOP, seed=1, device="cpu")
    made.prepare()
    return made


def inputs(tokens=T):
    gen = torch.Generator().manual_seed(2)
    return [torch.randn(tokens, H, generator=gen).bfloat16() for _ in range(4)]


def columns(t):
    """The same values as columns of a wider matrix, whose other columns are NaN."""
    wide = torch.full((t.shape[0], H + 40), float("nan"), dtype=t.dtype)
    wide[:, 16:16 + H] = t
    return wide[:, 16:16 + H]


def last(t):
    """... as the last columns of a matrix, behind which nothing follows."""
    wide = torch.full((t.shape[0], 2 * H), float("nan"), dtype=t.dtype)
    wide[:, H:] = t
    return wide[:, H:]


def transposed(t):
    return t.t().contiguous().t()


def every_other(t):
    return torch.stack([t, torch.full_like(t, float("nan"))], 2)[:, :, 0]


def same(a, b):
    a, b = vars(a), vars(b)
    assert a.keys() == b.keys()
    return all(torch.equal(a[n], b[n]) if isinstance(a[n], torch.Tensor) else n == "route" and same(a[n], b[n]) for n in a if a[n] is not None)


@pytest.mark.parametrize("lay", [columns, last, transposed, every_other])
@pytest.mark.parametrize("tokens", [1, T])
def test_matrices_of_any_layout(layer, lay, tokens):
    x, r, dout, dh = inputs(tokens)
    served, s = layer.serve(x, r), layer.train_forward(x, r)
    grads = layer.backward(s, dout, dh)
    x, r, dout, dh = map(lay, (x, r, dout, dh))
    assert same(layer.serve(x, r), served)
    s2 = layer.train_forward(x, r)
    assert same(s2, s) and same(layer.backward(s2, dout, dh), grads)


@pytest.mark.parametrize("shape", [(1, 1), (1, H), (T, 1)])
def test_expanded_gradients(layer, shape):
    """As the gradient of a sum comes: one element or row in place of all of them."""
    x, r, _, _ = inputs()
    s = layer.train_forward(x, r)
    d = torch.randn(shape, generator=torch.Generator().manual_seed(3)).bfloat16().expand(T, H)
    assert same(layer.backward(s, d, d), layer.backward(s, d.contiguous(), d.contiguous()))


def test_other_types_shapes_and_places_are_refused(layer):
    x, r, dout, dh = inputs()
    s = layer.train_forward(x, r)
    for bad in (lambda t: t.float(), lambda t: t.half(), lambda t: t[:, :-8], lambda t: t[None], lambda t: t.to("meta")):
        for call in (lambda b: layer.serve(b(x), r), lambda b: layer.serve(x, b(r)), lambda b: layer.train_forward(b(x), r), lambda b: layer.train_forward(x, b(r)),
                     lambda b: layer.backward(s, b(dout), dh), lambda b: layer.backward(s, dout, b(dh))):
            with pytest.raises(ValueError):
                call(bad)
    for call in (lambda: layer.serve(x, r[1:]), lambda: layer.backward(s, dout[1:], dh), lambda: layer.backward(s, dout, dh[1:])):
        with pytest.raises(ValueError):
            call()


def test_host_memory_is_no_operand():
    """Nothing is launched on tensors that no kernel could read."""
    made = expert_layer.ExpertLayer(H, F, E, TOP, device="cpu")
    x, r, _, _ = inputs()
    for call in (lambda: made.train_forward(x, r), made.prepare):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("lay", [lambda w: w, lambda w: w.transpose(-1, -2).contiguous().transpose(-1, -2), lambda w: w.expand(3, *w.shape[-2:]),
                                 lambda w: torch.cat([w, w], -1)[..., :w.shape[-1]]], ids=["contiguous", "transposed", "expanded", "columns"])
def test_weights_of_any_layout_are_quantised(layer, lay):
    w = lay(torch.randn(1, 136, 264, generator=torch.Generator().manual_seed(4)).bfloat16())
    got, want = expert_layer.quantize_weights(w), expert_layer.quantize_weights(w.clone(memory_format=torch.contiguous_format))
    assert torch.equal(got.q.view(torch.uint8), want.q.view(torch.uint8)) and torch.equal(got.scale, want.scale)
    assert torch.equal(expert_layer.quantize_weights(w[0]).scale, want.scale[0])


@pytest.mark.parametrize("name", ["up", "down", "shared_up", "shared_down", "gamma"])
def test_weights_that_are_no_weights_are_refused(layer, name):
    """A weight that was replaced by one of another type, shape or layout than products read."""
    x, r, dout, dh = inputs()
    s, good = layer.train_forward(x, r), getattr(layer, name)
    for bad in (good.float(), good[..., :-8], torch.stack([good, good], -1)[..., 0]):
        setattr(layer, name, bad)
        for call in (lambda: layer.train_forward(x, r), lambda: layer.backward(s, dout, dh)):
            with pytest.raises(ValueError):
                call()
    setattr(layer, name, good)
    layer.backward(layer.train_forward(x, r), dout, dh)


@pytest.mark.parametrize("lay", [columns, transposed])
def test_the_whole_derivative_adds_what_the_router_carries(layer, lay):
    x, r, dout, dh = inputs()
    s = layer.train_forward(x, r)
    held, whole = layer.backward(s, dout, dh), layer.train_backward(s, lay(dout), lay(dh))
    for name in ("up", "down", "shared_up", "shared_down", "weight"):
        assert torch.equal(getattr(held, name), getattr(whole, name)), name
    assert not hasattr(held, "router") and whole.router.shape == layer.router.shape and whole.router.dtype == torch.float32
    assert not torch.equal(held.x, whole.x) and not torch.equal(held.gamma, whole.gamma)
    # a shift of a token's logits changes nothing: the gradient of a token's logits sums to 0
    assert (whole.router.sum(1).abs() <= 1e-4 * whole.router.abs().sum(1)).all()


@pytest.mark.parametrize("hidden,ffn", [(264, 136), (256, 136), (264, 128), (256, 128), (8, 8)])
def test_e4m3_rows_begin_at_multiples_of_16(layer, monkeypatch, hidden, ffn):
    """Whatever the widths: the products' fast kernels need it of addresses, pitches and the experts' strides."""
    calls = []

    def watch(f):
        def g(*args):
            names = dict(zip(f.__code__.co_varnames, args))
            calls.append(f.__name__)
            for t in "AB":
                assert names["ld" + t.lower()] % 16 == 0 and names[t].data_ptr() % 16 == 0 and names.get("b_stride", 0) % 16 == 0
            return f(*args)
        return g
    for f in (ops_emulation.gemm_e4m3_block, ops_emulation.gemm_e4m3_block_grouped):
        monkeypatch.setattr(binding, f.__name__, watch(f))
    made = expert_layer.ExpertLayer(hidden, ffn, E, TOP, seed=1, device="cpu")
    made.prepare()
    made.serve(*(torch.randn(T, hidden).bfloat16() for _ in range(2)))
    assert calls.count("gemm_e4m3_block") == 2 and calls.count("gemm_e4m3_block_grouped") == 2


@pytest.mark.parametrize("exact", [False, True])
def test_exact_products_where_the_layer_asks_for_them(layer, monkeypatch, exact):
    types = []
    for f in (ops_emulation.gemm_e4m3_block, ops_emulation.gemm_e4m3_block_grouped):
        monkeypatch.setattr(binding, f.__name__, lambda *args, f=f: (types.append(args[-2]), f(*args))[1])
    made = expert_layer.ExpertLayer(H, F, E, TOP, seed=1, device="cpu", exact=exact)
    made.prepare()
    x, r, _, _ = inputs()
    assert same(made.serve(x, r), layer.serve(x, r))          # (which has no sums that could be cut off here)
    assert types[:4] == [binding.TYPE_BF16 | (binding.EXACT if exact else 0)] * 4
