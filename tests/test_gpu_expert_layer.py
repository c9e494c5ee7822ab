"""The operators of include/gemm_ops.h one after another, as paper_2108_13191_amd/expert_layer.py calls them, against the block's
definition in 64 bits on the host."""
import pytest
import torch

from paper_2108_13191_amd.expert_layer import ExpertLayer

pytestmark = pytest.mark.gpu


def definition(layer, x, r, route, params):
    """h, y and out in 64 bits with the layer's own choice of experts; `params`: the weights in 64 bits."""
    h = (x + r)
    h = h + (h.detach().to(layer.dtype).double() - h.detach())          # h is rounded as it is stored
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + layer.eps) * params["gamma"]

    def expert(rows, up, down):
        g, v = (rows @ up).chunk(2, dim=-1)
        return (torch.nn.functional.silu(g) * v) @ down
    rows = []
    for t in range(x.shape[0]):
        o = expert(y[t], params["shared_up"][0], params["shared_down"][0])
        for j, e in enumerate(route.expert[t].tolist()):
            o = o + route.weight[t, j] * expert(y[t], params["up"][e], params["down"][e])
        rows.append(o)
    return h, torch.stack(rows)


def setup(tokens, hidden, ffn, experts, top_k, dtype, grad=False):
    layer = ExpertLayer(hidden, ffn, experts, top_k, dtype=dtype, seed=3)
    gen = torch.Generator().manual_seed(5)
    x, r, dout, dh = (torch.randn(tokens, hidden, generator=gen).to(dtype) for _ in range(4))
    params = {n: getattr(layer, n).cpu().double().requires_grad_(grad) for n in ("gamma", "up", "down", "shared_up", "shared_down")}
    return layer, x, r, dout, dh, params


def off(got, want):
    return ((got.detach().cpu().double() - want.detach()).norm() / want.detach().norm()).item()


SIZES = [(1, 256, 136, 4, 2), (37, 264, 200, 8, 3), (300, 128, 384, 16, 2), (64, 1024, 256, 1, 1)]


@pytest.mark.parametrize("tokens,hidden,ffn,experts,top_k", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
def test_serve(tokens, hidden, ffn, experts, top_k, dtype):
    layer, x, r, _, _, params = setup(tokens, hidden, ffn, experts, top_k, dtype)
    layer.prepare()
    got = layer.serve(x.cuda(), r.cuda())
    route = got.route
    route.expert, route.weight = route.expert.cpu(), route.weight.cpu().double()
    h, out = definition(layer, x.double(), r.double(), route, params)
    assert torch.equal(got.h.cpu().double(), h)
    # rounding to e4m3: at most 2^-4 of a value, 0.036 of a matrix' norm (evenly spread errors).  Four matrices' errors reach the result
    # (y, W_up, the SwiGLU, W_down), those of the first product by up to twice (gate and value): sqrt(4 + 4 + 1 + 1) * 0.036 = 0.11
    assert off(got.out, out) <= 0.11


@pytest.mark.parametrize("tokens,hidden,ffn,experts,top_k", SIZES)
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
def test_training(tokens, hidden, ffn, experts, top_k, dtype):
    layer, x, r, dout, dh, params = setup(tokens, hidden, ffn, experts, top_k, dtype, grad=True)
    s = layer.train_forward(x.cuda(), r.cuda())
    d = layer.backward(s, dout.cuda(), dh.cuda())
    route = s.route
    route.expert, route.weight = route.expert.cpu(), route.weight.cpu().double().requires_grad_()
    x64, r64 = x.double().requires_grad_(), r.double().requires_grad_()
    h, out = definition(layer, x64, r64, route, params)
    (h * dh.double()).sum().add((out * dout.double()).sum()).backward()
    # at most ten roundings to 16 bits from the inputs to any of these, each up to half a unit in the last place
    bound = 10 * (2.0 ** -9 if dtype == torch.bfloat16 else 2.0 ** -12)
    assert torch.equal(s.h.cpu().double(), h.detach())
    assert off(s.out, out) <= bound
    assert torch.equal(x64.grad, r64.grad) and off(d.x, x64.grad) <= bound
    assert off(d.weight, route.weight.grad) <= bound
    for name, p in params.items():
        assert off(getattr(d, name), p.grad) <= bound, name


def test_on_a_stream_of_its_own():
    """Nothing is launched on another stream than the current one: work queued there in front of the layer is waited for."""
    layer, x, r, dout, dh, _ = setup(200, 256, 128, 8, 2, torch.bfloat16)
    layer.prepare()
    args = [t.cuda() for t in (x, r, dout, dh)]
    want = layer.serve(args[0], args[1])
    s = layer.train_forward(args[0], args[1])
    grads = vars(layer.backward(s, args[2], args[3]))
    torch.cuda.synchronize()
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        late = [torch.zeros_like(t) for t in args]
        busy = torch.randn(4096, 4096, device="cuda")
        for _ in range(8):
            busy = busy @ busy * 1e-2
        for t, a in zip(late, args):
            t.copy_(a)
        got = layer.serve(late[0], late[1])
        s2 = layer.train_forward(late[0], late[1])
        again = vars(layer.backward(s2, late[2], late[3]))
    stream.synchronize()
    assert torch.equal(got.h, want.h) and torch.equal(got.out, want.out) and torch.equal(s2.out, s.out)
    for name in grads:
        assert torch.equal(grads[name], again[name]), name
