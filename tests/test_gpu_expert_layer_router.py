"""The whole derivative of the feed-forward block with experts, through the router too: the choice of experts held, their weights a function of y."""
import pytest
import torch

from test_gpu_expert_layer import SIZES, definition, off, setup

pytestmark = pytest.mark.gpu

# Roundings to 16 bits on the way to a result, half a unit in the last place each: ten as for the block with its weights held (test_gpu_expert_layer.py), and
# those of the routing weights -- y's and the logits', of magnitudes up to 3, are errors of up to 2 x 3 of them relative to a weight.
ROUNDINGS = 16


def loss(layer, x, r, dout, dh, route, params):
    """sum(out dout) + sum(h dh) in 64 bits with the routing weights that y gives for the experts chosen; and out."""
    h = x + r
    h = h + (h.detach().to(layer.dtype).double() - h.detach())
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + layer.eps) * params["gamma"]
    p = torch.softmax(y @ params["router"], -1).gather(1, route.expert)
    route.weight = p / p.sum(-1, keepdim=True)
    h, out = definition(layer, x, r, route, params)
    return (h * dh.double()).sum() + (out * dout.double()).sum(), out


@pytest.mark.parametrize("tokens,hidden,ffn,experts,top_k", SIZES + [(50, 128, 64, 8, 8)])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
def test_whole_derivative(tokens, hidden, ffn, experts, top_k, dtype):
    layer, x, r, dout, dh, params = setup(tokens, hidden, ffn, experts, top_k, dtype, grad=True)
    params["router"] = layer.router.cpu().double().requires_grad_()
    s = layer.train_forward(x.cuda(), r.cuda())
    d = layer.train_backward(s, dout.cuda(), dh.cuda())
    route = s.route
    route.expert = route.expert.cpu()
    x64, r64 = x.double().requires_grad_(), r.double().requires_grad_()
    total, out = loss(layer, x64, r64, dout, dh, route, params)
    total.backward()
    bound = ROUNDINGS * (2.0 ** -9 if dtype == torch.bfloat16 else 2.0 ** -12)
    assert off(s.out, out) <= bound and off(d.x, x64.grad) <= bound
    for name, p in params.items():
        if name == "router" and top_k == 1:
            assert not d.router.any()                       # one expert's weight is 1 whatever the router says
        else:
            assert off(getattr(d, name), p.grad) <= bound, name


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
def test_against_differences(dtype):
    """Central differences of the definition in 64 bits along random directions of x, gamma and the router."""
    layer, x, r, dout, dh, params = setup(19, 128, 64, 6, 2, dtype)
    params["router"] = layer.router.cpu().double()
    s = layer.train_forward(x.cuda(), r.cuda())
    d = layer.train_backward(s, dout.cuda(), dh.cuda())
    route, gen, step = s.route, torch.Generator().manual_seed(1), 1e-6
    route.expert = route.expert.cpu()
    bound = ROUNDINGS * (2.0 ** -9 if dtype == torch.bfloat16 else 2.0 ** -12)
    # h's rounding is held where it is, as its derivative is taken to be 1
    r64 = (x + r).double() - x.double()
    for name in ("x", "gamma", "router"):
        grad = getattr(d, name).cpu().double()
        for _ in range(4):
            v = torch.randn(grad.shape, generator=gen, dtype=torch.float64)
            ends = []
            for sign in (step, -step):
                p = dict(params)
                if name != "x":
                    p[name] = p[name] + sign * v
                ends.append(unrounded(layer, x.double() + (sign * v if name == "x" else 0.0), r64, dout, dh, route, p))
            assert abs((grad * v).sum() - (ends[0] - ends[1]) / (2 * step)) <= bound * grad.norm() * v.norm(), name


def unrounded(layer, x, r, dout, dh, route, params):
    h = x + r
    y = h * torch.rsqrt((h * h).mean(-1, keepdim=True) + layer.eps) * params["gamma"]
    p = torch.softmax(y @ params["router"], -1).gather(1, route.expert)
    weight, out = p / p.sum(-1, keepdim=True), torch.zeros_like(h)

    def expert(rows, up, down):
        g, v = (rows @ up).chunk(2, dim=-1)
        return (torch.nn.functional.silu(g) * v) @ down
    for t in range(h.shape[0]):
        out[t] = expert(y[t], params["shared_up"][0], params["shared_down"][0])
        for j, e in enumerate(route.expert[t].tolist()):
            out[t] += weight[t, j] * expert(y[t], params["up"][e], params["down"][e])
    return float((h * dh.double()).sum() + (out * dout.double()).sum())
