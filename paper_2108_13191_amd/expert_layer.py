"""A feed-forward block with experts, built from the operators of include/gemm_ops.h: how they are called one after another.

    h = x + r,  y = rms_norm(h) * gamma
    out[t] = swiglu(y[t] W_up) W_down  of a shared expert  +  sum over the top_k experts e of token t:  weight[t, e] * (the same with W_up[e], W_down[e])

`serve` runs it in e4m3: the norm writes y quantised, the experts' products read it, SwiGLU writes its result quantised for the second
products.  `train_forward` and `train_backward` run it in 16 bits.  What is left to torch: the router's small product and
selection, moving rows into the experts' order and back, and SwiGLU in 16 bits.  Memory comes from torch; nothing synchronises with the host.

    python -m paper_2108_13191_amd.expert_layer --tokens 4096 --hidden 4096 --ffn 2048 --experts 8 --top-k 2
"""
from __future__ import annotations

import argparse
from types import SimpleNamespace

import torch

from . import binding
from .binding import check

TYPES = {torch.float16: binding.TYPE_F16, torch.bfloat16: binding.TYPE_BF16, torch.float32: binding.TYPE_F32}
E4M3 = torch.float8_e4m3fn


def _blocks(n):
    return (n + 127) // 128


def _stream(t):
    """The current stream, for kernels that take `t` and others beside it: memory of the current GPU."""
    if t.device.type != "cuda" or t.device.index != torch.cuda.current_device():
        raise ValueError(f"tensors of the current GPU expected, got one on {t.device}")
    return torch.cuda.current_stream().cuda_stream


def _pitch(t):
    """Elements from one row to the next (of a single row torch keeps any number)."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _e4m3(*shape, device):
    """Rows 16 bytes apart or a multiple of that, as the fast products read them (others take element loads: 4096 tokens with a hidden width of 4104 12.2 ms
    instead of 0.9)."""
    return torch.empty(*shape[:-1], (shape[-1] + 15) // 16 * 16, dtype=E4M3, device=device)[..., :shape[-1]]


def quantize_weights(w):
    """w (E x N x K or N x K) -> e4m3 of the same shape, scales E x ceil(N / 128) x ceil(K / 128)."""
    N, K = w.shape[-2:]
    w = w if w.stride(-1) == 1 and w.stride(-2) >= K else w.contiguous()
    q = _e4m3(*w.shape, device=w.device)
    scale = torch.empty(*w.shape[:-2], _blocks(N), _blocks(K), dtype=torch.float32, device=w.device)
    for m, qm, sm in zip(w.reshape(-1, N, K), q.view(-1, N, K), scale.view(-1, _blocks(N), _blocks(K))):
        check(binding.quantize_e4m3_blocks(N, K, TYPES[w.dtype], m, _pitch(m), qm, qm.stride(0), sm, _blocks(K), _stream(m)))
    return SimpleNamespace(q=q, scale=scale)


def swiglu(u):
    g, v = u.float().chunk(2, dim=-1)
    return (torch.nn.functional.silu(g) * v).to(u.dtype)


class ExpertLayer:
    """Weights as products read them: K x N (gemm_grouped) for training; N x K in e4m3 for serving, laid out once by `prepare`."""

    def __init__(self, hidden, ffn, experts, top_k, dtype=torch.bfloat16, eps=1e-5, seed=0, device="cuda", exact=False):
        """exact: e4m3 products exact however many tokens there are, at half the rate (binding.EXACT)."""
        if hidden % 8 or ffn % 8 or not 1 <= top_k <= experts:
            raise ValueError("hidden and ffn are multiples of 8, top_k at most the number of experts")
        self.hidden, self.ffn, self.experts, self.top_k, self.dtype, self.eps = hidden, ffn, experts, top_k, dtype, eps
        self.exact = binding.EXACT if exact else 0
        gen = torch.Generator(device=device).manual_seed(seed)

        def random(*shape, scale):
            return (torch.randn(*shape, generator=gen, device=device) * scale).to(dtype)
        self._shapes = {"gamma": (hidden,), "router": (hidden, experts), "up": (experts, hidden, 2 * ffn), "down": (experts, ffn, hidden), "shared_up": (1, hidden, 2 * ffn), "shared_down": (1, ffn, hidden)}
        self.gamma = (1.0 + 0.1 * torch.randn(hidden, generator=gen, device=device)).to(dtype)
        self.router = random(hidden, experts, scale=hidden ** -0.5)
        for name in ("up", "down", "shared_up", "shared_down"):
            shape = self._shapes[name]
            setattr(self, name, random(*shape, scale=shape[1] ** -0.5))

    def prepare(self):
        """The weights in e4m3, a row for each output."""
        self.quantized = SimpleNamespace(**{name: quantize_weights(getattr(self, name).transpose(1, 2).contiguous()) for name in ("up", "down", "shared_up", "shared_down")})

    def route(self, y):
        """The top_k experts of each token: `source`, the token of each of the tokens * top_k rows in the experts' order; `place`, where
        row j of token t went; `offsets`, the rows of each expert, and the weights."""
        weight, expert = torch.softmax((y @ self.router).float(), dim=-1).topk(self.top_k, dim=-1)
        order = expert.flatten().argsort(stable=True)
        place = torch.empty_like(order)
        place[order] = torch.arange(order.numel(), device=order.device)
        bounds = torch.arange(self.experts + 1, device=order.device)
        offsets = torch.searchsorted(expert.flatten()[order], bounds).to(torch.int32)
        return SimpleNamespace(weight=weight / weight.sum(-1, keepdim=True), expert=expert, source=order // self.top_k, place=place, offsets=offsets)

    def _combine(self, rows, route):
        """Sum over each token's rows, in a fixed order, f32."""
        return (rows[route.place].float().view(-1, self.top_k, rows.shape[1]) * route.weight[..., None]).sum(1)

    def _rows(self, name, t, tokens):
        """A caller's matrix as the kernels take it, which see an address, a pitch and the layer's type.  Rows of any pitch are taken
        as they lie; a copy is made where a row's elements are apart or rows overlap (an expanded gradient)."""
        if tuple(t.shape) != (tokens, self.hidden) or t.dtype != self.dtype or t.device != self.gamma.device:
            raise ValueError(f"{name}: {tokens} x {self.hidden} of {self.dtype} on {self.gamma.device} expected, got {tuple(t.shape)} of {t.dtype} on {t.device}")
        return t if t.stride(1) == 1 and _pitch(t) >= self.hidden else t.contiguous()

    def _check_weights(self, *names):
        """They may have been replaced: the kernels read them as the constructor lays them out."""
        for name in names:
            w = getattr(self, name)
            if tuple(w.shape) != self._shapes[name] or w.dtype != self.dtype or w.device != self.gamma.device or not w.is_contiguous():
                raise ValueError(f"{name}: {self._shapes[name]} of {self.dtype}, contiguous, on {self.gamma.device} expected")

    def _norm(self, x, r, quantized):
        self._check_weights("gamma")
        T, H = x.shape[0], self.hidden
        x, r = self._rows("x", x, T), self._rows("r", r, T)
        n = SimpleNamespace(h=torch.empty(T, H, dtype=x.dtype, device=x.device), y=torch.empty(T, H, dtype=x.dtype, device=x.device), rstd=torch.empty(T, dtype=torch.float32, device=x.device), q=None, scale=None)
        if quantized:
            n.q = _e4m3(T, H, device=x.device)
            n.scale = torch.empty(_blocks(H), T, dtype=torch.float32, device=x.device)
        check(binding.rms_norm(T, H, TYPES[x.dtype], x, _pitch(x), r, _pitch(r), self.gamma, self.eps, n.h, H, n.y, H, n.q, n.q.stride(0) if quantized else 0, n.scale, T, n.rstd, _stream(x)))
        return n

    def _product8(self, q, scale, w, offsets=None):
        rows, K = q.shape
        E, N = w.q.shape[:2]
        c = torch.empty(rows, N, dtype=self.dtype, device=q.device)
        if offsets is None:
            check(binding.gemm_e4m3_block(rows, N, K, q, q.stride(0), scale, rows, w.q, w.q.stride(1), w.scale, _blocks(K), c, N, TYPES[c.dtype] | self.exact, _stream(c)))
        else:
            check(binding.gemm_e4m3_block_grouped(rows, N, K, E, offsets, q, q.stride(0), scale, rows, w.q, w.q.stride(1), w.q.stride(0), w.scale, _blocks(K), w.scale.stride(0), c, N, TYPES[c.dtype] | self.exact, _stream(c)))
        return c

    def _swiglu8(self, u):
        rows, N = u.shape[0], u.shape[1] // 2
        q = _e4m3(rows, N, device=u.device)
        scale = torch.empty(_blocks(N), rows, dtype=torch.float32, device=u.device)
        check(binding.quantize_e4m3_rows(rows, N, TYPES[u.dtype], binding.ACT_SWIGLU, u, 2 * N, q, q.stride(0), scale, rows, _stream(u)))
        return q, scale

    def serve(self, x, r):
        """h and out of x and the residual r (tokens x hidden)."""
        w, n = self.quantized, self._norm(x, r, quantized=True)
        route = self.route(n.y)
        rows = _e4m3(route.source.numel(), self.hidden, device=x.device)
        rows.view(torch.uint8).copy_(n.q.view(torch.uint8)[route.source])
        up = self._product8(rows, n.scale[:, route.source].contiguous(), w.up, route.offsets)
        out = self._product8(*self._swiglu8(up), w.down, route.offsets)
        shared = self._product8(*self._swiglu8(self._product8(n.q, n.scale, w.shared_up)), w.shared_down)
        return SimpleNamespace(h=n.h, out=(self._combine(out, route) + shared.float()).to(self.dtype), route=route)

    def _product(self, a, w, offsets):
        (rows, K), (E, _, N) = a.shape, w.shape
        c = torch.empty(rows, N, dtype=a.dtype, device=a.device)
        check(binding.gemm_grouped(rows, N, K, E, offsets, TYPES[a.dtype], a, K, w, N, K * N, c, N, TYPES[c.dtype], _stream(c)))
        return c

    def _product_backward(self, a, w, dc, offsets):
        """Gradients of a (its type) and of w (f32, as an optimizer adds them up)."""
        (rows, K), (E, _, N) = a.shape, w.shape
        da, dw = torch.empty_like(a), torch.empty(w.shape, dtype=torch.float32, device=w.device)
        check(binding.gemm_grouped_grad_a(rows, N, K, E, offsets, TYPES[a.dtype], dc, _pitch(dc), w, N, K * N, da, K, TYPES[a.dtype], _stream(a)))
        check(binding.gemm_grouped_grad_b(rows, N, K, E, offsets, TYPES[a.dtype], a, K, dc, _pitch(dc), dw, N, K * N, TYPES[dw.dtype], _stream(a)))
        return da, dw

    def train_forward(self, x, r):
        """h, out and what `backward` needs."""
        self._check_weights(*self._shapes)
        s = self._norm(x, r, quantized=False)
        s.route = self.route(s.y)
        s.all = torch.arange(2, dtype=torch.int32, device=x.device) * x.shape[0]      # the shared expert: one group
        s.a, s.shared_a = s.y[s.route.source], s.y
        s.u, s.shared_u = self._product(s.a, self.up, s.route.offsets), self._product(s.shared_a, self.shared_up, s.all)
        s.s, s.shared_s = swiglu(s.u), swiglu(s.shared_u)
        s.d, shared = self._product(s.s, self.down, s.route.offsets), self._product(s.shared_s, self.shared_down, s.all)
        s.out = (self._combine(s.d, s.route) + shared.float()).to(self.dtype)
        return s

    def train_backward(self, s, dout, dh):
        """From the gradients of out and h: of x (and of r), gamma, the router, the experts' and the shared weights; and of the routing weights."""
        return self._backward(s, dout, dh, through_router=True)

    def backward(self, s, dout, dh):
        """The same with the routing weights held, as a router of the caller's own needs it: x and gamma without what reaches them through the
        weights, whose gradient is `weight`; none of the router."""
        return self._backward(s, dout, dh, through_router=False)

    def _backward(self, s, dout, dh, through_router):
        def expert(a, u, sw, up, down, dd, offsets):
            ds, ddown = self._product_backward(sw, down, dd, offsets)
            (g, v), d = u.float().chunk(2, dim=-1), ds.float()
            sig = torch.sigmoid(g)
            du = torch.cat([d * v * sig * (1.0 + g * (1.0 - sig)), d * g * sig], dim=-1).to(u.dtype)
            da, dup = self._product_backward(a, up, du, offsets)
            return da, dup, ddown
        self._check_weights(*self._shapes)
        route, tokens = s.route, s.h.shape[0]
        dout, dh = self._rows("dout", dout, tokens), self._rows("dh", dh, tokens)
        dweight = (s.d[route.place].view(-1, self.top_k, self.hidden).float() * dout[:, None].float()).sum(-1)
        weight = torch.empty(route.place.numel(), dtype=torch.float32, device=dout.device)
        weight[route.place] = route.weight.flatten()
        da, dup, ddown = expert(s.a, s.u, s.s, self.up, self.down, (dout[route.source].float() * weight[:, None]).to(self.dtype), route.offsets)
        dy, dshared_up, dshared_down = expert(s.shared_a, s.shared_u, s.shared_s, self.shared_up, self.shared_down, dout, s.all)
        dy, router = dy.float() + da[route.place].view(-1, self.top_k, self.hidden).float().sum(1), {}
        if through_router:
            # top-k of a softmax, divided by their sum: the softmax of the chosen logits alone.  dlogit = weight (dweight - sum(weight dweight)); others' are 0
            dchosen = route.weight * (dweight - (route.weight * dweight).sum(-1, keepdim=True))
            dlogits = torch.zeros(tokens, self.experts, device=dy.device).scatter_(1, route.expert, dchosen)
            dy, router = dy + dlogits @ self.router.float().t(), {"router": s.y.float().t() @ dlogits}
        dy = dy.to(self.dtype)
        T, H = dy.shape
        dx, dgamma = torch.empty_like(dy), torch.empty(H, dtype=torch.float32, device=dy.device)
        size = binding.rms_norm_grad_workspace_bytes(T, H)
        workspace = torch.empty(size, dtype=torch.uint8, device=dy.device)
        check(binding.rms_norm_grad(T, H, TYPES[dy.dtype], dy, H, s.h, H, self.gamma, s.rstd, dh, _pitch(dh), dx, H, dgamma, workspace, size, _stream(dy)))
        return SimpleNamespace(x=dx, gamma=dgamma, up=dup, down=ddown, shared_up=dshared_up, shared_down=dshared_down, weight=dweight, **router)


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("tokens", 4096), ("hidden", 4096), ("ffn", 2048), ("experts", 8), ("top-k", 2), ("steps", 10)):
        p.add_argument(f"--{name}", type=int, default=value)
    a = p.parse_args(argv)
    layer = ExpertLayer(a.hidden, a.ffn, a.experts, a.top_k)
    layer.prepare()
    x, r, dout, dh = (torch.randn(a.tokens, a.hidden, device="cuda").to(layer.dtype) for _ in range(4))

    def time(f):
        for _ in range(3):
            f()
        torch.cuda.synchronize()
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        for _ in range(a.steps):
            f()
        end.record()
        end.synchronize()
        return begin.elapsed_time(end) / a.steps
    products = 6.0 * a.tokens * (a.top_k + 1) * a.hidden * a.ffn
    forward, both = time(lambda: layer.serve(x, r)), time(lambda: layer.train_backward(layer.train_forward(x, r), dout, dh))
    print(f"{a.tokens} tokens, hidden {a.hidden}, ffn {a.ffn}, top {a.top_k} of {a.experts} experts and a shared one")
    print(f"serve, e4m3:               {forward:8.3f} ms, {products / forward * 1e-9:7.1f} TFLOP/s in the products")
    print(f"train, bf16, both ways:    {both:8.3f} ms, {3 * products / both * 1e-9:7.1f} TFLOP/s in the products")
    got, want = layer.serve(x, r).out.float(), layer.train_forward(x, r).out.float()
    print(f"e4m3 against bf16:         {((got - want).norm() / want.norm()).item():8.4f} of the result's norm")


if __name__ == "__main__":
    main()
