"""A feed-forward block with experts, built from the operators of include/gemm_ops.h and include/gemm_layer.h: how they are called one after another.

    h = x + r,  y = rms_norm(h) * gamma        (norm="layer": y = layer_norm(h) * gamma + beta)
    out[t] = swiglu(y[t] W_up) W_down  of a shared expert  +  sum over the top_k experts e of token t:  weight[t, e] * (the same with W_up[e], W_down[e])

`serve` runs it in 8 bits, e4m3 or integers as `prepare` laid the weights out: the norm writes y quantised, rows go to their experts, the experts' products read
them, SwiGLU writes its result quantised for the second products, and the way back adds up each token's rows and the shared expert's.  `train_forward`
and `train_backward` run it in 16 bits.  What is left to torch: the router's small product and selection, and SwiGLU in 16 bits.  Memory comes from torch; nothing
synchronises with the host.

    python -m paper_2108_13191_amd.expert_layer --tokens 4096 --hidden 4096 --ffn 2048 --experts 8 --top-k 2 --norm layer --format i8
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


def _bytes(*shape, dtype, device):
    """Rows 16 bytes apart or a multiple of that, as the fast products read them (others take element loads: 4096 tokens with a hidden width of 4104 12.2 ms
    instead of 0.9)."""
    return torch.empty(*shape[:-1], (shape[-1] + 15) // 16 * 16, dtype=dtype, device=device)[..., :shape[-1]]


def _e4m3(*shape, device):
    return _bytes(*shape, dtype=E4M3, device=device)


def _like(t, rows):
    """Room for as many rows as t has them."""
    return _bytes(rows, t.shape[1], dtype=t.dtype, device=t.device) if t.element_size() == 1 else torch.empty(rows, t.shape[1], dtype=t.dtype, device=t.device)


def _rows_of(source, rows, scale):
    """Rows and their scales in the order of `source`, by torch."""
    moved = _like(rows, source.numel())
    if rows.element_size() == 1:                       # torch has no indexing of e4m3
        moved.view(torch.uint8).copy_(rows.view(torch.uint8)[source])
    else:
        moved.copy_(rows[source])
    return moved, None if scale is None else scale[..., source].contiguous()


class _Route(SimpleNamespace):
    """A route that the layer has made itself: every row is some choice's."""


def _places(route, tokens, top_k, device):
    """The row of each choice (tokens x top_k), of which a router of the caller's own may have others than the kernels can read."""
    place = route.place
    if place.numel() != tokens * top_k or place.dtype == torch.bool or place.is_floating_point() or place.is_complex():
        raise ValueError(f"places of a route: {tokens} x {top_k} integers expected, got {tuple(place.shape)} of {place.dtype}")
    return place.reshape(tokens, top_k).to(device)


def _offsets(route, experts, device):
    """Where each expert's rows begin, as the products read it."""
    offsets = route.offsets
    if tuple(offsets.shape) != (experts + 1,) or offsets.dtype not in (torch.int32, torch.int64):
        raise ValueError(f"offsets of a route: {experts + 1} integers of 32 or 64 bits expected, got {tuple(offsets.shape)} of {offsets.dtype}")
    return (offsets if offsets.dtype == torch.int32 else offsets.clamp(0, 2 ** 31 - 1)).to(device, torch.int32).contiguous()


def _places32(place):
    """As the kernels read them; one outside the rows stays there."""
    return (place if place.dtype == torch.int32 else place.long().clamp(-1, place.numel()).to(torch.int32)).contiguous()


def _placed(rows, place):
    """Which choices have a row of `rows`, and each choice's row in f32, zeros without one."""
    there = (place >= 0) & (place < rows.shape[0])
    if rows.shape[0] == 0:
        rows = rows.new_zeros(1, rows.shape[1])
    return there, torch.where(there[..., None], rows[torch.where(there, place, 0).long()].float(), 0.0)


def _weight(w, tokens, top_k, device):
    """The weights of a route, as many as the kernels read.  A router of the caller's own may have one for each token, for each choice or for all."""
    if w is None:
        return None
    shape = (tokens, top_k)
    if w.is_complex() or w.dim() > 2 or any(n not in (1, of) for n, of in zip(w.shape[::-1], shape[::-1])):
        raise ValueError(f"weights of a route: {tokens} x {top_k} or what is broadcast to that expected, got {tuple(w.shape)} of {w.dtype}")
    return w.to(device, torch.float32).expand(shape).contiguous()


def _on_gpu(t):
    """Whether rows are moved by the library's kernels.  On the host, where its entry points have been replaced by others, torch moves them."""
    return t.is_cuda


def quantize_weights(w):
    """w (E x N x K or N x K) -> e4m3 of the same shape, scales E x ceil(N / 128) x ceil(K / 128)."""
    N, K = w.shape[-2:]
    w = w if w.stride(-1) == 1 and w.stride(-2) >= K else w.contiguous()
    q = _e4m3(*w.shape, device=w.device)
    scale = torch.empty(*w.shape[:-2], _blocks(N), _blocks(K), dtype=torch.float32, device=w.device)
    for m, qm, sm in zip(w.reshape(-1, N, K), q.view(-1, N, K), scale.view(-1, _blocks(N), _blocks(K))):
        check(binding.quantize_e4m3_blocks(N, K, TYPES[w.dtype], m, _pitch(m), qm, qm.stride(0), sm, _blocks(K), _stream(m)))
    return SimpleNamespace(q=q, scale=scale)


def quantize_weights_i8(w):
    """w (E x N x K or N x K) -> 8-bit integers of the same shape, scales E x N: one for each output."""
    N, K = w.shape[-2:]
    w = w.contiguous()
    q = _bytes(*w.shape, dtype=torch.int8, device=w.device)
    scale = torch.empty(w.shape[:-1], dtype=torch.float32, device=w.device)
    rows = scale.numel()
    check(binding.quantize_i8_rows(rows, K, TYPES[w.dtype], binding.ACT_NONE, w, K, q, q.stride(-2), scale, _stream(w)))
    return SimpleNamespace(q=q, scale=scale)


def swiglu(u):
    g, v = u.float().chunk(2, dim=-1)
    return (torch.nn.functional.silu(g) * v).to(u.dtype)


class ExpertLayer:
    """Weights as products read them: K x N (gemm_grouped) for training; N x K in e4m3 or 8-bit integers for serving, laid out once by `prepare`."""

    def __init__(self, hidden, ffn, experts, top_k, dtype=torch.bfloat16, eps=1e-5, seed=0, device="cuda", exact=False, norm="rms"):
        """exact: e4m3 products exact however many tokens there are, at half the rate (binding.EXACT); norm: "rms" or "layer", which has a beta beside gamma."""
        if hidden % 8 or ffn % 8 or not 1 <= top_k <= experts:
            raise ValueError("hidden and ffn are multiples of 8, top_k at most the number of experts")
        if norm not in ("rms", "layer"):
            raise ValueError(f"norm: rms or layer, not {norm!r}")
        self.norm, self.format = norm, "e4m3"
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
        if norm == "layer":
            self._shapes["beta"] = (hidden,)
            self.beta = random(hidden, scale=0.1)

    def prepare(self, format="e4m3"):
        """The weights in 8 bits, a row for each output; format: "e4m3" (a scale for 128 x 128) or "i8" (integers, a scale for each output), which `serve` then runs in."""
        if format not in ("e4m3", "i8"):
            raise ValueError(f"format: e4m3 or i8, not {format!r}")
        quantize = quantize_weights if format == "e4m3" else quantize_weights_i8
        self.format = format
        self.quantized = SimpleNamespace(**{name: quantize(getattr(self, name).transpose(1, 2).contiguous()) for name in ("up", "down", "shared_up", "shared_down")})

    def route(self, y):
        """The top_k experts of each token: `source`, the token of each of the tokens * top_k rows in the experts' order; `place`, where
        row j of token t went; `offsets`, the rows of each expert, and the weights.  Another one in its place decides itself; rows then move by its `source` and `place`, which
        may be more (groups filled up with rows of any token) or fewer than the choices: a choice whose place is no row (-1) adds nothing.  Places are different from each other.
        Its parts may be on the host (they are copied then, which waits for it)."""
        return SimpleNamespace(**vars(self._route(y)[0]))

    def _route(self, y, rows=None, scale=None):
        """route(y), and the tokens' rows and scales (blocks x tokens, or one for each token) in the experts' order."""
        if rows is not None and (type(self).route is not ExpertLayer.route or "route" in vars(self)):
            route = self.route(y)
            return route, *_rows_of(route.source, rows, scale)
        weight, expert = torch.softmax((y @ self.router).float(), dim=-1).topk(self.top_k, dim=-1)
        weight = weight / weight.sum(-1, keepdim=True)
        T, k, device = expert.shape[0], self.top_k, y.device
        if not _on_gpu(y):
            order = expert.flatten().argsort(stable=True)
            place = torch.empty_like(order)
            place[order] = torch.arange(order.numel(), device=device)
            bounds = torch.arange(self.experts + 1, device=device)
            offsets = torch.searchsorted(expert.flatten()[order], bounds).to(torch.int32)
            route = _Route(weight=weight, expert=expert, source=order // k, place=place, offsets=offsets)
            return route, *((None, None) if rows is None else _rows_of(route.source, rows, scale))
        expert = expert.contiguous()
        offsets, source, place = (torch.empty(n, dtype=torch.int32, device=device) for n in (self.experts + 1, T * k, T * k))
        N, size, blocks, moved, moved_scale = 0, 0, 0, None, None
        if rows is not None:
            N, size, moved = rows.shape[1], rows.element_size(), _like(rows, T * k)
        if scale is not None:
            blocks, moved_scale = scale.numel() // max(T, 1), scale.new_empty(*scale.shape[:-1], T * k)
        need = binding.expert_dispatch_workspace_bytes(T, k, self.experts)
        workspace = torch.empty(need, dtype=torch.uint8, device=device)
        check(binding.expert_dispatch(T, k, self.experts, binding.INDEX_I64, expert, offsets, source, place, N, size, rows, 0 if rows is None else _pitch(rows), blocks, scale, T,
                                      moved, 0 if rows is None else _pitch(moved), moved_scale, T * k, workspace, need, _stream(y)))
        return _Route(weight=weight, expert=expert, source=source, place=place, offsets=offsets), moved, moved_scale

    def _moved_by_torch(self, rows, place):
        """The kernels take as many rows as there are choices; a router of the caller's own may have more (groups filled up) or fewer."""
        return not _on_gpu(rows) or rows.shape[0] != place.numel()

    def _combine(self, rows, route, add, weight, dtype):
        """add + the sum over each token's rows (times its weights, if there are any), in a fixed order, f32, rounded to dtype.  A choice without a row adds nothing."""
        T, N = add.shape
        place, weight = _places(route, T, self.top_k, add.device), _weight(weight, T, self.top_k, add.device)
        if self._moved_by_torch(rows, place):
            rows = _placed(rows, place)[1]
            return ((rows if weight is None else rows * weight[..., None]).sum(1) + add.float()).to(dtype)
        out = torch.empty(T, N, dtype=dtype, device=rows.device)
        check(binding.expert_combine(T, self.top_k, N, TYPES[rows.dtype], _places32(place), rows, N, weight, add, _pitch(add), out, N, TYPES[dtype], _stream(out)))
        return out

    def _combine_grad(self, rows, route, dout):
        """The gradients of _combine's rows and weights; zeros for a row of no choice, as products over whole groups read it."""
        T, N = dout.shape
        place, weight = _places(route, T, self.top_k, dout.device), _weight(route.weight, T, self.top_k, dout.device)
        if self._moved_by_torch(rows, place):
            there, y = _placed(rows, place)
            drows = torch.zeros(rows.shape[0] + 1, N, dtype=self.dtype, device=rows.device)          # the last one: of choices without a row
            drows[torch.where(there, place, rows.shape[0]).long()] = (dout[:, None].float() * weight[..., None]).to(self.dtype)
            return drows[:-1], (y * dout[:, None].float()).sum(-1)
        drows, dweight = torch.empty_like(rows) if isinstance(route, _Route) else torch.zeros_like(rows), torch.empty(T, self.top_k, dtype=torch.float32, device=rows.device)
        check(binding.expert_combine_grad(T, self.top_k, N, TYPES[rows.dtype], _places32(place), dout, _pitch(dout), weight, rows, N, drows, N, dweight, _stream(rows)))
        return drows, dweight

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

    def _norm(self, x, r, format=None):
        self._check_weights(*(n for n in ("gamma", "beta") if n in self._shapes))
        T, H, dev = x.shape[0], self.hidden, x.device
        x, r = self._rows("x", x, T), self._rows("r", r, T)
        n = SimpleNamespace(h=torch.empty(T, H, dtype=x.dtype, device=dev), y=torch.empty(T, H, dtype=x.dtype, device=dev), mean=None, rstd=torch.empty(T, dtype=torch.float32, device=dev), q=None, scale=None)
        if format == "e4m3":
            n.q, n.scale = _e4m3(T, H, device=dev), torch.empty(_blocks(H), T, dtype=torch.float32, device=dev)
        elif format == "i8":
            n.q, n.scale = _bytes(T, H, dtype=torch.int8, device=dev), torch.empty(T, dtype=torch.float32, device=dev)
        ldq, type = n.q.stride(0) if format else 0, TYPES[x.dtype]
        if self.norm == "rms":
            q, scale = (n.q, n.scale) if format == "e4m3" else (None, None)
            check(binding.rms_norm(T, H, type, x, _pitch(x), r, _pitch(r), self.gamma, self.eps, n.h, H, n.y, H, q, ldq, scale, T, n.rstd, _stream(x)))
            if format == "i8":
                check(binding.quantize_i8_rows(T, H, type, binding.ACT_NONE, n.y, H, n.q, ldq, n.scale, _stream(x)))
            return n
        n.mean = torch.empty_like(n.rstd)
        q, scale = (n.q, n.scale) if format == "i8" else (None, None)
        check(binding.layer_norm(T, H, type, x, _pitch(x), r, _pitch(r), self.gamma, self.beta, self.eps, n.h, H, n.y, H, q, ldq, scale, n.mean, n.rstd, _stream(x)))
        if format == "e4m3":
            check(binding.quantize_e4m3_rows(T, H, type, binding.ACT_NONE, n.y, H, n.q, ldq, n.scale, T, _stream(x)))
        return n

    def _product8(self, q, scale, w, offsets=None):
        rows, K = q.shape
        E, N = w.q.shape[:2]
        c = torch.empty(rows, N, dtype=self.dtype, device=q.device)
        if q.dtype == torch.int8:
            if offsets is None:
                check(binding.gemm_i8(rows, N, K, q, q.stride(0), scale, w.q, w.q.stride(1), w.scale, c, N, TYPES[c.dtype], _stream(c)))
            else:
                check(binding.gemm_i8_grouped(rows, N, K, E, offsets, q, q.stride(0), scale, w.q, w.q.stride(1), w.q.stride(0), w.scale, w.scale.stride(0), c, N, TYPES[c.dtype], _stream(c)))
        elif offsets is None:
            check(binding.gemm_e4m3_block(rows, N, K, q, q.stride(0), scale, rows, w.q, w.q.stride(1), w.scale, _blocks(K), c, N, TYPES[c.dtype] | self.exact, _stream(c)))
        else:
            check(binding.gemm_e4m3_block_grouped(rows, N, K, E, offsets, q, q.stride(0), scale, rows, w.q, w.q.stride(1), w.q.stride(0), w.scale, _blocks(K), w.scale.stride(0), c, N, TYPES[c.dtype] | self.exact, _stream(c)))
        return c

    def _swiglu8(self, u):
        rows, N = u.shape[0], u.shape[1] // 2
        if self.format == "i8":
            q, scale = _bytes(rows, N, dtype=torch.int8, device=u.device), torch.empty(rows, dtype=torch.float32, device=u.device)
            check(binding.quantize_i8_rows(rows, N, TYPES[u.dtype], binding.ACT_SWIGLU, u, 2 * N, q, q.stride(0), scale, _stream(u)))
            return q, scale
        q = _e4m3(rows, N, device=u.device)
        scale = torch.empty(_blocks(N), rows, dtype=torch.float32, device=u.device)
        check(binding.quantize_e4m3_rows(rows, N, TYPES[u.dtype], binding.ACT_SWIGLU, u, 2 * N, q, q.stride(0), scale, rows, _stream(u)))
        return q, scale

    def serve(self, x, r):
        """h and out of x and the residual r (tokens x hidden)."""
        w, n = self.quantized, self._norm(x, r, self.format)
        route, rows, scale = self._route(n.y, n.q, n.scale)
        offsets = _offsets(route, self.experts, n.y.device)
        up = self._product8(rows, scale, w.up, offsets)
        out = self._product8(*self._swiglu8(up), w.down, offsets)
        shared = self._product8(*self._swiglu8(self._product8(n.q, n.scale, w.shared_up)), w.shared_down)
        return SimpleNamespace(h=n.h, out=self._combine(out, route, shared, route.weight, self.dtype), route=route)

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
        s = self._norm(x, r)
        s.route, s.a, _ = self._route(s.y, s.y)
        s.all = torch.arange(2, dtype=torch.int32, device=x.device) * x.shape[0]      # the shared expert: one group
        s.shared_a = s.y
        offsets = _offsets(s.route, self.experts, x.device)
        s.u, s.shared_u = self._product(s.a, self.up, offsets), self._product(s.shared_a, self.shared_up, s.all)
        s.s, s.shared_s = swiglu(s.u), swiglu(s.shared_u)
        s.d, shared = self._product(s.s, self.down, offsets), self._product(s.shared_s, self.shared_down, s.all)
        s.out = self._combine(s.d, s.route, shared, s.route.weight, self.dtype)
        return s

    def train_backward(self, s, dout, dh):
        """From the gradients of out and h: of x (and of r), gamma (and beta), the router, the experts' and the shared weights; and of the routing weights."""
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
        dd, dweight = self._combine_grad(s.d, route, dout)
        da, dup, ddown = expert(s.a, s.u, s.s, self.up, self.down, dd, _offsets(route, self.experts, dd.device))
        dy, dshared_up, dshared_down = expert(s.shared_a, s.shared_u, s.shared_s, self.shared_up, self.shared_down, dout, s.all)
        # what reaches y through its rows' copies, and through the shared expert
        dy, router = self._combine(da, route, dy, None, torch.float32 if through_router else self.dtype), {}
        if through_router:
            # top-k of a softmax, divided by their sum: the softmax of the chosen logits alone.  dlogit = weight (dweight - sum(weight dweight)); others' are 0
            dchosen = route.weight * (dweight - (route.weight * dweight).sum(-1, keepdim=True))
            dlogits = torch.zeros(tokens, self.experts, device=dy.device).scatter_(1, route.expert, dchosen)
            dy, router = dy + dlogits @ self.router.float().t(), {"router": s.y.float().t() @ dlogits}
        dy = dy.to(self.dtype)
        T, H = dy.shape
        dx, dgamma = torch.empty_like(dy), torch.empty(H, dtype=torch.float32, device=dy.device)
        grads = SimpleNamespace(x=dx, gamma=dgamma, up=dup, down=ddown, shared_up=dshared_up, shared_down=dshared_down, weight=dweight, **router)
        if self.norm == "layer":
            grads.beta = torch.empty_like(dgamma)
            size = binding.layer_norm_grad_workspace_bytes(T, H)
            workspace = torch.empty(size, dtype=torch.uint8, device=dy.device)
            check(binding.layer_norm_grad(T, H, TYPES[dy.dtype], dy, H, s.h, H, self.gamma, s.mean, s.rstd, dh, _pitch(dh), dx, H, dgamma, grads.beta, workspace, size, _stream(dy)))
            return grads
        size = binding.rms_norm_grad_workspace_bytes(T, H)
        workspace = torch.empty(size, dtype=torch.uint8, device=dy.device)
        check(binding.rms_norm_grad(T, H, TYPES[dy.dtype], dy, H, s.h, H, self.gamma, s.rstd, dh, _pitch(dh), dx, H, dgamma, workspace, size, _stream(dy)))
        return grads


def main(argv=None):
    p = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    for name, value in (("tokens", 4096), ("hidden", 4096), ("ffn", 2048), ("experts", 8), ("top-k", 2), ("steps", 10)):
        p.add_argument(f"--{name}", type=int, default=value)
    p.add_argument("--norm", choices=("rms", "layer"), default="rms")
    p.add_argument("--format", choices=("e4m3", "i8"), default="e4m3")
    a = p.parse_args(argv)
    layer = ExpertLayer(a.hidden, a.ffn, a.experts, a.top_k, norm=a.norm)
    layer.prepare(a.format)
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
    print(f"serve, {a.format + ':':<20}{forward:8.3f} ms, {products / forward * 1e-9:7.1f} TFLOP/s in the products")
    print(f"train, bf16, both ways:    {both:8.3f} ms, {3 * products / both * 1e-9:7.1f} TFLOP/s in the products")
    got, want = layer.serve(x, r).out.float(), layer.train_forward(x, r).out.float()
    print(f"{a.format + ' against bf16:':<27}{((got - want).norm() / want.norm()).item():8.4f} of the result's norm")


if __name__ == "__main__":
    main()
