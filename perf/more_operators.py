"""Operators of a transformer block served in 8-bit integers and trained in 16 bits, as cases to be timed: layer norm with the
residual's addition and its gradients; tokens sorted by expert with their rows moved there and back, weights applied, and the gradients of
that; quantisation to 8-bit integers with a scale for each row, and products of such matrices with scales for each token and channel, also grouped by expert.

`run` computes them in plain torch operations, or where `own` is set through `paper_2108_13191_amd.binding`.
"""
import math

import torch

own = False

F8, I8 = torch.float8_e4m3fn, torch.int8
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32, "e4m3": F8, "i8": I8}
EPS = 1e-5
BLOCK = 128                   # e4m3 elements of a row that share a scale
SCALE_FLOOR = 2.0 ** -96      # least magnitude that a row's scale stands for, so that no scale is zero

_lib = None


def _binding():
    global _lib
    if _lib is None:
        from paper_2108_13191_amd import binding
        _lib = binding
    return _lib


# ---- cases ------------------------------------------------------------------------------------------------------------------
# kind: which operator.  pad: elements between the rows' ends and the pitches.  M / T: rows (tokens).  drop: the share of a token's
# choices that belong to no expert here (padded tokens, experts of another process).


def _named(name, d):
    return dict(d, name=name) if name else d


def _norm(name, M, N, type, pad=0):
    return _named(name, {"kind": "norm", "M": M, "N": N, "type": type, "pad": pad})


def _norm_grad(name, M, N, type, residual, pad=0):
    return _named(name, {"kind": "norm_grad", "M": M, "N": N, "type": type, "residual": residual, "pad": pad})


def _dispatch(name, T, k, E, N, type, ids, skew, drop=0.0, pad=0):
    return _named(name, {"kind": "dispatch", "T": T, "k": k, "E": E, "N": N, "type": type, "ids": ids, "skew": skew, "drop": drop, "pad": pad})


def _combine(name, T, k, E, N, type, out, weighted, add, drop=0.0, pad=0):
    return _named(name, {"kind": "combine", "T": T, "k": k, "E": E, "N": N, "type": type, "out": out, "weighted": weighted, "add": add, "drop": drop, "pad": pad})


def _combine_grad(name, T, k, E, N, type, drop=0.0, pad=0):
    return _named(name, {"kind": "combine_grad", "T": T, "k": k, "E": E, "N": N, "type": type, "drop": drop, "pad": pad})


def _i8(name, M, N, K, c, pad=0):
    return _named(name, {"kind": "i8", "M": M, "N": N, "K": K, "c": c, "pad": pad})


def _i8_linear(name, M, N, K, type, act, c, pad=0):
    return _named(name, {"kind": "i8_linear", "M": M, "N": N, "K": K, "type": type, "act": act, "c": c, "pad": pad})


def _norm_linear(name, M, N, K, type):
    return _named(name, {"kind": "norm_linear", "M": M, "N": N, "K": K, "type": type})


def _i8_grouped(name, T, N, K, E, c, skew):
    return _named(name, {"kind": "i8_grouped", "T": T, "N": N, "K": K, "E": E, "c": c, "skew": skew})


def _i8_weights(name, M, N, type, pad=0):
    return _named(name, {"kind": "i8_weights", "M": M, "N": N, "type": type, "pad": pad})


def listed():
    return [
        # decoding, 16 sequences: latency of one norm in front of a layer of width 8192
        _norm("norm_decode", 16, 8192, "f16"),
        # a training step's norm over 16384 tokens, with what its backward pass reads: bandwidth
        _norm("norm_train", 16384, 4096, "bf16"),
        # its backward pass, a token count and a width that are no multiple of any tile
        _norm_grad("norm_grad_ragged", 8191, 4000, "bf16", True),
        # a small model's backward pass: latency and the reduction of the weights' gradients
        _norm_grad("norm_grad_small", 512, 768, "f16", False),
        # decoding: 32 tokens, two experts each, to 16 experts, rows in 8 bits with their scales
        _dispatch("dispatch_decode", 32, 2, 16, 2048, "i8", "i64", 0.5),
        # prefill or training: rows of 16 bits, uneven experts
        _dispatch("dispatch_prefill", 8192, 2, 16, 4096, "bf16", "i64", 0.7),
        # and back, six experts a token, a shared expert's result added, some choices of experts elsewhere
        _combine("combine_ragged", 5001, 6, 64, 2304, "f16", "f16", True, True, 0.1),
        # the way back's gradient: of the rows and of the weights
        _combine_grad("combine_grad", 8192, 2, 32, 2048, "bf16"),
        # decoding: 16 rows against a large weight matrix
        _i8("i8_decode16", 16, 8192, 8192, "f16"),
        # the headline square of this repository, in 8-bit integers
        _i8("i8_sq8192", 8192, 8192, 8192, "bf16"),
        # activations quantised in front of the product, no multiple of any tile
        _i8_linear("i8_linear_ragged", 4000, 4000, 4000, "bf16", "none", "f32"),
        # prefill with experts: uneven loads
        _i8_grouped("i8_experts_prefill", 16384, 4096, 2048, 16, "bf16", 0.7),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A width of a layer: most are multiples of 64 or 16, some of 8, some odd."""
    n, u = _log(rng, lo, hi), rng.random()
    step = 64 if u < 0.5 else 16 if u < 0.8 else 8 if u < 0.92 else 1
    return max(lo, n // step * step)


def draw(rng):
    while True:
        kind = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "dispatch", "dispatch", "combine", "combine", "combine_grad", "combine_grad",
                           "i8", "i8", "i8_linear", "norm_linear", "i8_grouped", "i8_grouped", "i8_weights"])
        type = rng.choice(["f16", "bf16"])
        pad = rng.choice([0, 0, 0, 16, 128])
        if kind in ("norm", "norm_grad", "i8_weights"):
            M, N = _log(rng, 1, 20000), _size(rng, 64, 16384)
            if M * N > 16384 * 4096:
                continue
            if kind == "norm":
                return _norm(None, M, N, type, pad)
            if kind == "norm_grad":
                return _norm_grad(None, M, N, type, rng.random() < 0.5, pad)
            return _i8_weights(None, M, N, type, pad)
        if kind in ("dispatch", "combine", "combine_grad"):
            T, k, N = _log(rng, 1, 20000), rng.randint(1, 8), _size(rng, 64, 8192)
            E, drop = rng.choice([4, 8, 16, 32, 64, 128, 256]), rng.choice([0.0, 0.0, 0.3])
            if k > E or T * k * N > 1 << 26:
                continue
            if kind == "dispatch":
                return _dispatch(None, T, k, E, N, rng.choice([type, "i8", "e4m3"]), rng.choice(["i32", "i64"]), rng.choice([0.0, 0.5, 1.0]), drop, pad)
            if kind == "combine":
                return _combine(None, T, k, E, N, type, rng.choice([type, "f32"]), rng.random() < 0.7, rng.random() < 0.5, drop, pad)
            return _combine_grad(None, T, k, E, N, type, drop, pad)
        N, K = _size(rng, 256, 16384), _size(rng, 256, 16384)
        c = rng.choice(["f16", "bf16", "f32"])
        if kind != "i8_grouped":
            M = _log(rng, 1, 256) if rng.random() < 0.5 else _log(rng, 256, 16384)
            if M * N * K > 8192 ** 3:
                continue
            if kind == "i8":
                return _i8(None, M, N, K, c, pad)
            if kind == "norm_linear":
                return _norm_linear(None, M, N, K, type)
            act = rng.choice(["none", "relu", "swiglu"])
            return _i8_linear(None, M, N, K, type, act, type if act == "swiglu" else c, pad)
        E = rng.choice([4, 8, 16, 32, 64, 128])
        T = _log(rng, 1, 512) if rng.random() < 0.4 else _log(rng, 512, 20000)
        N, K = min(N, 8192), min(K, 8192)
        if T * N * K > 16384 * 4096 * 2048 or E * N * K > 16 * 4096 * 4096:
            continue
        return _i8_grouped(None, T, N, K, E, c, rng.choice([0.0, 0.5, 1.0]))


# ---- inputs -----------------------------------------------------------------------------------------------------------------

def _up16(n):
    return (n + 15) // 16 * 16


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


class _Gen:
    """Draws tensors on the GPU; a matrix is a view of the first columns of rows of `ld` elements."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(self, *shape, std=1.0, mean=0.0, dtype=torch.float32, ld=None):
        out = torch.empty(*shape[:-1], ld or shape[-1], dtype=dtype, device="cuda")[..., :shape[-1]]
        flat = out if out.dim() < 3 else out.flatten(0, -2)
        rows = max(1, (1 << 26) // max(1, shape[-1]))
        if flat.dim() == 1:
            return flat.copy_(torch.randn(shape[-1], device="cuda", generator=self.g) * std + mean)
        for i in range(0, flat.shape[0], rows):          # in parts: no large temporary
            part = flat[i:i + rows]
            x = torch.randn(part.shape, device="cuda", generator=self.g).mul_(std).add_(mean)
            part.copy_(x.round_().clamp_(-127, 127) if dtype == I8 else x.clamp_(-448.0, 448.0) if dtype == F8 else x)
        return out

    def scales(self, *shape, typical):
        """Scales as a quantiser finds them: positive, spread by a factor of a few."""
        return torch.exp(torch.randn(*shape, device="cuda", generator=self.g) * 0.3) * typical

    def router(self, T, k, E, skew, drop):
        """Each token's k experts, all different, as an uneven router chooses them; -1 where a choice is of no expert here."""
        logits = skew * torch.randn(E, device="cuda", generator=self.g) + torch.randn(T, E, device="cuda", generator=self.g)
        ids = logits.topk(k, dim=1).indices
        return torch.where(torch.rand(T, k, device="cuda", generator=self.g) < drop, -1, ids)


def _out(*shape, dtype, ld=None):
    return torch.zeros(*shape[:-1], ld or shape[-1], dtype=dtype, device="cuda")[..., :shape[-1]]


def _places(ids, E):
    """Where the rows of each choice lie once they are sorted by expert: n (T x k), -1 for none."""
    flat = torch.where((ids >= 0) & (ids < E), ids, E).flatten()
    order = torch.argsort(flat, stable=True)
    place = torch.empty_like(order)
    place[order] = torch.arange(order.numel(), device=order.device)
    return torch.where(flat < E, place, -1).view(ids.shape).to(torch.int32)


def prepare(case, seed):
    g, kind = _Gen(seed), case["kind"]
    pad = case.get("pad", 0)
    s = {"case": case, "kind": kind, "stream": torch.cuda.current_stream().cuda_stream}
    if kind in ("norm", "norm_grad", "i8_weights"):
        M, N, dt = case["M"], case["N"], TYPES[case["type"]]
        ld = N + pad
        if kind == "i8_weights":
            s["x"] = g.normal(M, N, std=0.02, dtype=dt, ld=ld)
            s["q"], s["scale"] = _out(M, N, dtype=I8, ld=_up16(N)), _out(M, dtype=torch.float32)
            return s
        s["gamma"] = (1.0 + 0.1 * torch.randn(N, device="cuda", generator=g.g)).to(dt)
        if kind == "norm":
            s["beta"] = g.normal(N, std=0.1, dtype=dt)
            s["x"], s["r"] = g.normal(M, N, dtype=dt, ld=ld), g.normal(M, N, std=2.0, mean=0.25, dtype=dt, ld=ld)
            s["h"], s["y"] = _out(M, N, dtype=dt, ld=ld), _out(M, N, dtype=dt, ld=ld)
            s["mean"], s["rstd"] = _out(M, dtype=torch.float32), _out(M, dtype=torch.float32)
            return s
        s["dy"], s["h"] = g.normal(M, N, std=0.01, dtype=dt, ld=ld), g.normal(M, N, std=2.0, mean=0.25, dtype=dt, ld=ld)
        s["dh"] = g.normal(M, N, std=0.01, dtype=dt, ld=ld) if case["residual"] else None
        stats = [torch.var_mean(p.float(), 1, correction=0) for p in s["h"].split(4096)]
        s["mean"], s["rstd"] = torch.cat([m for _, m in stats]), torch.cat([torch.rsqrt(v + EPS) for v, _ in stats])
        s["dx"] = _out(M, N, dtype=dt, ld=ld)
        s["dgamma"], s["dbeta"] = _out(N, dtype=torch.float32), _out(N, dtype=torch.float32)
        s["workspace"] = None
        return s
    if kind in ("dispatch", "combine", "combine_grad"):
        T, k, E, N, dt = case["T"], case["k"], case["E"], case["N"], TYPES[case["type"]]
        ids = g.router(T, k, E, case.get("skew", 0.5), case["drop"])
        if kind == "dispatch":
            s["ids"] = ids.to(torch.int32 if case["ids"] == "i32" else torch.int64)
            ld = _up16(N) + pad if dt in (I8, F8) else N + pad
            s["x"] = g.normal(T, N, std=40.0 if dt == I8 else 100.0 if dt == F8 else 1.0, dtype=dt, ld=ld)
            # one scale a row in 8-bit integers; in e4m3 one for 128 elements, the rows' scales of a block of columns side by side
            blocks = 1 if dt == I8 else _blocks(N) if dt == F8 else 0
            s["blocks"] = blocks
            s["x_scale"] = g.scales(blocks, T, typical=0.01) if blocks else None
            s["rows"], s["rows_scale"] = _out(T * k, N, dtype=dt, ld=ld), _out(blocks, T * k, dtype=torch.float32) if blocks else None
            s["offsets"], s["source"], s["place"] = (_out(n, dtype=torch.int32) for n in (E + 1, T * k, T * k))
            s["workspace"] = None
            return s
        ld = N + pad
        s["place"] = _places(ids, E)
        s["y"] = g.normal(T * k, N, dtype=dt, ld=ld)
        w = torch.softmax(torch.randn(T, k, device="cuda", generator=g.g), 1)
        if kind == "combine":
            s["weight"] = w if case["weighted"] else None
            s["add"] = g.normal(T, N, dtype=dt, ld=ld) if case["add"] else None
            s["out"] = _out(T, N, dtype=TYPES[case["out"]], ld=ld)
            return s
        s["weight"], s["dout"] = w, g.normal(T, N, std=0.1, dtype=dt, ld=ld)
        s["dy"], s["dweight"] = _out(T * k, N, dtype=dt, ld=ld), _out(T, k, dtype=torch.float32)
        return s
    N, K = case["N"], case["K"]
    ld = _up16(K) + pad
    if kind == "i8_grouped":
        T, E = case["T"], case["E"]
        p = torch.softmax(case["skew"] * torch.randn(E, device="cuda", generator=g.g), 0)
        counts = torch.bincount(torch.multinomial(p, T, replacement=True, generator=g.g), minlength=E)
        s["offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
        s["counts"] = counts.tolist()      # for the plain form, which splits on the host
        s["a"], s["a_scale"] = g.normal(T, K, std=40.0, dtype=I8, ld=ld), g.scales(T, typical=1 / 40)
        s["b"], s["b_scale"] = g.normal(E, N, K, std=32.0, dtype=I8, ld=ld), g.scales(E, N, typical=K ** -0.5 / 32)
        s["c"] = _out(T, N, dtype=TYPES[case["c"]])
        return s
    M = case["M"]
    s["b"], s["b_scale"] = g.normal(N, K, std=32.0, dtype=I8, ld=ld), g.scales(N, typical=K ** -0.5 / 32)
    if kind == "norm_linear":
        dt = TYPES[case["type"]]
        s["gamma"], s["beta"] = (1.0 + 0.1 * torch.randn(K, device="cuda", generator=g.g)).to(dt), g.normal(K, std=0.1, dtype=dt)
        s["x"], s["r"] = g.normal(M, K, dtype=dt), g.normal(M, K, std=2.0, mean=0.25, dtype=dt)
        s["h"], s["c"] = _out(M, K, dtype=dt), _out(M, N, dtype=dt)
    else:
        s["c"] = _out(M, N, dtype=TYPES[case["c"]], ld=N + pad)
    if kind == "i8":
        s["a"], s["a_scale"] = g.normal(M, K, std=40.0, dtype=I8, ld=ld), g.scales(M, typical=1 / 40)
        return s
    if kind == "i8_linear":
        wide = 2 * K if case["act"] == "swiglu" else K
        s["x"] = g.normal(M, wide, dtype=TYPES[case["type"]], ld=wide + pad)
    s["q"], s["scale"] = _out(M, K, dtype=I8, ld=_up16(K)), _out(M, dtype=torch.float32)
    return s


# ---- the operators in plain operations --------------------------------------------------------------------------------------

def _layer_norm(s):
    h = (s["x"].float() + s["r"].float()).to(s["x"].dtype)
    hf = h.float()
    mean = hf.mean(1)
    centred = hf - mean[:, None]
    rstd = 1.0 / torch.sqrt(centred.square().mean(1) + EPS)
    return h, mean, rstd, centred * rstd[:, None] * s["gamma"].float() + s["beta"].float()


def _quantized(y):
    """Whole steps of the stored scale, the nearest ones (the quotient in 64 bits: rounded to 32 it falls on the border between two now and then)."""
    scale = y.abs().amax(1).clamp_min(SCALE_FLOOR) / 127.0
    return torch.round(y.double() / scale.double()[:, None]).float(), scale


def _activated(s):
    x, act = s["x"].float(), s["case"]["act"]
    if act == "swiglu":
        gate, up = x[:, :s["case"]["K"]], x[:, s["case"]["K"]:]
        return gate / (1.0 + torch.exp(-gate)) * up
    return torch.clamp_min(x, 0.0) if act == "relu" else x


def _product(a, a_scale, b, b_scale, dtype):
    return (a.float() @ b.float().t() * a_scale[:, None] * b_scale[None, :]).to(dtype)


def _gathered(y, place):
    """Rows of y in the tokens' order (T x k x N), zeros for a choice of no expert."""
    rows = y[place.flatten().clamp_min(0).long()].float()
    return torch.where((place.flatten() >= 0)[:, None], rows, 0.0).view(*place.shape, y.shape[1])


def _plain(s):
    kind, case = s["kind"], s["case"]
    if kind == "norm":
        h, mean, rstd, y = _layer_norm(s)
        return {"h": h, "y": y.to(h.dtype), "mean": mean, "rstd": rstd}
    if kind == "norm_grad":
        dy, rstd = s["dy"].float(), s["rstd"][:, None]
        xhat = (s["h"].float() - s["mean"][:, None]) * rstd
        g = dy * s["gamma"].float()
        dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return {"dx": dx.to(s["dy"].dtype), "dgamma": (dy * xhat).sum(0), "dbeta": dy.sum(0)}
    if kind == "i8_weights":
        q, scale = _quantized(s["x"].float())
        return {"q": q.to(I8), "scale": scale}
    if kind == "dispatch":
        k, E, x = case["k"], case["E"], s["x"]
        ids = s["ids"].flatten()
        valid = (ids >= 0) & (ids < E)
        key = torch.where(valid, ids, E)
        order = torch.argsort(key, stable=True)
        inverse = torch.empty_like(order)
        inverse[order] = torch.arange(order.numel(), device=order.device)
        offsets = torch.searchsorted(key[order], torch.arange(E + 1, device=order.device, dtype=key.dtype))
        there = key[order] < E
        token = order // k
        raw = x.view(torch.uint8) if x.dtype in (I8, F8) else x.view(torch.int16)
        rows = torch.where(there[:, None], raw[token], 0).view(x.dtype)
        got = {"offsets": offsets.to(torch.int32), "source": torch.where(there, token, -1).to(torch.int32),
               "place": torch.where(valid, inverse, -1).to(torch.int32), "rows": rows}
        if s["blocks"]:
            got["scale"] = torch.where(there[None, :], s["x_scale"][:, token], 0.0)
        return got
    if kind == "combine":
        rows = _gathered(s["y"], s["place"])
        out = (rows * s["weight"][:, :, None]).sum(1) if s["weight"] is not None else rows.sum(1)
        if s["add"] is not None:
            out = out + s["add"].float()
        return {"out": out.to(s["out"].dtype)}
    if kind == "combine_grad":
        place, dout = s["place"], s["dout"].float()
        spread = (s["weight"][:, :, None] * dout[:, None, :]).to(s["dy"].dtype).flatten(0, 1)
        at, n = place.flatten().long(), spread.shape[0]
        dy = torch.zeros(n + 1, spread.shape[1], dtype=spread.dtype, device=spread.device)
        dy[torch.where(at >= 0, at, n)] = spread
        return {"dy": dy[:n], "dweight": (_gathered(s["y"], place) * dout[:, None, :]).sum(2)}
    if kind == "i8":
        return {"c": _product(s["a"], s["a_scale"], s["b"], s["b_scale"], s["c"].dtype)}
    if kind == "i8_linear":
        q, scale = _quantized(_activated(s))
        return {"c": _product(q, scale, s["b"], s["b_scale"], s["c"].dtype)}
    if kind == "norm_linear":
        h, _, _, y = _layer_norm(s)
        q, scale = _quantized(y)
        return {"h": h, "c": _product(q, scale, s["b"], s["b_scale"], s["c"].dtype)}
    counts = s["counts"]
    a, sa = s["a"].split(counts), s["a_scale"].split(counts)
    return {"c": torch.cat([_product(x, xs, b, bs, s["c"].dtype) for x, xs, b, bs, n in zip(a, sa, s["b"], s["b_scale"], counts) if n])}


# ---- through the library ----------------------------------------------------------------------------------------------------

def _workspace(s, size, *of):
    """Made at the first call and kept, as a user's program would."""
    if s["workspace"] is None:
        s["workspace"] = torch.empty(max(16, size(*of)), dtype=torch.uint8, device="cuda")
    return s["workspace"], s["workspace"].numel()


def _own(s):
    lib, kind, case, st = _binding(), s["kind"], s["case"], s["stream"]
    code = {"f16": lib.TYPE_F16, "bf16": lib.TYPE_BF16, "f32": lib.TYPE_F32}
    if kind == "norm":
        x, r, h, y = s["x"], s["r"], s["h"], s["y"]
        lib.check(lib.layer_norm(case["M"], case["N"], code[case["type"]], x, x.stride(0), r, r.stride(0), s["gamma"], s["beta"], EPS, h, h.stride(0),
                                 y, y.stride(0), None, 0, None, s["mean"], s["rstd"], st))
        return {"h": h, "y": y, "mean": s["mean"], "rstd": s["rstd"]}
    if kind == "norm_grad":
        dy, h, dh, dx, M, N = s["dy"], s["h"], s["dh"], s["dx"], case["M"], case["N"]
        ws, size = _workspace(s, lib.layer_norm_grad_workspace_bytes, M, N)
        lib.check(lib.layer_norm_grad(M, N, code[case["type"]], dy, dy.stride(0), h, h.stride(0), s["gamma"], s["mean"], s["rstd"],
                                      dh, dh.stride(0) if dh is not None else 0, dx, dx.stride(0), s["dgamma"], s["dbeta"], ws, size, st))
        return {"dx": dx, "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    if kind == "i8_weights":
        x, q = s["x"], s["q"]
        lib.check(lib.quantize_i8_rows(case["M"], case["N"], code[case["type"]], lib.ACT_NONE, x, x.stride(0), q, q.stride(0), s["scale"], st))
        return {"q": q, "scale": s["scale"]}
    if kind == "dispatch":
        T, k, E, x, rows, ids = case["T"], case["k"], case["E"], s["x"], s["rows"], s["ids"]
        ws, size = _workspace(s, lib.expert_dispatch_workspace_bytes, T, k, E)
        lib.check(lib.expert_dispatch(T, k, E, lib.INDEX_I32 if case["ids"] == "i32" else lib.INDEX_I64, ids, s["offsets"], s["source"], s["place"],
                                      case["N"], x.element_size(), x, x.stride(0), s["blocks"], s["x_scale"], T, rows, rows.stride(0), s["rows_scale"], T * k, ws, size, st))
        got = {"offsets": s["offsets"], "source": s["source"], "place": s["place"], "rows": rows}
        if s["blocks"]:
            got["scale"] = s["rows_scale"]
        return got
    if kind == "combine":
        y, add, out = s["y"], s["add"], s["out"]
        lib.check(lib.expert_combine(case["T"], case["k"], case["N"], code[case["type"]], s["place"], y, y.stride(0), s["weight"],
                                     add, add.stride(0) if add is not None else 0, out, out.stride(0), code[case["out"]], st))
        return {"out": out}
    if kind == "combine_grad":
        dout, y, dy = s["dout"], s["y"], s["dy"]
        lib.check(lib.expert_combine_grad(case["T"], case["k"], case["N"], code[case["type"]], s["place"], dout, dout.stride(0), s["weight"],
                                          y, y.stride(0), dy, dy.stride(0), s["dweight"], st))
        return {"dy": dy, "dweight": s["dweight"]}
    N, K, b, c = case["N"], case["K"], s["b"], s["c"]
    if kind == "i8_grouped":
        a = s["a"]
        lib.check(lib.gemm_i8_grouped(case["T"], N, K, case["E"], s["offsets"], a, a.stride(0), s["a_scale"], b, b.stride(1), b.stride(0), s["b_scale"], N,
                                      c, c.stride(0), code[case["c"]], st))
        return {"c": c}
    M = case["M"]
    if kind == "i8":
        a = s["a"]
        lib.check(lib.gemm_i8(M, N, K, a, a.stride(0), s["a_scale"], b, b.stride(0), s["b_scale"], c, c.stride(0), code[case["c"]], st))
        return {"c": c}
    x, q = s["x"], s["q"]
    if kind == "norm_linear":
        r, h, type = s["r"], s["h"], code[case["type"]]
        lib.check(lib.layer_norm(M, K, type, x, x.stride(0), r, r.stride(0), s["gamma"], s["beta"], EPS, h, h.stride(0), None, 0, q, q.stride(0), s["scale"],
                                 None, None, st))
        lib.check(lib.gemm_i8(M, N, K, q, q.stride(0), s["scale"], b, b.stride(0), s["b_scale"], c, c.stride(0), type, st))
        return {"h": h, "c": c}
    act = {"none": lib.ACT_NONE, "relu": lib.ACT_RELU, "swiglu": lib.ACT_SWIGLU}[case["act"]]
    lib.check(lib.quantize_i8_rows(M, K, code[case["type"]], act, x, x.stride(0), q, q.stride(0), s["scale"], st))
    lib.check(lib.gemm_i8(M, N, K, q, q.stride(0), s["scale"], b, b.stride(0), s["b_scale"], c, c.stride(0), code[case["c"]], st))
    return {"c": c}


def run(s):
    return _own(s) if own else _plain(s)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    size = {"f16": 2, "bf16": 2, "f32": 4, "i8": 1, "e4m3": 1}
    if kind in ("norm", "norm_grad", "i8_weights"):
        M, N = case["M"], case["N"]
        if kind == "norm":
            return {"bytes": 8 * M * N + 4 * N + 8 * M, "flops": 9 * M * N}
        if kind == "norm_grad":
            return {"bytes": (8 if case["residual"] else 6) * M * N + 10 * N + 8 * M, "flops": 14 * M * N}
        return {"bytes": 3 * M * N + 4 * M, "flops": 3 * M * N}
    if kind in ("dispatch", "combine", "combine_grad"):
        T, k, E, N, item = case["T"], case["k"], case["E"], case["N"], size[case["type"]]
        rows = T * k * (1.0 - case["drop"])                # rows that belong to an expert
        if kind == "dispatch":
            scales = 4 * (1 if case["type"] == "i8" else _blocks(N) if case["type"] == "e4m3" else 0)
            return {"bytes": (item * N + scales) * (T + rows) + T * k * ((4 if case["ids"] == "i32" else 8) + 8) + 4 * (E + 1), "flops": T * k}
        if kind == "combine":
            each = item * rows * N + (item * T * N if case["add"] else 0) + size[case["out"]] * T * N
            return {"bytes": each + (8 if case["weighted"] else 4) * T * k, "flops": 2 * rows * N}
        return {"bytes": item * N * (T + 2 * rows) + 12 * T * k, "flops": 3 * rows * N}
    N, K = case["N"], case["K"]
    if kind == "i8_grouped":
        T, E = case["T"], case["E"]
        hit = E * (1.0 - (1.0 - 1.0 / E) ** T)          # experts that get a row, of even loads
        return {"bytes": T * K + 4 * T + hit * (N * K + 4 * N) + size[case["c"]] * T * N + 4 * (E + 1), "flops": 2 * T * N * K}
    M = case["M"]
    product = {"bytes": N * K + 4 * N, "flops": 2 * M * N * K}
    if kind == "i8":
        return {"bytes": product["bytes"] + M * K + 4 * M + size[case["c"]] * M * N, "flops": product["flops"]}
    if kind == "norm_linear":
        return {"bytes": product["bytes"] + 6 * M * K + 4 * K + 2 * M * N, "flops": product["flops"]}
    return {"bytes": product["bytes"] + (4 if case["act"] == "swiglu" else 2) * M * K + size[case["c"]] * M * N, "flops": product["flops"]}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    kind = s["kind"]

    def d(name):
        return s[name].double()

    def normed(x, r):
        stored = (x + r).to(s["x"].dtype).double()       # the definition norms the sum as it is stored
        m = torch.sum(stored, 1) / stored.shape[1]
        away = stored - m.unsqueeze(1)
        v = torch.sum(away * away, 1) / stored.shape[1]
        inv = (v + EPS) ** -0.5
        return x + r, m, inv, torch.addcmul(d("beta").unsqueeze(0), away * inv.unsqueeze(1), d("gamma").unsqueeze(0))

    def steps(y):
        """y in whole steps of its rows' scales, and those"""
        step = torch.maximum(torch.maximum(y.max(1).values, -y.min(1).values), torch.tensor(SCALE_FLOOR, dtype=torch.float64, device=y.device)) / 127.0
        return torch.round(y / step.unsqueeze(1)), step

    def stored_step(y):
        """The scale as it is stored, in f32: what the elements of rows that are held exactly go by"""
        return (y.abs().amax(1).float().clamp_min(SCALE_FLOOR) / 127.0).double()

    def times(a, sa, b, sb):
        return (a * sa.unsqueeze(1)) @ (b * sb.unsqueeze(1)).t()

    if kind == "norm":
        h, m, inv, y = normed(d("x"), d("r"))
        return {"h": h, "y": y, "mean": m, "rstd": inv}
    if kind == "norm_grad":
        n, inv = case["N"], d("rstd").unsqueeze(1)
        away = d("h") - d("mean").unsqueeze(1)
        up = d("dy") * d("gamma")
        dx = inv * up - inv * up.sum(1, keepdim=True) / n - inv ** 3 * away * (up * away).sum(1, keepdim=True) / n
        return {"dx": dx if s["dh"] is None else dx + d("dh"), "dgamma": torch.einsum("ij,ij->j", d("dy"), away * inv), "dbeta": torch.einsum("ij->j", d("dy"))}
    if kind == "i8_weights":
        return {"q": torch.round(d("x") / stored_step(d("x")).unsqueeze(1)).to(I8), "scale": d("x").abs().amax(1).clamp_min(SCALE_FLOOR) / 127.0}
    if kind == "dispatch":
        T, k, E, n = case["T"], case["k"], case["E"], case["T"] * case["k"]
        e = s["ids"].reshape(-1).to(torch.int64)
        e = torch.where(e < 0, torch.full_like(e, E), e)
        by = torch.sort(e * n + torch.arange(n, device="cuda")).values          # expert first, then the choice's place
        at, of = by % n, by // n
        total = int((e < E).sum())
        source = torch.full((n,), -1, dtype=torch.int64, device="cuda")
        source[:total] = at[:total] // k
        place = torch.full((n,), -1, dtype=torch.int64, device="cuda")
        place[at[:total]] = torch.arange(total, device="cuda")
        rows = torch.zeros(n, case["N"], dtype=torch.float64, device="cuda")
        rows[:total] = d("x")[source[:total]]
        got = {"offsets": torch.bincount(of, minlength=E + 1)[:E].cumsum(0).to(torch.int32), "source": source.to(torch.int32), "place": place.to(torch.int32), "rows": rows}
        got["offsets"] = torch.cat([got["offsets"].new_zeros(1), got["offsets"]])
        if s["blocks"]:
            got["scale"] = torch.zeros(s["blocks"], n, dtype=torch.float64, device="cuda")
            got["scale"][:, :total] = d("x_scale")[:, source[:total]]
        return got
    if kind in ("combine", "combine_grad"):
        T, k = case["T"], case["k"]
        place = s["place"].long()
        out = torch.zeros(T, case["N"], dtype=torch.float64, device="cuda") if kind == "combine" else torch.zeros_like(d("y"))
        dweight = torch.zeros(T, k, dtype=torch.float64, device="cuda")
        if kind == "combine" and s["add"] is not None:
            out += d("add")
        for j in range(k):                               # one choice of every token at a time
            t = (place[:, j] >= 0).nonzero().flatten()
            w = s["weight"][t, j].double().unsqueeze(1) if s["weight"] is not None else 1.0
            if kind == "combine":
                out[t] += w * s["y"][place[t, j]].double()
            else:
                out[place[t, j]] = w * s["dout"][t].double()
                dweight[t, j] = torch.einsum("ij,ij->i", s["dout"][t].double(), s["y"][place[t, j]].double())
        return {"out": out} if kind == "combine" else {"dy": out, "dweight": dweight}
    if kind == "i8":
        return {"c": times(d("a"), d("a_scale"), d("b"), d("b_scale"))}
    if kind == "i8_linear":
        y = d("x")
        if case["act"] == "swiglu":
            y = y[:, :case["K"]] * torch.sigmoid(y[:, :case["K"]]) * y[:, case["K"]:]
            return {"c": times(*steps(y), d("b"), d("b_scale"))}
        if case["act"] == "relu":
            y = torch.where(y > 0, y, torch.zeros_like(y))
        step = stored_step(y)
        return {"c": times(torch.round(y / step.unsqueeze(1)), step, d("b"), d("b_scale"))}
    if kind == "norm_linear":
        h, _, _, y = normed(d("x"), d("r"))
        return {"h": h, "c": times(*steps(y), d("b"), d("b_scale"))}
    c = torch.zeros(case["T"], case["N"], dtype=torch.float64, device="cuda")
    first = 0
    for e, n in enumerate(s["counts"]):
        if n:
            c[first:first + n] = times(s["a"][first:first + n].double(), s["a_scale"][first:first + n].double(), s["b"][e].double(), s["b_scale"][e].double())
        first += n
    return {"c": c}
