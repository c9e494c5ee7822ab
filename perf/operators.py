"""The operators around the products of a transformer layer, as cases to be timed: the RMS norm with the residual's addition (in
front of a layer, its output in 8 bits with scales or in 16 bits) and its gradients, quantisation to e4m3 with scales of activations and
weights, the product of e4m3 matrices with a scale for each block of 128, and products grouped by expert with ragged sizes, in e4m3 with block
scales (serving) and in 16 bits with both gradients (training).

`run` computes them in plain torch operations, or where `own` is set through `paper_2108_13191_amd.binding`.
"""
import math

import torch

own = False

F8 = torch.float8_e4m3fn
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-6
BLOCK = 128
SCALE_FLOOR = 2.0 ** -96      # least magnitude that a block's scale stands for, so that no scale is zero

_lib = None


def _binding():
    global _lib
    if _lib is None:
        from paper_2108_13191_amd import binding
        _lib = binding
    return _lib


# ---- cases ------------------------------------------------------------------------------------------------------------------
# kind: which operator.  pad: elements between the rows' ends and the pitches.  M / T: rows (tokens).


def _norm(name, M, N, type, out, pad=0):
    return _named(name, {"kind": "norm", "M": M, "N": N, "type": type, "out": out, "pad": pad})


def _norm_grad(name, M, N, type, residual, pad=0):
    return _named(name, {"kind": "norm_grad", "M": M, "N": N, "type": type, "residual": residual, "pad": pad})


def _quant(name, M, N, type, form, pad=0):
    return _named(name, {"kind": "quant", "M": M, "N": N, "type": type, "form": form, "pad": pad})


def _e4m3(name, M, N, K, c, pad=0):
    return _named(name, {"kind": "e4m3", "M": M, "N": N, "K": K, "c": c, "pad": pad})


def _grouped_e4m3(name, T, N, K, E, c, skew):
    return _named(name, {"kind": "grouped_e4m3", "T": T, "N": N, "K": K, "E": E, "c": c, "skew": skew})


def _grouped(name, kind, T, N, K, E, type, c, skew, pad=0):
    return _named(name, {"kind": kind, "T": T, "N": N, "K": K, "E": E, "type": type, "c": c, "skew": skew, "pad": pad})


def _named(name, d):
    return dict(d, name=name) if name else d


def listed():
    return [
        # decoding, 16 sequences: latency of one norm in front of a layer of width 8192
        _norm("norm_decode", 16, 8192, "f16", "e4m3"),
        # a prefill's norm over 16384 tokens: bandwidth
        _norm("norm_prefill", 16384, 4096, "bf16", "e4m3"),
        # the same norm's backward in training, a token count and a width that are no multiple of any tile
        _norm_grad("norm_grad_ragged", 8191, 4000, "bf16", True),
        # the hidden layer of a gated FFN on its way into the second product
        _quant("quant_swiglu", 4096, 8192, "bf16", "swiglu"),
        # a weight matrix on its way into 8 bits, once after each training step that is followed by generation
        _quant("quant_weights", 8192, 8192, "bf16", "blocks"),
        # decoding: 16 rows against a large weight matrix
        _e4m3("e4m3_decode16", 16, 8192, 8192, "f16"),
        # the headline square of this repository, in 8 bits
        _e4m3("e4m3_sq8192", 8192, 8192, 8192, "bf16"),
        # no multiple of any tile or scale block
        _e4m3("e4m3_ragged4000", 4000, 4000, 4000, "f32"),
        # decoding with experts: 64 rows (32 tokens, two experts each) over 16 experts
        _grouped_e4m3("experts_decode", 64, 4096, 2048, 16, "bf16", 0.5),
        # prefill with experts: uneven loads, some far from a multiple of a tile
        _grouped_e4m3("experts_prefill", 16384, 4096, 2048, 16, "bf16", 0.7),
        # training with experts: the forward product, and both gradients
        _grouped("experts_train_forward", "grouped", 16384, 2304, 768, 8, "f16", "f16", 0.7),
        _grouped("experts_train_backward", "grouped_grad", 16384, 2048, 1024, 32, "bf16", "f32", 0.7),
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
        kind = rng.choice(["norm", "norm_grad", "quant", "e4m3", "e4m3", "grouped_e4m3", "grouped_e4m3", "grouped", "grouped_grad"])
        type = rng.choice(["f16", "bf16"])
        pad = rng.choice([0, 0, 0, 16, 128])
        if kind in ("norm", "norm_grad", "quant"):
            M, N = _log(rng, 1, 20000), _size(rng, 128, 16384)
            if M * N > 16384 * 4096:
                continue
            if kind == "norm":
                return _norm(None, M, N, type, rng.choice(["e4m3", "e4m3", "16bit"]), pad)
            if kind == "norm_grad":
                return _norm_grad(None, M, N, type, rng.random() < 0.5, pad)
            return _quant(None, M, N, type, rng.choice(["rows", "relu", "swiglu", "blocks"]), pad)
        N, K = _size(rng, 256, 16384), _size(rng, 256, 16384)
        c = rng.choice(["f16", "bf16", "f32"])
        if kind == "e4m3":
            M = _log(rng, 1, 256) if rng.random() < 0.5 else _log(rng, 256, 16384)
            if M * N * K <= 8192 ** 3:
                return _e4m3(None, M, N, K, c, pad)
            continue
        E = rng.choice([4, 8, 16, 32, 64, 128])
        T = _log(rng, 1, 512) if rng.random() < 0.4 else _log(rng, 512, 20000)
        N, K = min(N, 8192), min(K, 8192)
        skew = rng.choice([0.0, 0.5, 1.0])
        if T * N * K > 16384 * 4096 * 2048 or E * N * K > 16 * 4096 * 4096:
            continue
        if kind == "grouped_e4m3":
            return _grouped_e4m3(None, T, N, K, E, c, skew)
        return _grouped(None, kind, T, N, K, E, type, rng.choice([type, "f32"]), skew, pad)


# ---- inputs -----------------------------------------------------------------------------------------------------------------

def _up16(n):
    return (n + 15) // 16 * 16


def _blocks(n):
    return (n + BLOCK - 1) // BLOCK


class _Gen:
    """Draws tensors on the GPU; a matrix is a view of the first columns of rows of `ld` elements."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(self, *shape, std=1.0, dtype=torch.float32, ld=None):
        out = torch.empty(*shape[:-1], ld or shape[-1], dtype=dtype, device="cuda")[..., :shape[-1]]
        flat = out if out.dim() < 3 else out.view(-1, shape[-1]) if out.is_contiguous() else out.flatten(0, -2)
        rows = max(1, (1 << 26) // max(1, shape[-1]))
        if flat.dim() == 1:
            return flat.copy_(torch.randn(shape[-1], device="cuda", generator=self.g) * std)
        for i in range(0, flat.shape[0], rows):          # in parts: no large temporary
            part = flat[i:i + rows]
            x = torch.randn(part.shape, device="cuda", generator=self.g).mul_(std)
            part.copy_(x.clamp_(-448.0, 448.0) if dtype == F8 else x)
        return out

    def scales(self, *shape, typical):
        """Scales as a quantiser finds them: positive, spread by a factor of a few."""
        return torch.exp(torch.randn(*shape, device="cuda", generator=self.g) * 0.3) * typical

    def counts(self, T, E, skew):
        """Rows of each expert, as a router deals them."""
        p = torch.softmax(skew * torch.randn(E, device="cuda", generator=self.g), 0)
        to = torch.multinomial(p, T, replacement=True, generator=self.g)
        return torch.bincount(to, minlength=E)


def _out(*shape, dtype, ld=None):
    return torch.zeros(*shape[:-1], ld or shape[-1], dtype=dtype, device="cuda")[..., :shape[-1]]


def prepare(case, seed):
    g, kind = _Gen(seed), case["kind"]
    pad = case.get("pad", 0)
    s = {"case": case, "kind": kind, "stream": torch.cuda.current_stream().cuda_stream}
    if kind in ("norm", "norm_grad", "quant"):
        M, N, dt = case["M"], case["N"], TYPES[case["type"]]
        ld, nb = N + pad, _blocks(N)
        if kind == "quant":
            wide = 2 * N if case["form"] == "swiglu" else N
            s["x"] = g.normal(M, wide, std=0.02 if case["form"] == "blocks" else 1.0, dtype=dt, ld=wide + pad)
            s["q"] = _out(M, N, dtype=F8, ld=_up16(N))
            s["scale"] = _out(*((_blocks(M), nb) if case["form"] == "blocks" else (nb, M)), dtype=torch.float32)
            return s
        s["gamma"] = (1.0 + 0.1 * torch.randn(N, device="cuda", generator=g.g)).to(dt)
        if kind == "norm":
            s["x"], s["r"] = g.normal(M, N, dtype=dt, ld=ld), g.normal(M, N, std=2.0, dtype=dt, ld=ld)
            s["h"] = _out(M, N, dtype=dt, ld=ld)
            if case["out"] == "e4m3":
                s["q"], s["scale"] = _out(M, N, dtype=F8, ld=_up16(N)), _out(nb, M, dtype=torch.float32)
            else:
                s["y"], s["rstd"] = _out(M, N, dtype=dt, ld=ld), _out(M, dtype=torch.float32)
            return s
        s["dy"], s["h"] = g.normal(M, N, std=0.01, dtype=dt, ld=ld), g.normal(M, N, std=2.0, dtype=dt, ld=ld)
        s["dh"] = g.normal(M, N, std=0.01, dtype=dt, ld=ld) if case["residual"] else None
        s["rstd"] = torch.cat([torch.rsqrt(p.float().square().mean(1) + EPS) for p in s["h"].split(4096)])
        s["dx"], s["dgamma"] = _out(M, N, dtype=dt, ld=ld), _out(N, dtype=torch.float32)
        s["workspace"] = torch.empty(max(1, 256 * N), dtype=torch.float32, device="cuda")
        return s
    N, K, kb = case["N"], case["K"], _blocks(case["K"])
    c = TYPES[case["c"]]
    if kind == "e4m3":
        M, ld = case["M"], _up16(K) + pad
        s["a"], s["a_scale"] = g.normal(M, K, std=150.0, dtype=F8, ld=ld), g.scales(kb, M, typical=1 / 150)
        s["b"], s["b_scale"] = g.normal(N, K, std=110.0, dtype=F8, ld=ld), g.scales(_blocks(N), kb, typical=K ** -0.5 / 110)
        s["c"] = _out(M, N, dtype=c, ld=N + pad)
        return s
    T, E = case["T"], case["E"]
    counts = g.counts(T, E, case["skew"])
    s["offsets"] = torch.cat([counts.new_zeros(1), counts.cumsum(0)]).to(torch.int32)
    s["counts"] = counts.tolist()      # for the plain form, which splits on the host
    if kind == "grouped_e4m3":
        s["a"], s["a_scale"] = g.normal(T, K, std=150.0, dtype=F8, ld=_up16(K)), g.scales(kb, T, typical=1 / 150)
        s["b"], s["b_scale"] = g.normal(E, N, K, std=110.0, dtype=F8, ld=_up16(K)), g.scales(E, _blocks(N), kb, typical=K ** -0.5 / 110)
        s["c"] = _out(T, N, dtype=c)
        return s
    dt = TYPES[case["type"]]
    s["b"] = g.normal(E, K, N, std=K ** -0.5, dtype=dt)
    s["a"] = g.normal(T, K, dtype=dt, ld=K + pad)
    if kind == "grouped":
        s["c"] = _out(T, N, dtype=c, ld=N + pad)
    else:
        s["dc"] = g.normal(T, N, std=0.1, dtype=dt, ld=N + pad)
        s["da"], s["db"] = _out(T, K, dtype=dt, ld=K + pad), _out(E, K, N, dtype=c)
    return s


# ---- the operators in plain operations --------------------------------------------------------------------------------------

def _row_blocks(y):
    """(values padded to whole blocks, as rows x blocks x 128)"""
    M, N = y.shape
    nb = _blocks(N)
    if nb * BLOCK != N:
        y = torch.cat([y, y.new_zeros(M, nb * BLOCK - N)], 1)
    return y.view(M, nb, BLOCK)


def _quantized_rows(y):
    M, N = y.shape
    t = _row_blocks(y)
    scale = t.abs().amax(2).clamp_min(SCALE_FLOOR) / 448.0
    return (t / scale[:, :, None]).view(M, -1)[:, :N].to(F8), scale.t().contiguous()


def _dequantized_rows(q, scale):
    return q.float() * scale.t().repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def _dequantized_blocks(q, scale):
    return q.float() * scale.repeat_interleave(BLOCK, 0)[:q.shape[0]].repeat_interleave(BLOCK, 1)[:, :q.shape[1]]


def _plain(s):
    kind, case = s["kind"], s["case"]
    if kind == "norm":
        h = (s["x"].float() + s["r"].float()).to(s["x"].dtype)
        hf = h.float()
        rstd = torch.rsqrt(hf.square().mean(1) + EPS)
        y = hf * rstd[:, None] * s["gamma"].float()
        if case["out"] == "e4m3":
            q, scale = _quantized_rows(y)
            return {"h": h, "q": q, "scale": scale}
        return {"h": h, "y": y.to(h.dtype), "rstd": rstd}
    if kind == "norm_grad":
        dy, xhat = s["dy"].float(), s["h"].float() * s["rstd"][:, None]
        g = dy * s["gamma"].float()
        dx = s["rstd"][:, None] * (g - xhat * (g * xhat).mean(1, keepdim=True))
        if s["dh"] is not None:
            dx = dx + s["dh"].float()
        return {"dx": dx.to(s["dy"].dtype), "dgamma": (dy * xhat).sum(0)}
    if kind == "quant":
        x, form = s["x"].float(), case["form"]
        if form == "blocks":
            M, N = x.shape
            t = _row_blocks(x)
            mb, nb = _blocks(M), t.shape[1]
            if mb * BLOCK != M:
                t = torch.cat([t, t.new_zeros(mb * BLOCK - M, nb, BLOCK)], 0)
            t = t.view(mb, BLOCK, nb, BLOCK)
            scale = t.abs().amax((1, 3)).clamp_min(SCALE_FLOOR) / 448.0
            return {"q": (t / scale[:, None, :, None]).view(mb * BLOCK, -1)[:M, :N].to(F8), "scale": scale}
        if form == "relu":
            x = torch.clamp_min(x, 0.0)
        elif form == "swiglu":
            gate, up = x[:, :case["N"]], x[:, case["N"]:]
            x = gate / (1.0 + torch.exp(-gate)) * up
        q, scale = _quantized_rows(x)
        return {"q": q, "scale": scale}
    if kind == "e4m3":
        return {"c": (_dequantized_rows(s["a"], s["a_scale"]) @ _dequantized_blocks(s["b"], s["b_scale"]).t()).to(s["c"].dtype)}
    counts = s["counts"]
    if kind == "grouped_e4m3":
        a = _dequantized_rows(s["a"], s["a_scale"]).split(counts)
        return {"c": torch.cat([(x @ _dequantized_blocks(b, bs).t()).to(s["c"].dtype) for x, b, bs, n in zip(a, s["b"], s["b_scale"], counts) if n])}
    a = s["a"].split(counts)
    if kind == "grouped":
        return {"c": torch.cat([(x.float() @ b.float()).to(s["c"].dtype) for x, b, n in zip(a, s["b"], counts) if n])}
    dc = s["dc"].split(counts)
    return {"da": torch.cat([(d.float() @ b.float().t()).to(s["da"].dtype) for d, b, n in zip(dc, s["b"], counts) if n]),
            "db": torch.stack([(x.float().t() @ d.float()).to(s["db"].dtype) for x, d in zip(a, dc)])}


# ---- through the library ----------------------------------------------------------------------------------------------------

def _own(s):
    lib, kind, case, st = _binding(), s["kind"], s["case"], s["stream"]
    if kind == "norm":
        x, r, h, type = s["x"], s["r"], s["h"], lib.TYPE_F16 if case["type"] == "f16" else lib.TYPE_BF16
        if case["out"] == "e4m3":
            q, scale = s["q"], s["scale"]
            lib.check(lib.rms_norm(case["M"], case["N"], type, x, x.stride(0), r, r.stride(0), s["gamma"], EPS, h, h.stride(0),
                                   None, 0, q, q.stride(0), scale, case["M"], None, st))
            return {"h": h, "q": q, "scale": scale}
        y = s["y"]
        lib.check(lib.rms_norm(case["M"], case["N"], type, x, x.stride(0), r, r.stride(0), s["gamma"], EPS, h, h.stride(0),
                               y, y.stride(0), None, 0, None, 0, s["rstd"], st))
        return {"h": h, "y": y, "rstd": s["rstd"]}
    if kind == "norm_grad":
        dy, h, dh, dx = s["dy"], s["h"], s["dh"], s["dx"]
        type, ws = lib.TYPE_F16 if case["type"] == "f16" else lib.TYPE_BF16, s["workspace"]
        lib.check(lib.rms_norm_grad(case["M"], case["N"], type, dy, dy.stride(0), h, h.stride(0), s["gamma"], s["rstd"],
                                    dh, dh.stride(0) if dh is not None else 0, dx, dx.stride(0), s["dgamma"], ws, 4 * ws.numel(), st))
        return {"dx": dx, "dgamma": s["dgamma"]}
    if kind == "quant":
        x, q, type = s["x"], s["q"], lib.TYPE_F16 if case["type"] == "f16" else lib.TYPE_BF16
        if case["form"] == "blocks":
            lib.check(lib.quantize_e4m3_blocks(case["M"], case["N"], type, x, x.stride(0), q, q.stride(0), s["scale"], s["scale"].stride(0), st))
        else:
            act = {"rows": lib.ACT_NONE, "relu": lib.ACT_RELU, "swiglu": lib.ACT_SWIGLU}[case["form"]]
            lib.check(lib.quantize_e4m3_rows(case["M"], case["N"], type, act, x, x.stride(0), q, q.stride(0), s["scale"], case["M"], st))
        return {"q": q, "scale": s["scale"]}
    c_type = {"f16": lib.TYPE_F16, "bf16": lib.TYPE_BF16, "f32": lib.TYPE_F32}[case["c"]]
    a, b = s["a"], s["b"]
    if kind == "e4m3":
        c = s["c"]
        lib.check(lib.gemm_e4m3_block(case["M"], case["N"], case["K"], a, a.stride(0), s["a_scale"], case["M"], b, b.stride(0),
                                      s["b_scale"], s["b_scale"].stride(0), c, c.stride(0), c_type, st))
        return {"c": c}
    T, N, K, E = case["T"], case["N"], case["K"], case["E"]
    if kind == "grouped_e4m3":
        c, bs = s["c"], s["b_scale"]
        lib.check(lib.gemm_e4m3_block_grouped(T, N, K, E, s["offsets"], a, a.stride(0), s["a_scale"], T, b, b.stride(1), b.stride(0),
                                              bs, bs.stride(1), bs.stride(0), c, c.stride(0), c_type, st))
        return {"c": c}
    type = lib.TYPE_F16 if case["type"] == "f16" else lib.TYPE_BF16
    if kind == "grouped":
        c = s["c"]
        lib.check(lib.gemm_grouped(T, N, K, E, s["offsets"], type, a, a.stride(0), b, b.stride(1), b.stride(0), c, c.stride(0), c_type, st))
        return {"c": c}
    dc, da, db = s["dc"], s["da"], s["db"]
    lib.check(lib.gemm_grouped_grad_a(T, N, K, E, s["offsets"], type, dc, dc.stride(0), b, b.stride(1), b.stride(0), da, da.stride(0), type, st))
    lib.check(lib.gemm_grouped_grad_b(T, N, K, E, s["offsets"], type, a, a.stride(0), dc, dc.stride(0), db, db.stride(1), db.stride(0), c_type, st))
    return {"da": da, "db": db}


def run(s):
    return _own(s) if own else _plain(s)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------

def work(case):
    kind = case["kind"]
    size = {"f16": 2, "bf16": 2, "f32": 4}
    if kind in ("norm", "norm_grad", "quant"):
        M, N, nb = case["M"], case["N"], _blocks(case["N"])
        if kind == "norm":
            out = M * N + 4 * M * nb if case["out"] == "e4m3" else 2 * M * N + 4 * M
            return {"bytes": 6 * M * N + 2 * N + out, "flops": 6 * M * N}
        if kind == "norm_grad":
            return {"bytes": (8 if case["residual"] else 6) * M * N + 6 * N + 4 * M, "flops": 10 * M * N}
        scales = _blocks(M) * nb if case["form"] == "blocks" else M * nb
        return {"bytes": (5 if case["form"] == "swiglu" else 3) * M * N + 4 * scales, "flops": 3 * M * N}
    N, K, kb = case["N"], case["K"], _blocks(case["K"])
    if kind == "e4m3":
        M = case["M"]
        return {"bytes": M * K + N * K + 4 * kb * (M + _blocks(N)) + size[case["c"]] * M * N, "flops": 2 * M * N * K}
    T, E = case["T"], case["E"]
    hit = E * (1.0 - (1.0 - 1.0 / E) ** T)          # experts that get a row, of even loads
    if kind == "grouped_e4m3":
        return {"bytes": T * K + 4 * kb * T + hit * (N * K + 4 * kb * _blocks(N)) + size[case["c"]] * T * N + 4 * (E + 1), "flops": 2 * T * N * K}
    if kind == "grouped":
        return {"bytes": 2 * T * K + 2 * hit * N * K + size[case["c"]] * T * N + 4 * (E + 1), "flops": 2 * T * N * K}
    return {"bytes": 2 * T * N + 2 * hit * N * K + 2 * T * K + 2 * T * K + 2 * T * N + size[case["c"]] * E * N * K + 8 * (E + 1), "flops": 4 * T * N * K}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------

def _block_max(y, rows):
    """Largest magnitude of each block of `rows` x 128 values."""
    M, N = y.shape
    mb, nb = -(-M // rows), _blocks(N)
    t = torch.zeros(mb * rows, nb * BLOCK, dtype=torch.float64, device=y.device)
    t[:M, :N] = y.abs()
    return torch.maximum(t.view(mb, rows, nb, BLOCK).amax(3).amax(1), torch.tensor(SCALE_FLOOR, dtype=torch.float64, device=y.device))


def _over(y, scale, rows):
    M, N = y.shape
    i = torch.arange(M, device=y.device) // rows
    j = torch.arange(N, device=y.device) // BLOCK
    return y / scale[i][:, j]


def exact(case, seed):
    s = prepare(case, seed)
    kind = s["kind"]

    def d(name):
        return s[name].double()

    if kind == "norm":
        h = d("x") + d("r")
        used = h.to(s["x"].dtype).double()               # the definition norms the sum as it is stored
        rstd = 1.0 / torch.sqrt((used * used).sum(1) / case["N"] + EPS)
        y = used * rstd[:, None] * d("gamma")[None, :]
        if case["out"] == "e4m3":
            scale = _block_max(y, 1) / 448.0
            return {"h": h, "q": _over(y, scale, 1), "scale": scale.t()}
        return {"h": h, "y": y, "rstd": rstd}
    if kind == "norm_grad":
        n, r = case["N"], d("rstd")[:, None]
        up = d("dy") * d("gamma")
        dot = (up * d("h")).sum(1, keepdim=True)
        dx = r * up - r ** 3 * d("h") * dot / n
        return {"dx": dx if s["dh"] is None else dx + d("dh"), "dgamma": torch.einsum("ij,ij->j", d("dy"), r * d("h"))}
    if kind == "quant":
        y = d("x")
        if case["form"] == "blocks":
            scale = _block_max(y, BLOCK) / 448.0
            return {"q": _over(y, scale, BLOCK), "scale": scale}
        if case["form"] == "relu":
            y = torch.where(y > 0, y, torch.zeros_like(y))
        elif case["form"] == "swiglu":
            y = y[:, :case["N"]] * torch.sigmoid(y[:, :case["N"]]) * y[:, case["N"]:]
        scale = _block_max(y, 1) / 448.0
        return {"q": _over(y, scale, 1), "scale": scale.t()}

    def wide(q, scale, rows):
        """e4m3 values times the scales of their blocks of `rows` x 128"""
        i = torch.arange(q.shape[0], device=q.device) // rows
        j = torch.arange(q.shape[1], device=q.device) // BLOCK
        return q.double() * scale.double()[i][:, j]

    if kind == "e4m3":
        return {"c": wide(s["a"], s["a_scale"].t(), 1) @ wide(s["b"], s["b_scale"], BLOCK).t()}
    ends = [sum(s["counts"][:e]) for e in range(case["E"] + 1)]
    if kind == "grouped_e4m3":
        c = torch.zeros(case["T"], case["N"], dtype=torch.float64, device="cuda")
        a = wide(s["a"], s["a_scale"].t(), 1)
        for e in range(case["E"]):
            if ends[e + 1] > ends[e]:
                c[ends[e]:ends[e + 1]] = a[ends[e]:ends[e + 1]] @ wide(s["b"][e], s["b_scale"][e], BLOCK).t()
        return {"c": c}
    c = torch.zeros(case["T"], case["K"] if kind == "grouped_grad" else case["N"], dtype=torch.float64, device="cuda")
    db = torch.zeros(case["E"], case["K"], case["N"], dtype=torch.float64, device="cuda") if kind == "grouped_grad" else None
    for e in range(case["E"]):
        rows = slice(ends[e], ends[e + 1])
        if kind == "grouped":
            c[rows] = d("a")[rows] @ s["b"][e].double()
        else:
            c[rows] = s["dc"][rows].double() @ s["b"][e].double().t()
            db[e] = s["a"][rows].double().t() @ s["dc"][rows].double()
    return {"c": c} if kind == "grouped" else {"da": c, "db": db}
