"""The operators of include/gemm_layer.h one after another, as a block with experts calls them: serving and the way back in graphs, on streams side by side, with
thousands of experts, and with rows that lie further than 2^32 bytes apart."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2108_13191_amd import binding                                    # noqa: E402
from ops_util import TYPE, stream                                           # noqa: E402
from layer_util import order, quantized                                     # noqa: E402

B16, F32 = torch.bfloat16, torch.float32
ok = binding.check


def empty(*shape, dtype=F32):
    return torch.zeros(shape, dtype=dtype, device="cuda")


class Block:
    """A block's weights, inputs and two calls: `serve` in 8-bit integers and `train`, the way there and back of rows through a norm, to experts (whose work is
    left out) and back."""

    def __init__(self, T, H, F, E, k, seed=7):
        self.T, self.H, self.F, self.E, self.k = T, H, F, E, k
        self.gen = torch.Generator(device="cuda").manual_seed(seed)
        self.x, self.r, self.dout, self.dh = (self.rand(T, H) for _ in range(4))
        self.gamma, self.beta = self.rand(H), self.rand(H)
        self.up, self.down = (self.integers(self.rand(E, n, m)) for n, m in ((2 * F, H), (H, F)))
        self.expert, self.weight = empty(T, k, dtype=torch.int64), empty(T, k)
        self.next()

    def rand(self, *s):
        return torch.randn(s, device="cuda", generator=self.gen).to(B16)

    def integers(self, w):
        E, n, m = w.shape
        q, s = empty(E, n, m, dtype=torch.int8), empty(E, n)
        ok(binding.quantize_i8_rows(E * n, m, TYPE["bf16"], binding.ACT_NONE, w, m, q, m, s, stream()))
        return q, s

    def next(self, one=None):
        """Other inputs and another choice of experts (-1: dropped); `one`: all to that expert."""
        for t in (self.x, self.r, self.dout, self.dh):
            t.copy_(self.rand(*t.shape))
        e = torch.randint(-1, self.E, (self.T, self.k), device="cuda", generator=self.gen)
        self.expert.copy_(e if one is None else torch.full_like(e, one))
        self.weight.copy_(torch.rand(self.T, self.k, device="cuda", generator=self.gen))

    def buffers(self):
        T, H, F, E, n = self.T, self.H, self.F, self.E, self.T * self.k
        need = binding.expert_dispatch_workspace_bytes(T, self.k, E)
        i8, i32 = torch.int8, torch.int32
        return dict(h=empty(T, H, dtype=B16), q=empty(T, H, dtype=i8), s=empty(T), mean=empty(T), rstd=empty(T), offsets=empty(E + 1, dtype=i32), source=empty(n, dtype=i32),
                    place=empty(n, dtype=i32), a=empty(n, H, dtype=i8), sa=empty(n), u=empty(n, 2 * F, dtype=B16), v=empty(n, F, dtype=i8), sv=empty(n), d=empty(n, H, dtype=B16),
                    out=empty(T, H, dtype=B16), y=empty(T, H, dtype=B16), rows=empty(n, H, dtype=B16), dd=empty(n, H, dtype=B16), dweight=empty(T, self.k),
                    dy=empty(T, H, dtype=B16), dx=empty(T, H, dtype=B16), dgamma=empty(H), dbeta=empty(H), work=empty(max(need, 16), dtype=torch.uint8),
                    work2=empty(binding.layer_norm_grad_workspace_bytes(T, H), dtype=torch.uint8))

    def serve(self, o):
        T, H, F, E, k, n, st, (qu, su), (qd, sd) = self.T, self.H, self.F, self.E, self.k, self.T * self.k, stream(), self.up, self.down
        ok(binding.layer_norm(T, H, TYPE["bf16"], self.x, H, self.r, H, self.gamma, self.beta, 1e-5, o["h"], H, None, 0, o["q"], H, o["s"], None, None, st))
        ok(binding.expert_dispatch(T, k, E, binding.INDEX_I64, self.expert, o["offsets"], o["source"], o["place"], H, 1, o["q"], H, 1, o["s"], T, o["a"], H, o["sa"], n,
                                   o["work"], o["work"].numel(), st))
        ok(binding.gemm_i8_grouped(n, 2 * F, H, E, o["offsets"], o["a"], H, o["sa"], qu, H, 2 * F * H, su, 2 * F, o["u"], 2 * F, TYPE["bf16"], st))
        ok(binding.quantize_i8_rows(n, F, TYPE["bf16"], binding.ACT_SWIGLU, o["u"], 2 * F, o["v"], F, o["sv"], st))
        ok(binding.gemm_i8_grouped(n, H, F, E, o["offsets"], o["v"], F, o["sv"], qd, F, H * F, sd, H, o["d"], H, TYPE["bf16"], st))
        ok(binding.expert_combine(T, k, H, TYPE["bf16"], o["place"], o["d"], H, self.weight, o["h"], H, o["out"], H, TYPE["bf16"], st))

    def train(self, o):
        T, H, E, k, n, st, b = self.T, self.H, self.E, self.k, self.T * self.k, stream(), TYPE["bf16"]
        ok(binding.layer_norm(T, H, b, self.x, H, self.r, H, self.gamma, self.beta, 1e-5, o["h"], H, o["y"], H, None, 0, None, o["mean"], o["rstd"], st))
        ok(binding.expert_dispatch(T, k, E, binding.INDEX_I64, self.expert, o["offsets"], o["source"], o["place"], H, 2, o["y"], H, 0, None, 0, o["rows"], H, None, 0,
                                   o["work"], o["work"].numel(), st))
        ok(binding.expert_combine(T, k, H, b, o["place"], o["rows"], H, self.weight, None, 0, o["out"], H, b, st))
        ok(binding.expert_combine_grad(T, k, H, b, o["place"], self.dout, H, self.weight, o["rows"], H, o["dd"], H, o["dweight"], st))
        ok(binding.expert_combine(T, k, H, b, o["place"], o["dd"], H, None, None, 0, o["dy"], H, b, st))
        ok(binding.layer_norm_grad(T, H, b, o["dy"], H, o["h"], H, self.gamma, o["mean"], o["rstd"], self.dh, H, o["dx"], H, o["dgamma"], o["dbeta"], o["work2"], o["work2"].numel(), st))


def same(a, b):
    for name in a:
        if not name.startswith("work"):
            assert torch.equal(a[name].view(torch.uint8), b[name].view(torch.uint8)), name


def clear(o):
    for t in o.values():
        t.view(torch.uint8).zero_()


SIZES = [(1, 256, 128, 4, 2), (5, 512, 256, 4, 2), (300, 1000, 384, 7, 3), (1200, 640, 128, 16, 2), (700, 4096, 512, 3, 1)]


@pytest.mark.parametrize("T,H,F,E,k", SIZES)
@pytest.mark.parametrize("what", ["serve", "train"])
def test_a_captured_graph(T, H, F, E, k, what):
    """Replays on new inputs and choices, with eager work between them, give the eager calls' bits; two graphs, each with a workspace of its own, side by side."""
    block = Block(T, H, F, E, k)
    call = getattr(block, what)
    first, second, eager = block.buffers(), block.buffers(), block.buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(first)
        call(second)
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for o in (first, second):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(o)
    for one in (None, 0, None, E - 1, -1, None):
        block.next(one)
        for o in (first, second, eager):
            clear(o)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graphs[1].replay()
        graphs[0].replay()
        torch.cuda.synchronize()
        call(eager)
        torch.cuda.synchronize()
        same(first, eager)
        same(second, eager)
        # nothing chosen: h itself (rounded once), or nothing
        if one == -1:
            assert torch.equal(eager["out"], eager["h"] if what == "serve" else torch.zeros_like(eager["out"]))
        else:
            assert bool((eager["out"] != 0).any())


@pytest.mark.parametrize("T,H,F,E,k", SIZES)
def test_serving_against_its_definition(T, H, F, E, k):
    """In 64 bits from the integers that the norm wrote: each step is held to its own definition by its own tests, their order and operands here."""
    block, o = Block(T, H, F, E, k, seed=11), None
    o = block.buffers()
    block.serve(o)
    torch.cuda.synchronize()
    host = {n: t.cpu() for n, t in o.items()}
    offsets, source, place = order(block.expert.cpu().numpy(), E)
    assert np.array_equal(host["offsets"].numpy(), offsets) and np.array_equal(host["place"].numpy().reshape(T, k), place)
    n = offsets[-1]
    a, sa = host["a"].double()[:n], host["sa"].double()
    assert torch.equal(host["a"][:n], host["q"][torch.from_numpy(source[:n])]) and torch.equal(host["sa"][:n], host["s"][torch.from_numpy(source[:n])])
    qu, su, qd, sd = (t.cpu().double() for t in (*block.up, *block.down))
    d = torch.zeros(T * k, H, dtype=torch.float64)
    half = 2.0 ** -9
    for e in range(E):
        lo, hi = offsets[e], offsets[e + 1]
        u = (a[lo:hi] @ qu[e].t()) * sa[lo:hi, None] * su[e]                 # sums of integers are exact: one of 0 is 0
        got = host["u"][lo:hi].double()
        assert bool(((got - u).abs() <= (half * 2 + 2.0 ** -22) * u.abs()).all())       # half a unit of bf16: 2^-8 of the value at most
        g, v = got[:, :F], got[:, F:]
        q, s = quantized((torch.nn.functional.silu(g) * v).numpy()) if hi > lo else (np.zeros((0, F)), np.zeros(0))
        # elements of a product in f32 that lies next to a border may differ by one
        assert hi == lo or np.abs(host["v"][lo:hi].numpy() - q).max() <= 1
        assert hi == lo or np.allclose(host["sv"][lo:hi].numpy(), s, rtol=1e-5, atol=0)
        d[lo:hi] = (host["v"][lo:hi].double() @ qd[e].t()) * host["sv"][lo:hi].double()[:, None] * sd[e]
    assert bool(((host["d"][:n].double() - d[:n]).abs() <= (half * 2 + 2.0 ** -22) * d[:n].abs()).all())
    assert not host["d"][n:].any() and not host["u"][n:].any()                          # rows behind the last are left alone
    out = host["h"].double()
    for j in range(k):
        p = torch.from_numpy(place[:, j].astype(np.int64))
        out = out + torch.where((p >= 0)[:, None], block.weight.cpu().double()[:, j, None] * host["d"].double()[p.clamp_min(0)], torch.zeros(()).double())
    most = host["h"].double().abs() + sum(block.weight.cpu().double()[:, j, None] * host["d"].double()[torch.from_numpy(place[:, j].astype(np.int64)).clamp_min(0)].abs() for j in range(k))
    assert bool(((host["out"].double() - out).abs() <= half * 2 * out.abs() + (2 * k + 1) * 2.0 ** -24 * most).all())


def test_side_by_side():
    """Two streams, each with blocks of its own sizes, at once: every result is that of a call by itself."""
    blocks = [Block(600, 512, 128, 8, 2, seed=1), Block(37, 4096, 256, 3, 3, seed=2)]
    want = []
    for b in blocks:
        o = b.buffers()
        b.serve(o)
        torch.cuda.synchronize()
        want.append(o)
    streams, got = [torch.cuda.Stream() for _ in blocks], [[b.buffers() for _ in range(6)] for b in blocks]
    torch.cuda.synchronize()
    for i in range(6):
        for b, s, o in zip(blocks, streams, got):
            with torch.cuda.stream(s):
                b.serve(o[i])
    torch.cuda.synchronize()
    for w, each in zip(want, got):
        for o in each:
            same(w, o)


@pytest.mark.parametrize("E,T", [(1000, 300), (5000, 2500)])
def test_thousands_of_experts(E, T):
    """To more experts than rows, most of them with none: each row against its own expert's product."""
    H, N = 64, 48
    gen = np.random.default_rng(3)
    expert = torch.from_numpy(gen.integers(0, E, (T, 1))).cuda()
    x = torch.from_numpy(gen.integers(-127, 128, (T, H)).astype(np.int8)).cuda()
    w = torch.from_numpy(gen.integers(-127, 128, (E, N, H)).astype(np.int8)).cuda()
    sx, sw = torch.rand(T, device="cuda") + 0.5, torch.rand(E, N, device="cuda") + 0.5
    rows, srows, offsets, source, place = empty(T, H, dtype=torch.int8), empty(T), empty(E + 1, dtype=torch.int32), empty(T, dtype=torch.int32), empty(T, dtype=torch.int32)
    need = binding.expert_dispatch_workspace_bytes(T, 1, E)
    work = empty(max(need, 16), dtype=torch.uint8)
    ok(binding.expert_dispatch(T, 1, E, binding.INDEX_I64, expert, offsets, source, place, H, 1, x, H, 1, sx, T, rows, H, srows, T, work, work.numel(), stream()))
    c, out = empty(T, N), empty(T, N)
    ok(binding.gemm_i8_grouped(T, N, H, E, offsets, rows, H, srows, w, H, N * H, sw, N, c, N, TYPE["f32"], stream()))
    ok(binding.expert_combine(T, 1, N, TYPE["f32"], place, c, N, None, None, 0, out, N, TYPE["f32"], stream()))
    e = expert[:, 0].cpu()
    sums = (w.cpu().long()[e] * x.cpu().long()[:, None]).sum(-1).to(F32)
    assert torch.equal(out.cpu(), sums * sx.cpu()[:, None] * sw.cpu()[e])


def test_rows_further_apart_than_32_bits():
    """Rows 3 * 2^29 elements apart: the norm, its gradients, the rows' way to experts and back, and products, against the same rows side by side."""
    T, H, E, k, ld = 3, 520, 2, 2, 3 << 29
    gen = torch.Generator(device="cuda").manual_seed(5)
    arena = torch.empty(6 * ld, dtype=B16, device="cuda")                     # room for six rows in 18 GiB
    out_arena = torch.empty(6 * ld, dtype=B16, device="cuda")

    def far(rows, dtype, a, at=0):
        return a.view(dtype).as_strided((rows, H), (ld, 1), at)
    b = TYPE["bf16"]
    x = torch.randn(T, H, device="cuda", generator=gen).to(B16)
    gamma = torch.randn(H, device="cuda", generator=gen).to(B16)
    n = k * T

    def run(X, ldx, H_, ldh, Q, ldq, rows, ldr, DY, DX):
        o = dict(s=empty(T), mean=empty(T), rstd=empty(T), offsets=empty(E + 1, dtype=torch.int32), place=empty(n, dtype=torch.int32), sr=empty(n), dgamma=empty(H), dbeta=empty(H),
                 c=empty(n, 32))
        expert = torch.tensor([[1, 0], [0, 1], [1, 1]], device="cuda")
        ok(binding.layer_norm(T, H, b, X, ldx, None, 0, gamma, None, 1e-5, H_, ldh, None, 0, Q, ldq, o["s"], o["mean"], o["rstd"], stream()))
        ok(binding.expert_dispatch(T, k, E, binding.INDEX_I64, expert, o["offsets"], None, o["place"], H, 1, Q, ldq, 1, o["s"], T, rows, ldr, o["sr"], n, None, 0, stream()))
        w, sw = torch.ones(E, 32, H, dtype=torch.int8, device="cuda"), torch.ones(E, 32, device="cuda")
        ok(binding.gemm_i8_grouped(n, 32, H, E, o["offsets"], rows, ldr, o["sr"], w, H, 32 * H, sw, 32, o["c"], 32, TYPE["f32"], stream()))
        work = empty(binding.layer_norm_grad_workspace_bytes(T, H), dtype=torch.uint8)
        ok(binding.layer_norm_grad(T, H, b, DY, ldx, H_, ldh, gamma, o["mean"], o["rstd"], None, 0, DX, ldx, o["dgamma"], o["dbeta"], work, work.numel(), stream()))
        torch.cuda.synchronize()
        o["rows"], o["DX"], o["h"] = rows[:n, :H].clone(), DX[:T, :H].clone(), H_[:T, :H].clone()
        return o

    near = run(x, H, empty(T, H, dtype=B16), H, empty(T, H, dtype=torch.int8), H, empty(n, H, dtype=torch.int8), H, x * 2, empty(T, H, dtype=B16))
    X, H_, DY, DX = far(T, B16, arena), far(T, B16, arena, 1024), far(T, B16, arena, 2048), far(T, B16, arena, 4096)
    Q, rows = far(T, torch.int8, arena, 16384), far(n, torch.int8, out_arena)
    X.copy_(x)
    DY.copy_(x * 2)
    got = run(X, ld, H_, ld, Q, ld, rows, ld, DY, DX)
    for name in near:
        assert torch.equal(near[name].view(torch.uint8), got[name].view(torch.uint8)), name

    Y, dY = far(n, B16, arena), far(n, B16, out_arena)
    y = torch.randn(n, H, device="cuda", generator=gen).to(B16)
    Y.copy_(y)
    weight = torch.rand(T, k, device="cuda", generator=gen)

    def back(Y_, ldy, D):
        out, dw = empty(T, H, dtype=B16), empty(T, k)
        ok(binding.expert_combine(T, k, H, b, near["place"], Y_, ldy, weight, None, 0, out, H, b, stream()))
        ok(binding.expert_combine_grad(T, k, H, b, near["place"], x, H, weight, Y_, ldy, D, ldy, dw, stream()))
        torch.cuda.synchronize()
        return out, dw, D.clone()
    for g, w in zip(back(Y, ld, dY), back(y, H, empty(n, H, dtype=B16))):
        assert torch.equal(g, w)
