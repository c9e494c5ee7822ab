"""The operators one after another in a HIP graph, and with thousands of experts."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2108_13191_amd import binding                                    # noqa: E402
from ops_util import DT, TYPE, ceil128, offsets_of, stream                 # noqa: E402


@pytest.mark.parametrize("T,H,F,E", [(5, 512, 256, 4), (300, 1024, 384, 4), (16, 17000, 128, 2)])
def test_a_captured_graph_of_the_serving_path(T, H, F, E):
    """Norm, product by expert, SwiGLU, product: replays on new inputs and offsets, with eager work between them, give the eager calls' bits."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    rand = lambda *s: torch.randn(s, device="cuda", generator=gen)         # noqa: E731
    b16 = torch.bfloat16
    x, r, gamma = rand(T, H).to(b16), rand(T, H).to(b16), rand(H).to(b16)
    up, down = rand(E, 2 * F, H).to(b16), rand(E, H, F).to(b16)
    off = torch.tensor([0] + [T] * E, dtype=torch.int32, device="cuda")

    def quantized(w):
        n, k = w.shape[1:]
        q, s = torch.empty(w.shape, dtype=DT["e4m3"], device="cuda"), torch.empty(E, ceil128(n), ceil128(k), device="cuda")
        for e in range(E):
            binding.check(binding.quantize_e4m3_blocks(n, k, TYPE["bf16"], w[e], k, q[e], k, s[e], ceil128(k), stream()))
        return q, s
    (qu, su), (qd, sd) = quantized(up), quantized(down)

    def buffers():
        return dict(h=torch.zeros(T, H, dtype=b16, device="cuda"), q=torch.zeros(T, H, dtype=DT["e4m3"], device="cuda"), s=torch.zeros(ceil128(H), T, device="cuda"),
                    u=torch.zeros(T, 2 * F, dtype=b16, device="cuda"), v=torch.zeros(T, F, dtype=DT["e4m3"], device="cuda"), t=torch.zeros(ceil128(F), T, device="cuda"),
                    c=torch.zeros(T, H, dtype=torch.float32, device="cuda"))

    def call(o):
        st = stream()
        binding.check(binding.rms_norm(T, H, TYPE["bf16"], x, H, r, H, gamma, 1e-5, o["h"], H, None, 0, o["q"], H, o["s"], T, None, st))
        binding.check(binding.gemm_e4m3_block_grouped(T, 2 * F, H, E, off, o["q"], H, o["s"], T, qu, H, 2 * F * H, su, ceil128(H), su.stride(0), o["u"], 2 * F, TYPE["bf16"], st))
        binding.check(binding.quantize_e4m3_rows(T, F, TYPE["bf16"], binding.ACT_SWIGLU, o["u"], 2 * F, o["v"], F, o["t"], T, st))
        binding.check(binding.gemm_e4m3_block_grouped(T, H, F, E, off, o["v"], F, o["t"], T, qd, F, H * F, sd, ceil128(F), sd.stride(0), o["c"], H, TYPE["f32"], st))

    replayed, eager = buffers(), buffers()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(replayed)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(replayed)
    for ends in ([0] + [T] * E, [0] * E + [T], np.linspace(0, T, E + 1).astype(int).tolist(), [T // 2] * E + [T]):
        off.copy_(torch.tensor(ends, dtype=torch.int32))
        x.copy_(rand(T, H))
        for o in (replayed, eager):
            for t in o.values():
                t.view(torch.uint8).zero_()
        graph.replay()
        torch.cuda.synchronize()
        call(eager)
        torch.cuda.synchronize()
        for name in eager:
            assert torch.equal(replayed[name].view(torch.uint8), eager[name].view(torch.uint8)), (ends, name)
        assert bool(eager["c"].isfinite().all()) and bool((eager["c"][off[0]:] != 0).any())


@pytest.mark.parametrize("E", [1000, 5000])
def test_thousands_of_experts(E):
    """Most of them without rows, the others with a few: integers, every product and both gradients exact."""
    rng = np.random.default_rng(E)
    counts = np.where(rng.random(E) < 0.1, rng.integers(1, 6, E), 0)
    counts[[0, 63, 64, E - 1]] = [1, 2, 40, 3]
    T, N, K = int(counts.sum()), 72, 48
    a, dc, b = (torch.from_numpy(rng.integers(-2, 3, s)).half().cuda() for s in ((T, K), (T, N), (E, K, N)))
    off = torch.from_numpy(offsets_of(counts)).cuda()
    owner = torch.from_numpy(np.repeat(np.arange(E), counts)).cuda()
    c, da, db = torch.zeros(T, N, device="cuda"), torch.zeros(T, K, device="cuda"), torch.full((E, K, N), 7.0, device="cuda")
    f, st = TYPE["f16"], stream()
    binding.check(binding.gemm_grouped(T, N, K, E, off, f, a, K, b, N, K * N, c, N, TYPE["f32"], st))
    binding.check(binding.gemm_grouped_grad_a(T, N, K, E, off, f, dc, N, b, N, K * N, da, K, TYPE["f32"], st))
    binding.check(binding.gemm_grouped_grad_b(T, N, K, E, off, f, a, K, dc, N, db, N, K * N, TYPE["f32"], st))
    rows = b[owner].float()
    assert torch.equal(c, (a.float()[:, :, None] * rows).sum(1)) and torch.equal(da, (rows * dc.float()[:, None, :]).sum(2))
    want = torch.zeros(E, K, N, device="cuda").index_add_(0, owner, a.float()[:, :, None] * dc.float()[:, None, :])
    assert torch.equal(db, want)
    # the e4m3 product: the same integers, scales 1
    q, w = a.float().to(DT["e4m3"]), b.float().transpose(1, 2).contiguous().to(DT["e4m3"])
    c8 = torch.zeros(T, N, device="cuda")
    binding.check(binding.gemm_e4m3_block_grouped(T, N, K, E, off, q, K, torch.ones(1, T, device="cuda"), T, w, K, N * K, torch.ones(E, 1, 1, device="cuda"), 1, 1, c8, N, TYPE["f32"], st))
    assert torch.equal(c8, c)
