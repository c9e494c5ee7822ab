"""The operators of include/gemm_ops.h where offsets pass 32 bits and where rows pass what one launch takes."""
import pytest
import torch

from paper_2108_13191_amd import binding
from tests.ops_util import DT, TYPE, assert_within, ceil128, result_bound, spread_blocks, spread_rows, stream

pytestmark = pytest.mark.gpu


def spread(t, ld):
    """The same matrix with rows `ld` elements apart."""
    out = torch.empty((t.shape[0] - 1) * ld + t.shape[1], dtype=t.dtype, device="cuda").as_strided(t.shape, (ld, 1))
    out.view(torch.uint8).as_strided((t.shape[0], t.shape[1] * t.element_size()), (ld * t.element_size(), 1)).copy_(t.view(torch.uint8))
    return out


def same(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


def test_rows_far_apart():
    """600 rows 2^23 elements apart: 10 GB, offsets beyond 2^32 elements."""
    M, N, ld = 600, 1000, 1 << 23
    gen = torch.Generator().manual_seed(1)
    x, r, g, dy = (torch.randn(*s, generator=gen).to(torch.bfloat16).cuda() for s in ((M, N), (M, N), (N,), (M, N)))
    q = [torch.empty(M, N, dtype=DT["e4m3"], device="cuda") for _ in range(2)]
    scale = [torch.empty(ceil128(N), M, dtype=torch.float32, device="cuda") for _ in range(2)]
    y = [torch.empty_like(x) for _ in range(2)]
    h = [torch.empty_like(x), spread(x, ld)]
    rstd = torch.empty(M, dtype=torch.float32, device="cuda")
    for i, xs in enumerate((x, h[1])):                      # the second time in place
        binding.check(binding.rms_norm(M, N, TYPE["bf16"], xs, xs.stride(0), r, N, g, 1e-5, h[i], h[i].stride(0), y[i], N, q[i], N, scale[i], M, rstd, stream()))
    assert same(h[0], h[1]) and same(y[0], y[1]) and same(q[0], q[1]) and torch.equal(scale[0], scale[1])
    dx, dg = [torch.empty_like(x) for _ in range(2)], [torch.empty(N, dtype=torch.float32, device="cuda") for _ in range(2)]
    size = binding.rms_norm_grad_workspace_bytes(M, N)
    ws = torch.empty(size, dtype=torch.uint8, device="cuda")
    for i in range(2):
        binding.check(binding.rms_norm_grad(M, N, TYPE["bf16"], dy, N, h[i], h[i].stride(0), g, rstd, None, 0, dx[i], N, dg[i], ws, size, stream()))
    assert same(dx[0], dx[1]) and torch.equal(dg[0], dg[1])
    for i in range(2):
        binding.check(binding.quantize_e4m3_rows(M, N // 2, TYPE["bf16"], binding.ACT_SWIGLU, h[i], h[i].stride(0), q[i], N, scale[i], M, stream()))
    assert same(q[0], q[1]) and torch.equal(scale[0][:4], scale[1][:4])
    blocks = [torch.empty(ceil128(M), ceil128(N), dtype=torch.float32, device="cuda") for _ in range(2)]
    for i in range(2):
        binding.check(binding.quantize_e4m3_blocks(M, N, TYPE["bf16"], h[i], h[i].stride(0), q[i], N, blocks[i], ceil128(N), stream()))
    assert same(q[0], q[1]) and torch.equal(blocks[0], blocks[1])


@pytest.mark.parametrize("ld", [1 << 22, (1 << 22) + 16])        # the tiled kernels' longest pitch, and one beyond it
@pytest.mark.parametrize("c", ["bf16", "f32"])
def test_e4m3_product_of_rows_far_apart(ld, c):
    M, N, K = 1200, 1100, 400
    gen = torch.Generator().manual_seed(2)
    a, b = (torch.randint(-8, 9, s, generator=gen).float().to(DT["e4m3"]).cuda() for s in ((M, K), (N, K)))
    sa, sb = torch.rand(ceil128(K), M, generator=gen).cuda(), torch.rand(ceil128(N), ceil128(K), generator=gen).cuda()
    c0 = torch.empty(M, N, dtype=DT[c], device="cuda")
    c1 = torch.empty((M - 1) * ld + N, dtype=DT[c], device="cuda").as_strided((M, N), (ld, 1))
    far = spread(a, ld), spread(b, ld)
    binding.check(binding.gemm_e4m3_block(M, N, K, a, K, sa, M, b, K, sb, ceil128(K), c0, N, TYPE[c], stream()))
    binding.check(binding.gemm_e4m3_block(M, N, K, far[0], ld, sa, M, far[1], ld, sb, ceil128(K), c1, ld, TYPE[c], stream()))
    if ld <= 1 << 22:
        assert same(c0, c1)                                 # the same kernel
    else:                                                   # another one, whose scaled sums have another order
        a64, b64 = a.double().cpu().numpy() * spread_rows(sa.cpu().double().numpy(), K), b.double().cpu().numpy() * spread_blocks(sb.cpu().double().numpy(), N, K)
        want, bound = a64 @ b64.T, result_bound(a64 @ b64.T, abs(a64) @ abs(b64.T), c)
        assert_within(c0.double().cpu().numpy(), want, bound, "rows next to each other")
        assert_within(c1.double().cpu().numpy(), want, bound, "rows far apart")


@pytest.mark.parametrize("ld", [1 << 22, (1 << 22) + 8])
def test_grouped_products_of_rows_far_apart(ld):
    """Rows and experts far apart: A and C 1100 rows (9 GB each), B of expert 2 behind 2^32 elements."""
    T, N, K, E, far = 1100, 136, 264, 3, (1 << 31) + 8
    gen = torch.Generator().manual_seed(3)
    offsets = torch.tensor([0, 500, 500, T], dtype=torch.int32).cuda()
    a, dc = (torch.randint(-4, 5, s, generator=gen).half().cuda() for s in ((T, K), (T, N)))
    b = torch.randint(-4, 5, (E, K, N), generator=gen).half().cuda()
    bf = torch.empty(2 * far + K * N, dtype=torch.float16, device="cuda").as_strided((E, K, N), (far, N, 1))
    bf.copy_(b)
    af, cf = spread(a, ld), spread(dc, ld)
    f = TYPE["f16"]

    def run(a, dc, b):
        c = spread(torch.zeros(T, N, dtype=torch.float16, device="cuda"), dc.stride(0))
        da = spread(torch.zeros(T, K, dtype=torch.float16, device="cuda"), a.stride(0))
        db = torch.empty(E, K, N, dtype=torch.float32, device="cuda")
        binding.check(binding.gemm_grouped(T, N, K, E, offsets, f, a, a.stride(0), b, N, b.stride(0), c, c.stride(0), f, stream()))
        binding.check(binding.gemm_grouped_grad_a(T, N, K, E, offsets, f, dc, dc.stride(0), b, N, b.stride(0), da, da.stride(0), f, stream()))
        binding.check(binding.gemm_grouped_grad_b(T, N, K, E, offsets, f, a, a.stride(0), dc, dc.stride(0), db, N, K * N, TYPE["f32"], stream()))
        return c, da, db
    for x, y in zip(run(a, dc, b), run(af, cf, bf)):
        assert same(x, y)


def test_more_rows_than_a_launch_takes():
    """5 million rows: as many results as in parts of a million."""
    M, N, part = 5_000_001, 16, 1_000_003
    x = torch.randn(M, N, device="cuda", generator=torch.Generator("cuda").manual_seed(4)).half()
    r, g = x.flip(0).contiguous(), torch.ones(N, device="cuda").half()

    def run(pieces):
        h, y, q = torch.empty_like(x), torch.empty_like(x), torch.empty(M, N, dtype=DT["e4m3"], device="cuda")
        q2, scale2 = torch.empty_like(q), torch.empty(1, M, dtype=torch.float32, device="cuda")
        scale, rstd = torch.empty(1, M, dtype=torch.float32, device="cuda"), torch.empty(M, dtype=torch.float32, device="cuda")
        for i, n in pieces:
            binding.check(binding.rms_norm(n, N, TYPE["f16"], x[i:], N, r[i:], N, g, 1e-5, h[i:], N, y[i:], N, q[i:], N, scale[0, i:], M, rstd[i:], stream()))
            binding.check(binding.quantize_e4m3_rows(n, N, TYPE["f16"], binding.ACT_NONE, x[i:], N, q2[i:], N, scale2[0, i:], M, stream()))
        return h, y, q, scale, rstd, q2, scale2
    for a, b in zip(run([(0, M)]), run([(i, min(part, M - i)) for i in range(0, M, part)])):
        assert same(a, b)
