"""Each kernel form of the products of include/gemm_ops.h on shapes that reach it (ops_form_cases.py; which form a shape runs on is asked here too): integers, whose every
sum is exact, remainders in every dimension, NaN between the rows, and launches repeated to the bit."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import ops_form_cases as cases                                             # noqa: E402
from paper_2108_13191_amd import binding                                    # noqa: E402
from ops_util import DT, TYPE, ceil128, offsets_of, stream                 # noqa: E402

LAUNCHES = 12


def padded(t, ld):
    """The same matrices with rows `ld` elements apart, NaN between them."""
    wide = torch.full((*t.shape[:-1], ld), float("nan"), device="cuda").to(t.dtype)
    wide[..., :t.shape[-1]] = t
    return wide


def up(n, to):
    return (n + to - 1) // to * to


def canary(rows, cols, kind, batch=()):
    return torch.full((*batch, rows, cols), -77.0, device="cuda").to(DT[kind])


def repeat(out, want, call):
    for i in range(LAUNCHES):
        out.fill_(-77.0)
        binding.check(call())
        assert torch.equal(out, want), f"launch {i}"


@pytest.mark.parametrize("form,rows,N,K,c", cases.E4M3)
def test_e4m3(form, rows, N, K, c):
    counts = [rows] if isinstance(rows, int) else rows
    T, E, kb, nb, ld = sum(counts), len(counts), ceil128(K), ceil128(N), up(K, 16) + 16
    lone = isinstance(rows, int)
    T += 0 if lone else cases.EXTRA
    assert binding.product_form(binding.PRODUCT_E4M3, T, N, K, -1 if lone else E, ld, ld, TYPE[c]) == form
    g = torch.Generator("cuda").manual_seed(N + K)
    a, b = (torch.randint(-4, 5, s, device="cuda", generator=g).float() for s in ((T, K), (E, N, K)))
    sa, sb = (2.0 ** torch.randint(-2, 3, s, device="cuda", generator=g).float() for s in ((kb, T), (E, nb, kb)))
    A, B = padded(a.to(DT["e4m3"]), ld), padded(b.to(DT["e4m3"]), ld)
    off = torch.from_numpy(offsets_of(counts)).cuda()
    want = torch.full((T + 1, N + 3), -77.0, device="cuda").to(DT[c])
    x = a * sa.t().repeat_interleave(128, 1)[:, :K]
    ends = off.tolist()
    for e in range(E):
        w = b[e] * sb[e].repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
        r = slice(ends[e], ends[e + 1])
        want[r, :N] = (x[r].double() @ w.double().t().contiguous()).float().to(DT[c])
    C = torch.empty_like(want)
    if lone:
        repeat(C, want, lambda: binding.gemm_e4m3_block(T, N, K, A, ld, sa, T, B, ld, sb, kb, C, N + 3, TYPE[c], stream()))
    else:
        repeat(C, want, lambda: binding.gemm_e4m3_block_grouped(T, N, K, E, off, A, ld, sa, T, B, ld, N * ld, sb, kb, nb * kb, C, N + 3, TYPE[c], stream()))


def operands(counts, N, K, type, pad):
    g = torch.Generator("cuda").manual_seed(N + K)
    T, E = sum(counts) + cases.EXTRA, len(counts)
    a, d, b = (torch.randint(-2, 3, s, device="cuda", generator=g).to(DT[type]) for s in ((T, K), (T, N), (E, K, N)))
    off = torch.from_numpy(offsets_of(counts)).cuda()
    ln, lk = up(N, pad) + (8 if pad > 1 else 0), up(K, pad) + (8 if pad > 1 else 0)
    return T, E, a, d, b, off, ln, lk, [slice(*x) for x in zip(off.tolist(), off.tolist()[1:])]


def form_of(product, counts, N, K, lda, ldb, out):
    return binding.product_form(product, sum(counts) + cases.EXTRA, N, K, len(counts), lda, ldb, TYPE[out])


@pytest.mark.parametrize("type,out", [("f16", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("form,counts,N,K,pad", [(*c, 8) for c in cases.FORWARD] + [(*c, 1) for c in cases.UNALIGNED])
def test_forward(form, counts, N, K, pad, type, out):
    T, E, a, d, b, off, ln, lk, rows = operands(counts, N, K, type, pad)
    assert form_of(binding.PRODUCT_FORWARD, counts, N, K, lk, ln, out) == form
    A, B, want = padded(a, lk), padded(b, ln), canary(T + 1, ln, out)
    for e, r in enumerate(rows):
        want[r, :N] = (a[r].float() @ b[e].float()).to(want.dtype)
    C = torch.empty_like(want)
    repeat(C, want, lambda: binding.gemm_grouped(T, N, K, E, off, TYPE[type], A, lk, B, ln, K * ln, C, ln, TYPE[out], stream()))


@pytest.mark.parametrize("type,out", [("f16", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("form,counts,N,K,pad", [(*c, 8) for c in cases.GRAD_A] + [(*c, 1) for c in cases.UNALIGNED])
def test_gradient_of_a(form, counts, N, K, pad, type, out):
    T, E, a, d, b, off, ln, lk, rows = operands(counts, N, K, type, pad)
    assert form_of(binding.PRODUCT_GRAD_A, counts, N, K, ln, ln, out) == form
    D, B, want = padded(d, ln), padded(b, ln), canary(T + 1, lk, out)
    for e, r in enumerate(rows):
        want[r, :K] = (d[r].float() @ b[e].float().t()).to(want.dtype)
    dA = torch.empty_like(want)
    repeat(dA, want, lambda: binding.gemm_grouped_grad_a(T, N, K, E, off, TYPE[type], D, ln, B, ln, K * ln, dA, lk, TYPE[out], stream()))


@pytest.mark.parametrize("type,out", [("f16", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("form,counts,N,K,pad", [(*c, 8) for c in cases.GRAD_B] + [(*c, 1) for c in cases.UNALIGNED])
def test_gradient_of_b(form, counts, N, K, pad, type, out):
    T, E, a, d, b, off, ln, lk, rows = operands(counts, N, K, type, pad)
    assert form_of(binding.PRODUCT_GRAD_B, counts, N, K, lk, ln, out) == form
    A, D, want = padded(a, lk), padded(d, ln), canary(K, ln, out, (E,))
    for e, r in enumerate(rows):
        want[e, :, :N] = (a[r].float().t() @ d[r].float()).to(want.dtype)
    dB = torch.empty_like(want)
    repeat(dB, want, lambda: binding.gemm_grouped_grad_b(T, N, K, E, off, TYPE[type], A, lk, D, ln, dB, ln, K * ln, TYPE[out], stream()))


def test_e4m3_tiles_of_rows_far_apart():
    """Rows 2^22 elements apart, the tiled kernels' longest pitch: offsets within a tile pass 2^28 bytes, within a matrix 2^32."""
    M, N, K, ld = 1300, 1200, 400, 1 << 22
    assert binding.product_form(binding.PRODUCT_E4M3, M, N, K, -1, ld, ld, TYPE["f32"]) == "widened_128x128"
    g = torch.Generator("cuda").manual_seed(1)
    a, b = (torch.randint(-8, 9, s, device="cuda", generator=g).float() for s in ((M, K), (N, K)))
    sa, sb = (2.0 ** torch.randint(-2, 3, s, device="cuda", generator=g).float() for s in ((4, M), (10, 4)))

    def far(t):
        wide = torch.empty((t.shape[0] - 1) * ld + up(K, 16), dtype=torch.uint8, device="cuda").as_strided(t.shape, (ld, 1))
        return wide.copy_(t.to(DT["e4m3"]).view(torch.uint8)).view(DT["e4m3"])
    A, B, C = far(a), far(b), torch.empty(M, N, device="cuda")
    binding.check(binding.gemm_e4m3_block(M, N, K, A, ld, sa, M, B, ld, sb, 4, C, N, TYPE["f32"], stream()))
    want = (a * sa.t().repeat_interleave(128, 1)[:, :K]).double() @ (b * sb.repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]).double().t().contiguous()
    assert torch.equal(C, want.float())


@pytest.mark.parametrize("c", ["bf16", "f32"])
def test_many_experts_of_a_row_and_a_million_columns(c):
    """More tiles of few rows than a launch has workgroups: larger ones are taken."""
    E, N, K = 256, 1 << 20, 16
    assert binding.product_form(binding.PRODUCT_E4M3, E, N, K, E, K, K, TYPE[c]) in ("e4m3_128x128", "widened_128x128_short_groups")
    g = torch.Generator("cuda").manual_seed(1)
    a, b = (torch.randint(-4, 5, s, device="cuda", generator=g).float() for s in ((E, K), (N, K)))
    off, C = torch.arange(E + 1, dtype=torch.int32, device="cuda"), torch.empty(E, N, dtype=DT[c], device="cuda")
    binding.check(binding.gemm_e4m3_block_grouped(E, N, K, E, off, a.to(DT["e4m3"]), K, torch.ones(1, E, device="cuda"), E, b.to(DT["e4m3"]), K, 0, torch.ones(N // 128, 1, device="cuda"), 1, 0,
                                                  C, N, TYPE[c], stream()))
    assert torch.equal(C, (a @ b.t().contiguous()).to(DT[c]))
