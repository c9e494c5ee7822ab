"""Products of e4m3 matrices with block scales and products grouped by expert, with their gradients, against their definitions
in 64 bits: sizes around the tiles, short last blocks, odd sizes and pitches, experts without rows, rows without an expert, one row."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2108_13191_amd import binding                                                                   # noqa: E402
from ops_util import (LEAST, TYPE, UNIT, Mat, assert_within, ceil128, e4m3_values, offsets_of, result_bound, spread_blocks,   # noqa: E402
                      spread_rows, stream)


def up16(n):
    return (n + 15) // 16 * 16


def run_e4m3(M, N, K, c, counts=None, pad=0, offset=0, integers=False, seed=0, ldc=None, c_offset=0):
    """Runs the (grouped) e4m3 product and checks it; returns the result.  counts: rows of each expert, less than M leaves rows over."""
    rng = np.random.default_rng(seed)
    E = 1 if counts is None else len(counts)
    lda, kb, nb = (up16(K) + pad if offset % 16 == 0 and pad % 16 == 0 else K + pad), ceil128(K), ceil128(N)
    A = Mat("e4m3", M, K, lda, offset, e4m3_values(rng, M, K, integers=integers))
    B = Mat("e4m3", N, K, lda, offset, e4m3_values(rng, E, N, K, integers=integers), batch=E)
    if integers:
        sa, sb = 2.0 ** rng.integers(-2, 3, size=(kb, M)), 2.0 ** rng.integers(-2, 3, size=(E, nb, kb))
    else:
        sa, sb = np.exp(rng.standard_normal((kb, M))) / 100, np.exp(rng.standard_normal((E, nb, kb))) / 100
    SA, SB = Mat("f32", kb, M, M + 3, 1, sa), Mat("f32", nb, kb, kb + 1, 2, sb, batch=E)
    C = Mat(c, M, N, ldc or N + 5, c_offset)
    if counts is None:
        rc = binding.gemm_e4m3_block(M, N, K, A.ptr, A.ld, SA.ptr, SA.ld, B.ptr, B.ld, SB.ptr, SB.ld, C.ptr, C.ld, TYPE[c], stream())
        off = [0, M]
    else:
        off = offsets_of(counts)
        dev = torch.from_numpy(off).cuda()
        rc = binding.gemm_e4m3_block_grouped(M, N, K, E, dev, A.ptr, A.ld, SA.ptr, SA.ld, B.ptr, B.ld, B.stride, SB.ptr, SB.ld, SB.stride,
                                             C.ptr, C.ld, TYPE[c], stream())
    assert rc == binding.OK, binding.strerror(rc)
    torch.cuda.synchronize()
    a = A.values() * spread_rows(SA.values(), K)
    b, s = B.values().reshape(E, N, K), SB.values().reshape(E, nb, kb)
    want, mag = np.full((M, N), float(Mat(c, 1, 1).values()[0, 0])), np.zeros((M, N))
    for e in range(E):
        rows = slice(off[e], off[e + 1])
        w = b[e] * spread_blocks(s[e], N, K)
        want[rows], mag[rows] = a[rows] @ w.T, np.abs(a[rows]) @ np.abs(w).T
    got = C.fetch()
    if integers:
        # every product and sum is exact in f32; the result rounds once
        assert np.array_equal(got, torch.from_numpy(want).to(torch.float32).to({"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[c]).double().numpy())
    else:
        assert_within(got, want, result_bound(want, mag, c), f"e4m3 {(M, N, K)} {counts}")
    return got


SIZES = [(1, 1, 1), (1, 16, 128), (1, 4096, 2048), (3, 7, 5), (16, 256, 512), (17, 250, 384), (40, 512, 1024), (64, 129, 260), (100, 1000, 1000),
         (128, 128, 128), (129, 257, 200), (255, 256, 256), (257, 300, 384), (300, 520, 1000), (512, 512, 2048), (513, 770, 640)]


@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("c", ["f16", "bf16", "f32"])
def test_e4m3_product(M, N, K, c):
    run_e4m3(M, N, K, c, seed=M + N + K)


@pytest.mark.parametrize("M,N,K", SIZES)
def test_e4m3_product_of_integers_is_exact(M, N, K):
    run_e4m3(M, N, K, "f32", integers=True, seed=M)


@pytest.mark.parametrize("M,N,K", [(9, 33, 130), (200, 300, 257), (300, 264, 512), (33, 130, 1024)])
@pytest.mark.parametrize("pad,offset", [(16, 0), (48, 16), (1, 0), (0, 3), (7, 5)])
def test_e4m3_pitches_and_addresses(M, N, K, pad, offset):
    run_e4m3(M, N, K, "f32", pad=pad, offset=offset, seed=pad)


@pytest.mark.parametrize("ldc,c_offset", [(301, 1), (304, 0), (300, 3)])
@pytest.mark.parametrize("c", ["f16", "f32"])
def test_e4m3_result_of_any_pitch(ldc, c_offset, c):
    run_e4m3(260, 299, 384, c, ldc=ldc, c_offset=c_offset)
    run_e4m3(20, 299, 384, c, ldc=ldc, c_offset=c_offset)


COUNTS = [[5], [0, 0, 3, 0], [1, 1, 1, 1], [16, 17, 0, 15], [256, 0, 300, 1], [130, 127, 129, 0, 64], [0, 0, 0], [2] * 70 + [0] * 59 + [33]]


@pytest.mark.parametrize("counts", COUNTS, ids=str)
@pytest.mark.parametrize("N,K", [(64, 128), (300, 520), (130, 77)])
def test_e4m3_grouped(counts, N, K):
    run_e4m3(sum(counts), N, K, "bf16", counts, seed=N)
    run_e4m3(sum(counts) + 9, N, K, "f32", counts, seed=K)            # nine rows without an expert


# Large products, of 2^22 results and more: 16-bit results come from the e4m3 matrix instructions, which add products with the bits below
# 2^-13 of the largest one's exponent of a group cut off.  A product of a group of 8 is then off by at most 2^-13 of the group's largest,
# a sum by 8 * 2^-13 of its magnitudes at the very most; over many results errors of random sign stay below 2^-15 of their norm.
LARGE = [(3400, 3700, 300), (4096, 3585, 640), (3333, 4500, 129), (4730, 4400, 272), (2048, 2050, 200)]
MIDDLE = [(1200, 1300, 300), (1025, 1601, 520), (900, 2000, 128)]         # between those and the ones for few rows: 128 x 128 tiles


def large_e4m3(M, N, K, c, counts=None, integers=False):
    """Runs and returns (result, expected, magnitudes) in 64 bits, computed on the GPU."""
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    E, kb, nb, ld = (1 if counts is None else len(counts)), ceil128(K), ceil128(N), up16(K) + 16
    if integers:
        draw = lambda *s: torch.randint(-8, 9, s, device="cuda", generator=g).float()                          # noqa: E731
        scale = lambda *s: 2.0 ** torch.randint(-2, 3, s, device="cuda", generator=g).float()                 # noqa: E731
    else:
        draw = lambda *s: (torch.randn(s, device="cuda", generator=g) * 100).clamp(-448, 448)                  # noqa: E731
        scale = lambda *s: torch.exp(torch.randn(s, device="cuda", generator=g)) / 100                         # noqa: E731
    a, b = draw(M, K).to(torch.float8_e4m3fn), draw(E, N, K).to(torch.float8_e4m3fn)
    # what lies between the rows' ends and the pitch is NaN (0x7f)
    A = torch.full((M, ld), 0x7F, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    B = torch.full((E, N, ld), 0x7F, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    A[:, :K], B[:, :, :K] = a, b
    sa, sb = scale(kb, M), scale(E, nb, kb)
    C = torch.full((M + 1, N + 3), -77.0, device="cuda").to({"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[c])
    off = [0, M] if counts is None else offsets_of(counts).tolist()
    if counts is None:
        rc = binding.gemm_e4m3_block(M, N, K, A, ld, sa, M, B, ld, sb, kb, C, N + 3, TYPE[c], stream())
    else:
        dev = torch.tensor(off, dtype=torch.int32, device="cuda")
        rc = binding.gemm_e4m3_block_grouped(M, N, K, E, dev, A, ld, sa, M, B, ld, N * ld, sb, kb, nb * kb, C, N + 3, TYPE[c], stream())
    assert rc == binding.OK, binding.strerror(rc)
    want, mag = torch.full((M, N), -77.0, dtype=torch.float64, device="cuda"), torch.zeros(M, N, dtype=torch.float64, device="cuda")
    x = a.double() * sa.double().t().repeat_interleave(128, 1)[:, :K]
    for e in range(E):
        rows = slice(off[e], off[e + 1])
        w = b[e].double() * sb[e].double().repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
        want[rows], mag[rows] = x[rows] @ w.t().contiguous(), x[rows].abs() @ w.abs().t().contiguous()
    assert bool((C[M] == -77.0).all()) and bool((C[:, N:] == -77.0).all()), "memory outside the result was written"
    return C[:M, :N].double().cpu().numpy(), want.cpu().numpy(), mag.cpu().numpy()


@pytest.mark.parametrize("M,N,K", LARGE)
@pytest.mark.parametrize("c", ["f16", "bf16", "f32"])
def test_e4m3_large_product(M, N, K, c):
    got, want, mag = large_e4m3(M, N, K, c)
    if c == "f32":
        assert_within(got, want, result_bound(want, mag, c), f"e4m3 {(M, N, K)}")
    else:
        # beyond what the type holds the result is infinite: 65520 and up in f16
        over = np.abs(want) >= 65520.0 if c == "f16" else np.zeros(want.shape, bool)
        near = np.abs(np.abs(want) - 65520.0) <= 2.0 ** -10 * mag
        assert np.array_equal(np.isinf(got) & ~near, over & ~near if c == "f16" else over)
        got, want, mag = got[~over & np.isfinite(got)], want[~over & np.isfinite(got)], mag[~over & np.isfinite(got)]
        assert_within(got, want, 2.0 ** -10 * mag * 1.01 + np.abs(want) * UNIT[c] + LEAST[c], f"e4m3 {(M, N, K)}")
        assert np.linalg.norm(got - want) <= (UNIT[c] + 2.0 ** -15) * np.linalg.norm(want)


@pytest.mark.parametrize("M,N,K", LARGE)
@pytest.mark.parametrize("c", ["f16", "bf16", "f32"])
def test_e4m3_large_product_of_integers(M, N, K, c):
    """Products of integers up to 8 lie within 13 bits of each other: nothing is cut off, every sum is exact, the result rounds once."""
    got, want, _ = large_e4m3(M, N, K, c, integers=True)
    assert np.array_equal(got, torch.from_numpy(want).float().to({"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[c]).double().numpy())


@pytest.mark.parametrize("M,N,K", MIDDLE)
@pytest.mark.parametrize("c", ["f16", "bf16", "f32"])
def test_e4m3_middle_product(M, N, K, c):
    """Exact products and f32 sums whatever the result's type."""
    got, want, mag = large_e4m3(M, N, K, c)
    inside = np.abs(want) < (65504.0 if c == "f16" else np.inf)
    assert_within(got[inside], want[inside], result_bound(want, mag, c)[inside], f"e4m3 {(M, N, K)}")
    got, want, mag = large_e4m3(M, N, K, c, integers=True)
    assert np.array_equal(got, torch.from_numpy(want).float().to({"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[c]).double().numpy())


@pytest.mark.parametrize("counts", [[1000, 0, 700, 1300, 33], [257, 256, 1, 2900], [3000], [100, 90, 0, 64, 129, 128] * 2, [30, 0, 41, 25] * 5,
                                    [100, 90, 0, 64, 129, 128] * 8], ids=str)
@pytest.mark.parametrize("c,extra", [("bf16", 0), ("f32", 11)])
def test_e4m3_large_grouped(counts, c, extra):
    got, want, mag = large_e4m3(sum(counts) + extra, 4100, 390, c, counts, integers=True)
    want = torch.from_numpy(want).float().to({"bf16": torch.bfloat16, "f32": torch.float32}[c]).double().numpy()
    assert np.array_equal(got, want)


def test_e4m3_nan_stays_in_its_row_and_column():
    M, N, K = 300, 300, 260
    rng = np.random.default_rng(0)
    a, b = e4m3_values(rng, M, K), e4m3_values(rng, N, K)
    a[7, 259] = np.nan
    b[299, 0] = np.nan
    sa, sb = np.ones((3, M)), np.ones((3, 3))
    sa[1, 40] = np.nan
    for rows in (M, 20):
        A, B, SA, SB, C = Mat("e4m3", rows, K, 272, 0, a[:rows]), Mat("e4m3", N, K, 272, 0, b), Mat("f32", 3, rows, None, 0, sa[:, :rows]), Mat("f32", 3, 3, None, 0, sb), Mat("f32", rows, N)
        assert binding.gemm_e4m3_block(rows, N, K, A.ptr, 272, SA.ptr, rows, B.ptr, 272, SB.ptr, 3, C.ptr, N, TYPE["f32"], stream()) == binding.OK
        torch.cuda.synchronize()
        want = np.zeros((rows, N), bool)
        want[7, :], want[:, 299] = True, True
        if rows > 40:
            want[40, :] = True
        assert np.array_equal(np.isnan(C.fetch()), want)


def test_e4m3_without_a_sum_is_zeros():
    C = Mat("f16", 70, 33)
    assert binding.gemm_e4m3_block(70, 33, 0, None, 0, None, 0, None, 0, None, 0, C.ptr, 33, TYPE["f16"], stream()) == binding.OK
    torch.cuda.synchronize()
    assert not C.fetch().any()


def test_e4m3_block_gradient_by_the_same_operator():
    """dC B as a product with B transposed, whose block scales transpose with it."""
    M, N, K = 70, 384, 256
    rng = np.random.default_rng(3)
    dc, b = e4m3_values(rng, M, N), e4m3_values(rng, N, K)
    s_dc, sb = np.exp(rng.standard_normal((3, M))), np.exp(rng.standard_normal((3, 2)))
    D, BT, S, SB, dA = Mat("e4m3", M, N, None, 0, dc), Mat("e4m3", K, N, None, 0, b.T.copy()), Mat("f32", 3, M, None, 0, s_dc), Mat("f32", 2, 3, None, 0, sb.T.copy()), Mat("f32", M, K)
    assert binding.gemm_e4m3_block(M, K, N, D.ptr, N, S.ptr, M, BT.ptr, N, SB.ptr, 3, dA.ptr, K, TYPE["f32"], stream()) == binding.OK
    torch.cuda.synchronize()
    x, w = dc * spread_rows(S.values(), N), b * spread_blocks(SB.values().T, N, K)
    assert_within(dA.fetch(), x @ w, result_bound(x @ w, np.abs(x) @ np.abs(w), "f32"), "gradient")


# ---- 16 bits: forward, gradient of A, gradient of B -------------------------------------------------------------------------

def run_grouped(counts, N, K, type, out, extra=0, pad=0, offset=0, seed=0, integers=False):
    rng = np.random.default_rng(seed)
    T, E, off = sum(counts) + extra, len(counts), offsets_of(counts)
    draw = (lambda *s: rng.integers(-2, 3, size=s).astype(np.float64)) if integers else (lambda *s: rng.standard_normal(s))
    A, D = Mat(type, T, K, K + pad, offset, draw(T, K)), Mat(type, T, N, N + pad, offset, draw(T, N))
    B = Mat(type, K, N, N + pad, offset, draw(E, K, N), batch=E)
    C, dA, dB = Mat(out, T, N, N + pad, offset), Mat(out, T, K, K + pad, offset), Mat(out, K, N, N + pad, offset, batch=E)
    dev = torch.from_numpy(off).cuda()
    s = stream()
    for rc in (binding.gemm_grouped(T, N, K, E, dev, TYPE[type], A.ptr, A.ld, B.ptr, B.ld, B.stride, C.ptr, C.ld, TYPE[out], s),
               binding.gemm_grouped_grad_a(T, N, K, E, dev, TYPE[type], D.ptr, D.ld, B.ptr, B.ld, B.stride, dA.ptr, dA.ld, TYPE[out], s),
               binding.gemm_grouped_grad_b(T, N, K, E, dev, TYPE[type], A.ptr, A.ld, D.ptr, D.ld, dB.ptr, dB.ld, dB.stride, TYPE[out], s)):
        assert rc == binding.OK, binding.strerror(rc)
    torch.cuda.synchronize()
    a, d, b = A.values(), D.values(), B.values().reshape(E, K, N)
    untouched = float(Mat(out, 1, 1).values()[0, 0])
    c, da, db = np.full((T, N), untouched), np.full((T, K), untouched), np.zeros((E, K, N))
    mc, mda, mdb = np.zeros((T, N)), np.zeros((T, K)), np.zeros((E, K, N))
    for e in range(E):
        r = slice(off[e], off[e + 1])
        c[r], mc[r] = a[r] @ b[e], np.abs(a[r]) @ np.abs(b[e])
        da[r], mda[r] = d[r] @ b[e].T, np.abs(d[r]) @ np.abs(b[e]).T
        db[e], mdb[e] = a[r].T @ d[r], np.abs(a[r]).T @ np.abs(d[r])
    for name, got, want, mag in (("C", C.fetch(), c, mc), ("dA", dA.fetch(), da, mda), ("dB", dB.fetch().reshape(E, K, N), db, mdb)):
        if integers:
            assert np.array_equal(got, want), name
        else:
            assert_within(got, want, result_bound(want, mag, out), f"{name} {counts} {(N, K)}")


@pytest.mark.parametrize("counts", COUNTS, ids=str)
@pytest.mark.parametrize("N,K", [(64, 128), (264, 328), (130, 77), (512, 256)])
def test_grouped_and_gradients(counts, N, K):
    run_grouped(counts, N, K, "bf16", "f32", seed=N)
    run_grouped(counts, N, K, "f16", "f16", extra=5, seed=K)


@pytest.mark.parametrize("type", ["f16", "bf16"])
@pytest.mark.parametrize("N,K", [(1, 1), (8, 8), (24, 72), (256, 64), (384, 640), (1000, 24)])
def test_grouped_integers_are_exact(type, N, K):
    run_grouped([40, 0, 1, 300], N, K, type, "f32", extra=3, integers=True, seed=N)


@pytest.mark.parametrize("type,out", [("f16", "f16"), ("bf16", "f32")])
@pytest.mark.parametrize("counts,N,K", [([1000, 0, 700, 1300, 33], 4104, 392), ([3000], 3700, 130), ([257, 256, 1, 2900], 392, 4200)], ids=str)
def test_grouped_large(type, out, counts, N, K):
    """Tiles that fill the chip, forward and both gradients, on integers (exact sums; f16 results round once)."""
    g = torch.Generator(device="cuda").manual_seed(N + K)
    T, E, off = sum(counts) + 7, len(counts), offsets_of(counts).tolist()
    dt, do = {"f16": torch.float16, "bf16": torch.bfloat16}[type], {"f16": torch.float16, "f32": torch.float32}[out]
    ln, lk = (N + 15) // 8 * 8, (K + 15) // 8 * 8

    def operand(*shape):
        buf = torch.full(shape, float("nan"), device="cuda").to(dt)
        return buf
    A, D, B = operand(T, lk), operand(T, ln), operand(E, K, ln)
    for t, n in ((A, K), (D, N), (B, N)):
        t[..., :n] = torch.randint(-2, 3, (*t.shape[:-1], n), device="cuda", generator=g).to(dt)
    C, dA, dB = (torch.full(s, -77.0, device="cuda").to(do) for s in ((T + 1, ln), (T + 1, lk), (E, K, ln)))
    dev, s = torch.tensor(off, dtype=torch.int32, device="cuda"), stream()
    binding.check(binding.gemm_grouped(T, N, K, E, dev, TYPE[type], A, lk, B, ln, K * ln, C, ln, TYPE[out], s))
    binding.check(binding.gemm_grouped_grad_a(T, N, K, E, dev, TYPE[type], D, ln, B, ln, K * ln, dA, lk, TYPE[out], s))
    binding.check(binding.gemm_grouped_grad_b(T, N, K, E, dev, TYPE[type], A, lk, D, ln, dB, ln, K * ln, TYPE[out], s))
    c, da, db = (torch.full(t.shape, -77.0, device="cuda", dtype=torch.float64) for t in (C, dA, dB))
    for e in range(E):
        r = slice(off[e], off[e + 1])
        a, d, b = A[r, :K].double(), D[r, :N].double(), B[e, :, :N].double()
        c[r, :N], da[r, :K], db[e, :, :N] = a @ b, d @ b.t().contiguous(), a.t().contiguous() @ d
    for name, got, want in (("C", C, c), ("dA", dA, da), ("dB", dB, db)):
        assert torch.equal(got, want.float().to(do)), name


@pytest.mark.parametrize("pad,offset", [(8, 0), (24, 8), (1, 0), (0, 1), (3, 2)])
@pytest.mark.parametrize("N,K", [(72, 136), (33, 65)])
def test_grouped_pitches_and_addresses(pad, offset, N, K):
    run_grouped([20, 0, 133, 5], N, K, "bf16", "bf16", pad=pad, offset=offset, seed=pad)


def test_grouped_gradients_are_those_of_the_forward_product():
    """Differences of a scalar of the forward product, L = sum(C * D), in A and in B, against the gradients (f32 results;
    L is linear in each, so a difference of any step is exact up to the sums' rounding)."""
    counts, N, K, type = [7, 0, 20], 24, 40, "f16"
    rng = np.random.default_rng(11)
    T, E = sum(counts), len(counts)
    a, d, b = (rng.integers(-3, 4, size=s).astype(np.float64) for s in ((T, K), (T, N), (E, K, N)))
    dev = torch.from_numpy(offsets_of(counts)).cuda()

    def forward(a, b):
        A, B, C = Mat(type, T, K, None, 0, a), Mat(type, K, N, None, 0, b, batch=E), Mat("f32", T, N)
        assert binding.gemm_grouped(T, N, K, E, dev, TYPE[type], A.ptr, K, B.ptr, N, B.stride, C.ptr, N, TYPE["f32"], stream()) == binding.OK
        torch.cuda.synchronize()
        return float((C.fetch() * d).sum())

    A, B, D = Mat(type, T, K, None, 0, a), Mat(type, K, N, None, 0, b, batch=E), Mat(type, T, N, None, 0, d)
    dA, dB = Mat("f32", T, K), Mat("f32", K, N, batch=E)
    assert binding.gemm_grouped_grad_a(T, N, K, E, dev, TYPE[type], D.ptr, N, B.ptr, N, B.stride, dA.ptr, K, TYPE["f32"], stream()) == binding.OK
    assert binding.gemm_grouped_grad_b(T, N, K, E, dev, TYPE[type], A.ptr, K, D.ptr, N, dB.ptr, N, dB.stride, TYPE["f32"], stream()) == binding.OK
    torch.cuda.synchronize()
    ga, gb = dA.fetch(), dB.fetch()
    for _ in range(6):
        i, k, e, n = rng.integers(T), rng.integers(K), rng.integers(E), rng.integers(N)
        up, down = a.copy(), a.copy()
        up[i, k] += 1
        down[i, k] -= 1
        assert (forward(up, b) - forward(down, b)) / 2 == ga[i, k]          # small integers: exact
        up, down = b.copy(), b.copy()
        up[e, k, n] += 1
        down[e, k, n] -= 1
        assert (forward(a, up) - forward(a, down)) / 2 == gb[e, k, n]


@pytest.mark.parametrize("counts,N,K,type", [([257, 256, 1, 2900], 392, 4200, "bf16"), ([3000, 1000], 3000, 200, "f16"), ([90] * 40, 1000, 640, "f16")], ids=str)
def test_grouped_repeats_to_the_bit(counts, N, K, type):
    """Forty launches of each product in a row, on integers (every order of sums exact): a copy into LDS that is read before it has
    arrived would show in some of them."""
    g = torch.Generator(device="cuda").manual_seed(1)
    T, E, dt = sum(counts), len(counts), {"f16": torch.float16, "bf16": torch.bfloat16}[type]
    A, D, B = (torch.randint(-2, 3, s, device="cuda", generator=g).to(dt) for s in ((T, K), (T, N), (E, K, N)))
    out = [[torch.zeros(s, device="cuda") for s in ((T, N), (T, K), (E, K, N))] for _ in range(2)]
    off = offsets_of(counts).tolist()
    for e in range(E):
        r = slice(off[e], off[e + 1])
        a, d, b = A[r].float(), D[r].float(), B[e].float()
        out[1][0][r], out[1][1][r], out[1][2][e] = a @ b, d @ b.t().contiguous(), a.t().contiguous() @ d
    dev, s = torch.tensor(off, dtype=torch.int32, device="cuda"), stream()
    C, dA, dB = out[0]
    for i in range(40):
        for t in out[0]:
            t.zero_()
        binding.check(binding.gemm_grouped(T, N, K, E, dev, TYPE[type], A, K, B, N, K * N, C, N, TYPE["f32"], s))
        binding.check(binding.gemm_grouped_grad_a(T, N, K, E, dev, TYPE[type], D, N, B, N, K * N, dA, K, TYPE["f32"], s))
        binding.check(binding.gemm_grouped_grad_b(T, N, K, E, dev, TYPE[type], A, K, D, N, dB, N, K * N, TYPE["f32"], s))
        for name, got, want in zip(("C", "dA", "dB"), out[0], out[1]):
            assert torch.equal(got, want), f"{name} in launch {i}"


@pytest.mark.parametrize("M,N,K,c", [(4096, 3585, 640, "bf16"), (4096, 3585, 640, "f32"), (1200, 1300, 2000, "f32"), (24, 8192, 4096, "f32")])
def test_e4m3_repeats_to_the_bit(M, N, K, c):
    g = torch.Generator(device="cuda").manual_seed(1)
    a, b = (torch.randint(-4, 5, s, device="cuda", generator=g).float().to(torch.float8_e4m3fn) for s in ((M, K), (N, K)))
    ld = up16(K)
    A, B = torch.zeros(M, ld, dtype=torch.float8_e4m3fn, device="cuda"), torch.zeros(N, ld, dtype=torch.float8_e4m3fn, device="cuda")
    A[:, :K], B[:, :K] = a, b
    sa, sb = torch.ones(ceil128(K), M, device="cuda"), torch.ones(ceil128(N), ceil128(K), device="cuda")
    want = (a.float() @ b.float().t().contiguous()).to({"bf16": torch.bfloat16, "f32": torch.float32}[c])
    C = torch.zeros_like(want)
    for i in range(40):
        C.zero_()
        binding.check(binding.gemm_e4m3_block(M, N, K, A, ld, sa, M, B, ld, sb, sb.stride(0), C, N, TYPE[c], stream()))
        assert torch.equal(C, want), f"launch {i}"


def test_offsets_out_of_range_and_decreasing_stay_inside():
    """Offsets below 0, above T and decreasing: what is in range is computed, nothing else is touched."""
    T, N, K = 50, 40, 64
    rng = np.random.default_rng(5)
    a, b = rng.integers(-2, 3, size=(T, K)).astype(np.float64), rng.integers(-2, 3, size=(3, K, N)).astype(np.float64)
    A, B, C = Mat("f16", T, K, None, 0, a), Mat("f16", K, N, None, 0, b, batch=3), Mat("f32", T, N)
    off = torch.tensor([-7, 20, 10, 2_000_000_000], dtype=torch.int32, device="cuda")       # groups 0 .. 20, none, 10 .. 50
    assert binding.gemm_grouped(10, N, K, 1, off, TYPE["f16"], A.ptr, K, B.ptr, N, B.stride, C.ptr, N, TYPE["f32"], stream()) == binding.OK
    torch.cuda.synchronize()
    got = C.fetch()
    assert np.array_equal(got[:10], a[:10] @ b[0]) and (got[10:] == -1234.0).all()
    off = torch.tensor([30, 20, 20, 2_000_000_000], dtype=torch.int32, device="cuda")       # none, none, 20 .. 50
    C = Mat("f32", T, N)
    assert binding.gemm_grouped(T, N, K, 3, off, TYPE["f16"], A.ptr, K, B.ptr, N, B.stride, C.ptr, N, TYPE["f32"], stream()) == binding.OK
    torch.cuda.synchronize()
    got = C.fetch()
    assert np.array_equal(got[20:], a[20:] @ b[2]) and (got[:20] == -1234.0).all()


def test_one_matrix_for_all_experts():
    """A stride of 0: every group reads the same B."""
    counts, N, K = [30, 3], 72, 64
    rng = np.random.default_rng(8)
    a, b = rng.integers(-2, 3, size=(33, K)).astype(np.float64), rng.integers(-2, 3, size=(K, N)).astype(np.float64)
    A, B, C = Mat("bf16", 33, K, None, 0, a), Mat("bf16", K, N, None, 0, b), Mat("f32", 33, N)
    dev = torch.from_numpy(offsets_of(counts)).cuda()
    assert binding.gemm_grouped(33, N, K, 2, dev, TYPE["bf16"], A.ptr, K, B.ptr, N, 0, C.ptr, N, TYPE["f32"], stream()) == binding.OK
    torch.cuda.synchronize()
    assert np.array_equal(C.fetch(), a @ b)


def test_a_captured_graph_gives_the_eager_results():
    """The grouped product in a HIP graph, replayed on new inputs and new offsets, with eager work between the replays."""
    T, N, K, E = 200, 264, 256, 4
    g = torch.Generator(device="cuda").manual_seed(2)
    a = torch.randn(T, K, device="cuda", generator=g).half()
    b = torch.randn(E, K, N, device="cuda", generator=g).half()
    off = torch.tensor([0, 50, 50, 120, 200], dtype=torch.int32, device="cuda")
    c, eager = torch.zeros(T, N, device="cuda"), torch.zeros(T, N, device="cuda")

    def call(out):
        binding.check(binding.gemm_grouped(T, N, K, E, off, TYPE["f16"], a, K, b, N, K * N, out, N, TYPE["f32"], stream()))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(c)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(c)
    for ends in ([0, 50, 50, 120, 200], [0, 0, 200, 200, 200], [0, 1, 2, 199, 200]):
        off.copy_(torch.tensor(ends, dtype=torch.int32))
        a.copy_(torch.randn(T, K, device="cuda", generator=g))
        c.zero_()
        graph.replay()
        torch.cuda.synchronize()
        call(eager)
        torch.cuda.synchronize()
        assert torch.equal(c, eager)
