"""Products of 8-bit integer matrices with scales for each token and channel, plain and by expert: sums are exact, so results are held to their definition's roundings."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2108_13191_amd import binding                                                  # noqa: E402
from ops_util import DT, LEAST, TYPE, UNIT, Mat, assert_within, offsets_of, stream            # noqa: E402
from layer_util import Ints                                                               # noqa: E402
from i8_form_cases import FORMS, GROUPED, up                                              # noqa: E402

I8 = torch.int8


def scales(rng, *shape):
    return (np.exp(rng.standard_normal(shape)) * 0.01).astype(np.float32).astype(np.float64)


def expected(a, sa, b, sb):
    """(sums below 2^31: exact in 64-bit floating point)"""
    return (a.astype(np.float64) @ b.astype(np.float64).T) * sa[:, None] * sb[None, :]


def bound(want, c):
    """The sum becomes f32, and is multiplied twice: three roundings; then one to the result's type."""
    off = np.abs(want) * 3.1 * 2.0 ** -24 + 2.0 ** -149
    return off + (np.abs(want) + off) * UNIT[c] + LEAST[c]


def run(M, N, K, c, lda, ldb, ldc, a_off=0, b_off=0, c_off=0, seed=0, low=-127):
    rng = np.random.default_rng(seed + M * N + K)
    a, b = rng.integers(low, 128, (M, K)), rng.integers(low, 128, (N, K))
    A, B, C = Ints(I8, M, K, lda, a_off, a), Ints(I8, N, K, ldb, b_off, b), Mat(c, M, N, ldc, c_off)
    SA, SB = Mat("f32", 1, M, None, 1, scales(rng, 1, M)), Mat("f32", 1, N, None, 3, scales(rng, 1, N))
    rc = binding.gemm_i8(M, N, K, A.ptr, A.ld, SA.ptr, B.ptr, B.ld, SB.ptr, C.ptr, C.ld, TYPE[c], stream())
    assert rc == binding.OK, binding.strerror(rc)
    torch.cuda.synchronize()
    want = expected(a, SA.values()[0], b, SB.values()[0])
    got = C.fetch()
    assert_within(got, want, bound(want, c), f"{M}x{N}x{K} {c}")
    return got


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 16, 16), (3, 5, 7), (16, 32, 128), (17, 33, 127), (15, 31, 129), (64, 64, 64), (65, 63, 65), (128, 128, 256), (129, 127, 255),
                                   (40, 1000, 300), (256, 256, 128), (257, 255, 640), (300, 520, 1000), (5, 4100, 2000)])
@pytest.mark.parametrize("c", ["f16", "bf16", "f32"])
def test_small_and_odd_sizes(M, N, K, c):
    run(M, N, K, c, up(K, 16), up(K, 16) + 16, N + 8)


@pytest.mark.parametrize("lda,ldb,a_off,b_off", [(201, 203, 0, 0), (208, 208, 1, 0), (208, 208, 0, 8), (216, 208, 0, 0), (208, 216, 3, 5)])
@pytest.mark.parametrize("M,N,c", [(1, 1, "f32"), (70, 66, "bf16"), (300, 200, "f16")])
def test_any_alignment(lda, ldb, a_off, b_off, M, N, c):
    assert "any_alignment" not in binding.i8_form(M, N, 200, -1, 208, 208, TYPE[c])
    run(M, N, 200, c, lda, ldb, N + 3, a_off, b_off, 1)
    run(M, N, 190, c, lda, ldb, N, a_off, b_off, 2)


@pytest.mark.parametrize("form,M,N,K", FORMS)
@pytest.mark.parametrize("c", ["f32", "bf16"])
def test_each_form(form, M, N, K, c):
    """With -128 among the values, remainders in every dimension; launches repeat to the bit."""
    assert binding.i8_form(M, N, K, -1, up(K, 16), up(K, 16), TYPE[c]) == form
    first = run(M, N, K, c, up(K, 16), up(K, 16), N, low=-128)
    assert np.array_equal(first, run(M, N, K, c, up(K, 16), up(K, 16), N, low=-128))


@pytest.mark.parametrize("M,N,K", [(2, 3, 131071), (70, 130, 131071), (300, 264, 131071), (600, 600, 70001)])
@pytest.mark.parametrize("ld", [131072, 131073 + 6])
def test_the_longest_sums_of_the_largest_products(M, N, K, ld):
    """-128 by -128: sums of 2147467264, the next K would leave 32 bits."""
    a, b = torch.full((M, ld), -128, dtype=I8, device="cuda"), torch.full((N, ld), -128, dtype=I8, device="cuda")
    b[1] = 127
    sa, sb, c = torch.ones(M, device="cuda"), torch.ones(N, device="cuda"), torch.zeros(M, N, device="cuda")
    binding.check(binding.gemm_i8(M, N, K, a, ld, sa, b, ld, sb, c, N, TYPE["f32"], stream()))
    want = torch.full((M, N), float(np.float32(K * 16384)), device="cuda")
    want[:, 1] = float(np.float32(-K * 16256))
    assert torch.equal(c, want)


def test_scales_beyond_each_others_range():
    """The scales' product would be zero or infinite in f32, the result is neither: the sum is multiplied by one, then by the other."""
    M, N, K = 4, 20, 64
    a, b = torch.full((M, K), 127, dtype=I8, device="cuda"), torch.full((N, K), 127, dtype=I8, device="cuda")
    c = torch.zeros(M, N, device="cuda")
    for x, y in ((2.0 ** -100, 2.0 ** -30), (2.0 ** 100, 2.0 ** -120)):
        binding.check(binding.gemm_i8(M, N, K, a, K, torch.full((M,), x, device="cuda"), b, K, torch.full((N,), y, device="cuda"), c, N, TYPE["f32"], stream()))
        assert bool((c == K * 127 * 127 * x * y).all()) and bool((c > 0).all())


@pytest.mark.parametrize("M,N,K", [(5, 40, 100), (300, 300, 200), (700, 900, 256)])
def test_a_nan_scale_reaches_its_row_or_column_alone(M, N, K):
    rng = np.random.default_rng(4)
    a, b = (torch.from_numpy(rng.integers(-9, 10, s)).to(I8).cuda() for s in ((M, up(K, 16)), (N, up(K, 16))))
    sa, sb = torch.ones(M, device="cuda"), torch.ones(N, device="cuda")
    sa[3], sb[7] = float("nan"), float("nan")
    a[3] = 0
    c = torch.zeros(M, N, device="cuda")
    binding.check(binding.gemm_i8(M, N, K, a, a.stride(0), sa, b, b.stride(0), sb, c, N, TYPE["f32"], stream()))
    want = a[:, :K].double() @ b[:, :K].double().t()
    assert bool(c[3].isnan().all()) and bool(c[:, 7].isnan().all())
    c[3], c[:, 7] = 0, 0
    want[3], want[:, 7] = 0, 0
    assert torch.equal(c.double(), want)


def test_no_sum():
    sa, sb, c = torch.ones(40, device="cuda"), torch.ones(50, device="cuda"), torch.full((40, 50), 7.0, device="cuda")
    binding.check(binding.gemm_i8(40, 50, 0, None, 0, sa, None, 0, sb, c, 50, TYPE["f32"], stream()))
    assert bool((c == 0).all())


def grouped(counts, N, K, c, rest=0, ld_pad=0, c_pad=0, seed=0, b_stride=None):
    E, T = len(counts), int(sum(counts)) + rest
    rng = np.random.default_rng(seed + T + N + K)
    a, b = rng.integers(-127, 128, (T, K)), rng.integers(-127, 128, (E, N, K))
    ld = up(K, 16) + ld_pad
    A, B, C = Ints(I8, T, K, ld, 0, a), Ints(I8, N, K, ld, 0, b, batch=E), Mat(c, T, N, N + c_pad)
    SA, SB = Mat("f32", 1, T, None, 1, scales(rng, 1, T)), Mat("f32", E, N, N + 1, 0, scales(rng, E, N))
    off = torch.from_numpy(offsets_of(counts)).cuda()
    rc = binding.gemm_i8_grouped(T, N, K, E, off, A.ptr, ld, SA.ptr, B.ptr, ld, B.stride, SB.ptr, N + 1, C.ptr, C.ld, TYPE[c], stream())
    assert rc == binding.OK, binding.strerror(rc)
    torch.cuda.synchronize()
    got, at = C.fetch(), 0
    bv = B.values().reshape(E, N, K)
    for e, n in enumerate(counts):
        want = expected(a[at:at + n], SA.values()[0][at:at + n], bv[e], SB.values().reshape(E, N)[e])
        assert_within(got[at:at + n], want, bound(want, c), f"expert {e}")
        at += n
    untouched = Mat(c, T, N, N + c_pad).fetch()
    assert np.array_equal(got[at:], untouched[at:])                              # rows of no group
    return got


@pytest.mark.parametrize("counts", [[1], [0, 3, 0, 1], [16, 17, 0, 33, 1], [128, 129, 127, 0], [300, 0, 513, 40], [2] * 70, [0] * 63 + [5, 0, 7] + [0] * 10])
@pytest.mark.parametrize("N,K,c", [(40, 100, "f32"), (264, 384, "bf16"), (130, 129, "f16")])
def test_grouped(counts, N, K, c):
    grouped(counts, N, K, c, rest=3, ld_pad=16, c_pad=4)


@pytest.mark.parametrize("form,counts,N,K", GROUPED)
def test_each_form_grouped(form, counts, N, K):
    assert binding.i8_form(sum(counts), N, K, len(counts), up(K, 16), up(K, 16), TYPE["bf16"]) == form
    assert np.array_equal(grouped(counts, N, K, "bf16"), grouped(counts, N, K, "bf16"))


@pytest.mark.parametrize("counts", [[1, 5, 0, 64, 70]])
def test_grouped_at_any_alignment(counts):
    grouped(counts, 77, 90, "f32", rest=2, ld_pad=3)


@pytest.mark.parametrize("ends", [[0, 40, 10, 5], [-5, 10, 20, 90], [50, 60, 60, 60], [0, 0, 0, 0], [-2**31, 30, 2**31 - 1, 2**31 - 1]])
@pytest.mark.parametrize("N,K", [(48, 64), (300, 300)])
def test_offsets_out_of_range_or_order(ends, N, K):
    """Taken within 0 .. T, decreasing ones as empty groups; nothing outside C is written, rows of no group stay."""
    T, E = 60, 3
    rng = np.random.default_rng(9)
    A, B, C = Ints(I8, T, K, up(K, 16), 0, rng.integers(-5, 6, (T, K))), Ints(I8, N, K, up(K, 16), 0, np.ones((E, N, K)), batch=E), Mat("f32", T, N)
    sa, sb = torch.ones(T, device="cuda"), torch.ones(E, N, device="cuda")
    off = torch.tensor(ends, dtype=torch.int64).clamp(-2**31, 2**31 - 1).to(torch.int32).cuda()
    binding.check(binding.gemm_i8_grouped(T, N, K, E, off, A.ptr, A.ld, sa, B.ptr, B.ld, B.stride, sb, N, C.ptr, N, TYPE["f32"], stream()))
    torch.cuda.synchronize()
    got, rows = C.fetch(), A.values().sum(1)
    covered = np.zeros(T, bool)
    for lo, hi in zip(ends, ends[1:]):
        lo = min(max(lo, 0), T)
        covered[lo:min(max(hi, lo), T)] = True
    assert np.array_equal(got[covered], np.repeat(rows[covered][:, None], N, 1)) and (got[~covered] == -1234.0).all()


def test_one_matrix_for_all_experts_and_strides_of_scales():
    T, N, K, E = 90, 72, 96, 3
    rng = np.random.default_rng(2)
    a, b = (torch.from_numpy(rng.integers(-9, 10, s)).to(I8).cuda() for s in ((T, K), (N, K)))
    sa, sb, c = torch.ones(T, device="cuda"), torch.full((N,), 2.0, device="cuda"), torch.zeros(T, N, device="cuda")
    off = torch.tensor([0, 20, 50, 90], dtype=torch.int32, device="cuda")
    binding.check(binding.gemm_i8_grouped(T, N, K, E, off, a, K, sa, b, K, 0, sb, 0, c, N, TYPE["f32"], stream()))
    assert torch.equal(c.double(), 2 * (a.double() @ b.double().t()))


# every form, small sums, and operands that only the kernel for any alignment takes
@pytest.mark.parametrize("form,M,N,K,odd", [f + (0,) for f in FORMS if f[1] * f[2] * f[3] < 2e10] + 
                         [("few_rows_64x64_any_alignment", 700, 1700, 1100, 1), ("few_rows_64x64_any_alignment", 300, 2100, 4099, 7), ("few_rows_32x32_any_alignment", 5, 40, 17, 3),
                          ("few_rows_32x32_any_alignment", 40, 300, 9, 1), ("few_rows_32x32_any_alignment", 33, 70, 9001, 2), ("any_alignment_64x64", 70, 130, 300, 1 << 22)])
@pytest.mark.parametrize("c", ["f16", "bf16", "f32"])
def test_every_form_gives_the_same_bits(form, M, N, K, odd, c):
    """Those of the definition: the exact sum to f32, times the row's scale, times the column's, each rounded to f32, and once to the result's type."""
    gen = torch.Generator(device="cuda").manual_seed(M + N + K)
    lda, ldb = up(K, 16) + odd, up(K, 16)
    assert binding.i8_form(M, N, K, -1, lda, ldb, TYPE[c]) == form
    a, b = (torch.randint(-128, 128, (rows, ld), dtype=I8, device="cuda", generator=gen) for rows, ld in ((M, lda), (N, ldb)))
    sa, sb = (torch.rand(n, device="cuda", generator=gen) * s for n, s in ((M, 1.0), (N, 1e-3)))
    out = torch.zeros(M, N, dtype=DT[c], device="cuda")
    binding.check(binding.gemm_i8(M, N, K, a, lda, sa, b, ldb, sb, out, N, TYPE[c], stream()))
    sums = (a[:, :K].double() @ b[:, :K].double().t()).float()              # exact in 64 bits
    assert torch.equal(out, (sums * sa[:, None] * sb).to(DT[c]))
