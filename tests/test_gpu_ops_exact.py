"""How exact e4m3 products are.  The e4m3 matrix instructions, which large 16-bit results come from where the caller does not ask for exact products, lose at most 2^-10 of the sum of
magnitudes: tested with operands that come near that, and with grouped products of normal values.  Exact products are held to the bound of f32 sums at the same sizes."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2108_13191_amd import binding                                    # noqa: E402
from ops_util import DT, LEAST, TYPE, UNIT, assert_within, ceil128, result_bound, stream      # noqa: E402
from test_gpu_ops_products import large_e4m3                                # noqa: E402

COUNTS = [[1000, 257, 0, 1500, 1001], [70, 90, 0, 131, 128] * 8, [30, 0, 41, 25] * 5]


@pytest.mark.parametrize("counts", COUNTS, ids=["large", "middle", "short"])
@pytest.mark.parametrize("c", ["f16", "bf16"])
@pytest.mark.parametrize("exact", [False, True])
def test_grouped_normal_values(monkeypatch, counts, c, exact):
    if exact:
        monkeypatch.setitem(TYPE, c, TYPE[c] | binding.EXACT)
    N = 6001 if sum(counts) > 1000 else 14001
    assert binding.product_form(binding.PRODUCT_E4M3, sum(counts), N, 390, len(counts), 416, 416, TYPE[c]).startswith("widened" if exact else "e4m3")
    got, want, mag = large_e4m3(sum(counts), N, 390, c, counts)
    inside = np.abs(want) < (65504.0 - 2.0 ** -9 * mag if c == "f16" else np.inf)
    got, want, mag = got[inside], want[inside], mag[inside]
    if exact:
        assert_within(got, want, result_bound(want, mag, c), "exact")
    else:
        assert_within(got, want, 2.0 ** -10 * mag * 1.01 + np.abs(want) * UNIT[c] + LEAST[c], "e4m3 instructions")
        assert np.linalg.norm(got - want) <= (UNIT[c] + 2.0 ** -15) * np.linalg.norm(want)


def product(a, b, c_type, dtype, scale=1.0):
    (M, K), N = a.shape, b.shape[0]
    C = torch.empty(M, N, dtype=dtype, device="cuda")
    one = lambda *s: torch.ones(s, device="cuda")                                            # noqa: E731
    binding.check(binding.gemm_e4m3_block(M, N, K, a.to(DT["e4m3"]).cuda(), K, scale * one(ceil128(K), M), M, b.to(DT["e4m3"]).cuda(), K, one(ceil128(N), ceil128(K)), ceil128(K), C, N, c_type, stream()))
    return C.double().cpu()


# one product of each 8 is 256 * 256 = 2^16, cut off below 2^3 then; the other seven are 2.5 * 3 = 7.5: together 52.5 of 65588.5, or 2^-10.3
NEAR = [(256.0, 256.0, 2.5, 3.0), (-256.0, 256.0, 2.5, 3.0), (448.0, 448.0, 3.5, 4.5)]


@pytest.mark.parametrize("large_a,large_b,small_a,small_b", NEAR)
@pytest.mark.parametrize("at", [0, 3, 7])
@pytest.mark.parametrize("c", ["f16", "bf16"])
def test_small_products_beside_a_large_one(large_a, large_b, small_a, small_b, at, c):
    """In one row of A and one of B of a large problem; all other products are zeros."""
    M = N = 2048
    a, b = torch.zeros(M, 128), torch.zeros(N, 128)
    a[5, 16:24], b[7, 16:24] = small_a, small_b
    a[5, 16 + at], b[7, 16 + at] = large_a, large_b
    want, mag = (a[5].double() * b[7].double()).sum(), (a[5].double() * b[7].double()).abs().sum()
    scale = 2.0 ** -6 if c == "f16" else 1.0               # within f16's range
    w, m = want.item() * scale, mag.item() * scale
    for exact in (0, binding.EXACT):
        got = product(a, b, TYPE[c] | exact, DT[c], scale)[5, 7].item()
        assert abs(got - w) <= (1e-5 if exact else 2.0 ** -10) * m + abs(w) * UNIT[c] + LEAST[c], (exact, got, w)


@pytest.mark.parametrize("c", ["f16", "bf16", "f32"])
def test_rows_do_not_depend_on_the_rows_beside_them(c):
    """448 * 448 - 448 * 448 and 126 ones: 126 whatever the number of rows, where exact products are asked for; f32 results always have them."""
    a, b = torch.ones(2048, 128), torch.ones(2048, 128)
    a[:, :2], b[:, 0], b[:, 1] = 448.0, 448.0, -448.0
    exact = TYPE[c] | binding.EXACT
    for rows in (1, 64, 700, 2048):
        assert (product(a[:rows], b, exact, DT[c]) == 126.0).all()
    without = product(a, b, TYPE[c], DT[c])
    assert (without - 126.0).abs().max() <= (0.0 if c == "f32" else 2.0 ** -10 * (2 * 448.0 ** 2 + 126.0))
