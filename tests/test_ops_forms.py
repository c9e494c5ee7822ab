"""Which kernel form a product of include/gemm_ops.h runs on, without a GPU: that the shapes which the GPU tests hold for a form reach it, that every form has some, and the
lines between the forms."""
import pytest

import ops_form_cases as cases
from paper_2108_13191_amd import binding
from paper_2108_13191_amd.binding import PRODUCT_E4M3, PRODUCT_FORWARD, PRODUCT_GRAD_A, PRODUCT_GRAD_B, TYPE_BF16, TYPE_F16, TYPE_F32, product_form

TYPE = {"f16": TYPE_F16, "bf16": TYPE_BF16, "f32": TYPE_F32}


def up(n, to):
    return (n + to - 1) // to * to


def e4m3(rows, N, K, c):
    T, E = (rows, -1) if isinstance(rows, int) else (sum(rows) + cases.EXTRA, len(rows))
    return product_form(PRODUCT_E4M3, T, N, K, E, up(K, 16), up(K, 16), TYPE[c])


def grouped(product, rows, N, K, pad=8):
    lda, ldb = {PRODUCT_FORWARD: (K, N), PRODUCT_GRAD_A: (N, N), PRODUCT_GRAD_B: (K, N)}[product]
    return product_form(product, sum(rows) + cases.EXTRA, N, K, len(rows), up(lda, pad), up(ldb, pad), TYPE_F32)


@pytest.mark.parametrize("form,rows,N,K,c", cases.E4M3)
def test_e4m3_forms(form, rows, N, K, c):
    assert e4m3(rows, N, K, c) == form


@pytest.mark.parametrize("product,form,rows,N,K", [(p, *c) for p, some in ((PRODUCT_FORWARD, cases.FORWARD), (PRODUCT_GRAD_A, cases.GRAD_A), (PRODUCT_GRAD_B, cases.GRAD_B)) for c in some])
def test_16_bit_forms(product, form, rows, N, K):
    assert grouped(product, rows, N, K) == form


@pytest.mark.parametrize("form,rows,N,K", cases.UNALIGNED)
def test_forms_of_any_alignment(form, rows, N, K):
    for product in (PRODUCT_FORWARD, PRODUCT_GRAD_A, PRODUCT_GRAD_B):
        assert grouped(product, rows, N, K, pad=1) == form


def test_every_form_has_shapes_that_reach_it():
    few = [f"few_rows_{t}" for t in ("16x16", "16x32", "32x16", "32x32", "32x64")]
    wide = ["widened_128x128", "widened_128x128_short_groups", "widened_128x128_two", "widened_256x128", "e4m3_128x128", "e4m3_256x256"]
    assert {c[0] for c in cases.E4M3} == {*few, *wide}
    assert {c[0] for c in cases.FORWARD} == {"256x256", "128x256", "128x128"}
    assert {c[0] for c in cases.GRAD_A} == {c[0] for c in cases.GRAD_B} == {"256x256", "128x128"}


def test_forms_of_what_the_tiles_do_not_take():
    far = (1 << 22) + 16
    assert product_form(PRODUCT_E4M3, 1300, 1200, 400, -1, 1 << 22, 1 << 22, TYPE_F32) == "widened_128x128"
    for lda, ldb in ((far, 400), (400, far), (401, 400), (400, 408)):
        assert product_form(PRODUCT_E4M3, 1300, 1200, 400, -1, lda, ldb, TYPE_F32) == "any_alignment_64x64"
    assert product_form(PRODUCT_FORWARD, 100, 7, 64, 2, 64, 7, TYPE_F32) == "any_alignment_64x64"
    assert product_form(PRODUCT_FORWARD, 100, 9, 64, 2, 64, 9, TYPE_F32) == "any_alignment_128x128"


def test_nothing_to_run():
    for args in ((PRODUCT_E4M3, 0, 8, 8, -1), (PRODUCT_E4M3, 8, 0, 8, -1), (PRODUCT_FORWARD, 8, 8, 8, 0), (PRODUCT_FORWARD, 8, 8, 8, -1), (PRODUCT_GRAD_B, 8, 8, 8, 65536), (4, 8, 8, 8, 1),
                 (-1, 8, 8, 8, 1), (PRODUCT_GRAD_A, 2**31, 8, 8, 1)):
        assert product_form(*args, 8, 8, TYPE_F32) is None
    assert product_form(PRODUCT_FORWARD, 8, 8, 8, 1, 8, 8, 3) is None


def test_forms_that_a_launch_has_no_workgroups_for_give_way_to_larger_tiles():
    def short(E, N, c, T=None):
        return product_form(PRODUCT_E4M3, T or E, N, 16, E, 16, 16, c)
    assert short(256, 1 << 18, TYPE_BF16) == short(256, 1 << 18, TYPE_F32) == "few_rows_16x32"
    assert short(256, 1 << 20, TYPE_BF16) == "e4m3_128x128" and short(256, 1 << 20, TYPE_F32) == "widened_128x128_short_groups"
    assert short(65535, 14000, TYPE_F32, 65535 * 30) == "widened_256x128"           # 80894 tiles of 128 rows, 73214 of 256, 110 columns of them
    assert short(65535, 33000, TYPE_BF16) is None                                   # 65535 + 255 of 256 rows, 129 columns of them
    grad_a = lambda N: product_form(PRODUCT_GRAD_A, 65535, 64, N, 65535, 64, 64, TYPE_F32)          # noqa: E731
    assert grad_a(16000) == "128x128" and grad_a(32000) == "256x256" and grad_a(33000) is None


def test_exact_e4m3_products_never_run_on_the_e4m3_instructions():
    for rows, N, K, c in ((8192, 8192, 8192, TYPE_BF16), (8192, 8192, 8192, TYPE_F16), (4730, 4399, 1300, TYPE_BF16), ([1000, 257, 0, 1500, 1001], 6001, 1300, TYPE_F16)):
        T, E = (rows, -1) if isinstance(rows, int) else (sum(rows), len(rows))
        form = lambda c: product_form(PRODUCT_E4M3, T, N, K, E, up(K, 16), up(K, 16), c)                    # noqa: E731
        assert form(c).startswith("e4m3_") and form(c | binding.EXACT).startswith("widened_")
        assert form(TYPE_F32 | binding.EXACT) == form(TYPE_F32) == form(c | binding.EXACT)                  # as f32 results do
    assert product_form(PRODUCT_E4M3, 8, 8, 8, -1, 16, 16, 3 | binding.EXACT) is None and product_form(PRODUCT_FORWARD, 8, 8, 8, 1, 8, 8, binding.EXACT) is None


def test_exactness_beside_the_type_of_a_result():
    """Taken by the e4m3 products alone; whatever else is refused stays so."""
    P, exact = 4096, binding.EXACT
    lone = dict(M=4, N=8, K=16, A=P, lda=16, a_scale=P, ld_as=4, B=P, ldb=16, b_scale=P, ld_bs=1, C=P, ldc=8)
    for c in (exact | 3, exact << 1, -1, exact | -32):
        assert binding.gemm_e4m3_block(**lone, c_type=c) == binding.ERR_CONFIG
    assert binding.gemm_e4m3_block(**{**lone, "C": P + 1}, c_type=exact | TYPE_BF16) == binding.ERR_ALIGN
    assert binding.gemm_e4m3_block(**{**lone, "C": P + 2}, c_type=exact | TYPE_F32) == binding.ERR_ALIGN
    assert binding.gemm_e4m3_block(**{**lone, "M": 0}, c_type=exact | TYPE_F32) == binding.OK
    assert binding.gemm_grouped(T=4, N=8, K=16, E=2, offsets=P, type=TYPE_F16, A=P, lda=16, B=P, ldb=8, b_stride=128, C=P, ldc=8, c_type=exact | TYPE_F16) == binding.ERR_CONFIG


def test_large_tiles_only_where_matrices_fill_them():
    grad_b = lambda T, K, N, E: product_form(PRODUCT_GRAD_B, T, N, K, E, up(K, 8), up(N, 8), TYPE_F32)        # noqa: E731
    for T, K, N, E in ((8192, 304, 304, 128), (16384, 264, 1032, 64), (16384, 640, 640, 64), (16384, 128, 4096, 64), (2000, 48, 72, 1000), (8192, 300, 300, 128)):
        assert grad_b(T, K, N, E) == "128x128"
    for T, K, N, E in ((16384, 1024, 2048, 32), (16384, 1032, 2056, 32), (16384, 512, 512, 128), (16384, 776, 1032, 64), (16384, 4096, 4096, 1)):
        assert grad_b(T, K, N, E) == "256x256"
    forward = lambda T, N, E: product_form(PRODUCT_FORWARD, T, N, 1024, E, 1024, up(N, 8), TYPE_F16)         # noqa: E731
    for T, N, E in ((8192, 72, 512), (8192, 264, 128), (8192, 520, 64), (2000, 1032, 128)):
        assert forward(T, N, E) == "128x128"
    for T, N, E in ((8192, 2048, 64), (64, 4096, 16), (4000, 1160, 128)):
        assert forward(T, N, E) == "128x256"
