"""Layer norm of rows near f32's range: what a row gives does not depend on how its elements are dealt to threads, so on how many rows and columns a call has."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2108_13191_amd import binding                                                       # noqa: E402
from ops_util import TYPE, Mat, assert_within, stream                                          # noqa: E402
from layer_util import F32, Ints, layer_norm, quantized, rounding                              # noqa: E402

EPS = 1e-5
BIG = 3e38


def rows_near_the_range(M, N, rng):
    """Of M rows the first eight: halves of either sign (the sum of a part passes the range, the row's is 0), the same turned round, three elements whose differences from the
    mean pass it, runs of 8 of one sign; then rows whose sum passes it: all of one sign, three quarters, the last two elements; and one with an infinity in the last place."""
    x = rng.standard_normal((M, N))
    half = N // 2
    x[0, :half], x[0, half:2 * half], x[0, 2 * half:] = BIG, -BIG, 0
    x[1] = -x[0]
    x[2] = 0
    x[2, :3] = BIG, -BIG, -BIG
    x[3] = np.where(np.arange(N) // 8 % 2, -BIG, BIG)
    x[3, N // 16 * 16:] = 0
    x[4] = -BIG
    x[5, :3 * N // 4], x[5, 3 * N // 4:] = BIG, -BIG
    x[6, -2:] = BIG
    x[7, -1] = np.inf
    return x


@pytest.mark.parametrize("N", [24, 40, 100, 136, 250, 512, 700, 1024, 2001, 4000, 4096, 8000, 8191, 16000, 16384, 17000, 30011])
@pytest.mark.parametrize("M", [9, 600])
@pytest.mark.parametrize("residual", [False, True])
def test_rows_near_the_range(M, N, residual):
    type, rng = "bf16", np.random.default_rng(N)
    x = rows_near_the_range(M, N, rng)
    X, R = Mat(type, M, N, N + 3, 1, x), Mat(type, M, N, N + 1, 0, np.zeros((M, N)))
    G, B = Mat(type, 1, N, None, 0, 1 + 0.2 * rng.standard_normal((1, N))), Mat(type, 1, N, None, 0, rng.standard_normal((1, N)))
    Y, Q, S, mu, rs = Mat(type, M, N), Ints(torch.int8, M, N), Mat("f32", 1, M), Mat("f32", 1, M), Mat("f32", 1, M)
    assert binding.layer_norm(M, N, TYPE[type], X.ptr, X.ld, R.ptr if residual else None, R.ld, G.ptr, B.ptr, EPS, None, 0, Y.ptr, N, Q.ptr, N, S.ptr, mu.ptr, rs.ptr, stream()) == binding.OK
    torch.cuda.synchronize()
    y, q, s, mean, rstd = Y.fetch(), Q.fetch(), S.fetch()[0], mu.fetch()[0], rs.fetch()[0]
    h = X.values()
    beta_q, beta_s = quantized(B.values())
    for i in range(4):
        assert rstd[i] == 0 and np.array_equal(y[i], B.values()[0]) and np.array_equal(q[i], beta_q[0]) and s[i] == beta_s[0], i
        assert abs(mean[i] - h[i].mean()) <= F32 * np.abs(h[i]).mean(), i
    for i in range(4, 8):
        assert np.isnan(y[i]).all() and np.isnan(s[i]) and np.isnan(rstd[i]) and np.isnan(mean[i]) and (q[i] == 0).all(), i
    m, r, want, off = layer_norm(h[8:], G.values(), B.values(), EPS)
    assert_within(y[8:], want, rounding(want, off, type), "y")
    assert_within(mean[8:], m[:, 0], F32 * np.abs(h[8:]).mean(1), "mean")
