"""RMS norm with the residual's addition, its gradients, and quantisation to e4m3, against their definitions in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2108_13191_amd import binding                                                                   # noqa: E402
from ops_util import DT, LEAST, TYPE, UNIT, Mat, assert_within, ceil128, spread_blocks, spread_rows, stream   # noqa: E402

EPS = 1e-6
F32 = 1e-5           # relative: f32 sums of up to 20000 squares and a few operations
SHAPES = [(1, 1), (1, 128), (2, 7), (5, 130), (16, 512), (3, 520), (17, 1024), (33, 2047), (4, 2048), (9, 4000), (2, 4096), (7, 8192), (3, 8200),
          (2, 16384), (2, 16400), (1, 20001)]


def rounded(x, kind):
    return torch.from_numpy(np.ascontiguousarray(x)).to(torch.float32).to(DT[kind]).double().numpy()


def check_quantized(y, y_err, q, scale, what):
    """y: values in 64 bits of known error (absolute), q and its scale spread over them."""
    got = q * scale
    assert_within(got, y, np.abs(y) * UNIT["e4m3"] * 1.001 + scale * LEAST["e4m3"] * 1.001 + 2 * y_err, what)


def block_scale(y):
    """Scales in rows form of y (M x N), 64 bits."""
    M, N = y.shape
    t = np.zeros((M, ceil128(N) * 128))
    t[:, :N] = np.abs(y)
    return (np.maximum(t.reshape(M, -1, 128).max(2), 2.0 ** -96) / 448.0).T


@pytest.mark.parametrize("M,N", SHAPES)
@pytest.mark.parametrize("type", ["f16", "bf16"])
@pytest.mark.parametrize("residual", [True, False])
def test_norm(M, N, type, residual):
    rng = np.random.default_rng(M + N)
    X, R = Mat(type, M, N, N + 3, 1, rng.standard_normal((M, N))), Mat(type, M, N, N + 8, 0, 3 * rng.standard_normal((M, N)))
    G = Mat(type, 1, N, None, 1, 1 + 0.2 * rng.standard_normal((1, N)))
    H, Y, Q, S, rs = Mat(type, M, N, N + 1, 3), Mat(type, M, N, N + 8, 8), Mat("e4m3", M, N, N + 5, 1), Mat("f32", ceil128(N), M, M + 2, 1), Mat("f32", 1, M)
    rc = binding.rms_norm(M, N, TYPE[type], X.ptr, X.ld, R.ptr if residual else None, R.ld, G.ptr, EPS, H.ptr, H.ld, Y.ptr, Y.ld, Q.ptr, Q.ld,
                          S.ptr, S.ld, rs.ptr, stream())
    assert rc == binding.OK, binding.strerror(rc)
    torch.cuda.synchronize()
    h = rounded(X.values() + R.values(), type) if residual else X.values()
    assert np.array_equal(H.fetch(), h)
    rstd = 1 / np.sqrt((h * h).mean(1, keepdims=True) + EPS)
    assert_within(rs.fetch(), rstd.T, rstd.T * F32, "rstd")
    y = h * rstd * G.values()
    assert_within(Y.fetch(), y, np.abs(y) * (F32 + UNIT[type] * 1.001) + LEAST[type], "y")
    s = S.fetch()
    assert_within(s, block_scale(y), block_scale(y) * F32, "scale")
    check_quantized(y, np.abs(y) * F32, Q.fetch(), spread_rows(s, N), "q")


@pytest.mark.parametrize("outputs", ["h", "y", "q", "rstd", "yq", ""])
@pytest.mark.parametrize("N", [300, 17000])
def test_norm_outputs_alone(outputs, N):
    M, type = 5, "bf16"
    rng = np.random.default_rng(N)
    x, r = rng.standard_normal((M, N)), rng.standard_normal((M, N))
    X, R, G = Mat(type, M, N, None, 0, x), Mat(type, M, N, None, 0, r), Mat(type, 1, N, None, 0, np.ones((1, N)))
    full = [Mat(type, M, N), Mat(type, M, N), Mat("e4m3", M, N), Mat("f32", ceil128(N), M), Mat("f32", 1, M)]
    some = [Mat(m.kind, m.rows, m.cols) for m in full]

    def call(m, want):
        H, Y, Q, S, rs = (t.ptr if on else None for t, on in zip(m, ["h" in want, "y" in want, "q" in want, "q" in want, "rstd" in want]))
        assert binding.rms_norm(M, N, TYPE[type], X.ptr, N, R.ptr, N, G.ptr, EPS, H, N, Y, N, Q, N, S, M, rs, stream()) == binding.OK

    call(full, "h y q rstd")
    call(some, outputs)
    torch.cuda.synchronize()
    names = ["h", "y", "q", "q", "rstd"]
    for a, b, name in zip(full, some, names):
        if name in outputs:
            assert np.array_equal(a.fetch(), b.fetch()), name
        else:
            assert torch.equal(b.dev.cpu().view(torch.uint8), b.host.view(torch.uint8)), f"{name} was written"


@pytest.mark.parametrize("N", [256, 4000, 16400])
@pytest.mark.parametrize("into", ["x", "r"])
def test_norm_in_place(N, into):
    M, type = 6, "f16"
    rng = np.random.default_rng(N)
    x, r = rng.standard_normal((M, N)), rng.standard_normal((M, N))
    X, R, G, Y, Y2, H = Mat(type, M, N, None, 0, x), Mat(type, M, N, None, 0, r), Mat(type, 1, N, None, 0, np.ones((1, N))), Mat(type, M, N), Mat(type, M, N), Mat(type, M, N)
    assert binding.rms_norm(M, N, TYPE[type], X.ptr, N, R.ptr, N, G.ptr, EPS, H.ptr, N, Y.ptr, N, None, 0, None, 0, None, stream()) == binding.OK
    target = X if into == "x" else R
    assert binding.rms_norm(M, N, TYPE[type], X.ptr, N, R.ptr, N, G.ptr, EPS, target.ptr, N, Y2.ptr, N, None, 0, None, 0, None, stream()) == binding.OK
    torch.cuda.synchronize()
    assert np.array_equal(Y.fetch(), Y2.fetch()) and np.array_equal(target._view(target.dev.cpu())[0].double().numpy(), H.fetch())


def test_norm_of_zeros_large_values_and_nans():
    M, N, type = 5, 384, "bf16"
    x = np.zeros((M, N))
    x[1] = 1e30                       # squares that f32 does not hold: h^2 is infinite, rstd 0, y 0
    x[2, 5] = np.inf                  # h * 0 is NaN there, 0 elsewhere
    x[3, 200] = np.nan                # the whole row
    x[4] = 2.0
    X, G = Mat(type, M, N, None, 0, x), Mat(type, 1, N, None, 0, np.ones((1, N)))
    Y, Q, S = Mat(type, M, N), Mat("e4m3", M, N), Mat("f32", 3, M)
    assert binding.rms_norm(M, N, TYPE[type], X.ptr, N, None, 0, G.ptr, EPS, None, 0, Y.ptr, N, Q.ptr, N, S.ptr, M, None, stream()) == binding.OK
    torch.cuda.synchronize()
    y, q, s = Y.fetch(), Q.fetch(), S.fetch()
    assert (y[0] == 0).all() and (q[0] == 0).all() and np.allclose(s[:, 0], 2.0 ** -96 / 448, rtol=1e-6)
    assert (y[1] == 0).all() and (q[1] == 0).all()
    assert np.isnan(y[2, 5]) and (np.delete(y[2], 5) == 0).all() and np.isnan(s[0, 2]) and np.isnan(q[2, :128]).all() and (q[2, 128:] == 0).all()
    assert np.isnan(y[3]).all() and np.isnan(s[:, 3]).all() and np.isnan(q[3]).all()
    assert (y[4] == 1).all() and (q[4] == 448).all() and np.allclose(s[:, 4], 1 / 448, rtol=1e-5)


@pytest.mark.parametrize("M,N", SHAPES + [(600, 64), (1030, 264), (5000, 8), (530, 8192)])
@pytest.mark.parametrize("type,residual", [("f16", True), ("bf16", False), ("bf16", True)])
def test_norm_gradients(M, N, type, residual):
    rng = np.random.default_rng(M * N)
    D, H = Mat(type, M, N, N + 3, 1, rng.standard_normal((M, N))), Mat(type, M, N, N + 8, 0, 2 * rng.standard_normal((M, N)))
    U, G = Mat(type, M, N, N + 1, 2, rng.standard_normal((M, N))), Mat(type, 1, N, None, 1, 1 + 0.2 * rng.standard_normal((1, N)))
    dy, h, up, gamma = D.values(), H.values(), U.values(), G.values()
    R = Mat("f32", 1, M, None, 0, 1 / np.sqrt((h * h).mean(1) + EPS))
    rstd = R.values().reshape(M, 1)
    need = binding.rms_norm_grad_workspace_bytes(M, N)
    assert 0 < need <= 1024 * N
    ws = torch.full((need // 4 + 4,), float("nan"), device="cuda")
    dX, dG = Mat(type, M, N, N + 2, 1), Mat("f32", 1, N)
    results = []
    for _ in range(2):
        rc = binding.rms_norm_grad(M, N, TYPE[type], D.ptr, D.ld, H.ptr, H.ld, G.ptr, R.ptr, U.ptr if residual else None, U.ld, dX.ptr, dX.ld, dG.ptr, ws, need, stream())
        assert rc == binding.OK, binding.strerror(rc)
        torch.cuda.synchronize()
        results.append((dX.fetch(), dG.fetch()))
    assert np.array_equal(results[0][0], results[1][0]) and np.array_equal(results[0][1], results[1][1])      # a fixed order of sums
    assert bool(torch.isnan(ws[need // 4:]).all())
    g, xhat = dy * gamma, h * rstd
    want = rstd * (g - xhat * (g * xhat).mean(1, keepdims=True)) + (up if residual else 0)
    mag = rstd * (np.abs(g) + np.abs(xhat) * np.abs(g * xhat).mean(1, keepdims=True)) + (np.abs(up) if residual else 0)
    assert_within(results[0][0], want, mag * F32 + np.abs(want) * UNIT[type] * 1.001 + LEAST[type], "dX")
    want, mag = (dy * xhat).sum(0, keepdims=True), np.abs(dy * xhat).sum(0, keepdims=True)
    assert_within(results[0][1], want, mag * F32, "dgamma")


def test_norm_gradients_against_differences():
    """A scalar of the definition, differentiated by central differences in 64 bits: its gradient is what the kernel gives."""
    M, N = 3, 40
    rng = np.random.default_rng(2)
    D, H, G = (Mat("f16", r, N, None, 0, v) for r, v in ((M, rng.standard_normal((M, N))), (M, rng.standard_normal((M, N))), (1, 1 + 0.2 * rng.standard_normal((1, N)))))
    dy, h, gamma = D.values(), H.values(), G.values()

    def scalar(h, gamma):
        return float((dy * h / np.sqrt((h * h).mean(1, keepdims=True) + EPS) * gamma).sum())

    R, dX, dG = Mat("f32", 1, M, None, 0, 1 / np.sqrt((h * h).mean(1) + EPS)), Mat("f16", M, N), Mat("f32", 1, N)
    need = binding.rms_norm_grad_workspace_bytes(M, N)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    assert binding.rms_norm_grad(M, N, TYPE["f16"], D.ptr, N, H.ptr, N, G.ptr, R.ptr, None, 0, dX.ptr, N, dG.ptr, ws, need, stream()) == binding.OK
    torch.cuda.synchronize()
    gx, gg, step = dX.fetch(), dG.fetch(), 1e-5
    for i in range(M):
        for j in range(0, N, 7):
            a, b = h.copy(), h.copy()
            a[i, j] += step
            b[i, j] -= step
            d = (scalar(a, gamma) - scalar(b, gamma)) / (2 * step)
            assert abs(gx[i, j] - d) <= 1e-6 + 2 ** -10 * (abs(d) + 1e-3)            # the result's rounding to f16
    for j in range(0, N, 7):
        a, b = gamma.copy(), gamma.copy()
        a[0, j] += step
        b[0, j] -= step
        d = (scalar(h, a) - scalar(h, b)) / (2 * step)
        assert abs(gg[0, j] - d) <= 1e-4 * (1 + abs(d))


@pytest.mark.parametrize("into", ["dy", "dh"])
@pytest.mark.parametrize("N", [512, 5000, 17000])
def test_norm_gradient_in_place_and_without_dgamma(into, N):
    M, type = 37, "bf16"
    rng = np.random.default_rng(N)
    D, H, U, G = (Mat(type, r, N, None, 0, rng.standard_normal((r, N))) for r in (M, M, M, 1))
    R, dX = Mat("f32", 1, M, None, 0, np.full((1, M), 0.9)), Mat(type, M, N)
    assert binding.rms_norm_grad(M, N, TYPE[type], D.ptr, N, H.ptr, N, G.ptr, R.ptr, U.ptr, N, dX.ptr, N, None, None, 0, stream()) == binding.OK
    target = D if into == "dy" else U
    assert binding.rms_norm_grad(M, N, TYPE[type], D.ptr, N, H.ptr, N, G.ptr, R.ptr, U.ptr, N, target.ptr, N, None, None, 0, stream()) == binding.OK
    torch.cuda.synchronize()
    assert np.array_equal(dX.fetch(), target._view(target.dev.cpu())[0].double().numpy())


def test_dgamma_of_no_rows_is_zeros():
    dG = Mat("f32", 1, 100)
    assert binding.rms_norm_grad(0, 100, TYPE["f16"], None, 0, None, 0, None, None, None, 0, None, 0, dG.ptr, None, 0, stream()) == binding.OK
    torch.cuda.synchronize()
    assert not dG.fetch().any()


@pytest.mark.parametrize("M,N", [(1, 1), (1, 128), (2, 130), (16, 256), (17, 520), (40, 1000), (130, 384), (3, 7001)])
@pytest.mark.parametrize("type", ["f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu", "swiglu"])
def test_quantize_rows(M, N, type, act):
    rng = np.random.default_rng(M + N)
    wide = 2 * N if act == "swiglu" else N
    X = Mat(type, M, wide, wide + 3, 1, rng.standard_normal((M, wide)) * np.exp(3 * rng.standard_normal((M, 1))))
    Q, S = Mat("e4m3", M, N, N + 3, 1), Mat("f32", ceil128(N), M, M + 1, 1)
    code = {"none": binding.ACT_NONE, "relu": binding.ACT_RELU, "swiglu": binding.ACT_SWIGLU}[act]
    rc = binding.quantize_e4m3_rows(M, N, TYPE[type], code, X.ptr, X.ld, Q.ptr, Q.ld, S.ptr, S.ld, stream())
    assert rc == binding.OK, binding.strerror(rc)
    torch.cuda.synchronize()
    x = X.values()
    with np.errstate(over="ignore"):
        y = np.maximum(x, 0) if act == "relu" else x[:, :N] / (1 + np.exp(-x[:, :N])) * x[:, N:] if act == "swiglu" else x
    # exp(-g) of g down to -300 loses relative precision with |g|: half a unit of the exponent's argument
    rel = 1e-6 if act != "swiglu" else 1e-5 * (1 + np.abs(x[:, :N]) / 10)
    s = S.fetch()
    assert_within(s, block_scale(y), block_scale(y) * (1e-6 if act != "swiglu" else 1e-4) + 1e-37, "scale")
    check_quantized(y, np.abs(y) * rel + 1e-37, Q.fetch(), spread_rows(s, N), "q")


@pytest.mark.parametrize("M,N", [(1, 1), (128, 128), (129, 127), (300, 520), (7, 1000), (256, 384)])
@pytest.mark.parametrize("type", ["f16", "bf16"])
def test_quantize_blocks(M, N, type):
    rng = np.random.default_rng(M + N)
    X = Mat(type, M, N, N + 3, 1, rng.standard_normal((M, N)))
    Q, S = Mat("e4m3", M, N, N + 3, 1), Mat("f32", ceil128(M), ceil128(N), ceil128(N) + 2, 1)
    rc = binding.quantize_e4m3_blocks(M, N, TYPE[type], X.ptr, X.ld, Q.ptr, Q.ld, S.ptr, S.ld, stream())
    assert rc == binding.OK, binding.strerror(rc)
    torch.cuda.synchronize()
    x, s = X.values(), S.fetch()
    want = np.zeros((ceil128(M), ceil128(N)))
    for a in range(ceil128(M)):
        for b in range(ceil128(N)):
            want[a, b] = np.abs(x[128 * a:128 * a + 128, 128 * b:128 * b + 128]).max() / 448
    assert_within(s, want, want * 1e-6, "scale")
    check_quantized(x, np.abs(x) * 1e-6, Q.fetch(), spread_blocks(s, M, N), "q")


def test_quantize_poisons_the_block_of_a_nan_or_infinity_alone():
    for bad in (np.nan, np.inf, -np.inf):
        x = np.ones((20, 300))
        x[3, 130] = bad
        x[5] = 0.0
        X, Q, S = Mat("bf16", 20, 300, None, 0, x), Mat("e4m3", 20, 300), Mat("f32", 3, 20)
        assert binding.quantize_e4m3_rows(20, 300, TYPE["bf16"], binding.ACT_NONE, X.ptr, 300, Q.ptr, 300, S.ptr, 20, stream()) == binding.OK
        torch.cuda.synchronize()
        q, s = Q.fetch(), S.fetch()
        want = np.zeros((20, 300), bool)
        want[3, 128:256] = True
        assert np.array_equal(np.isnan(q), want) and np.isnan(s[1, 3]) and np.isnan(s).sum() == 1
        assert (q[5] == 0).all() and (s[:, 5] > 0).all()
        S2 = Mat("f32", 1, 3)
        assert binding.quantize_e4m3_blocks(20, 300, TYPE["bf16"], X.ptr, 300, Q.ptr, 300, S2.ptr, 3, stream()) == binding.OK
        torch.cuda.synchronize()
        s2 = S2.fetch()
        assert np.isnan(s2[0, 1]) and np.isnan(s2).sum() == 1 and np.isnan(Q.fetch()[:, 128:256]).all()


def test_quantize_every_e4m3_value_is_kept():
    """A block whose largest magnitude is 448 has the scale 1: every value that e4m3 holds comes back, and ties go to even."""
    codes = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    x = codes[~np.isnan(codes)]
    mid = np.array([1.0625, 1.1875, -17.0, 0.0009765625, 3 * 0.0009765625, 440.0])       # halfway between neighbours
    even = np.array([1.0, 1.25, -16.0, 0.0, 2 * 0.001953125, 448.0])
    row = np.concatenate([x, [448.0, 0.0]])[:256]
    block = np.concatenate([mid, [448.0], np.zeros(121)])
    X, Q, S = Mat("f16", 1, 384, None, 0, np.concatenate([row, block])), Mat("e4m3", 1, 384), Mat("f32", 3, 1)
    assert binding.quantize_e4m3_rows(1, 384, TYPE["f16"], binding.ACT_NONE, X.ptr, 384, Q.ptr, 384, S.ptr, 1, stream()) == binding.OK
    torch.cuda.synchronize()
    q, s = Q.fetch()[0], S.fetch()[:, 0]
    for b in range(3):
        if s[b] == 1.0:
            part = np.concatenate([row, np.concatenate([even, [448.0], np.zeros(121)])])[128 * b:128 * b + 128]
            assert np.array_equal(q[128 * b:128 * b + 128], part)
    assert s[2] == 1.0 and (s == 1.0).sum() == 3
