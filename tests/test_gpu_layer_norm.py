"""Layer norm with the residual's addition, its gradients, and rows quantised to 8-bit integers, against their definitions in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2108_13191_amd import binding                                                       # noqa: E402
from ops_util import LEAST, TYPE, UNIT, Mat, assert_within, stream                             # noqa: E402
from layer_util import F32, Ints, layer_norm, quantized, rounded, rounding, row_scales         # noqa: E402

EPS = 1e-5
I8 = torch.int8
# each number of wavefronts and chunks a row and both ends of it, more rows than few, rows longer than registers
SHAPES = [(1, 1), (1, 8), (2, 7), (5, 130), (16, 512), (3, 520), (17, 1024), (33, 2047), (4, 2048), (9, 4000), (600, 2056), (2, 4096), (7, 8192), (520, 8191), (3, 8200),
          (2, 16384), (2, 16400), (1, 20001)]


def operands(type, M, N, seed, beta=True):
    rng = np.random.default_rng(seed)
    return (Mat(type, M, N, N + 3, 1, rng.standard_normal((M, N))), Mat(type, M, N, N + 8, 0, 3 * rng.standard_normal((M, N)) + 0.7),
            Mat(type, 1, N, None, 1, 1 + 0.2 * rng.standard_normal((1, N))), Mat(type, 1, N, None, 3, 0.3 * rng.standard_normal((1, N))) if beta else None)


def check_steps(y, off, q, s, what):
    """Integers of rows whose values are known within `off`: scale within what the largest may be off, elements the nearest but at borders."""
    most = np.maximum(np.abs(y).max(1), 2.0 ** -96)
    assert_within(s, most / 127, (off.max(1) + most * 2.0 ** -23) / 127, what + " scale")
    assert_within(q * s[:, None], y, 0.5 * s[:, None] * (1 + 2.0 ** -20) + off, what)
    assert np.abs(q).max() <= 127


@pytest.mark.parametrize("M,N", SHAPES)
@pytest.mark.parametrize("type,residual,beta", [("f16", True, True), ("bf16", True, True), ("bf16", False, False), ("f16", False, True)])
def test_norm(M, N, type, residual, beta):
    X, R, G, B = operands(type, M, N, M + N, beta)
    H, Y, Q, S = Mat(type, M, N, N + 1, 3), Mat(type, M, N, N + 8, 8), Ints(I8, M, N, N + 5, 1), Mat("f32", 1, M, None, 1)
    mu, rs = Mat("f32", 1, M), Mat("f32", 1, M, None, 2)
    rc = binding.layer_norm(M, N, TYPE[type], X.ptr, X.ld, R.ptr if residual else None, R.ld, G.ptr, B.ptr if beta else None, EPS, H.ptr, H.ld, Y.ptr, Y.ld,
                            Q.ptr, Q.ld, S.ptr, mu.ptr, rs.ptr, stream())
    assert rc == binding.OK, binding.strerror(rc)
    torch.cuda.synchronize()
    h = rounded(X.values() + R.values(), type) if residual else X.values()
    assert np.array_equal(H.fetch(), h)
    mean, rstd, y, off = layer_norm(h, G.values(), B.values() if beta else np.zeros((1, N)), EPS)
    assert_within(mu.fetch(), mean.T, F32 * np.abs(h).mean(1)[None] + 2.0 ** -149, "mean")
    # (the mean's own error adds its square to the variance)
    assert_within(rs.fetch(), rstd.T, rstd.T * (F32 + (F32 * np.abs(h).mean(1)[None]) ** 2 * rstd.T ** 2), "rstd")
    assert_within(Y.fetch(), y, rounding(y, off, type), "y")
    check_steps(y, off, Q.fetch(), S.fetch()[0], "q")


@pytest.mark.parametrize("outputs", ["h", "y", "q", "mean", "rstd", "yq", "hq", ""])
@pytest.mark.parametrize("M,N", [(5, 300), (5, 3000), (700, 5000), (3, 17000)])
def test_norm_outputs_alone(outputs, M, N):
    type = "bf16"
    X, R, G, B = operands(type, M, N, N)

    def make():
        return [Mat(type, M, N), Mat(type, M, N), Ints(I8, M, N), Mat("f32", 1, M), Mat("f32", 1, M), Mat("f32", 1, M)]

    def call(m, want):
        H, Y, Q, S, mu, rs = (t.ptr if on else None for t, on in zip(m, ["h" in want, "y" in want, "q" in want, "q" in want, "mean" in want, "rstd" in want]))
        assert binding.layer_norm(M, N, TYPE[type], X.ptr, X.ld, R.ptr, R.ld, G.ptr, B.ptr, EPS, H, N, Y, N, Q, N, S, mu, rs, stream()) == binding.OK

    full, some = make(), make()
    call(full, "h y q mean rstd")
    call(some, outputs)
    torch.cuda.synchronize()
    for a, b, name in zip(full, some, ["h", "y", "q", "q", "mean", "rstd"]):
        if name in outputs:
            assert np.array_equal(a.fetch(), b.fetch()), name
        else:
            assert torch.equal(b.dev.cpu().view(torch.uint8), b.host.view(torch.uint8)), f"{name} was written"


@pytest.mark.parametrize("N", [256, 4000, 16400])
@pytest.mark.parametrize("into", ["x", "r"])
def test_norm_in_place(N, into):
    M, type = 6, "f16"
    X, R, G, B = operands(type, M, N, N)
    H, Y, Y2 = Mat(type, M, N), Mat(type, M, N), Mat(type, M, N)
    assert binding.layer_norm(M, N, TYPE[type], X.ptr, X.ld, R.ptr, R.ld, G.ptr, B.ptr, EPS, H.ptr, N, Y.ptr, N, None, 0, None, None, None, stream()) == binding.OK
    target = X if into == "x" else R
    assert binding.layer_norm(M, N, TYPE[type], X.ptr, X.ld, R.ptr, R.ld, G.ptr, B.ptr, EPS, target.ptr, target.ld, Y2.ptr, N, None, 0, None, None, None, stream()) == binding.OK
    torch.cuda.synchronize()
    assert np.array_equal(Y.fetch(), Y2.fetch()) and np.array_equal(target._view(target.dev.cpu())[0].double().numpy(), H.fetch())


@pytest.mark.parametrize("N", [384, 3000, 17000])
def test_norm_far_from_zero_constant_rows_infinities_and_nans(N):
    M, type = 7, "bf16"
    rng = np.random.default_rng(N)
    x = np.zeros((M, N))
    x[0] = 3.0                                   # constant: the variance is 0 to the bit (sums of 3s are exact), y = beta
    x[1] = 256 + 2.0 * rng.integers(0, 2, N)     # far from zero: the squares about the mean, not their difference
    x[2, 5] = np.inf
    x[3, 200] = np.nan
    x[4, ::2], x[4, 1::2] = 1e30, -1e30          # squares that f32 does not hold: rstd 0, y = beta
    x[5] = 0.0
    x[6] = 1e-20 * rng.standard_normal(N)
    X = Mat(type, M, N, None, 0, x)
    G, B = Mat(type, 1, N, None, 0, np.ones((1, N))), Mat(type, 1, N, None, 0, np.full((1, N), 0.5))
    Y, Q, S, mu, rs = Mat(type, M, N), Ints(I8, M, N), Mat("f32", 1, M), Mat("f32", 1, M), Mat("f32", 1, M)
    assert binding.layer_norm(M, N, TYPE[type], X.ptr, N, None, 0, G.ptr, B.ptr, EPS, None, 0, Y.ptr, N, Q.ptr, N, S.ptr, mu.ptr, rs.ptr, stream()) == binding.OK
    torch.cuda.synchronize()
    y, q, s, rstd = Y.fetch(), Q.fetch(), S.fetch()[0], rs.fetch()[0]
    for i in (0, 4, 5):
        assert (y[i] == 0.5).all() and (q[i] == 127).all()
    assert rstd[4] == 0 and np.isclose(rstd[0], EPS ** -0.5, rtol=1e-6)
    h = X.values()
    _, want_rstd, want, off = layer_norm(h[[1, 6]], np.ones((1, N)), np.full((1, N), 0.5), EPS)
    assert_within(rstd[[1, 6]], want_rstd[:, 0], want_rstd[:, 0] * F32 * (1 + F32 * 256 ** 2), "rstd far from zero")
    assert_within(y[[1, 6]], want, rounding(want, off, type), "y far from zero")
    for i in (2, 3):
        assert np.isnan(y[i]).all() and np.isnan(s[i]) and (q[i] == 0).all() and np.isnan(rstd[i])


GRADS = [(1, 1), (1, 8), (2, 7), (5, 130), (16, 512), (3, 520), (17, 1024), (33, 2047), (9, 4000), (2, 4096), (7, 8192), (3, 8200), (2, 16384), (3, 16400), (1, 20001),
         (600, 64), (1030, 264), (5000, 8), (530, 8192)]


def grad_inputs(type, M, N, seed):
    rng = np.random.default_rng(seed)
    D, H = Mat(type, M, N, N + 3, 1, rng.standard_normal((M, N))), Mat(type, M, N, N + 8, 0, 2 * rng.standard_normal((M, N)) + 0.5)
    U, G = Mat(type, M, N, N + 1, 2, rng.standard_normal((M, N))), Mat(type, 1, N, None, 1, 1 + 0.2 * rng.standard_normal((1, N)))
    h = H.values()
    mean, var = h.mean(1), h.var(1)
    return D, H, U, G, Mat("f32", 1, M, None, 0, mean), Mat("f32", 1, M, None, 0, 1 / np.sqrt(var + EPS))


def check_gradients(inputs, residual, dx, dgamma, dbeta):
    """Against the formula, of the operands as they are stored."""
    D, H, U, G, MU, RS = inputs
    M, type = D.rows, D.kind
    dy, h, up, gamma, mean, rstd = D.values(), H.values(), U.values(), G.values(), MU.values().reshape(M, 1), RS.values().reshape(M, 1)
    g, xhat = dy * gamma, (h - mean) * rstd
    m1, m2 = g.mean(1, keepdims=True), (g * xhat).mean(1, keepdims=True)
    want = rstd * (g - m1 - xhat * m2) + (up if residual else 0)
    # sums of g and g xhat by F32 of their magnitudes, xhat by the roundings of h - mean and its product, the others by a few 2^-24
    xoff = 2.0 ** -22 * (np.abs(h) + np.abs(mean)) * rstd
    off = rstd * (F32 * (np.abs(g) + np.abs(g).mean(1, keepdims=True) + np.abs(xhat) * np.abs(g * xhat).mean(1, keepdims=True)) +
                  np.abs(xhat) * (np.abs(g) * xoff).mean(1, keepdims=True) + xoff * np.abs(m2)) + (2.0 ** -23 * np.abs(up) if residual else 0)
    assert_within(dx, want, rounding(want, off, type), "dx")
    # a workgroup adds up to M / 256 + 1 rows in a row, then up to 16 of its slots and 16 + 16 of all
    depth = (M / 256 + 64) * 2.0 ** -24
    assert_within(dgamma, (dy * xhat).sum(0), (depth * np.abs(dy * xhat) + np.abs(dy) * xoff).sum(0) + 2.0 ** -149, "dgamma")
    assert_within(dbeta, dy.sum(0), depth * np.abs(dy).sum(0) + 2.0 ** -149, "dbeta")


@pytest.mark.parametrize("M,N", GRADS)
@pytest.mark.parametrize("type,residual", [("f16", True), ("bf16", False), ("bf16", True)])
def test_gradients(M, N, type, residual):
    inputs = D, H, U, G, MU, RS = grad_inputs(type, M, N, M * N)
    need = binding.layer_norm_grad_workspace_bytes(M, N)
    assert 0 < need <= 2048 * N
    ws = torch.full((need // 4 + 4,), float("nan"), device="cuda")
    results = []
    for _ in range(2):
        dX, dG, dB = Mat(type, M, N, N + 2, 1), Mat("f32", 1, N), Mat("f32", 1, N, None, 1)
        rc = binding.layer_norm_grad(M, N, TYPE[type], D.ptr, D.ld, H.ptr, H.ld, G.ptr, MU.ptr, RS.ptr, U.ptr if residual else None, U.ld, dX.ptr, dX.ld, dG.ptr, dB.ptr,
                                     ws, need, stream())
        assert rc == binding.OK, binding.strerror(rc)
        torch.cuda.synchronize()
        results.append((dX.fetch(), dG.fetch()[0], dB.fetch()[0]))
    assert all(np.array_equal(a, b) for a, b in zip(*results))               # a fixed order of sums
    assert bool(torch.isnan(ws[need // 4:]).all())
    check_gradients(inputs, residual, *results[0])


@pytest.mark.parametrize("wanted", ["gamma", "beta", "none"])
@pytest.mark.parametrize("M,N", [(3, 40), (300, 136), (40, 17000)])
def test_gradients_of_one_of_gamma_and_beta(wanted, M, N):
    type = "f16"
    D, H, U, G, MU, RS = grad_inputs(type, M, N, 3)
    need = binding.layer_norm_grad_workspace_bytes(M, N)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out = []
    for want in ("gamma beta", wanted):
        dX, dG, dB = Mat(type, M, N), Mat("f32", 1, N), Mat("f32", 1, N)
        assert binding.layer_norm_grad(M, N, TYPE[type], D.ptr, D.ld, H.ptr, H.ld, G.ptr, MU.ptr, RS.ptr, U.ptr, U.ld, dX.ptr, N, dG.ptr if "gamma" in want else None,
                                       dB.ptr if "beta" in want else None, ws if want != "none" else None, need if want != "none" else 0, stream()) == binding.OK
        torch.cuda.synchronize()
        out.append((dX.fetch(), dG.fetch(), dB.fetch()))
    assert np.array_equal(out[0][0], out[1][0])
    for i, name in ((1, "gamma"), (2, "beta")):
        assert np.array_equal(out[1][i], out[0][i] if name == wanted else np.full((1, N), -1234.0))


@pytest.mark.parametrize("M,N", [(300, 264), (900, 264), (20, 9000), (300, 17000)])
@pytest.mark.parametrize("into", ["dy", "dh"])
def test_gradients_in_place(M, N, into):
    """(Not to the bits of other places: dY is read twice by the form for few rows, so that one is not taken where dX takes its place.)"""
    type = "bf16"
    inputs = D, H, U, G, MU, RS = grad_inputs(type, M, N, 5)
    need = binding.layer_norm_grad_workspace_bytes(M, N)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    dG, dB = torch.zeros(N, device="cuda"), torch.zeros(N, device="cuda")
    t = D if into == "dy" else U
    assert binding.layer_norm_grad(M, N, TYPE[type], D.ptr, D.ld, H.ptr, H.ld, G.ptr, MU.ptr, RS.ptr, U.ptr, U.ld, t.ptr, t.ld, dG, dB, ws, need, stream()) == binding.OK
    torch.cuda.synchronize()
    check_gradients(inputs, True, t._view(t.dev.cpu())[0].double().numpy(), dG.double().cpu().numpy(), dB.double().cpu().numpy())


def test_gradients_of_no_rows():
    N = 300
    dG, dB = torch.full((N,), 3.0, device="cuda"), torch.full((N,), 3.0, device="cuda")
    assert binding.layer_norm_grad(0, N, TYPE["f16"], None, N, None, N, None, None, None, None, 0, None, N, dG, dB, None, 0, stream()) == binding.OK
    assert bool((dG == 0).all()) and bool((dB == 0).all())


@pytest.mark.parametrize("M,N", [(3, 40), (2, 700)])
def test_gradients_against_differences(M, N):
    """Of the loss <dy, y> + <dh, h>, by central differences of the norm's definition in 64 bits."""
    type = "f16"
    D, H, U, G, MU, RS = grad_inputs(type, M, N, 11)
    dy, h, up, gamma = D.values(), H.values(), U.values(), G.values()
    beta = np.zeros((1, N))
    dX, dG, dB = Mat(type, M, N), Mat("f32", 1, N), Mat("f32", 1, N)
    need = binding.layer_norm_grad_workspace_bytes(M, N)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    assert binding.layer_norm_grad(M, N, TYPE[type], D.ptr, D.ld, H.ptr, H.ld, G.ptr, MU.ptr, RS.ptr, U.ptr, U.ld, dX.ptr, N, dG.ptr, dB.ptr, ws, need, stream()) == binding.OK
    torch.cuda.synchronize()

    def loss(h, gamma, beta):
        return (dy * layer_norm(h, gamma, beta, EPS)[2]).sum() + (up * h).sum()
    rng, step = np.random.default_rng(1), 1e-5
    for got, at in ((dX.fetch(), 0), (dG.fetch(), 1), (dB.fetch(), 2)):
        for _ in range(8):
            args = [h, gamma, beta]
            v = rng.standard_normal(args[at].shape)
            ends = []
            for sign in (1, -1):
                moved = list(args)
                moved[at] = args[at] + sign * step * v
                ends.append(loss(*moved))
            slope = (ends[0] - ends[1]) / (2 * step)
            # the rounding of each element of dx to f16, differences' own error far below
            assert abs((got * v).sum() - slope) <= np.abs(v * got).sum() * (2 * UNIT[type]) + 1e-6 * abs(slope) + 1e-4


ROWS = [(1, 1), (3, 7), (5, 130), (16, 512), (9, 1000), (17, 2048), (600, 2050), (4, 4000), (3, 8192), (520, 8192), (2, 16384), (2, 16400), (1, 40001)]


@pytest.mark.parametrize("M,N", ROWS)
@pytest.mark.parametrize("type", ["f16", "bf16"])
@pytest.mark.parametrize("act", [binding.ACT_NONE, binding.ACT_RELU])
def test_rows_to_integers_to_the_bit(M, N, type, act):
    rng = np.random.default_rng(M * N + act)
    X = Mat(type, M, N, N + 3, 1, rng.standard_normal((M, N)) * np.exp(3 * rng.standard_normal((M, 1))))
    Q, S = Ints(I8, M, N, N + 1, 3), Mat("f32", 1, M, None, 1)
    assert binding.quantize_i8_rows(M, N, TYPE[type], act, X.ptr, X.ld, Q.ptr, Q.ld, S.ptr, stream()) == binding.OK
    torch.cuda.synchronize()
    x = X.values()
    q, s = quantized(np.maximum(x, 0) if act else x)
    assert np.array_equal(S.fetch()[0], s.astype(np.float64), equal_nan=True) and np.array_equal(Q.fetch(), q)


@pytest.mark.parametrize("type", ["f16", "bf16"])
def test_borders_between_integers_to_the_bit(type):
    """Every value of the type from a quarter to 127 steps, under 40 largest values: those next to a border are told from those on it."""
    bits = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(torch.float16 if type == "f16" else torch.bfloat16).double().numpy()
    values = bits[np.isfinite(bits) & (np.abs(bits) >= 2.0 ** -6) & (np.abs(bits) <= 64)]
    tops = rounded(np.concatenate([[64.0, 127.0, 63.5, 31.75, 95.25], 64 + 64 * np.random.default_rng(0).random(35)]), type)
    x = np.concatenate([np.tile(values, (len(tops), 1)), tops[:, None]], 1)
    M, N = x.shape
    X, Q, S = Mat(type, M, N, None, 0, x), Ints(I8, M, N), Mat("f32", 1, M)
    assert binding.quantize_i8_rows(M, N, TYPE[type], 0, X.ptr, N, Q.ptr, N, S.ptr, stream()) == binding.OK
    torch.cuda.synchronize()
    q, s = quantized(x)
    assert np.array_equal(S.fetch()[0], s.astype(np.float64), equal_nan=True) and np.array_equal(Q.fetch(), q)


@pytest.mark.parametrize("M,N", [(1, 1), (5, 130), (17, 1000), (600, 4096), (3, 9000), (2, 17000)])
@pytest.mark.parametrize("type", ["f16", "bf16"])
def test_swiglu_rows_to_integers(M, N, type):
    rng = np.random.default_rng(M * N)
    X = Mat(type, M, 2 * N, 2 * N + 5, 1, 3 * rng.standard_normal((M, 2 * N)))
    Q, S = Ints(I8, M, N, N + 1), Mat("f32", 1, M)
    assert binding.quantize_i8_rows(M, N, TYPE[type], binding.ACT_SWIGLU, X.ptr, X.ld, Q.ptr, Q.ld, S.ptr, stream()) == binding.OK
    torch.cuda.synchronize()
    g, u = X.values()[:, :N], X.values()[:, N:]
    y = g / (1 + np.exp(-g)) * u
    check_steps(y, np.abs(y) * 1e-6, Q.fetch(), S.fetch()[0], "swiglu")


@pytest.mark.parametrize("N", [200, 3000, 17000])
def test_integers_of_zeros_infinities_nans_and_extremes(N):
    M, type = 6, "bf16"
    x = np.ones((M, N))
    x[0] = 0
    x[1, 3] = np.inf
    x[2, 100] = np.nan
    x[3] = 3e38
    x[4] = 2.0 ** -120                                       # below the floor: zeros
    x[5, 1:] = -1.0
    X, Q, S = Mat(type, M, N, None, 0, x), Ints(I8, M, N), Mat("f32", 1, M)
    assert binding.quantize_i8_rows(M, N, TYPE[type], 0, X.ptr, N, Q.ptr, N, S.ptr, stream()) == binding.OK
    torch.cuda.synchronize()
    q, s = Q.fetch(), S.fetch()[0]
    assert (q[[0, 1, 2, 4]] == 0).all() and (q[3] == 127).all() and q[5, 0] == 127 and (q[5, 1:] == -127).all()
    assert np.isnan(s[[1, 2]]).all() and np.array_equal(s[[0, 3, 4, 5]], row_scales(X.values()[[0, 3, 4, 5]]).astype(np.float64))


def test_more_rows_than_a_launch():
    M, N, type = (1 << 21) + 5, 8, "bf16"
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(M, N, device="cuda", generator=g).bfloat16()
    gamma = torch.ones(N, device="cuda").bfloat16()
    h, y, q = torch.zeros_like(x), torch.zeros_like(x), torch.zeros(M, N, dtype=I8, device="cuda")
    mean, rstd, scale, scale2 = (torch.zeros(M, device="cuda") for _ in range(4))
    q2 = torch.zeros_like(q)
    binding.check(binding.layer_norm(M, N, TYPE[type], x, N, x, N, gamma, None, EPS, h, N, y, N, q, N, scale, mean, rstd, stream()))
    binding.check(binding.quantize_i8_rows(M, N, TYPE[type], 0, h, N, q2, N, scale2, stream()))
    assert torch.equal(h, (x.float() * 2).bfloat16())
    rows = torch.cat([torch.arange(1000), torch.arange(M - 1000, M)]).cuda()
    hd = h[rows].double().cpu().numpy()
    m, r, want, off = layer_norm(hd, np.ones((1, N)), np.zeros((1, N)), EPS)
    assert_within(y[rows].double().cpu().numpy(), want, rounding(want, off, type), "y")
    assert_within(mean[rows].double().cpu().numpy(), m[:, 0], F32 * np.abs(hd).mean(1), "mean")
    qw, sw = quantized(hd)
    assert np.array_equal(q2[rows].cpu().numpy(), qw) and np.array_equal(scale2[rows].cpu().numpy(), sw)
    assert bool((scale > 0).all()) and bool((scale2 > 0).all()) and bool((rstd > 0).all())
    assert LEAST[type] > 0


def test_rows_beyond_the_range():
    """Sums that pass f32's range: NaN; squares only: beta.  Neighbouring rows keep their values."""
    M, N, type = 5, 300, "bf16"
    rng = np.random.default_rng(4)
    x = rng.standard_normal((M, N))
    x[1] = 3e38                                              # the sum
    x[3] = rng.choice([-1e30, 1e30], N)                      # squares
    X, G, B = Mat(type, M, N, None, 0, x), Mat(type, 1, N, None, 0, rng.standard_normal((1, N))), Mat(type, 1, N, None, 0, rng.standard_normal((1, N)))
    Y, Q, S, mean, rstd = Mat(type, M, N), Ints(I8, M, N), Mat("f32", 1, M), Mat("f32", 1, M), Mat("f32", 1, M)
    assert binding.layer_norm(M, N, TYPE[type], X.ptr, N, None, 0, G.ptr, B.ptr, EPS, None, 0, Y.ptr, N, Q.ptr, N, S.ptr, mean.ptr, rstd.ptr, stream()) == binding.OK
    torch.cuda.synchronize()
    y, q, s, r = Y.fetch(), Q.fetch(), S.fetch()[0], rstd.fetch()[0]
    assert np.isnan(y[1]).all() and np.isnan(s[1]) and (q[1] == 0).all()
    assert r[3] == 0 and np.array_equal(y[3], B.values()[0]) and np.array_equal(q[3:4], quantized(B.values())[0])
    rows = [0, 2, 4]
    _, _, want, off = layer_norm(X.values()[rows], G.values(), B.values(), EPS)
    assert_within(y[rows], want, rounding(want, off, type), "y")


def test_more_columns_than_a_launch():
    """The columns' sums of one row of more than 2^28, 16 threads a column."""
    N, type = (1 << 28) + 72, "bf16"
    h = torch.randint(-3, 4, (N,), dtype=torch.int8, device="cuda").bfloat16()
    dy = torch.roll(h, 1) + 0.5
    gamma, dx = torch.ones_like(h), torch.zeros_like(h)
    mean, rstd = torch.full((1,), 0.25, device="cuda"), torch.full((1,), 0.5, device="cuda")
    dgamma, dbeta = torch.zeros(N, device="cuda"), torch.zeros(N, device="cuda")
    need = binding.layer_norm_grad_workspace_bytes(1, N)
    work = torch.zeros(need, dtype=torch.uint8, device="cuda")
    binding.check(binding.layer_norm_grad(1, N, TYPE[type], dy, N, h, N, gamma, mean, rstd, None, 0, dx, N, dgamma, dbeta, work, need, stream()))
    assert torch.equal(dbeta, dy.float()) and torch.equal(dgamma, dy.float() * ((h.float() - 0.25) * 0.5))       # exact: few bits each
    assert bool(dx.isfinite().all()) and bool((dx[-72:] != 0).any())
