"""Layer norm of many rows: how many additions follow one another in f32 in its gradients' sums over rows, and rows beyond what one launch takes."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2108_13191_amd import binding                                                       # noqa: E402
from layer_util import F32, layer_norm, quantized, rounding                                    # noqa: E402
from ops_util import TYPE, assert_within, stream                                               # noqa: E402
from test_gpu_layer_norm import EPS, check_steps                                               # noqa: E402


@pytest.mark.parametrize("M,N", [(20000, 8200), (20000, 8193), (9000, 16384), (20000, 4000), (20000, 8192), (40000, 768), (40000, 100), (9000, 16400)])
@pytest.mark.parametrize("in_place", [False, True])
def test_small_terms_behind_large_ones(M, N, in_place):
    """Rows of 2^24 in front of rows of 1, each of which a sum that has reached 2^24 loses: the error is what follows one another.  At most M / 256 + 64 additions do, each off by
    half a unit of what it gives."""
    dy = torch.ones(M, N, dtype=torch.bfloat16, device="cuda")
    dy[:64] = 2.0 ** 24
    h, gamma, dx = torch.ones_like(dy), torch.ones(N, dtype=torch.bfloat16, device="cuda"), dy if in_place else torch.empty_like(dy)
    mean, rstd = torch.zeros(M, device="cuda"), torch.ones(M, device="cuda")
    dgamma, dbeta = torch.zeros(N, device="cuda"), torch.zeros(N, device="cuda")
    need = binding.layer_norm_grad_workspace_bytes(M, N)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    binding.check(binding.layer_norm_grad(M, N, TYPE["bf16"], dy, N, h, N, gamma, mean, rstd, None, 0, dx, N, dgamma, dbeta, work, need, stream()))
    want = 64 * 2 ** 24 + M - 64
    for name, got in (("dgamma", dgamma), ("dbeta", dbeta)):
        off = (got.double() - want).abs().max().item()
        assert off <= (M / 256 + 64) * 2.0 ** -24 * want, f"{name} off by {off}"


@pytest.mark.parametrize("type", ["bf16", "f16"])
def test_both_sides_of_a_launchs_last_row(type):
    """Everything that a row gives, of rows at both ends and around row 2^21, where the second launch begins; what lies behind the last row stays."""
    M, N, launch = (1 << 21) + 700, 12, 1 << 21
    dtype = torch.bfloat16 if type == "bf16" else torch.float16
    g = torch.Generator(device="cuda").manual_seed(2)
    x, r = ((torch.randn(M, N, device="cuda", generator=g) * 2 + 0.5).to(dtype) for _ in range(2))
    gamma, beta = (1 + 0.2 * torch.randn(N, device="cuda", generator=g)).to(dtype), (0.3 * torch.randn(N, device="cuda", generator=g)).to(dtype)
    h, y, q, q2 = (torch.full((M + 2, N), 77, dtype=t, device="cuda") for t in (dtype, dtype, torch.int8, torch.int8))
    mean, rstd, scale, scale2 = (torch.full((M + 2,), -7.0, device="cuda") for _ in range(4))
    binding.check(binding.layer_norm(M, N, TYPE[type], x, N, r, N, gamma, beta, EPS, h, N, y, N, q, N, scale, mean, rstd, stream()))
    binding.check(binding.quantize_i8_rows(M, N, TYPE[type], binding.ACT_NONE, x, N, q2, N, scale2, stream()))
    for t in (h, y, q, q2):
        assert bool((t[M:] == 77).all())
    for t in (mean, rstd, scale, scale2):
        assert bool((t[M:] == -7).all())
    assert torch.equal(h[:M], (x.float() + r.float()).to(dtype))
    at = torch.cat([torch.arange(600), torch.arange(launch - 600, M)]).cuda()

    def take(t):
        return t[at].double().cpu().numpy()
    m, s, want, off = layer_norm(take(h), gamma.double().cpu().numpy()[None], beta.double().cpu().numpy()[None], EPS)
    magnitude = abs(take(h)).mean(1)
    assert_within(take(mean), m[:, 0], F32 * magnitude, "mean")
    assert_within(take(rstd), s[:, 0], s[:, 0] * (F32 + (F32 * magnitude * s[:, 0]) ** 2), "rstd")
    assert_within(take(y), want, rounding(want, off, type), "y")
    check_steps(want, off, take(q), take(scale), "q")
    qw, sw = quantized(take(x))
    assert (take(q2) == qw).all() and (take(scale2) == sw).all()
    # and the gradients, which take any number of rows in one launch
    dy = torch.randn(M, N, device="cuda", generator=g).to(dtype)
    dx, dgamma, dbeta = torch.full((M + 2, N), 77, dtype=dtype, device="cuda"), torch.zeros(N, device="cuda"), torch.zeros(N, device="cuda")
    need = binding.layer_norm_grad_workspace_bytes(M, N)
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    binding.check(binding.layer_norm_grad(M, N, TYPE[type], dy, N, h, N, gamma, mean, rstd, None, 0, dx, N, dgamma, dbeta, work, need, stream()))
    assert bool((dx[M:] == 77).all())
    d, xhat = take(dy), (take(h) - take(mean)[:, None]) * take(rstd)[:, None]
    gd = d * gamma.double().cpu().numpy()
    want = take(rstd)[:, None] * (gd - gd.mean(1, keepdims=True) - xhat * (gd * xhat).mean(1, keepdims=True))
    # twelve terms and a few operations, each by 2^-24 of what it has: below F32 of the largest terms
    off = F32 * take(rstd)[:, None] * (abs(gd) + abs(gd).mean(1, keepdims=True) + abs(xhat) * abs(gd * xhat).mean(1, keepdims=True)) * (1 + magnitude[:, None] * take(rstd)[:, None])
    assert_within(take(dx), want, rounding(want, off, type), "dx")
    full = (h[:M].double() - mean[:M, None].double()) * rstd[:M, None].double() * dy.double()
    assert bool(((dgamma.double() - full.sum(0)).abs() <= (M / 256 + 64) * 2.0 ** -24 * full.abs().sum(0) * 1.01).all())
    assert bool(((dbeta.double() - dy.double().sum(0)).abs() <= (M / 256 + 64) * 2.0 ** -24 * dy.double().abs().sum(0)).all())
