"""Sums over the rows of layer norm's gradients: how many additions follow one another in f32."""
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2108_13191_amd import binding                                                       # noqa: E402
from ops_util import TYPE, stream                                                              # noqa: E402


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
