"""What the quantisers round, to the bit: an element is the e4m3 value nearest to its f32 value divided by the scale that is stored beside it, ties
to even; and SwiGLU in f32 to a few units in the last place whatever the gate."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2108_13191_amd import binding                                    # noqa: E402
from ops_util import DT, TYPE, ceil128, stream                              # noqa: E402


def bits(t):
    return t.contiguous().view(torch.uint8)


def quotients(y, scale):
    """e4m3(y / scale) on the host: both roundings to nearest even."""
    return (y / scale).to(DT["e4m3"])


@pytest.mark.parametrize("M,N", [(64, 4096), (300, 1000), (129, 8200)])
@pytest.mark.parametrize("type", ["f16", "bf16"])
@pytest.mark.parametrize("act", ["none", "relu"])
def test_rows_hold_the_nearest_quotients(M, N, type, act):
    x = (torch.randn(M, N, generator=torch.Generator().manual_seed(M)) * 3.0).to(DT[type])
    q, s = torch.empty(M, N, dtype=DT["e4m3"], device="cuda"), torch.empty(ceil128(N), M, device="cuda")
    code = binding.ACT_RELU if act == "relu" else binding.ACT_NONE
    binding.check(binding.quantize_e4m3_rows(M, N, TYPE[type], code, x.cuda(), N, q, N, s, M, stream()))
    y = x.float().clamp_min(0.0) if act == "relu" else x.float()
    most = torch.nn.functional.pad(y, (0, -N % 128)).view(M, -1, 128).abs().amax(2).clamp_min(2.0 ** -96)
    assert torch.equal(s.cpu().t(), most / 448.0)
    want = quotients(y, s.cpu().t().repeat_interleave(128, 1)[:, :N])
    assert torch.equal(bits(q.cpu()), bits(want))


@pytest.mark.parametrize("M,N", [(256, 2048), (300, 1000)])
@pytest.mark.parametrize("type", ["f16", "bf16"])
def test_blocks_hold_the_nearest_quotients(M, N, type):
    x = (torch.randn(M, N, generator=torch.Generator().manual_seed(N)) * 0.02).to(DT[type])
    q, s = torch.empty(M, N, dtype=DT["e4m3"], device="cuda"), torch.empty(ceil128(M), ceil128(N), device="cuda")
    binding.check(binding.quantize_e4m3_blocks(M, N, TYPE[type], x.cuda(), N, q, N, s, ceil128(N), stream()))
    want = quotients(x.float(), s.cpu().repeat_interleave(128, 0)[:M].repeat_interleave(128, 1)[:, :N])
    assert torch.equal(bits(q.cpu()), bits(want))


@pytest.mark.parametrize("N", [2048, 4096, 8192, 16384, 32768])
def test_the_norm_holds_the_nearest_quotients(N):
    """Rows of +-1 and +-7, 11 to 5, have the mean square 16: rstd is 1/4 and y exact in f32, whatever the order of the sum."""
    M, gen = 24, torch.Generator().manual_seed(N)
    row = torch.tensor([1.0] * 11 + [7.0] * 5).repeat(N // 16)
    x = torch.stack([row[torch.randperm(N, generator=gen)] for _ in range(M)]) * (torch.randint(0, 2, (M, N), generator=gen) * 2 - 1)
    gamma = (1.0 + 0.1 * torch.randn(N, generator=gen)).bfloat16()
    q, s = torch.empty(M, N, dtype=DT["e4m3"], device="cuda"), torch.empty(N // 128, M, device="cuda")
    binding.check(binding.rms_norm(M, N, TYPE["bf16"], x.bfloat16().cuda(), N, None, 0, gamma.cuda(), 0.0, None, 0, None, 0, q, N, s, M, None, stream()))
    want = quotients(x * 0.25 * gamma.float(), s.cpu().t().repeat_interleave(128, 1))
    assert torch.equal(bits(q.cpu()), bits(want))


@pytest.mark.parametrize("type", ["f16", "bf16"])
def test_swiglu_is_as_exact_for_every_gate(type):
    """A block of one gate value and one u: its scale is the magnitude of the result over 448.  f32 has 6e-8 of relative error in each of exp, its
    argument's correction, 1 + exp, the reciprocal (two units), three products and the scale's division: below 1e-6 together."""
    g = torch.linspace(-86.0, 86.0, 4001).to(DT[type])
    M = g.numel()
    x = torch.cat([g[:, None].expand(M, 128), torch.full((M, 128), 3.0, dtype=DT[type])], 1).contiguous().cuda()
    q, s = torch.empty(M, 128, dtype=DT["e4m3"], device="cuda"), torch.empty(1, M, device="cuda")
    binding.check(binding.quantize_e4m3_rows(M, 128, TYPE[type], binding.ACT_SWIGLU, x, 256, q, 128, s, M, stream()))
    y = g.double().numpy()
    want = np.maximum(np.abs(y / (1.0 + np.exp(-y)) * 3.0), 2.0 ** -96) / 448.0
    assert (np.abs(s.cpu().double().numpy()[0] - want) <= 1e-6 * want).all()


def test_swiglu_of_the_largest_gates_and_infinities():
    """exp beyond f32's range: 0 below, the gate itself above; an infinite gate shows in its block."""
    g = torch.tensor([-3e38, -1e4, -200.0, 200.0, 1e4, 3e38, float("-inf"), float("inf"), float("nan")]).bfloat16()
    M = g.numel()
    x = torch.cat([g[:, None].expand(M, 128), torch.ones(M, 128, dtype=torch.bfloat16)], 1).contiguous().cuda()
    q, s = torch.empty(M, 128, dtype=DT["e4m3"], device="cuda"), torch.empty(1, M, device="cuda")
    binding.check(binding.quantize_e4m3_rows(M, 128, TYPE["bf16"], binding.ACT_SWIGLU, x, 256, q, 128, s, M, stream()))
    q, s = q.float().cpu(), s.cpu()[0]
    assert (q[:3] == 0).all() and (q[3:6] == 448).all() and q[6:].isnan().all() and s[6:].isnan().all()
    assert torch.equal(s[:3], torch.full((3,), 2.0 ** -96) / 448.0) and torch.equal(s[3:6], g[3:6].float() / 448.0)
