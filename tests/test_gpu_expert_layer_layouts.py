"""paper_2108_13191_amd/expert_layer.py on callers' matrices of other layouts: the bits of contiguous copies."""
import pytest
import torch

from paper_2108_13191_amd.expert_layer import ExpertLayer

pytestmark = pytest.mark.gpu


def columns(t):
    wide = torch.full((t.shape[0], t.shape[1] + 40), float("nan"), dtype=t.dtype, device=t.device)
    wide[:, 16:16 + t.shape[1]] = t
    return wide[:, 16:16 + t.shape[1]]


@pytest.mark.parametrize("lay", [columns, lambda t: t.t().contiguous().t()], ids=["columns", "transposed"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16], ids=["bf16", "f16"])
def test_matrices_of_any_layout(lay, dtype):
    layer = ExpertLayer(264, 200, 8, 3, dtype=dtype, seed=3)
    layer.prepare()
    gen = torch.Generator().manual_seed(5)
    x, r, dout, dh = (torch.randn(37, 264, generator=gen).to(dtype).cuda() for _ in range(4))
    for a, b in (((x, r, dout, dh), tuple(map(lay, (x, r, dout, dh)))), ((x, r, dout[:1].expand(37, 264).contiguous(), dh), (x, r, dout[:1].expand(37, 264), dh))):
        served, s = [layer.serve(*t[:2]) for t in (a, b)], [layer.train_forward(*t[:2]) for t in (a, b)]
        assert torch.equal(served[0].out, served[1].out) and torch.equal(s[0].out, s[1].out) and torch.equal(s[0].h, s[1].h)
        one, two = vars(layer.backward(s[0], *a[2:])), vars(layer.backward(s[1], *b[2:]))
        for name in one:
            assert torch.equal(one[name], two[name]), name
