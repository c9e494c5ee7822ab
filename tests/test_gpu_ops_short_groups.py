"""The e4m3 product of many short groups of rows, whose tiles leave out the quarters of 128 rows that a group does not have: groups that end at,
before and behind the quarters, against the definition in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from ops_util import assert_within, result_bound                            # noqa: E402
from test_gpu_ops_products import large_e4m3                                # noqa: E402

EDGES = [1, 31, 32, 33, 0, 63, 64, 65, 95, 96, 97, 127, 128, 129, 160, 161]
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("counts", [EDGES + [3, 21, 0] * 12, [32] * 13, [0] * 40 + [400], [40, 24] * 7 + [5]], ids=["edges", "quarters", "one", "uneven"])
@pytest.mark.parametrize("K", [100, 256, 392, 1040])
@pytest.mark.parametrize("c", ["bf16", "f32"])
def test_quarters_of_a_tile(counts, K, c):
    N = 1 + 1_500_000 // sum(counts)                    # more results than the kernel for few rows takes, fewer than 2^22
    got, want, mag = large_e4m3(sum(counts) + 7, N, K, c, counts)
    assert_within(got, want, result_bound(want, mag, c), f"{counts} {N} {K}")
    got, want, _ = large_e4m3(sum(counts) + 7, N, K, c, counts, integers=True)
    assert np.array_equal(got, torch.from_numpy(want).float().to(TYPES[c]).double().numpy())
