"""Every kernel form of the row operators of include/gemm_layer.h (the CPU test reads the rules between them) against the definitions: norms, gradients row by row and in one launch, 8-bit
rows, rows back from experts and the gradients of that, dispatched rows past the caches; in place where the header allows it."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

import test_gpu_experts as experts                                                             # noqa: E402
import test_gpu_layer_norm as rows                                                             # noqa: E402
from layer_form_cases import COMBINE, COMBINE_GRAD, GRAD, GRAD_FEW, GRAD_ONLY_IN_PLACE, NORM   # noqa: E402
from layer_util import Ints                                                                    # noqa: E402
from ops_util import LEAST, TYPE, UNIT, Mat, assert_within, stream                             # noqa: E402
from paper_2108_13191_amd import binding                                                       # noqa: E402

I32 = torch.int32
TYPES = pytest.mark.parametrize("type", ["f16", "bf16"])


@pytest.mark.parametrize("M,N", NORM)
@TYPES
def test_norm(M, N, type):
    rows.test_norm(M, N, type, True, True)


@pytest.mark.parametrize("M,N", NORM)
@TYPES
def test_rows_to_integers(M, N, type):
    rows.test_rows_to_integers_to_the_bit(M, N, type, binding.ACT_NONE)
    rows.test_swiglu_rows_to_integers(M, N, type)


def gradients(M, N, type, into):
    inputs = D, H, U, G, MU, RS = rows.grad_inputs(type, M, N, M + N)
    need = binding.layer_norm_grad_workspace_bytes(M, N)
    ws = torch.full((need // 4 + 4,), float("nan"), device="cuda")
    dG, dB = Mat("f32", 1, N), Mat("f32", 1, N, None, 1)
    dX = {"dy": D, "dh": U, None: Mat(type, M, N, N + 2, 1)}[into]
    rc = binding.layer_norm_grad(M, N, TYPE[type], D.ptr, D.ld, H.ptr, H.ld, G.ptr, MU.ptr, RS.ptr, U.ptr, U.ld, dX.ptr, dX.ld, dG.ptr, dB.ptr, ws, need, stream())
    assert rc == binding.OK, binding.strerror(rc)
    torch.cuda.synchronize()
    assert bool(torch.isnan(ws[need // 4:]).all())
    if into:
        back = dX.dev.cpu()
        dx = dX._view(back)[0].double().numpy().copy()
        dX._view(back).copy_(dX._view(dX.host))
        assert torch.equal(back.view(torch.uint8), dX.host.view(torch.uint8)), "memory outside the result was written"
    else:
        dx = dX.fetch()
    rows.check_gradients(inputs, True, dx, dG.fetch()[0], dB.fetch()[0])


@pytest.mark.parametrize("M,N", GRAD)
@pytest.mark.parametrize("type,into", [("bf16", None), ("f16", "dy"), ("bf16", "dh")])
def test_gradients_row_by_row(M, N, type, into):
    gradients(M, N, type, into)


@pytest.mark.parametrize("M,N", GRAD_ONLY_IN_PLACE)
@TYPES
def test_gradients_of_long_rows_in_place(M, N, type):
    gradients(M, N, type, "dy")


@pytest.mark.parametrize("M,N", GRAD_FEW)
@pytest.mark.parametrize("type,into", [("bf16", None), ("f16", "dh")])
def test_gradients_in_one_launch(M, N, type, into):
    gradients(M, N, type, into)


@pytest.mark.parametrize("T,k,N", COMBINE)
@pytest.mark.parametrize("type,out_type", [("f16", "f16"), ("bf16", "f32"), ("f32", "f32")])
def test_rows_back_from_experts(T, k, N, type, out_type):
    experts.test_combine(T, k, N, type, out_type, True, True, 0.2)


@pytest.mark.parametrize("T,k,N", COMBINE_GRAD)
@TYPES
def test_gradients_of_rows_back(T, k, N, type):
    experts.test_gradients(T, k, N, type, True, "rows weight", 0.2)


@pytest.mark.parametrize("T,k,N", COMBINE_GRAD)
def test_gradients_of_rows_back_in_their_place(T, k, N):
    """dY is Y: dropped choices' rows stay as they are."""
    type, rng = "bf16", np.random.default_rng(T + k + N)
    at = experts.places(rng, T, k, 0.2)
    P, W = Ints(I32, T, k, None, 1, at), Mat("f32", T, k, None, 1, rng.random((T, k)))
    Y, D, dW = Mat(type, T * k, N, N + 3, 1, rng.standard_normal((T * k, N))), Mat(type, T, N, N + 5, 3, rng.standard_normal((T, N))), Mat("f32", T, k, None, 1)
    assert binding.expert_combine_grad(T, k, N, TYPE[type], P.ptr, D.ptr, D.ld, W.ptr, Y.ptr, Y.ld, Y.ptr, Y.ld, dW.ptr, stream()) == binding.OK
    torch.cuda.synchronize()
    valid = (at >= 0) & (at < T * k)
    d, y, w = D.values().reshape(T, 1, N), Y.values().reshape(T * k, N), W.values().reshape(T, k, 1)
    want, off = y.copy(), np.zeros_like(y)
    want[at[valid]] = np.broadcast_to(w * d, (T, k, N))[valid]
    off[at[valid]] = (np.abs(w * d) * (2.0 ** -24 + (1 + 2.0 ** -24) * UNIT[type]) + LEAST[type])[valid]
    assert_within(Y._view(Y.dev.cpu())[0].double().numpy(), want, off, "dy")
    products = np.where(valid[..., None], d * y[np.where(valid, at, 0)], 0)
    depth = max(32, N / 512) + 15                            # up to 32 (or N / 512) products in a row in a lane, 6 sums of lanes and 8 of wavefronts
    assert_within(dW.fetch().reshape(T, k), products.sum(2), depth * 2.0 ** -24 * np.abs(products).sum(2), "dweight")


def test_dispatched_rows_past_the_caches():
    """134 MB of rows by part: the largest calls store past the caches."""
    T, k, E, N = 8200, 2, 16, 4099
    g = torch.Generator(device="cuda").manual_seed(7)
    expert = torch.randint(-1, E + 1, (T, k), device="cuda", generator=g)
    x = torch.randint(-2 ** 15, 2 ** 15, (T, N), dtype=torch.int16, device="cuda", generator=g)
    scale = torch.rand(1, T, device="cuda", generator=g)
    off, src, at = (torch.full((n,), 85, dtype=I32, device="cuda") for n in (E + 1, T * k, T * k))
    out, out_scale = torch.full((T * k + 1, N + 3), 85, dtype=torch.int16, device="cuda"), torch.full((1, T * k), -3.0, device="cuda")
    need = binding.expert_dispatch_workspace_bytes(T, k, E)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    for _ in range(3):
        binding.check(binding.expert_dispatch(T, k, E, binding.INDEX_I64, expert, off, src, at, N, 2, x, N, 1, scale, T, out, N + 3, out_scale, T * k, ws, need, stream()))
    key = torch.where((expert >= 0) & (expert < E), expert, E).flatten()
    by = torch.argsort(key, stable=True)
    total = int((key < E).sum())
    assert torch.equal(off.long(), torch.searchsorted(key[by], torch.arange(E + 1, device="cuda")))
    place = torch.empty_like(by)
    place[by] = torch.where(torch.arange(T * k, device="cuda") < total, torch.arange(T * k, device="cuda"), -1)
    assert torch.equal(at.long(), place) and torch.equal(src[:total].long(), by[:total] // k) and bool((src[total:] == -1).all())
    assert torch.equal(out[:total, :N], x[by[:total] // k]) and bool((out[total:] == 85).all()) and bool((out[:, N:] == 85).all())
    assert torch.equal(out_scale[0, :total], scale[0, by[:total] // k]) and bool((out_scale[0, total:] == -3.0).all())
