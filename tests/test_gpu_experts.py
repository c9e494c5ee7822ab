"""Tokens sorted by expert, their rows moved there and back with weights applied, and the gradients of that, against numpy's stable sort and sums in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
if not torch.cuda.is_available():
    pytest.skip("no GPU", allow_module_level=True)

from paper_2108_13191_amd import binding                                                  # noqa: E402
from ops_util import LEAST, TYPE, UNIT, Mat, assert_within, stream                        # noqa: E402
from layer_util import Ints, order                                                        # noqa: E402

I32, I64 = torch.int32, torch.int64
ELEMENT = {1: torch.int8, 2: torch.int16, 4: torch.int32}


def choices(rng, T, k, E, drop):
    e = rng.integers(0, max(E, 1), (T, k))
    bad = rng.choice([-1, E, -2**31, 2**31 - 1], (T, k))
    return np.where((rng.random((T, k)) < drop) | (E == 0), bad, e)


def dispatch(expert, E, index=I64, N=0, size=2, blocks=0, seed=0, with_source=True, pad=0, offset=0):
    """Runs it and checks everything that it writes, and that it writes nothing else."""
    T, k = expert.shape
    n = T * k
    rng = np.random.default_rng(seed)
    ids = Ints(index, T, k, None, 1, expert)
    offsets, source, place = Ints(I32, 1, E + 1, None, 1), Ints(I32, 1, n, None, 1), Ints(I32, 1, n, None, 2)
    info = torch.iinfo(ELEMENT[size])
    X = Ints(ELEMENT[size], T, N, N + pad, offset, rng.integers(info.min, info.max + 1, (T, N)))
    rows = Ints(ELEMENT[size], n, N, N + 2 * pad, offset)
    S, RS = Mat("f32", blocks, T, T + 1, 1, rng.standard_normal((blocks, T))), Mat("f32", blocks, n, n + 2, 3)
    need = binding.expert_dispatch_workspace_bytes(T, k, E)
    assert 0 <= need <= 8 * n + (1 << 22)
    ws = torch.full((need + 16,), 0x5a, dtype=torch.uint8, device="cuda")
    rc = binding.expert_dispatch(T, k, E, binding.INDEX_I64 if index == I64 else binding.INDEX_I32, ids.ptr, offsets.ptr, source.ptr if with_source else None, place.ptr,
                                 N, size, X.ptr if N else None, X.ld, blocks, S.ptr, S.ld, rows.ptr, rows.ld, RS.ptr, RS.ld, ws, need, stream())
    assert rc == binding.OK, binding.strerror(rc)
    torch.cuda.synchronize()
    assert bool((ws[need:] == 0x5a).all())
    off, src, at = order(expert, E)
    assert np.array_equal(offsets.fetch()[0], off)
    assert np.array_equal(place.fetch()[0], at.ravel())
    assert np.array_equal(source.fetch()[0], src if with_source else np.full(n, 85))
    total = off[-1]
    want = np.full((n, N), 85)
    want[:total] = X.values().reshape(T, N)[src[:total]]
    assert np.array_equal(rows.fetch().reshape(n, N), want)
    if blocks:
        scale = np.full((blocks, n), -1234.0)
        scale[:, :total] = S.values().reshape(blocks, T)[:, src[:total]]
        assert np.array_equal(RS.fetch().reshape(blocks, n), scale)


SIZES = [(300, 3, 5000), (10, 70, 9), (256, 1, 7), (16, 4, 3), (8, 8, 2047), (65, 64, 2047), (64, 64, 1), (1000, 4, 256), (2049, 2, 30), (4096, 1, 2047), (4097, 1, 2047), (1, 1, 1), (1, 4, 4), (3, 2, 5), (7, 1, 300), (32, 2, 16), (64, 1, 8), (13, 5, 7), (128, 2, 64), (257, 1, 3), (300, 3, 1000), (128, 8, 256), (1023, 1, 5), (512, 2, 65535),
         (1025, 1, 5), (205, 5, 64), (700, 2, 2047), (700, 2, 2048), (5000, 3, 17), (4096, 8, 64), (3000, 2, 65535), (20000, 4, 128), (40000, 6, 5000), (70001, 1, 1)]


@pytest.mark.parametrize("T,k,E", SIZES)
@pytest.mark.parametrize("index,drop", [(I64, 0.0), (I32, 0.3)])
def test_order(T, k, E, index, drop):
    dispatch(choices(np.random.default_rng(T + k + E), T, k, E, drop), E, index, N=5, size=2)


# parts of more than 64 choices, whose 64s end within a token's; the first ones' experts have few rows each and many, and the last part is short
@pytest.mark.parametrize("T,k,E", [(20000, 3, 2047), (50000, 5, 300), (60000, 7, 1000), (33000, 10, 2000), (9000, 50, 2047)])
@pytest.mark.parametrize("drop", [0.0, 0.3])
def test_parts_that_end_within_a_token(T, k, E, drop):
    expert = choices(np.random.default_rng(T + k), T, k, E, drop)
    dispatch(expert, E, N=5, size=2)
    dispatch(np.minimum(expert, expert % 3), E, N=0)


# a token's choices: more than a lane each, more than are placed by part, all that a call takes
@pytest.mark.parametrize("T,k,E", [(20, 65, 9), (30, 256, 9), (30, 257, 9), (1, 1024, 5), (1, 1100, 5), (3, 700, 64), (1, 65535, 70), (2, 65535, 3000)])
def test_long_lists_of_choices(T, k, E):
    dispatch(choices(np.random.default_rng(T + k), T, k, E, 0.2), E, N=9, size=2, blocks=1)


def test_the_longest_list_comes_back():
    T, k, N = 2, 65535, 16
    gen = torch.Generator(device="cuda").manual_seed(3)
    Y, weight = torch.randn(T * k, N, device="cuda", generator=gen), torch.rand(T, k, device="cuda", generator=gen)
    place = torch.randperm(T * k, device="cuda", generator=gen).to(I32)
    out = torch.zeros(T, N, device="cuda")
    binding.check(binding.expert_combine(T, k, N, TYPE["f32"], place, Y, N, weight, None, 0, out, N, TYPE["f32"], stream()))
    terms = Y.double()[place.long()].view(T, k, N) * weight.double()[..., None]
    # each of k additions and each product rounded once in f32
    assert bool(((out.double() - terms.sum(1)).abs() <= (k + 1) * 2.0 ** -24 * terms.abs().sum(1)).all())
    b16, dY, dweight = Y.bfloat16(), torch.zeros(T * k, N, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, k, device="cuda")
    dout = torch.randn(T, N, device="cuda", generator=gen).bfloat16()
    binding.check(binding.expert_combine_grad(T, k, N, TYPE["bf16"], place, dout, N, weight, b16, N, dY, N, dweight, stream()))
    dots = b16.double()[place.long()].view(T, k, N) * dout.double()[:, None]
    assert bool(((dweight.double() - dots.sum(-1)).abs() <= (N + 1) * 2.0 ** -24 * dots.abs().sum(-1)).all())
    assert torch.equal(dY[place.long()].view(T, k, N), (weight[..., None] * dout[:, None].float()).bfloat16())


@pytest.mark.parametrize("T,k", [(5, 2), (64, 4), (700, 3), (1500, 3)])
@pytest.mark.parametrize("case", ["all one", "none", "last", "reversed", "the same twice"])
def test_orders_at_the_edges(T, k, case):
    E = 9
    expert = {"all one": np.full((T, k), 4), "none": np.full((T, k), -1), "last": np.full((T, k), E - 1),
              "reversed": np.tile((E - 1 - np.arange(T) * E // T)[:, None], (1, k)), "the same twice": np.repeat(np.arange(T)[:, None] % E, k, 1)}[case]
    dispatch(expert, E, N=33, size=1, blocks=1)


def test_no_tokens_no_choices_and_no_experts():
    for T, k in ((0, 2), (3, 0), (0, 0)):
        offsets = torch.full((301,), 7, dtype=I32, device="cuda")
        assert binding.expert_dispatch(T, k, 300, binding.INDEX_I32, None, offsets, None, None, 8, 2, None, 8, 0, None, 0, None, 8, None, 0, None, 0, stream()) == binding.OK
        assert bool((offsets == 0).all())
    dispatch(np.zeros((3, 2), int), 0, N=8, size=2)
    dispatch(np.zeros((3000, 2), int), 0, N=8, size=2)


# bytes a row: below a chunk, at its ends, at a piece's ends (4096), odd ones
@pytest.mark.parametrize("N,size", [(1, 1), (1, 2), (7, 1), (7, 2), (15, 1), (3, 4), (16, 1), (17, 1), (31, 1), (9, 2), (2048, 1), (1000, 2), (2047, 2), (2048, 2), (2049, 2), (1024, 4),
                                    (4097, 1), (3001, 4), (10007, 1)])
@pytest.mark.parametrize("T,k", [(9, 3), (3, 20), (600, 2), (2100, 2)])
def test_rows_of_any_width(N, size, T, k):
    dispatch(choices(np.random.default_rng(N), T, k, 6, 0.2), 6, N=N, size=size, pad=3, offset=1)


@pytest.mark.parametrize("blocks", [1, 3, 64, 65, 130])
@pytest.mark.parametrize("T,k", [(9, 3), (3, 20), (600, 2), (2100, 2)])
def test_scales_go_with_their_rows(blocks, T, k):
    dispatch(choices(np.random.default_rng(blocks), T, k, 6, 0.2), 6, N=40, size=1, blocks=blocks, with_source=False)


def test_only_the_order():
    dispatch(choices(np.random.default_rng(1), 40, 3, 6, 0.2), 6, N=0)
    dispatch(choices(np.random.default_rng(1), 1000, 3, 6, 0.2), 6, N=0)
    dispatch(choices(np.random.default_rng(1), 4000, 3, 6, 0.2), 6, N=0, with_source=False)


def places(rng, T, k, drop):
    """Places of T x k choices as a sort by expert leaves them: a permutation, -1 (or out of range) for some."""
    at = rng.permutation(T * k).reshape(T, k)
    return np.where(rng.random((T, k)) < drop, rng.choice([-1, T * k, -2**31, 2**31 - 1], (T, k)), at)


COMBINE = [(1, 1, 1), (3, 2, 7), (17, 3, 130), (5, 8, 512), (9, 6, 520), (300, 2, 1025), (40, 1, 2048), (33, 5, 3000), (4, 2, 8200), (2, 3, 17001), (2000, 2, 64)]


@pytest.mark.parametrize("T,k,N", COMBINE)
@pytest.mark.parametrize("type,out_type", [("f16", "f16"), ("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32")])
@pytest.mark.parametrize("weighted,add,drop", [(True, True, 0.2), (False, False, 0.0), (True, False, 0.5)])
def test_combine(T, k, N, type, out_type, weighted, add, drop):
    rng = np.random.default_rng(T * k + N)
    at = places(rng, T, k, drop)
    P, W = Ints(I32, T, k, None, 1, at), Mat("f32", T, k, None, 1, rng.random((T, k)))
    Y, A, O = Mat(type, T * k, N, N + 3, 1, rng.standard_normal((T * k, N))), Mat(type, T, N, N + 5, 0, rng.standard_normal((T, N))), Mat(out_type, T, N, N + 1, 2)
    rc = binding.expert_combine(T, k, N, TYPE[type], P.ptr, Y.ptr, Y.ld, W.ptr if weighted else None, A.ptr if add else None, A.ld, O.ptr, O.ld, TYPE[out_type], stream())
    assert rc == binding.OK, binding.strerror(rc)
    torch.cuda.synchronize()
    valid = (at >= 0) & (at < T * k)
    rows = np.where(valid[..., None], Y.values().reshape(T * k, N)[np.where(valid, at, 0)], 0) * (W.values().reshape(T, k, 1) if weighted else 1)
    want = rows.sum(1) + (A.values().reshape(T, N) if add else 0)
    # k products and k + 1 sums, each rounded once
    off = (2 * k + 1) * 2.0 ** -24 * (np.abs(rows).sum(1) + (np.abs(A.values().reshape(T, N)) if add else 0))
    assert_within(O.fetch().reshape(T, N), want, off + (np.abs(want) + off) * UNIT[out_type] + LEAST[out_type], "out")


def test_the_order_of_a_sum():
    """The choices in their order, `add` last, products rounded before they are added: the same bits as these steps in f32."""
    T, k, N = 50, 7, 300
    g = torch.Generator(device="cuda").manual_seed(3)
    y, w, add = torch.randn(T * k, N, device="cuda", generator=g), torch.rand(T, k, device="cuda", generator=g), torch.randn(T, N, device="cuda", generator=g)
    at = torch.randperm(T * k, generator=g, device="cuda").view(T, k).to(I32)
    out = torch.zeros(T, N, device="cuda")
    binding.check(binding.expert_combine(T, k, N, TYPE["f32"], at, y, N, w, add, N, out, N, TYPE["f32"], stream()))
    want = torch.zeros(T, N, device="cuda")
    for j in range(k):
        want = want + w[:, j:j + 1] * y[at[:, j].long()]
    assert torch.equal(out, want + add)


def test_combine_into_add_and_of_no_choices():
    T, k, N = 40, 2, 200
    rng = np.random.default_rng(5)
    P, Y = Ints(I32, T, k, None, 0, places(rng, T, k, 0.3)), Mat("bf16", T * k, N, None, 0, rng.standard_normal((T * k, N)))
    A, O = Mat("bf16", T, N, None, 0, rng.standard_normal((T, N))), Mat("bf16", T, N)
    for out in (O, A):
        assert binding.expert_combine(T, k, N, TYPE["bf16"], P.ptr, Y.ptr, N, None, A.ptr, N, out.ptr, N, TYPE["bf16"], stream()) == binding.OK
    torch.cuda.synchronize()
    assert np.array_equal(A._view(A.dev.cpu())[0].double().numpy(), O.fetch())
    for add in (None, A.ptr):
        O = Mat("bf16", T, N)
        assert binding.expert_combine(T, 0, N, TYPE["bf16"], None, None, 0, None, add, N, O.ptr, N, TYPE["bf16"], stream()) == binding.OK
        torch.cuda.synchronize()
        assert np.array_equal(O.fetch(), A._view(A.dev.cpu())[0].double().numpy() if add else np.zeros((T, N)))


@pytest.mark.parametrize("T,k,N", COMBINE + [(3, 70, 5000)])
@pytest.mark.parametrize("type", ["f16", "bf16"])
@pytest.mark.parametrize("weighted,wanted,drop", [(True, "rows weight", 0.2), (False, "rows weight", 0.0), (True, "rows", 0.5), (True, "weight", 0.5), (False, "rows", 0.2)])
def test_gradients(T, k, N, type, weighted, wanted, drop):
    rng = np.random.default_rng(T * k + N + 1)
    at = places(rng, T, k, drop)
    P, W = Ints(I32, T, k, None, 1, at), Mat("f32", T, k, None, 1, rng.random((T, k)))
    Y, D = Mat(type, T * k, N, N + 3, 1, rng.standard_normal((T * k, N))), Mat(type, T, N, N + 5, 3, rng.standard_normal((T, N)))
    dY, dW = Mat(type, T * k, N, N + 1, 2), Mat("f32", T, k, None, 1)
    rc = binding.expert_combine_grad(T, k, N, TYPE[type], P.ptr, D.ptr, D.ld, W.ptr if weighted else None, Y.ptr if "weight" in wanted else None, Y.ld,
                                     dY.ptr if "rows" in wanted else None, dY.ld, dW.ptr if "weight" in wanted else None, stream())
    assert rc == binding.OK, binding.strerror(rc)
    torch.cuda.synchronize()
    valid = (at >= 0) & (at < T * k)
    d, y, w = D.values().reshape(T, 1, N), Y.values().reshape(T * k, N), W.values().reshape(T, k, 1) if weighted else np.ones((T, k, 1))
    untouched, got = Mat(type, T * k, N, N + 1, 2).fetch().reshape(T * k, N), dY.fetch().reshape(T * k, N)
    want, off = untouched.copy(), np.zeros_like(untouched)
    if "rows" in wanted:
        want[at[valid]] = np.broadcast_to(w * d, (T, k, N))[valid]
        off = np.abs(want) * 2.0 ** -24 + (np.abs(want) * (1 + 2.0 ** -24)) * UNIT[type] + LEAST[type]
    assert_within(got, want, off, "dy")
    products = np.where(valid[..., None], d * y[np.where(valid, at, 0)], 0)
    want = products.sum(2) if "weight" in wanted else np.full((T, k), -1234.0)
    # up to 32 (or N / 512) products in a row in a lane, 6 sums of lanes and 8 of wavefronts
    depth = max(32, N / 512) + 15
    assert_within(dW.fetch().reshape(T, k), want, depth * 2.0 ** -24 * np.abs(products).sum(2), "dweight")


def test_gradient_in_place_and_of_empty_rows():
    T, k, N = 30, 3, 600
    rng = np.random.default_rng(8)
    P, W = Ints(I32, T, k, None, 0, places(rng, T, k, 0.2)), Mat("f32", T, k, None, 0, rng.random((T, k)))
    Y, D = Mat("bf16", T * k, N, None, 0, rng.standard_normal((T * k, N))), Mat("bf16", T, N, None, 0, rng.standard_normal((T, N)))
    dY, dW = Mat("bf16", T * k, N, None, 0, Y.values()), [torch.full((T, k), 5.0, device="cuda") for _ in range(3)]
    for i, out in enumerate((dY, Y)):
        assert binding.expert_combine_grad(T, k, N, TYPE["bf16"], P.ptr, D.ptr, N, W.ptr, Y.ptr, N, out.ptr, N, dW[i], stream()) == binding.OK
    torch.cuda.synchronize()
    assert torch.equal(dY.dev.view(torch.int16)[:T * k * N], Y.dev.view(torch.int16)[:T * k * N]) and torch.equal(dW[0], dW[1])
    assert binding.expert_combine_grad(T, k, 0, TYPE["bf16"], P.ptr, None, 0, W.ptr, None, 0, None, 0, dW[2], stream()) == binding.OK
    assert bool((dW[2] == 0).all())


def test_the_gradient_is_the_adjoint():
    """<combine(y, w, add), d> changes with y and w as the gradients say, and dispatch's rows come back as the unweighted sum."""
    T, k, N, E = 60, 4, 256, 8
    g = torch.Generator(device="cuda").manual_seed(3)
    expert = torch.rand(T, E, device="cuda", generator=g).topk(k, 1).indices
    x = torch.randn(T, N, device="cuda", generator=g).half()
    off, src, at = torch.zeros(E + 1, dtype=I32, device="cuda"), torch.zeros(T * k, dtype=I32, device="cuda"), torch.zeros(T * k, dtype=I32, device="cuda")
    rows, back = torch.zeros(T * k, N, device="cuda").half(), torch.zeros(T, N, device="cuda")
    binding.check(binding.expert_dispatch(T, k, E, binding.INDEX_I64, expert, off, src, at, N, 2, x, N, 0, None, 0, rows, N, None, 0, None, 0, stream()))
    binding.check(binding.expert_combine(T, k, N, TYPE["f16"], at, rows, N, None, None, 0, back, N, TYPE["f32"], stream()))
    assert torch.equal(back, x.float() * k)
    # on small integers everything is exact
    y, w = torch.randint(-4, 5, (T * k, N), device="cuda", generator=g).half(), torch.randint(-4, 5, (T, k), device="cuda", generator=g).float()
    d = torch.randint(-4, 5, (T, N), device="cuda", generator=g).half()
    dy, dw, out = torch.zeros_like(y), torch.zeros_like(w), torch.zeros(T, N, device="cuda")
    binding.check(binding.expert_combine_grad(T, k, N, TYPE["f16"], at, d, N, w, y, N, dy, N, dw, stream()))
    binding.check(binding.expert_combine(T, k, N, TYPE["f16"], at, y, N, w, None, 0, out, N, TYPE["f32"], stream()))
    total = (out.double() * d.double()).sum()
    assert total == (y.double() * dy.double()).sum() == (w.double() * dw.double()).sum()


def test_many_tokens():
    """More tokens than one launch of the way back or of the rows has wavefronts for (2^24 pieces of a row)."""
    T, N, E = (1 << 24) + 3, 2, 3
    expert = (torch.arange(T, device="cuda") % 4 - (torch.arange(T, device="cuda") == 7).long() * 9)
    x = torch.arange(2 * T, device="cuda").remainder_(30000).to(torch.int16).view(T, N)
    off, at = torch.zeros(E + 1, dtype=I32, device="cuda"), torch.zeros(T, dtype=I32, device="cuda")
    rows = torch.zeros(T, N, dtype=torch.int16, device="cuda")
    need = binding.expert_dispatch_workspace_bytes(T, 1, E)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    binding.check(binding.expert_dispatch(T, 1, E, binding.INDEX_I64, expert, off, None, at, N, 2, x, N, 0, None, 0, rows, N, None, 0, ws, need, stream()))
    key = torch.where((expert >= 0) & (expert < E), expert, E)
    by = torch.argsort(key, stable=True)
    total = int((key < E).sum())
    assert off.tolist() == [0] + torch.bincount(key, minlength=4)[:3].cumsum(0).tolist() and off[-1] == total
    assert torch.equal(rows[:total], x[by[:total]]) and bool((rows[total:] == 0).all())
    y, out = (rows.float() / 16).half(), torch.zeros(T, N, device="cuda")
    binding.check(binding.expert_combine(T, 1, N, TYPE["f16"], at, y, N, None, None, 0, out, N, TYPE["f32"], stream()))
    valid = at >= 0
    assert torch.equal(out[valid], y[at[valid].long()].float()) and bool((out[~valid] == 0).all()) and torch.equal(valid, key < E)
