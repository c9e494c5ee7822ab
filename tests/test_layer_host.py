"""Host-side checks of the operators of include/gemm_layer.h that need no GPU: the header's prototypes against the binding's table, what each entry point refuses and with which
code, what it takes as empty, that both ways of the binding pass the same arguments, workspaces' sizes, and which kernel a product of 8-bit integers runs on."""
import ctypes
import os
import re

import pytest

from i8_form_cases import FORMS, GROUPED, up
from paper_2108_13191_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
I64, VP, CI, DB = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_double
KINDS = {"i": I64, "p": VP, "d": DB}
SIZE, PITCH, NULL, CONFIG, ALIGN, WORKSPACE = (binding.ERR_SIZE, binding.ERR_PITCH, binding.ERR_NULL, binding.ERR_CONFIG, binding.ERR_ALIGN, binding.ERR_WORKSPACE)
F16, BF16, F32 = binding.TYPE_F16, binding.TYPE_BF16, binding.TYPE_F32


def text():
    return open(os.path.join(ROOT, "include", "gemm_layer.h")).read()


def test_the_binding_calls_what_the_header_declares():
    found = {}
    for ret, name, args in re.findall(r"\b(int|int64_t)\s+(\w+)\s*\(([^)]*)\)\s*;", re.sub(r"/\*.*?\*/", "", text(), flags=re.S)):
        found[name] = (ret, [a.strip() for a in args.split(",")])
    assert set(found) == set(binding._LAYER_OPS) | {"layer_norm_grad_workspace_bytes", "expert_dispatch_workspace_bytes"}
    raw = ctypes.CDLL(binding.LIB_PATH)
    for name, letters in binding._LAYER_OPS.items():
        ret, args = found[name]
        assert ret == "int" and "".join("p" if "*" in a else "d" if a.startswith("double") else "i" for a in args) == letters and hasattr(raw, name)
        f = getattr(binding, name)
        assert f.__code__.co_varnames[:f.__code__.co_argcount] == tuple(re.findall(r"(\w+)$", a)[0] for a in args)
        assert f.__defaults__ == (0,) and f.__doc__
    assert "GEMM_INDEX_I32 = %d, GEMM_INDEX_I64 = %d" % (binding.INDEX_I32, binding.INDEX_I64) in text()
    assert not set(binding._OPS) & set(binding._LAYER_OPS)


# A call of each entry point that is refused for nothing; pointers are multiples of 16 that nothing reads: every call below ends before a launch.
P = 4096
GOOD = {
    "layer_norm": dict(M=4, N=8, type=F16, X=P, ldx=8, R=P, ldr=8, gamma=P, beta=P, eps=1e-5, H=P, ldh=8, Y=P, ldy=8, Q=P, ldq=8, scale=P, mean=P, rstd=P),
    "layer_norm_grad": dict(M=4, N=8, type=BF16, dY=P, lddy=8, H=P, ldh=8, gamma=P, mean=P, rstd=P, dH=P, lddh=8, dX=P, lddx=8, dgamma=P, dbeta=P, workspace=P, workspace_bytes=1 << 20),
    "quantize_i8_rows": dict(M=4, N=8, type=F16, act=2, X=P, ldx=16, Q=P, ldq=8, scale=P),
    "gemm_i8": dict(M=4, N=8, K=16, A=P, lda=16, a_scale=P, B=P, ldb=16, b_scale=P, C=P, ldc=8, c_type=F32),
    "gemm_i8_grouped": dict(T=4, N=8, K=16, E=2, offsets=P, A=P, lda=16, a_scale=P, B=P, ldb=16, b_stride=128, b_scale=P, bs_stride=8, C=P, ldc=8, c_type=BF16),
    "expert_dispatch": dict(T=3000, top_k=2, E=5, index_type=1, expert=P, offsets=P, source=P, place=P, N=8, size=2, X=P, ldx=8, blocks=1, scale=P, ld_scale=3000, rows=P, ld_rows=8,
                            row_scale=P, ld_row_scale=6000, workspace=P, workspace_bytes=1 << 24),
    "expert_combine": dict(T=4, top_k=2, N=8, type=F16, place=P, Y=P, ldy=8, weight=P, add=P, ld_add=8, out=P, ldo=8, out_type=F32),
    "expert_combine_grad": dict(T=4, top_k=2, N=8, type=BF16, place=P, dOut=P, lddo=8, weight=P, Y=P, ldy=8, dY=P, lddy=8, dweight=P),
}
BIG = 2**31


def each(code, **values):
    """(code, {name: value}) for each value of each name."""
    return [(code, {n: x}) for n, v in values.items() for x in (v if isinstance(v, (list, tuple)) else [v])]


REFUSED = {
    "layer_norm": each(SIZE, M=[-1, BIG], N=[-1, BIG]) + each(CONFIG, type=[F32, 3, -1], eps=[-1e-9, float("nan")]) + each(PITCH, ldx=[7, BIG], ldr=7, ldh=7, ldy=7, ldq=7) +
                  each(NULL, X=0, gamma=0, Q=0, scale=0) + each(ALIGN, X=P + 1, R=P + 1, gamma=P + 1, beta=P + 1, H=P + 1, Y=P + 1, scale=P + 2, mean=P + 2, rstd=P + 1),
    "layer_norm_grad": each(SIZE, M=[-1, BIG], N=[-1, BIG]) + each(CONFIG, type=[F32, 3]) + each(PITCH, lddy=7, ldh=7, lddh=7, lddx=[7, BIG]) +
                       each(NULL, dY=0, H=0, gamma=0, mean=0, rstd=0, dX=0, workspace=0) + [(NULL, dict(dbeta=0, workspace=0)), (NULL, dict(dgamma=0, workspace=0))] +
                       each(ALIGN, dY=P + 1, H=P + 1, gamma=P + 1, dH=P + 1, dX=P + 1, mean=P + 2, rstd=P + 2, dgamma=P + 2, dbeta=P + 2, workspace=P + 8) +
                       [(ALIGN, dict(M=0, dbeta=P + 2))] + each(WORKSPACE, workspace_bytes=[0, 63, -1]),
    "quantize_i8_rows": each(SIZE, M=[-1, BIG], N=[-1, BIG]) + each(CONFIG, type=[F32, 3], act=[3, -1]) + each(PITCH, ldx=[15, BIG], ldq=7) + [(PITCH, dict(act=1, ldx=7))] +
                        each(NULL, X=0, Q=0, scale=0) + each(ALIGN, X=P + 1, scale=P + 2),
    "gemm_i8": each(SIZE, M=[-1, BIG], N=[-1, BIG], K=[-1, BIG]) + [(SIZE, dict(K=131072, lda=131072, ldb=131072)), (SIZE, dict(M=BIG - 1, N=BIG - 1, ldc=BIG - 1))] +
               each(CONFIG, c_type=[3, -1, 16]) + each(PITCH, lda=[15, BIG], ldb=15, ldc=7) + each(NULL, A=0, B=0, C=0, a_scale=0, b_scale=0) +
               each(ALIGN, C=P + 2, a_scale=P + 2, b_scale=P + 1) + [(ALIGN, dict(c_type=F16, C=P + 1)), (NULL, dict(K=0, lda=0, ldb=0, A=0, B=0, b_scale=0))],
    "gemm_i8_grouped": each(SIZE, T=[-1, BIG], N=[-1, BIG], K=[-1, 131072], E=[-1, 65536]) + each(CONFIG, c_type=[3, 5]) + each(PITCH, lda=15, ldb=15, b_stride=-1, bs_stride=-1, ldc=7) +
                       each(NULL, offsets=0, A=0, B=0, C=0, a_scale=0, b_scale=0) + each(ALIGN, offsets=P + 2, C=P + 1, a_scale=P + 1, b_scale=P + 2),
    "expert_dispatch": each(SIZE, T=[-1, BIG, BIG // 2], top_k=[-1, 65536, BIG], E=[-1, 65536], N=[-1, BIG], blocks=[-1, BIG]) + each(CONFIG, index_type=[2, -1], size=[0, 3, 8]) +
                       each(PITCH, ldx=7, ld_rows=[7, BIG], ld_scale=2999, ld_row_scale=5999) + each(NULL, expert=0, offsets=0, place=0, rows=0, scale=0, row_scale=0, workspace=0) +
                       each(ALIGN, expert=P + 4, offsets=P + 2, source=P + 2, place=P + 2, X=P + 1, rows=P + 1, scale=P + 2, row_scale=P + 2, workspace=P + 8) +
                       [(ALIGN, dict(index_type=0, expert=P + 2)), (ALIGN, dict(size=4, X=P + 2)), (NULL, dict(T=0, offsets=0)), (ALIGN, dict(top_k=0, offsets=P + 1))] +
                       each(WORKSPACE, workspace_bytes=[0, -1, 100]),
    "expert_combine": each(SIZE, T=[-1, BIG, BIG // 2], top_k=[-1, 65536, BIG], N=[-1, BIG]) + each(CONFIG, type=[3, -1], out_type=[BF16, 3]) + [(CONFIG, dict(type=F32, out_type=F16))] +
                      each(PITCH, ldy=7, ld_add=7, ldo=[7, BIG]) + each(NULL, place=0, Y=0, out=0) + each(ALIGN, place=P + 2, Y=P + 1, weight=P + 2, add=P + 1, out=P + 2) +
                      [(ALIGN, dict(type=F32, Y=P + 2))],
    "expert_combine_grad": each(SIZE, T=[-1, BIG], top_k=[-1, 65536, BIG], N=[-1, BIG]) + each(CONFIG, type=[F32, 3]) + each(PITCH, lddo=7, ldy=7, lddy=7) + each(NULL, place=0, dOut=0, Y=0) +
                           each(ALIGN, place=P + 2, dOut=P + 1, weight=P + 2, Y=P + 1, dY=P + 1, dweight=P + 2) + [(NULL, dict(N=0, place=0))],
}
# nothing to compute: no pointer is looked at
EMPTY = {
    "layer_norm": [dict(M=0, X=0, gamma=0), dict(N=0, H=0)],
    "layer_norm_grad": [dict(N=0, dY=0, dX=0), dict(M=0, dgamma=0, dbeta=0, dY=0)],
    "quantize_i8_rows": [dict(M=0, X=0, Q=0, scale=0), dict(N=0, ldx=0)],
    "gemm_i8": [dict(M=0, A=0, C=0), dict(N=0, ldc=0, C=0)],
    "gemm_i8_grouped": [dict(T=0, A=0), dict(N=0, C=0), dict(E=0, offsets=0)],
    "expert_dispatch": [],
    "expert_combine": [dict(T=0, Y=0, out=0), dict(N=0, Y=0, out=0)],
    "expert_combine_grad": [dict(T=0, dOut=0), dict(top_k=0, dweight=0, place=0), dict(dweight=0, dY=0, place=0), dict(N=0, dweight=0, place=0)],
}


def use(monkeypatch, way):
    if way == "ctypes":
        monkeypatch.setattr(binding, "_layer_words", binding._no_fast_way)
        monkeypatch.setattr(binding, "_layer_norm", binding._no_fast_way)
    elif binding._fastcall is None:
        pytest.skip("no extension")


@pytest.mark.parametrize("name", GOOD)
@pytest.mark.parametrize("way", ["extension", "ctypes"])
def test_refusals(monkeypatch, name, way):
    use(monkeypatch, way)
    f = getattr(binding, name)
    for code, change in REFUSED[name]:
        args = {**GOOD[name], **change}
        assert f(**args) == code, change
        with pytest.raises(binding.GemmError) as e:
            binding.check(f(*args.values()))
        assert e.value.code == code
    for change in EMPTY[name]:
        assert f(**{**GOOD[name], **change}) == binding.OK, change


class Tensor:
    def __init__(self, address):
        self.address = address

    def data_ptr(self):
        return self.address


@pytest.mark.parametrize("name", GOOD)
@pytest.mark.parametrize("way", ["extension", "ctypes"])
def test_each_operator_reaches_its_own_entry_point(monkeypatch, name, way):
    use(monkeypatch, way)
    letters, seen, through = binding._LAYER_OPS[name], [], []
    f = ctypes.CFUNCTYPE(CI, *[KINDS[k] for k in letters])(lambda *a: (seen.append(a), -77)[1])

    class Library:
        pass
    lib = Library()
    setattr(lib, name, lambda *a: (through.append(name), f(*a))[1])
    setattr(lib, name + "_address", ctypes.cast(f, VP).value)
    monkeypatch.setattr(binding, "load", lambda: lib)
    args = [101 + i if k == "i" else Tensor(4096 * (i + 1)) if k == "p" else 0.25 for i, k in enumerate(letters)]
    want = tuple(x.address if isinstance(x, Tensor) else x for x in args)
    assert getattr(binding, name)(*args) == -77 and seen.pop() == want
    assert getattr(binding, name)(*args[:-1]) == -77 and seen.pop() == want[:-1] + (None,)      # the stream defaults to 0
    args[letters.index("p")] = None
    assert getattr(binding, name)(*args) == -77 and seen.pop()[letters.index("p")] is None
    assert len(through) == (3 if way == "ctypes" else 0) and not seen


def test_what_the_extension_leaves_goes_through_ctypes():
    if binding._fastcall is None:
        pytest.skip("no extension")
    known = {len(letters) for name, letters in binding._LAYER_OPS.items() if name != "layer_norm"}
    for n in range(0, 25):
        seen = []
        f = ctypes.CFUNCTYPE(CI, *[I64] * n)(lambda *a: (seen.append(a), 5)[1])
        args = [(i + 1) * 0x100000001 for i in range(n)]
        rc = binding._fastcall.layer_words(ctypes.cast(f, VP).value, "i" * n, *args)
        assert (rc == 5 and seen == [tuple(args)]) if n in known else (rc is NotImplemented and not seen)
    norm = list(GOOD["layer_norm"].values()) + [0]
    for bad in (1, None, "x"):
        assert binding._layer_norm(0, *norm[:9], bad, *norm[10:]) is NotImplemented
    assert binding.layer_norm(**{**GOOD["layer_norm"], "eps": 0, "ldx": 7}) == PITCH            # an integer eps goes through ctypes
    with pytest.raises(ctypes.ArgumentError):
        binding.layer_norm(**{**GOOD["layer_norm"], "eps": "x"})


def test_workspaces():
    w = binding.layer_norm_grad_workspace_bytes
    assert w(0, 8) == w(8, 0) == w(-1, 8) == w(8, -1) == w(2**31, 8) == w(8, 2**31) == 0
    for M in (1, 2, 15, 16, 17, 255, 256, 257, 4096, 2**31 - 1):
        for N in (1, 8, 1000, 4096, 16384, 17000, 2**31 - 1):
            assert 8 * N <= w(M, N) <= 8 * N * min(M, 256)
    d = binding.expert_dispatch_workspace_bytes
    assert d(0, 2, 8) == d(2, 0, 8) == d(-1, 2, 8) == d(2**31 - 1, 2, 8) == d(5000, 2, 65536) == d(5000, 2, -1) == 0 == d(32, 2, 16)
    assert d(1, 65536, 8) == 0
    for T, k in ((5000, 2), (16384, 8), (2**30, 1), (2**31 - 1, 1), (1, 65535), (2000, 256), (2000, 257)):
        for E in (0, 1, 64, 2047, 2048, 65535):
            assert 0 < d(T, k, E) <= 8 * T * k + (1 << 22) and d(T, k, E) % 16 == 0


@pytest.mark.parametrize("form,M,N,K", FORMS)
def test_forms(form, M, N, K):
    assert binding.i8_form(M, N, K, -1, up(K, 16), up(K, 16), BF16) == form
    assert binding.i8_form(M, N, K, -1, up(K, 16) + 1, up(K, 16), BF16) in ("few_rows_32x32_any_alignment", "few_rows_64x64_any_alignment")


def test_forms_by_expert_and_of_nothing():
    for form, counts, N, K in GROUPED:
        assert binding.i8_form(sum(counts), N, K, len(counts), up(K, 16), up(K, 16), F32) == form
    assert {f for f, *_ in FORMS} >= {f for f, *_ in GROUPED}
    for bad in (dict(T=0), dict(N=0), dict(E=0), dict(K=131072), dict(T=-1), dict(N=BIG), dict(c_type=3), dict(E=65536)):
        args = {**dict(T=100, N=100, K=100, E=-1, lda=112, ldb=112, c_type=F32), **bad}
        assert binding.i8_form(*args.values()) is None
    # thousands of experts with a wide N: larger tiles where smaller ones would be more than a launch has workgroups
    assert binding.i8_form(60000, 1 << 17, 128, 60000, 128, 128, F16) in ("256x256", None)
