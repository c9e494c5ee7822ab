"""Host-side checks of the operators of include/gemm_ops.h that need no GPU: the header's prototypes against the binding's tables, what
each entry point refuses and with which code, what it takes as empty, and that both ways of the binding pass the same arguments."""
import ctypes
import os
import re

import pytest

from paper_2108_13191_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
I64, VP, CI, DB = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int, ctypes.c_double
KINDS = {"i": I64, "p": VP, "d": DB}
SIZE, PITCH, NULL, CONFIG, ALIGN, WORKSPACE = (binding.ERR_SIZE, binding.ERR_PITCH, binding.ERR_NULL, binding.ERR_CONFIG, binding.ERR_ALIGN, binding.ERR_WORKSPACE)
F16, BF16, F32 = binding.TYPE_F16, binding.TYPE_BF16, binding.TYPE_F32


def prototypes():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "gemm_ops.h")).read(), flags=re.S)
    out = {}
    for ret, name, args in re.findall(r"\b(int|int64_t)\s+(\w+)\s*\(([^)]*)\)\s*;", text):
        out[name] = (ret, [a.strip() for a in args.split(",")])
    return out


def letter(arg):
    return "p" if "*" in arg else "d" if arg.startswith("double") else "i" if arg.startswith("int64_t") else "?"


def test_the_binding_calls_what_the_header_declares():
    found = prototypes()
    assert set(found) == set(binding._OPS) | {"rms_norm_grad_workspace_bytes"}
    raw = ctypes.CDLL(binding.LIB_PATH)
    for name, letters in binding._OPS.items():
        ret, args = found[name]
        assert ret == "int" and "".join(map(letter, args)) == letters and hasattr(raw, name)
        f = getattr(binding, name)
        # the function's own argument names, in the header's order
        assert f.__code__.co_varnames[:f.__code__.co_argcount] == tuple(re.findall(r"(\w+)$", a)[0] for a in args)
        assert f.__defaults__ == (0,) and f.__doc__
    text = open(os.path.join(ROOT, "include", "gemm_ops.h")).read()
    for name, value in {"GEMM_TYPE_F16": F16, "GEMM_TYPE_BF16": BF16, "GEMM_TYPE_F32": F32, "GEMM_OPS_ACT_NONE": binding.ACT_NONE,
                        "GEMM_OPS_ACT_RELU": binding.ACT_RELU, "GEMM_OPS_ACT_SWIGLU": binding.ACT_SWIGLU}.items():
        assert re.search(rf"\b{name} = {value}\b", text)


# A call of each entry point that is refused for nothing: 4 x 8 problems, K = 16, 2 experts.  Pointers are multiples of 16 that nothing reads:
# every call below ends before a launch.
P = 4096
GOOD = {
    "quantize_e4m3_rows": dict(M=4, N=8, type=F16, act=2, X=P, ldx=16, Q=P, ldq=8, scale=P, ld_scale=4),
    "quantize_e4m3_blocks": dict(M=4, N=8, type=BF16, X=P, ldx=8, Q=P, ldq=8, scale=P, ld_scale=1),
    "rms_norm": dict(M=4, N=8, type=F16, X=P, ldx=8, R=P, ldr=8, gamma=P, eps=1e-5, H=P, ldh=8, Y=P, ldy=8, Q=P, ldq=8, scale=P, ld_scale=4, rstd=P),
    "rms_norm_grad": dict(M=4, N=8, type=BF16, dY=P, lddy=8, H=P, ldh=8, gamma=P, rstd=P, dH=P, lddh=8, dX=P, lddx=8, dgamma=P, workspace=P, workspace_bytes=1 << 20),
    "gemm_e4m3_block": dict(M=4, N=8, K=16, A=P, lda=16, a_scale=P, ld_as=4, B=P, ldb=16, b_scale=P, ld_bs=1, C=P, ldc=8, c_type=F32),
    "gemm_e4m3_block_grouped": dict(T=4, N=8, K=16, E=2, offsets=P, A=P, lda=16, a_scale=P, ld_as=4, B=P, ldb=16, b_stride=128, b_scale=P, ld_bs=1, bs_stride=1,
                                    C=P, ldc=8, c_type=BF16),
    "gemm_grouped": dict(T=4, N=8, K=16, E=2, offsets=P, type=F16, A=P, lda=16, B=P, ldb=8, b_stride=128, C=P, ldc=8, c_type=F16),
    "gemm_grouped_grad_a": dict(T=4, N=8, K=16, E=2, offsets=P, type=F16, dC=P, lddc=8, B=P, ldb=8, b_stride=128, dA=P, ldda=16, a_type=F32),
    "gemm_grouped_grad_b": dict(T=4, N=8, K=16, E=2, offsets=P, type=BF16, A=P, lda=16, dC=P, lddc=8, dB=P, lddb=8, db_stride=128, b_type=BF16),
}
BIG = 2**31
REFUSED = {
    "quantize_e4m3_rows": [(SIZE, dict(M=-1)), (SIZE, dict(N=BIG)), (CONFIG, dict(type=F32)), (CONFIG, dict(type=3)), (CONFIG, dict(act=3)), (CONFIG, dict(act=-1)),
                           (PITCH, dict(ldx=15)), (PITCH, dict(act=1, ldx=7)), (PITCH, dict(ldq=7)), (PITCH, dict(ld_scale=3)), (PITCH, dict(ldx=BIG)),
                           (NULL, dict(X=0)), (NULL, dict(Q=0)), (NULL, dict(scale=0)), (ALIGN, dict(X=P + 1)), (ALIGN, dict(scale=P + 2)),
                           (SIZE, dict(act=0, N=BIG - 1, ldx=BIG - 1, ldq=BIG - 1))],
    "quantize_e4m3_blocks": [(SIZE, dict(M=BIG)), (SIZE, dict(N=-1)), (CONFIG, dict(type=2)), (PITCH, dict(ldx=7)), (PITCH, dict(ldq=7)), (PITCH, dict(ld_scale=0)),
                             (PITCH, dict(N=129, ldx=136, ldq=136, ld_scale=1)), (NULL, dict(X=0)), (NULL, dict(Q=0)), (NULL, dict(scale=0)), (ALIGN, dict(X=P + 1)),
                             (ALIGN, dict(scale=P + 1)), (SIZE, dict(M=BIG - 1, N=BIG - 1, ldx=BIG - 1, ldq=BIG - 1, ld_scale=BIG // 128))],
    "rms_norm": [(SIZE, dict(M=-1)), (SIZE, dict(N=BIG)), (CONFIG, dict(type=F32)), (CONFIG, dict(eps=-1e-9)), (CONFIG, dict(eps=float("nan"))),
                 (PITCH, dict(ldx=7)), (PITCH, dict(ldr=7)), (PITCH, dict(ldh=7)), (PITCH, dict(ldy=7)), (PITCH, dict(ldq=7)), (PITCH, dict(ld_scale=3)),
                 (NULL, dict(X=0)), (NULL, dict(gamma=0)), (NULL, dict(Q=0)), (NULL, dict(scale=0)),
                 (ALIGN, dict(X=P + 1)), (ALIGN, dict(R=P + 1)), (ALIGN, dict(gamma=P + 1)), (ALIGN, dict(H=P + 1)), (ALIGN, dict(Y=P + 1)), (ALIGN, dict(scale=P + 2)),
                 (ALIGN, dict(rstd=P + 2))],
    "rms_norm_grad": [(SIZE, dict(M=-1)), (SIZE, dict(N=BIG)), (CONFIG, dict(type=F32)), (PITCH, dict(lddy=7)), (PITCH, dict(ldh=7)), (PITCH, dict(lddh=7)), (PITCH, dict(lddx=7)),
                      (NULL, dict(dY=0)), (NULL, dict(H=0)), (NULL, dict(gamma=0)), (NULL, dict(rstd=0)), (NULL, dict(dX=0)), (NULL, dict(workspace=0)),
                      (ALIGN, dict(dY=P + 1)), (ALIGN, dict(H=P + 1)), (ALIGN, dict(gamma=P + 1)), (ALIGN, dict(dH=P + 1)), (ALIGN, dict(dX=P + 1)), (ALIGN, dict(rstd=P + 2)),
                      (ALIGN, dict(workspace=P + 8)), (ALIGN, dict(dgamma=P + 2)), (ALIGN, dict(M=0, dgamma=P + 2)), (WORKSPACE, dict(workspace_bytes=31)), (WORKSPACE, dict(workspace_bytes=0))],
    "gemm_e4m3_block": [(SIZE, dict(M=-1)), (SIZE, dict(N=BIG)), (SIZE, dict(K=BIG)), (CONFIG, dict(c_type=3)), (CONFIG, dict(c_type=-1)), (PITCH, dict(lda=15)), (PITCH, dict(ldb=15)),
                        (PITCH, dict(ldc=7)), (PITCH, dict(ld_as=3)), (PITCH, dict(ld_bs=0)), (NULL, dict(A=0)), (NULL, dict(B=0)), (NULL, dict(C=0)), (NULL, dict(a_scale=0)),
                        (NULL, dict(b_scale=0)), (ALIGN, dict(C=P + 2)), (ALIGN, dict(c_type=F16, C=P + 1)), (ALIGN, dict(a_scale=P + 2)), (ALIGN, dict(b_scale=P + 1)),
                        (SIZE, dict(M=BIG - 1, N=BIG - 1, ldc=BIG - 1, ld_as=BIG - 1)), (NULL, dict(K=0, lda=0, ldb=0, C=0))],
    "gemm_e4m3_block_grouped": [(SIZE, dict(T=-1)), (SIZE, dict(E=-1)), (SIZE, dict(E=65536)), (SIZE, dict(K=-1)), (CONFIG, dict(c_type=5)), (PITCH, dict(lda=15)), (PITCH, dict(ldb=15)),
                                (PITCH, dict(b_stride=-1)), (PITCH, dict(bs_stride=-1)), (PITCH, dict(ldc=7)), (PITCH, dict(ld_as=3)), (PITCH, dict(ld_bs=0)), (NULL, dict(offsets=0)),
                                (NULL, dict(A=0)), (NULL, dict(B=0)), (NULL, dict(C=0)), (NULL, dict(a_scale=0)), (NULL, dict(b_scale=0)), (ALIGN, dict(offsets=P + 2)), (ALIGN, dict(C=P + 1))],
    "gemm_grouped": [(SIZE, dict(T=BIG)), (SIZE, dict(N=-1)), (SIZE, dict(E=-1)), (SIZE, dict(E=65536)), (CONFIG, dict(type=F32)), (CONFIG, dict(type=F16, c_type=BF16)), (CONFIG, dict(c_type=3)),
                     (PITCH, dict(lda=15)), (PITCH, dict(ldb=7)), (PITCH, dict(ldc=7)), (PITCH, dict(b_stride=-8)), (NULL, dict(A=0)), (NULL, dict(B=0)), (NULL, dict(C=0)), (NULL, dict(offsets=0)),
                     (ALIGN, dict(A=P + 1)), (ALIGN, dict(B=P + 1)), (ALIGN, dict(C=P + 1)), (ALIGN, dict(c_type=F32, C=P + 2)), (ALIGN, dict(offsets=P + 1))],
    "gemm_grouped_grad_a": [(SIZE, dict(T=BIG)), (SIZE, dict(K=-1)), (SIZE, dict(E=65536)), (CONFIG, dict(type=2)), (CONFIG, dict(a_type=BF16)), (PITCH, dict(lddc=7)), (PITCH, dict(ldb=7)),
                            (PITCH, dict(ldda=15)), (PITCH, dict(b_stride=-8)), (NULL, dict(dC=0)), (NULL, dict(B=0)), (NULL, dict(dA=0)), (NULL, dict(offsets=0)), (ALIGN, dict(dC=P + 1)),
                            (ALIGN, dict(B=P + 1)), (ALIGN, dict(dA=P + 2)), (ALIGN, dict(offsets=P + 2))],
    "gemm_grouped_grad_b": [(SIZE, dict(T=-1)), (SIZE, dict(N=BIG)), (SIZE, dict(E=-1)), (CONFIG, dict(type=2)), (CONFIG, dict(b_type=F16)), (PITCH, dict(lda=15)), (PITCH, dict(lddc=7)),
                            (PITCH, dict(lddb=7)), (PITCH, dict(db_stride=127)), (PITCH, dict(db_stride=0)), (NULL, dict(A=0)), (NULL, dict(dC=0)), (NULL, dict(dB=0)), (NULL, dict(offsets=0)),
                            (ALIGN, dict(A=P + 1)), (ALIGN, dict(dC=P + 1)), (ALIGN, dict(dB=P + 1)), (ALIGN, dict(b_type=F32, dB=P + 2)), (ALIGN, dict(offsets=P + 2))],
}
# nothing to compute: no pointer is looked at
EMPTY = {
    "quantize_e4m3_rows": [dict(M=0, X=0, Q=0, scale=0), dict(N=0, X=0, Q=0, scale=0)],
    "quantize_e4m3_blocks": [dict(M=0, X=0, Q=0, scale=0), dict(N=0, ldx=0)],
    "rms_norm": [dict(M=0, X=0, gamma=0), dict(N=0, H=0)],
    "rms_norm_grad": [dict(N=0, dY=0, dX=0), dict(M=0, dgamma=0, dY=0)],
    "gemm_e4m3_block": [dict(M=0, A=0, C=0), dict(N=0, ldc=0, C=0)],
    "gemm_e4m3_block_grouped": [dict(T=0, A=0), dict(N=0, C=0), dict(E=0, offsets=0)],
    "gemm_grouped": [dict(T=0, A=0), dict(N=0, C=0), dict(E=0, offsets=0)],
    "gemm_grouped_grad_a": [dict(T=0, dC=0), dict(K=0, dA=0), dict(E=0, offsets=0)],
    "gemm_grouped_grad_b": [dict(N=0, dB=0), dict(K=0, dB=0), dict(E=0, offsets=0)],
}


@pytest.mark.parametrize("name", GOOD)
@pytest.mark.parametrize("way", ["extension", "ctypes"])
def test_refusals(monkeypatch, name, way):
    if way == "ctypes":
        monkeypatch.setattr(binding, "_words", binding._no_fast_way)
        monkeypatch.setattr(binding, "_norm", binding._no_fast_way)
    f = getattr(binding, name)
    for code, change in REFUSED[name]:
        args = {**GOOD[name], **change}
        assert f(**args) == code, change
        with pytest.raises(binding.GemmError) as e:
            binding.check(f(*args.values()))
        assert e.value.code == code
    for change in EMPTY[name]:
        assert f(**{**GOOD[name], **change}) == binding.OK, change


def test_workspace_of_the_gradient():
    w = binding.rms_norm_grad_workspace_bytes
    assert w(0, 8) == w(8, 0) == w(-1, 8) == w(8, -1) == w(2**31, 8) == w(8, 2**31) == 0
    last = 0
    for M in (1, 2, 15, 16, 17, 255, 256, 257, 4096, 2**31 - 1):
        for N in (1, 8, 1000, 4096, 16384, 17000, 2**31 - 1):
            assert 4 * N <= w(M, N) <= 4 * N * min(M, 256)
        assert w(M, 1000) >= last                       # more rows never need less
        last = w(M, 1000)


def recorder(letters):
    seen = []
    f = ctypes.CFUNCTYPE(CI, *[KINDS[k] for k in letters])(lambda *a: (seen.append(a), -77)[1])
    return seen, f, ctypes.cast(f, VP).value


class Tensor:
    def __init__(self, address):
        self.address = address

    def data_ptr(self):
        return self.address


@pytest.mark.parametrize("name", GOOD)
@pytest.mark.parametrize("way", ["extension", "ctypes"])
def test_each_operator_reaches_its_own_entry_point(monkeypatch, name, way):
    letters = binding._OPS[name]
    seen, f, address = recorder(letters)
    through = []

    class Library:
        pass
    lib = Library()
    setattr(lib, name, lambda *a: (through.append(name), f(*a))[1])
    setattr(lib, name + "_address", address)
    monkeypatch.setattr(binding, "load", lambda: lib)
    if way == "ctypes":
        monkeypatch.setattr(binding, "_words", binding._no_fast_way)
        monkeypatch.setattr(binding, "_norm", binding._no_fast_way)
    elif binding._fastcall is None:
        pytest.skip("no extension")
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
    np = pytest.importorskip("numpy")
    letters = binding._OPS["quantize_e4m3_blocks"]
    seen, f, address = recorder(letters)
    good = [1, 2, 3, 16, 8, None, 8, Tensor(32), 9, 0]
    assert binding._words(address, letters, *good) == -77 and seen.pop() == (1, 2, 3, 16, 8, None, 8, 32, 9, None)
    for i, k in enumerate(letters):
        for bad in (1.5, "7", object(), Tensor("x")) + (() if k == "p" else (None,)):
            assert binding._words(address, letters, *good[:i], bad, *good[i + 1:]) is NotImplemented
    assert binding._words(address, letters, *good[:-1]) is NotImplemented and binding._words(address, letters, *good, 1) is NotImplemented
    norm = list(GOOD["rms_norm"].values()) + [0]
    nseen, nf, naddress = recorder(binding._OPS["rms_norm"])
    assert binding._norm(naddress, *norm) == -77 and nseen.pop()[8] == 1e-5
    for bad in (1, None, "x", np.float32(1e-5)):
        assert binding._norm(naddress, *norm[:8], bad, *norm[9:]) is NotImplemented
    assert not seen and not nseen
    # and answers as ever: an integer eps, numpy integers
    assert binding.rms_norm(**{**GOOD["rms_norm"], "eps": 0, "ldx": np.int64(7)}) == PITCH
    with pytest.raises(ctypes.ArgumentError):
        binding.rms_norm(**{**GOOD["rms_norm"], "eps": "x"})
