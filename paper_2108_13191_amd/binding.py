"""Thin binding of the C ABIs in include/gemm_f16.h and include/gemm_ops.h: ctypes, and for the GEMM entry points themselves a small extension
(csrc/fastcall.c) in front of it that marshals the usual arguments in native code.

Argument marshalling only: every step of the GEMM runs in the HIP kernels of
libgemm_f16.so.  There is no fallback: if the library has not been built (run
`python -m paper_2108_13191_amd.build`), loading raises.
Functions take raw device pointers (ints) or objects with `data_ptr()` (torch
tensors); nothing here computes.
"""
from __future__ import annotations

import ctypes
import os

import contextlib

try:
    from . import _fastcall
except ImportError:                     # not built, or for another Python: everything goes through ctypes
    _fastcall = None

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libgemm_f16.so")
# the same library plus the comparison kernels and ablation rows (never selected; reached by
# forcing their configuration ids, which follow the product's): see build.py
LADDER_LIB_PATH = os.path.join(_HERE, "libgemm_f16_ladder.so")
_libs = {}
_active = "product"


@contextlib.contextmanager
def library(kind: str):
    """Within the block every function of this module calls into the named build
    ("product" or "ladder").  The two keep separate forced-configuration state."""
    global _active
    prev, _active = _active, kind
    try:
        yield
    finally:
        _active = prev

OK = 0
ERR_SIZE, ERR_PITCH, ERR_NULL, ERR_LAUNCH, ERR_CONFIG, ERR_ALIGN, ERR_WORKSPACE = -1, -2, -3, -4, -5, -6, -7


class GemmConfig(ctypes.Structure):
    _fields_ = [("id", ctypes.c_int32), ("block_m", ctypes.c_int32), ("block_n", ctypes.c_int32),
                ("block_k", ctypes.c_int32), ("waves", ctypes.c_int32), ("wave_m", ctypes.c_int32),
                ("wave_n", ctypes.c_int32), ("lds_bytes", ctypes.c_int32), ("grid", ctypes.c_int64),
                ("split_rows", ctypes.c_int32), ("id2", ctypes.c_int32), ("name", ctypes.c_char * 48)]

    def as_dict(self):
        d = {k: getattr(self, k) for k, _ in self._fields_}
        d["name"] = self.name.decode()
        return d


class GemmError(RuntimeError):
    def __init__(self, code: int):
        self.code = code
        super().__init__(f"gemm_f16 error {code}: {strerror(code)}")


# The entry points of gemm_ops.h and the kinds of their arguments: "i" an int64_t, "p" a pointer, "d" a double.
_OPS = {
    "quantize_e4m3_rows": "iiiipipipip",
    "quantize_e4m3_blocks": "iiipipipip",
    "rms_norm": "iiipipipdpipipipipp",
    "rms_norm_grad": "iiipipipppipippip",
    "gemm_e4m3_block": "iiipipipipipiip",
    "gemm_e4m3_block_grouped": "iiiippipipiipiipiip",
    "gemm_grouped": "iiiipipipiipiip",
    "gemm_grouped_grad_a": "iiiipipipiipiip",
    "gemm_grouped_grad_b": "iiiipipipipiiip",
}


def load() -> ctypes.CDLL:
    """Load the active library (built in-tree); raise if it is missing."""
    if _active not in _libs:
        path = {"product": LIB_PATH, "ladder": LADDER_LIB_PATH}[_active]
        if not os.path.exists(path):
            raise ImportError(
                f"{path} is missing: build the HIP library first "
                "(python -m paper_2108_13191_amd.build); there is no CPU fallback")
        lib = ctypes.CDLL(path)
        i64, vp, ci = ctypes.c_int64, ctypes.c_void_p, ctypes.c_int
        for name in ("gemm_f16_f32acc", "gemm_f16_f16acc", "gemm_f16_f16acc_static_workspace"):
            f = getattr(lib, name)
            f.argtypes = [i64, i64, i64, vp, i64, vp, i64, vp, i64, vp]
            f.restype = ci
        for name in ("gemm_f16_f32acc_bias_act", "gemm_f16_f16acc_bias_act"):
            f = getattr(lib, name)
            f.argtypes = [i64, i64, i64, vp, i64, vp, i64, vp, i64, vp, ci, vp]
            f.restype = ci
        lib.gemm_f16_f16acc_workspace_bytes.argtypes = [i64, i64, i64]
        lib.gemm_f16_f16acc_workspace_bytes.restype = i64
        lib.gemm_f16_f16acc_workspace.argtypes = [i64, i64, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp]
        lib.gemm_f16_f16acc_workspace.restype = ci
        lib.gemm_strerror.argtypes = [ci]
        lib.gemm_strerror.restype = ctypes.c_char_p
        lib.gemm_f16_query_config.argtypes = [ci, i64, i64, i64, vp, i64, vp, i64, vp, i64,
                                              ctypes.POINTER(GemmConfig)]
        lib.gemm_f16_query_config.restype = ci
        lib.gemm_f16_num_configs.argtypes = []
        lib.gemm_f16_num_configs.restype = ci
        lib.gemm_f16_describe_config.argtypes = [ci, ctypes.POINTER(GemmConfig)]
        lib.gemm_f16_describe_config.restype = ci
        lib.gemm_f16_force_config.argtypes = [ci]
        lib.gemm_f16_force_config.restype = ci
        kinds = {"i": i64, "p": vp, "d": ctypes.c_double}
        for name, letters in _OPS.items():
            f = getattr(lib, name)
            f.argtypes = [kinds[k] for k in letters]
            f.restype = ci
            setattr(lib, name + "_address", ctypes.cast(f, vp).value)
        lib.rms_norm_grad_workspace_bytes.argtypes = [i64, i64]
        lib.rms_norm_grad_workspace_bytes.restype = i64
        lib.gemm_ops_form.argtypes = [i64] * 8
        lib.gemm_ops_form.restype = ctypes.c_char_p
        # where the entry points are, for _fastcall
        for name in ("gemm_f16_f32acc", "gemm_f16_f16acc", "gemm_f16_f16acc_static_workspace", "gemm_f16_f32acc_bias_act",
                     "gemm_f16_f16acc_bias_act", "gemm_f16_f16acc_workspace"):
            setattr(lib, name + "_address", ctypes.cast(getattr(lib, name), vp).value)
        _libs[_active] = lib
    return _libs[_active]


def _ptr(x) -> int:
    if x is None:
        return 0
    if hasattr(x, "data_ptr"):
        return int(x.data_ptr())
    return int(x)


def _no_fast_way(*args):
    return NotImplemented


# The entry points below first ask one of these, which takes ints, None and objects with data_ptr() and returns NotImplemented, having
# called nothing, for anything else.
_plain, _bias_act, _workspace = (_fastcall.plain, _fastcall.bias_act, _fastcall.workspace) if _fastcall else (_no_fast_way,) * 3
_words, _norm = (_fastcall.words, _fastcall.norm) if _fastcall else (_no_fast_way,) * 2


def gemm_f16_f32acc(M, N, K, A, lda, B, ldb, C, ldc, stream=0) -> int:
    """C (f32) += A (f16) @ B (f16); returns the library's status code."""
    lib = load()
    rc = _plain(lib.gemm_f16_f32acc_address, M, N, K, A, lda, B, ldb, C, ldc, stream)
    return rc if rc is not NotImplemented else lib.gemm_f16_f32acc(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc, _ptr(stream))


def gemm_f16_f16acc(M, N, K, A, lda, B, ldb, C, ldc, stream=0) -> int:
    """C (f16) += A (f16) @ B (f16), f32 accumulation, one rounding on store."""
    lib = load()
    rc = _plain(lib.gemm_f16_f16acc_address, M, N, K, A, lda, B, ldb, C, ldc, stream)
    return rc if rc is not NotImplemented else lib.gemm_f16_f16acc(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc, _ptr(stream))


def gemm_f16_f16acc_workspace_bytes(M, N, K) -> int:
    """Bytes of workspace that let gemm_f16_f16acc_workspace cut this problem along k (0: none needed)."""
    return load().gemm_f16_f16acc_workspace_bytes(M, N, K)


def gemm_f16_f16acc_workspace(M, N, K, A, lda, B, ldb, C, ldc, workspace, workspace_bytes, stream=0) -> int:
    """gemm_f16_f16acc with caller-provided scratch memory (device, 16-byte aligned) for split-k plans."""
    lib = load()
    rc = _workspace(lib.gemm_f16_f16acc_workspace_address, M, N, K, A, lda, B, ldb, C, ldc, workspace, workspace_bytes, stream)
    return rc if rc is not NotImplemented else lib.gemm_f16_f16acc_workspace(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc, _ptr(workspace), workspace_bytes, _ptr(stream))


def gemm_f16_f16acc_static_workspace(M, N, K, A, lda, B, ldb, C, ldc, stream=0) -> int:
    """gemm_f16_f16acc_workspace on the library's own fixed scratch array: allocates nothing."""
    lib = load()
    rc = _plain(lib.gemm_f16_f16acc_static_workspace_address, M, N, K, A, lda, B, ldb, C, ldc, stream)
    return rc if rc is not NotImplemented else lib.gemm_f16_f16acc_static_workspace(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc, _ptr(stream))


ACT_NONE, ACT_RELU = 0, 1


def gemm_f16_f32acc_bias_act(M, N, K, A, lda, B, ldb, C, ldc, bias, act, stream=0) -> int:
    """C (f32) = act(C + A @ B + bias[None, :]); bias f32 device vector or None."""
    lib = load()
    rc = _bias_act(lib.gemm_f16_f32acc_bias_act_address, M, N, K, A, lda, B, ldb, C, ldc, bias, act, stream)
    return rc if rc is not NotImplemented else lib.gemm_f16_f32acc_bias_act(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc, _ptr(bias), act, _ptr(stream))


def gemm_f16_f16acc_bias_act(M, N, K, A, lda, B, ldb, C, ldc, bias, act, stream=0) -> int:
    """C (f16) = act(C + A @ B + bias[None, :]), f32 arithmetic, one rounding on store; bias f16 or None."""
    lib = load()
    rc = _bias_act(lib.gemm_f16_f16acc_bias_act_address, M, N, K, A, lda, B, ldb, C, ldc, bias, act, stream)
    return rc if rc is not NotImplemented else lib.gemm_f16_f16acc_bias_act(M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc, _ptr(bias), act, _ptr(stream))


# ---- include/gemm_ops.h: the operators around the products of a transformer layer.  Matrices and pitches in elements; every function
# but the last two returns the library's status code.

TYPE_F16, TYPE_BF16, TYPE_F32 = 0, 1, 2
ACT_SWIGLU = 2
EXACT = 16              # beside the c_type of an e4m3 product: exact products whatever the result's size


def _general(name, args) -> int:
    """The way through ctypes, for what _fastcall leaves: pointers as ints, None or objects with data_ptr()."""
    return getattr(load(), name)(*[_ptr(x) if k == "p" else x for x, k in zip(args, _OPS[name], strict=True)])


def _call(name, *args) -> int:
    rc = _words(getattr(load(), name + "_address"), _OPS[name], *args)
    return rc if rc is not NotImplemented else _general(name, args)


def quantize_e4m3_rows(M, N, type, act, X, ldx, Q, ldq, scale, ld_scale, stream=0) -> int:
    """Q (e4m3), scale[k block][row] = X (M x N of `type`; M x 2N for ACT_SWIGLU) after `act`, a scale for 128 elements of a row."""
    return _call("quantize_e4m3_rows", M, N, type, act, X, ldx, Q, ldq, scale, ld_scale, stream)


def quantize_e4m3_blocks(M, N, type, X, ldx, Q, ldq, scale, ld_scale, stream=0) -> int:
    """Q (e4m3), scale[row block][column block] = X (M x N of `type`), a scale for 128 x 128 elements."""
    return _call("quantize_e4m3_blocks", M, N, type, X, ldx, Q, ldq, scale, ld_scale, stream)


def rms_norm(M, N, type, X, ldx, R, ldr, gamma, eps, H, ldh, Y, ldy, Q, ldq, scale, ld_scale, rstd, stream=0) -> int:
    """H = X + R, Y = H * rstd * gamma in 16 bits and / or quantised into Q and scale; R and any output may be None."""
    args = (M, N, type, X, ldx, R, ldr, gamma, eps, H, ldh, Y, ldy, Q, ldq, scale, ld_scale, rstd, stream)
    rc = _norm(load().rms_norm_address, *args)
    return rc if rc is not NotImplemented else _general("rms_norm", args)


def rms_norm_grad(M, N, type, dY, lddy, H, ldh, gamma, rstd, dH, lddh, dX, lddx, dgamma, workspace, workspace_bytes, stream=0) -> int:
    """dX (of x and of the residual alike) and dgamma (f32, None: not formed) from dY and dH (None: no gradient of h itself)."""
    return _call("rms_norm_grad", M, N, type, dY, lddy, H, ldh, gamma, rstd, dH, lddh, dX, lddx, dgamma, workspace, workspace_bytes, stream)


def gemm_e4m3_block(M, N, K, A, lda, a_scale, ld_as, B, ldb, b_scale, ld_bs, C, ldc, c_type, stream=0) -> int:
    """C (M x N of `c_type`, which may be | EXACT) = A (M x K e4m3, scales in rows) @ B (N x K e4m3, scales in blocks) transposed."""
    return _call("gemm_e4m3_block", M, N, K, A, lda, a_scale, ld_as, B, ldb, b_scale, ld_bs, C, ldc, c_type, stream)


def gemm_e4m3_block_grouped(T, N, K, E, offsets, A, lda, a_scale, ld_as, B, ldb, b_stride, b_scale, ld_bs, bs_stride, C, ldc, c_type, stream=0) -> int:
    """gemm_e4m3_block of rows offsets[e] .. offsets[e + 1] (int32 on the device) with B[e], for E experts."""
    return _call("gemm_e4m3_block_grouped", T, N, K, E, offsets, A, lda, a_scale, ld_as, B, ldb, b_stride, b_scale, ld_bs, bs_stride, C, ldc, c_type, stream)


def gemm_grouped(T, N, K, E, offsets, type, A, lda, B, ldb, b_stride, C, ldc, c_type, stream=0) -> int:
    """C (T x N) = rows of A (T x K) @ B[e] (K x N), rows offsets[e] .. offsets[e + 1] with expert e."""
    return _call("gemm_grouped", T, N, K, E, offsets, type, A, lda, B, ldb, b_stride, C, ldc, c_type, stream)


def gemm_grouped_grad_a(T, N, K, E, offsets, type, dC, lddc, B, ldb, b_stride, dA, ldda, a_type, stream=0) -> int:
    """dA (T x K) = rows of dC (T x N) @ B[e] (K x N) transposed."""
    return _call("gemm_grouped_grad_a", T, N, K, E, offsets, type, dC, lddc, B, ldb, b_stride, dA, ldda, a_type, stream)


def gemm_grouped_grad_b(T, N, K, E, offsets, type, A, lda, dC, lddc, dB, lddb, db_stride, b_type, stream=0) -> int:
    """dB[e] (K x N) = A_e transposed @ dC_e, summed over the expert's rows; zeros for an expert without rows."""
    return _call("gemm_grouped_grad_b", T, N, K, E, offsets, type, A, lda, dC, lddc, dB, lddb, db_stride, b_type, stream)


def rms_norm_grad_workspace_bytes(M, N) -> int:
    """Bytes of workspace that rms_norm_grad needs to form dgamma."""
    return load().rms_norm_grad_workspace_bytes(M, N)


PRODUCT_E4M3, PRODUCT_FORWARD, PRODUCT_GRAD_A, PRODUCT_GRAD_B = 0, 1, 2, 3


def product_form(product, T, N, K, E, lda, ldb, c_type):
    """The name of the kernel that a product would run on (E < 0: gemm_e4m3_block), None where there is nothing to run."""
    name = load().gemm_ops_form(product, T, N, K, E, lda, ldb, c_type)
    return name.decode() if name else None


def strerror(code: int) -> str:
    return load().gemm_strerror(code).decode()


def query_config(c_is_f16, M, N, K, A, lda, B, ldb, C, ldc) -> dict:
    out = GemmConfig()
    rc = load().gemm_f16_query_config(int(c_is_f16), M, N, K, _ptr(A), lda, _ptr(B), ldb, _ptr(C), ldc,
                                      ctypes.byref(out))
    if rc != OK:
        raise GemmError(rc)
    return out.as_dict()


def num_configs() -> int:
    return load().gemm_f16_num_configs()


def describe_config(cfg_id: int) -> dict:
    out = GemmConfig()
    rc = load().gemm_f16_describe_config(cfg_id, ctypes.byref(out))
    if rc != OK:
        raise GemmError(rc)
    return out.as_dict()


def force_config(cfg_id: int) -> int:
    return load().gemm_f16_force_config(cfg_id)


def check(rc: int) -> None:
    if rc != OK:
        raise GemmError(rc)
