"""The entry points of include/gemm_layer.h that expert_layer.py calls, on the host, as ops_emulation.py has those of gemm_ops.h.  ROW_ENTRY_POINTS: those that move
rows, for tests that have expert_layer.py call them (its `_on_gpu` replaced); elsewhere torch moves rows on the host."""
import torch

from ops_emulation import KIND, at, mat
from paper_2108_13191_amd import binding


def quantize(y, Q, ldq, scale):
    M, N = y.shape
    s = y.abs().amax(1).clamp_min(2.0 ** -96) * torch.tensor(1 / 127.0)
    at(scale, torch.float32, (M, 1)).copy_(s)
    mat(Q, torch.int8, M, N, ldq).copy_((y.double() / s.double()[:, None]).round())


def quantize_i8_rows(M, N, type, act, X, ldx, Q, ldq, scale, stream=0):
    x = mat(X, KIND[type], M, 2 * N if act == binding.ACT_SWIGLU else N, ldx).float()
    quantize(torch.nn.functional.silu(x[:, :N]) * x[:, N:] if act == binding.ACT_SWIGLU else x, Q, ldq, scale)
    return binding.OK


def layer_norm(M, N, type, X, ldx, R, ldr, gamma, beta, eps, H, ldh, Y, ldy, Q, ldq, scale, mean, rstd, stream=0):
    kind = KIND[type]
    h = (mat(X, kind, M, N, ldx).float() + mat(R, kind, M, N, ldr).float()).to(kind)
    mat(H, kind, M, N, ldh).copy_(h)
    m = h.float().mean(1)
    d = h.float() - m[:, None]
    s = torch.rsqrt(d.square().mean(1) + eps)
    at(mean, torch.float32, (M, 1)).copy_(m)
    at(rstd, torch.float32, (M, 1)).copy_(s)
    y = d * s[:, None] * at(gamma, kind, (N, 1)).float() + at(beta, kind, (N, 1)).float()
    mat(Y, kind, M, N, ldy).copy_(y)
    if Q is not None:
        quantize(y, Q, ldq, scale)
    return binding.OK


def layer_norm_grad_workspace_bytes(M, N):
    return 16


def layer_norm_grad(M, N, type, dY, lddy, H, ldh, gamma, mean, rstd, dH, lddh, dX, lddx, dgamma, dbeta, workspace, workspace_bytes, stream=0):
    kind = KIND[type]
    r, m = at(rstd, torch.float32, (M, 1))[:, None], at(mean, torch.float32, (M, 1))[:, None]
    dy, x = mat(dY, kind, M, N, lddy).float(), (mat(H, kind, M, N, ldh).float() - m) * r
    g = dy * at(gamma, kind, (N, 1)).float()
    mat(dX, kind, M, N, lddx).copy_(r * (g - g.mean(1, keepdim=True) - x * (g * x).mean(1, keepdim=True)) + mat(dH, kind, M, N, lddh).float())
    at(dgamma, torch.float32, (N, 1)).copy_((dy * x).sum(0))
    at(dbeta, torch.float32, (N, 1)).copy_(dy.sum(0))
    return binding.OK


def gemm_i8_grouped(T, N, K, E, offsets, A, lda, a_scale, B, ldb, b_stride, b_scale, bs_stride, C, ldc, c_type, stream=0):
    a, c = mat(A, torch.int8, T, K, lda).double(), mat(C, KIND[c_type], T, N, ldc)
    b, s, r = at(B, torch.int8, (E, b_stride), (N, ldb), (K, 1)).double(), at(b_scale, torch.float32, (E, bs_stride), (N, 1)), at(a_scale, torch.float32, (T, 1))
    off = at(offsets, torch.int32, (E + 1, 1)).tolist()
    for e in range(E):
        lo, hi = off[e], off[e + 1]
        c[lo:hi] = ((a[lo:hi] @ b[e].t()).float() * r[lo:hi, None] * s[e]).to(c.dtype)
    return binding.OK


def gemm_i8(M, N, K, A, lda, a_scale, B, ldb, b_scale, C, ldc, c_type, stream=0):
    return gemm_i8_grouped(M, N, K, 1, torch.tensor([0, M], dtype=torch.int32), A, lda, a_scale, B, ldb, 0, b_scale, 0, C, ldc, c_type)


ENTRY_POINTS = (quantize_i8_rows, layer_norm, layer_norm_grad_workspace_bytes, layer_norm_grad, gemm_i8, gemm_i8_grouped)


def combined(rows, at_, weight, add):
    """What expert_combine gives, in f32, of places T x k; those outside the T * k rows add nothing."""
    there = (at_ >= 0) & (at_ < at_.numel())
    terms = torch.where(there[..., None], rows[torch.where(there, at_, 0).long()].float(), 0.0)
    total = (terms if weight is None else terms * weight[..., None]).sum(1)
    return total if add is None else total + add.float()


def expert_combine(T, top_k, N, type, place, Y, ldy, weight, add, ld_add, out, ldo, out_type, stream=0):
    w = None if weight is None else mat(weight, torch.float32, T, top_k, top_k)
    a = None if add is None else mat(add, KIND[type], T, N, ld_add)
    mat(out, KIND[out_type], T, N, ldo).copy_(combined(mat(Y, KIND[type], T * top_k, N, ldy), mat(place, torch.int32, T, top_k, top_k), w, a))
    return binding.OK


def expert_combine_grad(T, top_k, N, type, place, dOut, lddo, weight, Y, ldy, dY, lddy, dweight, stream=0):
    at_, d = mat(place, torch.int32, T, top_k, top_k), mat(dOut, KIND[type], T, N, lddo).float()
    y, w = mat(Y, KIND[type], T * top_k, N, ldy), torch.ones(T, top_k) if weight is None else mat(weight, torch.float32, T, top_k, top_k)
    there = (at_ >= 0) & (at_ < at_.numel())
    dots = (y[torch.where(there, at_, 0).long()].float() * d[:, None]).sum(-1)
    mat(dweight, torch.float32, T, top_k, top_k).copy_(torch.where(there, dots, 0.0))
    mat(dY, KIND[type], T * top_k, N, lddy)[at_[there].long()] = (w[..., None] * d[:, None])[there].to(KIND[type])
    return binding.OK


def expert_dispatch_workspace_bytes(T, top_k, E):
    return 16


def expert_dispatch(T, top_k, E, index_type, expert, offsets, source, place, N, size, X, ldx, blocks, scale, ld_scale, rows, ld_rows, row_scale, ld_row_scale, workspace, workspace_bytes, stream=0):
    n = T * top_k
    flat = mat(expert, torch.int64 if index_type == binding.INDEX_I64 else torch.int32, T, top_k, top_k).flatten()
    key = torch.where((flat >= 0) & (flat < E), flat, E)
    by = key.argsort(stable=True)
    total = int((key < E).sum())
    valid = torch.arange(n) < total
    at(offsets, torch.int32, (E + 1, 1)).copy_(torch.searchsorted(key[by], torch.arange(E + 1)))
    at(source, torch.int32, (n, 1)).copy_(torch.where(valid, by // top_k, -1))
    at(place, torch.int32, (n, 1))[by] = torch.where(valid, torch.arange(n), -1).int()
    if X is not None:
        kind = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[size]
        assert X.element_size() == rows.element_size() == size
        mat(rows.view(kind), kind, n, N, ld_rows)[:total] = mat(X.view(kind), kind, T, N, ldx)[by[:total] // top_k]
        if blocks:
            mat(row_scale, torch.float32, blocks, n, ld_row_scale)[:, :total] = mat(scale, torch.float32, blocks, T, ld_scale)[:, by[:total] // top_k]
    return binding.OK


ROW_ENTRY_POINTS = (expert_combine, expert_combine_grad, expert_dispatch_workspace_bytes, expert_dispatch)
