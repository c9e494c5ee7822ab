"""The entry points of paper_2108_13191_amd.binding that expert_layer.py calls, on the host: each reads and writes its operands as the kernels do, from an
address by pitches, strides and the type it is told.  An operand of another type, or one that ends before its last element, is an error here."""
import torch

from paper_2108_13191_amd import binding

KIND = {binding.TYPE_F16: torch.float16, binding.TYPE_BF16: torch.bfloat16, binding.TYPE_F32: torch.float32}
E4M3 = torch.float8_e4m3fn


def at(t, kind, *shape_and_strides):
    """The operand as a kernel sees it: ((rows, pitch), (columns, 1)) behind its address."""
    assert t.dtype == kind, f"a matrix of {t.dtype} is read as {kind}"
    shape, strides = zip(*shape_and_strides)
    return t.as_strided(shape, strides, t.storage_offset())          # raises where it leaves the storage


def mat(t, kind, rows, cols, pitch):
    return at(t, kind, (rows, pitch), (cols, 1))


def ceil128(n):
    return (n + 127) // 128


def quotients(y, scale):
    return (y / scale).to(E4M3)


def block_max(y):
    """Largest magnitudes of 128 neighbours of each row."""
    return torch.nn.functional.pad(y, (0, -y.shape[1] % 128)).view(y.shape[0], ceil128(y.shape[1]), 128).abs().amax(2).clamp_min(2.0 ** -96)


def quantize_e4m3_rows(M, N, type, act, X, ldx, Q, ldq, scale, ld_scale, stream=0):
    x = mat(X, KIND[type], M, 2 * N if act == binding.ACT_SWIGLU else N, ldx).float()
    if act == binding.ACT_SWIGLU:
        x = torch.nn.functional.silu(x[:, :N]) * x[:, N:]
    s = block_max(x) / 448.0
    mat(scale, torch.float32, ceil128(N), M, ld_scale).copy_(s.t())
    mat(Q, E4M3, M, N, ldq).copy_(quotients(x, s.repeat_interleave(128, 1)[:, :N]))
    return binding.OK


def quantize_e4m3_blocks(M, N, type, X, ldx, Q, ldq, scale, ld_scale, stream=0):
    x = mat(X, KIND[type], M, N, ldx).float()
    s = torch.nn.functional.pad(block_max(x), (0, 0, 0, -M % 128)).view(ceil128(M), 128, -1).amax(1).clamp_min(2.0 ** -96) / 448.0
    mat(scale, torch.float32, ceil128(M), ceil128(N), ld_scale).copy_(s)
    mat(Q, E4M3, M, N, ldq).copy_(quotients(x, s.repeat_interleave(128, 0)[:M].repeat_interleave(128, 1)[:, :N]))
    return binding.OK


def rms_norm(M, N, type, X, ldx, R, ldr, gamma, eps, H, ldh, Y, ldy, Q, ldq, scale, ld_scale, rstd, stream=0):
    kind = KIND[type]
    h = (mat(X, kind, M, N, ldx).float() + mat(R, kind, M, N, ldr).float()).to(kind)
    mat(H, kind, M, N, ldh).copy_(h)
    s = torch.rsqrt(h.float().square().mean(1) + eps)
    at(rstd, torch.float32, (M, 1)).copy_(s)
    y = h.float() * s[:, None] * at(gamma, kind, (N, 1)).float()
    mat(Y, kind, M, N, ldy).copy_(y)
    if Q is not None:
        b = block_max(y) / 448.0
        mat(scale, torch.float32, ceil128(N), M, ld_scale).copy_(b.t())
        mat(Q, E4M3, M, N, ldq).copy_(quotients(y, b.repeat_interleave(128, 1)[:, :N]))
    return binding.OK


def rms_norm_grad(M, N, type, dY, lddy, H, ldh, gamma, rstd, dH, lddh, dX, lddx, dgamma, workspace, workspace_bytes, stream=0):
    kind = KIND[type]
    r = at(rstd, torch.float32, (M, 1))[:, None]
    dy, x = mat(dY, kind, M, N, lddy).float(), mat(H, kind, M, N, ldh).float() * r
    g = dy * at(gamma, kind, (N, 1)).float()
    mat(dX, kind, M, N, lddx).copy_(r * (g - x * (g * x).mean(1, keepdim=True)) + mat(dH, kind, M, N, lddh).float())
    at(dgamma, torch.float32, (N, 1)).copy_((dy * x).sum(0))
    return binding.OK


def spread(Q, scale, rows, K, ld, ld_scale):
    return mat(Q, E4M3, rows, K, ld).float() * mat(scale, torch.float32, ceil128(K), rows, ld_scale).t().repeat_interleave(128, 1)[:, :K]


def gemm_e4m3_block_grouped(T, N, K, E, offsets, A, lda, a_scale, ld_as, B, ldb, b_stride, b_scale, ld_bs, bs_stride, C, ldc, c_type, stream=0):
    a, c = spread(A, a_scale, T, K, lda, ld_as), mat(C, KIND[c_type & ~binding.EXACT], T, N, ldc)
    b = at(B, E4M3, (E, b_stride), (N, ldb), (K, 1)).float()
    s = at(b_scale, torch.float32, (E, bs_stride), (ceil128(N), ld_bs), (ceil128(K), 1))
    off = at(offsets, torch.int32, (E + 1, 1)).tolist()
    for e in range(E):
        w = b[e] * s[e].repeat_interleave(128, 0)[:N].repeat_interleave(128, 1)[:, :K]
        c[off[e]:off[e + 1]] = (a[off[e]:off[e + 1]] @ w.t()).to(c.dtype)
    return binding.OK


def gemm_e4m3_block(M, N, K, A, lda, a_scale, ld_as, B, ldb, b_scale, ld_bs, C, ldc, c_type, stream=0):
    return gemm_e4m3_block_grouped(M, N, K, 1, torch.tensor([0, M], dtype=torch.int32), A, lda, a_scale, ld_as, B, ldb, 0, b_scale, ld_bs, 0, C, ldc, c_type)


def gemm_grouped(T, N, K, E, offsets, type, A, lda, B, ldb, b_stride, C, ldc, c_type, stream=0):
    a, b, c = mat(A, KIND[type], T, K, lda).float(), at(B, KIND[type], (E, b_stride), (K, ldb), (N, 1)).float(), mat(C, KIND[c_type], T, N, ldc)
    off = at(offsets, torch.int32, (E + 1, 1)).tolist()
    for e in range(E):
        c[off[e]:off[e + 1]] = (a[off[e]:off[e + 1]] @ b[e]).to(c.dtype)
    return binding.OK


def gemm_grouped_grad_a(T, N, K, E, offsets, type, dC, lddc, B, ldb, b_stride, dA, ldda, a_type, stream=0):
    d, b, a = mat(dC, KIND[type], T, N, lddc).float(), at(B, KIND[type], (E, b_stride), (K, ldb), (N, 1)).float(), mat(dA, KIND[a_type], T, K, ldda)
    off = at(offsets, torch.int32, (E + 1, 1)).tolist()
    for e in range(E):
        a[off[e]:off[e + 1]] = (d[off[e]:off[e + 1]] @ b[e].t()).to(a.dtype)
    return binding.OK


def gemm_grouped_grad_b(T, N, K, E, offsets, type, A, lda, dC, lddc, dB, lddb, db_stride, b_type, stream=0):
    a, d, b = mat(A, KIND[type], T, K, lda).float(), mat(dC, KIND[type], T, N, lddc).float(), at(dB, KIND[b_type], (E, db_stride), (K, lddb), (N, 1))
    off = at(offsets, torch.int32, (E + 1, 1)).tolist()
    for e in range(E):
        b[e] = (a[off[e]:off[e + 1]].t() @ d[off[e]:off[e + 1]]).to(b.dtype)
    return binding.OK


ENTRY_POINTS = (quantize_e4m3_rows, quantize_e4m3_blocks, rms_norm, rms_norm_grad, gemm_e4m3_block, gemm_e4m3_block_grouped, gemm_grouped, gemm_grouped_grad_a,
                gemm_grouped_grad_b)
