// The C ABI of include/gemm_layer.h: checks of arguments.
#include "ops_common.h"
#include "../../include/gemm_layer.h"

namespace {

constexpr int64_t MOST_K_I8 = 131071;                      // 2^14 K < 2^31: no sum of products leaves 32 bits

bool bad_index(int64_t type) { return type != GEMM_INDEX_I32 && type != GEMM_INDEX_I64; }
// T tokens of top_k choices, whose number fits an int.  A token's choices go one after another, which takes a wavefront some 20 ms at 65535 and would not end for minutes at 2^31
bool bad_choices(int64_t T, int64_t top_k) { return bad_size(T) || top_k < 0 || top_k > 65535 || (T > 0 && top_k > INT32_MAX / T); }

OpsGemm shaped_i8(int64_t M, int64_t N, int64_t K, int64_t E, const int32_t* offsets, int64_t c_type, void* stream)
{
    OpsGemm g = {};
    g.M = (int)M; g.N = (int)N; g.K = (int)K; g.E = E < 0 ? 1 : (int)E;
    g.offsets = offsets;
    g.elem = ELEM_I8;
    g.c_type = (int)c_type;
    g.a_kc = g.b_kc = true;
    g.num_xcd = chip().xcds;
    g.stream = (hipStream_t)stream;
    return g;
}

// E < 0: one product, nothing grouped
int run_i8(int64_t M, int64_t N, int64_t K, int64_t E, const int32_t* offsets, const void* A, int64_t lda, const float* sa,
           const void* B, int64_t ldb, int64_t b_stride, const float* sb, int64_t bs_stride, void* C, int64_t ldc, int64_t c_type, void* stream)
{
    if (bad_size(M) || bad_size(N) || bad_size(K) || K > MOST_K_I8 || E > 65535) return GEMM_F16_ERR_SIZE;
    if (!is_16bit(c_type) && c_type != GEMM_TYPE_F32) return GEMM_F16_ERR_CONFIG;
    if (M == 0 || N == 0 || E == 0) return GEMM_F16_OK;
    if (bad_pitch(lda, K) || bad_pitch(ldb, K) || bad_pitch(ldc, N) || b_stride < 0 || bs_stride < 0) return GEMM_F16_ERR_PITCH;
    if (!C || !sa || !sb || (E > 0 && !offsets) || (K > 0 && (!A || !B))) return GEMM_F16_ERR_NULL;
    if (unaligned(C, type_size(c_type)) || unaligned(sa, 4) || unaligned(sb, 4) || unaligned(offsets, 4)) return GEMM_F16_ERR_ALIGN;
    OpsGemm g = shaped_i8(M, N, K, E, offsets, c_type, stream);
    g.A = (const char*)A; g.lda = lda; g.B = (const char*)B; g.ldb = ldb; g.b_stride = b_stride;
    g.C = (char*)C; g.ldc = ldc;
    g.sa = sa; g.sb = sb; g.sb_stride = bs_stride;
    return ops_run_product(g);
}

}  // namespace

extern "C" {

int layer_norm(int64_t M, int64_t N, int64_t type, const void* X, int64_t ldx, const void* R, int64_t ldr, const void* gamma, const void* beta, double eps,
               void* H, int64_t ldh, void* Y, int64_t ldy, void* Q, int64_t ldq, float* scale, float* mean, float* rstd, void* stream)
{
    if (bad_size(M) || bad_size(N)) return GEMM_F16_ERR_SIZE;
    if (!is_16bit(type) || !(eps >= 0.0)) return GEMM_F16_ERR_CONFIG;
    if (M == 0 || N == 0) return GEMM_F16_OK;
    if (bad_pitch(ldx, N) || (R && bad_pitch(ldr, N)) || (H && bad_pitch(ldh, N)) || (Y && bad_pitch(ldy, N)) || (Q && bad_pitch(ldq, N))) return GEMM_F16_ERR_PITCH;
    if (!X || !gamma || !Q != !scale) return GEMM_F16_ERR_NULL;
    if (unaligned(X, 2) || unaligned(R, 2) || unaligned(gamma, 2) || unaligned(beta, 2) || unaligned(H, 2) || unaligned(Y, 2) || unaligned(scale, 4) || unaligned(mean, 4) ||
        unaligned(rstd, 4)) return GEMM_F16_ERR_ALIGN;
    return ops_launch_layer_norm((int)type, {(int)M, (int)N, X, R, gamma, beta, ldx, ldr, H, Y, ldh, ldy, (uint8_t*)Q, ldq, scale, mean, rstd, (float)eps}, (hipStream_t)stream);
}

int64_t layer_norm_grad_workspace_bytes(int64_t M, int64_t N)
{
    if (M <= 0 || N <= 0 || M > INT32_MAX || N > INT32_MAX) return 0;
    return 8 * N * ops_layer_norm_grad_parts(M, N);
}

int layer_norm_grad(int64_t M, int64_t N, int64_t type, const void* dY, int64_t lddy, const void* H, int64_t ldh, const void* gamma, const float* mean, const float* rstd,
                    const void* dH, int64_t lddh, void* dX, int64_t lddx, float* dgamma, float* dbeta, void* workspace, int64_t workspace_bytes, void* stream)
{
    if (bad_size(M) || bad_size(N)) return GEMM_F16_ERR_SIZE;
    if (!is_16bit(type)) return GEMM_F16_ERR_CONFIG;
    const bool columns = dgamma || dbeta;
    if (N == 0 || (M == 0 && !columns)) return GEMM_F16_OK;
    if (M > 0) {
        if (bad_pitch(lddy, N) || bad_pitch(ldh, N) || bad_pitch(lddx, N) || (dH && bad_pitch(lddh, N))) return GEMM_F16_ERR_PITCH;
        if (!dY || !H || !gamma || !mean || !rstd || !dX || (columns && !workspace)) return GEMM_F16_ERR_NULL;
        if (unaligned(dY, 2) || unaligned(H, 2) || unaligned(gamma, 2) || unaligned(dH, 2) || unaligned(dX, 2) || unaligned(mean, 4) || unaligned(rstd, 4) ||
            (columns && unaligned(workspace, 16))) return GEMM_F16_ERR_ALIGN;
        if (columns && workspace_bytes < layer_norm_grad_workspace_bytes(M, N)) return GEMM_F16_ERR_WORKSPACE;
    }
    if (unaligned(dgamma, 4) || unaligned(dbeta, 4)) return GEMM_F16_ERR_ALIGN;
    return ops_launch_layer_norm_grad((int)type, {(int)M, (int)N, dY, H, gamma, dH, mean, rstd, lddy, ldh, lddh, dX, lddx, dgamma, dbeta, (float*)workspace}, (hipStream_t)stream);
}

int quantize_i8_rows(int64_t M, int64_t N, int64_t type, int64_t act, const void* X, int64_t ldx, void* Q, int64_t ldq, float* scale, void* stream)
{
    if (bad_size(M) || bad_size(N)) return GEMM_F16_ERR_SIZE;
    if (!is_16bit(type) || (act != GEMM_OPS_ACT_NONE && act != GEMM_OPS_ACT_RELU && act != GEMM_OPS_ACT_SWIGLU)) return GEMM_F16_ERR_CONFIG;
    if (M == 0 || N == 0) return GEMM_F16_OK;
    if (bad_pitch(ldx, act == GEMM_OPS_ACT_SWIGLU ? 2 * N : N) || bad_pitch(ldq, N)) return GEMM_F16_ERR_PITCH;
    if (!X || !Q || !scale) return GEMM_F16_ERR_NULL;
    if (unaligned(X, 2) || unaligned(scale, 4)) return GEMM_F16_ERR_ALIGN;
    return ops_launch_quant_i8((int)type, {(int)M, (int)N, (int)act, X, ldx, (uint8_t*)Q, ldq, scale, 0}, (hipStream_t)stream);
}

int gemm_i8(int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const float* a_scale, const void* B, int64_t ldb, const float* b_scale,
            void* C, int64_t ldc, int64_t c_type, void* stream)
{
    return run_i8(M, N, K, -1, nullptr, A, lda, a_scale, B, ldb, 0, b_scale, 0, C, ldc, c_type, stream);
}

int gemm_i8_grouped(int64_t T, int64_t N, int64_t K, int64_t E, const int32_t* offsets, const void* A, int64_t lda, const float* a_scale,
                    const void* B, int64_t ldb, int64_t b_stride, const float* b_scale, int64_t bs_stride, void* C, int64_t ldc, int64_t c_type, void* stream)
{
    if (E < 0) return GEMM_F16_ERR_SIZE;
    return run_i8(T, N, K, E, offsets, A, lda, a_scale, B, ldb, b_stride, b_scale, bs_stride, C, ldc, c_type, stream);
}

const char* gemm_i8_form(int64_t T, int64_t N, int64_t K, int64_t E, int64_t lda, int64_t ldb, int64_t c_type)
{
    if (bad_size(T) || bad_size(N) || bad_size(K) || K > MOST_K_I8 || E > 65535 || E == 0 || T == 0 || N == 0 || (!is_16bit(c_type) && c_type != GEMM_TYPE_F32)) return nullptr;
    static const int32_t some_offsets = 0;
    OpsGemm g = shaped_i8(T, N, K, E, E < 0 ? nullptr : &some_offsets, c_type, nullptr);
    g.lda = lda; g.ldb = ldb;
    return ops_product_form(g);
}

int64_t expert_dispatch_workspace_bytes(int64_t T, int64_t top_k, int64_t E)
{
    if (bad_choices(T, top_k) || E < 0 || E > 65535) return 0;
    return ops_dispatch_workspace_bytes(T, top_k, E);
}

int expert_dispatch(int64_t T, int64_t top_k, int64_t E, int64_t index_type, const void* expert, int32_t* offsets, int32_t* source, int32_t* place,
                    int64_t N, int64_t size, const void* X, int64_t ldx, int64_t blocks, const float* scale, int64_t ld_scale,
                    void* rows, int64_t ld_rows, float* row_scale, int64_t ld_row_scale, void* workspace, int64_t workspace_bytes, void* stream)
{
    if (bad_choices(T, top_k) || E < 0 || E > 65535 || bad_size(N) || bad_size(blocks)) return GEMM_F16_ERR_SIZE;
    if (bad_index(index_type) || (X && size != 1 && size != 2 && size != 4)) return GEMM_F16_ERR_CONFIG;
    const int64_t n = T * top_k;
    const bool moved = X && N > 0;
    if (n > 0 && moved && (bad_pitch(ldx, N) || bad_pitch(ld_rows, N) || (blocks > 0 && (bad_pitch(ld_scale, T) || bad_pitch(ld_row_scale, n))))) return GEMM_F16_ERR_PITCH;
    if (!offsets) return GEMM_F16_ERR_NULL;
    if (n > 0 && (!expert || !place || (moved && (!rows || (blocks > 0 && (!scale || !row_scale)))))) return GEMM_F16_ERR_NULL;
    if (unaligned(offsets, 4)) return GEMM_F16_ERR_ALIGN;
    if (n > 0) {
        if (unaligned(expert, index_type == GEMM_INDEX_I64 ? 8 : 4) || unaligned(source, 4) || unaligned(place, 4) ||
            (moved && (unaligned(X, (uintptr_t)size) || unaligned(rows, (uintptr_t)size) || (blocks > 0 && (unaligned(scale, 4) || unaligned(row_scale, 4)))))) return GEMM_F16_ERR_ALIGN;
        const int64_t need = ops_dispatch_workspace_bytes(T, top_k, E);
        if (need > 0) {
            if (!workspace) return GEMM_F16_ERR_NULL;
            if (unaligned(workspace, 16)) return GEMM_F16_ERR_ALIGN;
            if (workspace_bytes < need) return GEMM_F16_ERR_WORKSPACE;
        }
    }
    DispatchArgs a = {};
    a.T = T; a.top_k = (int)top_k; a.E = (int)E; a.index64 = index_type == GEMM_INDEX_I64; a.expert = expert;
    a.offsets = offsets; a.source = source; a.place = place;
    if (moved) {
        a.N = (int)N; a.size = (int)size; a.X = X; a.ldx = ldx; a.rows = rows; a.ld_rows = ld_rows;
        a.blocks = blocks; a.scale = scale; a.ld_scale = ld_scale; a.row_scale = row_scale; a.ld_row_scale = ld_row_scale;
    }
    return ops_launch_dispatch(a, workspace, (hipStream_t)stream);
}

int expert_combine(int64_t T, int64_t top_k, int64_t N, int64_t type, const int32_t* place, const void* Y, int64_t ldy, const float* weight,
                   const void* add, int64_t ld_add, void* out, int64_t ldo, int64_t out_type, void* stream)
{
    if (bad_choices(T, top_k) || bad_size(N)) return GEMM_F16_ERR_SIZE;
    if ((!is_16bit(type) && type != GEMM_TYPE_F32) || (out_type != type && out_type != GEMM_TYPE_F32)) return GEMM_F16_ERR_CONFIG;
    if (T == 0 || N == 0) return GEMM_F16_OK;
    if ((top_k > 0 && bad_pitch(ldy, N)) || (add && bad_pitch(ld_add, N)) || bad_pitch(ldo, N)) return GEMM_F16_ERR_PITCH;
    if (!out || (top_k > 0 && (!place || !Y))) return GEMM_F16_ERR_NULL;
    if (unaligned(place, 4) || unaligned(Y, type_size(type)) || unaligned(weight, 4) || unaligned(add, type_size(type)) || unaligned(out, type_size(out_type))) return GEMM_F16_ERR_ALIGN;
    return ops_launch_combine((int)type, (int)out_type, {T, T * top_k, (int)top_k, (int)N, place, Y, ldy, weight, add, ld_add, out, ldo}, (hipStream_t)stream);
}

int expert_combine_grad(int64_t T, int64_t top_k, int64_t N, int64_t type, const int32_t* place, const void* dOut, int64_t lddo, const float* weight,
                        const void* Y, int64_t ldy, void* dY, int64_t lddy, float* dweight, void* stream)
{
    if (bad_choices(T, top_k) || bad_size(N)) return GEMM_F16_ERR_SIZE;
    if (!is_16bit(type)) return GEMM_F16_ERR_CONFIG;
    if (T == 0 || top_k == 0 || (!dweight && (N == 0 || !dY))) return GEMM_F16_OK;
    if (bad_pitch(lddo, N) || (dweight && bad_pitch(ldy, N)) || (dY && bad_pitch(lddy, N))) return GEMM_F16_ERR_PITCH;
    if (!place || (N > 0 && (!dOut || (dweight && !Y)))) return GEMM_F16_ERR_NULL;
    if (unaligned(place, 4) || unaligned(dOut, 2) || unaligned(weight, 4) || unaligned(Y, 2) || unaligned(dY, 2) || unaligned(dweight, 4)) return GEMM_F16_ERR_ALIGN;
    return ops_launch_combine_grad((int)type, {T, T * top_k, (int)top_k, (int)N, place, dOut, lddo, weight, Y, ldy, dY, lddy, dweight}, (hipStream_t)stream);
}

}  // extern "C"
