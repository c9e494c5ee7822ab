/*
 * gemm_layer.h -- C ABI of further operators around the products of a transformer layer (MI355X, gfx950), in the same library as
 * gemm_f16.h and gemm_ops.h: layer norm with the residual's addition and its gradients, quantisation to 8-bit integers and products of
 * such matrices, and tokens' rows moved to their experts' order and back, with the gradients of that.
 *
 * Conventions are those of gemm_ops.h: row-major matrices in device memory of the current HIP device, pitches in ELEMENTS, sizes
 * from 0 to 2^31-1, work only enqueued on `stream` (a hipStream_t as void*), arguments checked on the host before anything is launched,
 * the GEMM_F16_* return codes, nothing allocated, nothing thrown, no state kept.  An output must not overlap an input unless said
 * otherwise.  No call writes between a row's end and the pitch; an aligned 16-byte fetch may read there.  All entry points may be
 * captured into a HIP graph.  A workspace serves one call at a time: calls (or graphs) that may run at once have one each; what
 * it holds means nothing between calls.
 */
#ifndef GEMM_LAYER_H
#define GEMM_LAYER_H

#include <stdint.h>
#include "gemm_ops.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Layer norm of M rows of N elements with the residual's addition:
 *     h = x + r                    rounded to `type` (f16 or bf16); r NULL: h = x
 *     mean = sum(h) / N,  rstd = 1 / sqrt(sum((h - mean)^2) / N + eps)      of the rounded h, in f32 (sums about the mean: no cancellation of squares)
 *     y = (h - mean) * rstd * gamma + beta                                  beta NULL: 0
 * Outputs, each of which may be NULL: H (h), Y (y in `type`), Q with scale (y as 8-bit integers with a scale for each row, as
 * quantize_i8_rows has them, from the f32 value), mean and rstd (M f32 each, as layer_norm_grad takes them).  H may be X or R
 * themselves.  gamma, beta: N elements of `type`.  Q without scale or scale without Q is GEMM_F16_ERR_NULL; eps that is
 * negative or no number is GEMM_F16_ERR_CONFIG.  N = 0 writes nothing.  A row that holds a NaN or an infinity, or whose sum passes f32's range, is
 * NaN (Q: the scale NaN, elements 0; mean and rstd too); where only its sum of squares does, or sums of parts of it or differences from its mean, rstd is 0 and y is beta.  Pointers of 16-bit matrices: 2-byte aligned, any pitch.
 */
int layer_norm(int64_t M, int64_t N, int64_t type,
               const void* X, int64_t ldx, const void* R, int64_t ldr,
               const void* gamma, const void* beta, double eps,
               void* H, int64_t ldh, void* Y, int64_t ldy,
               void* Q, int64_t ldq, float* scale,
               float* mean, float* rstd, void* stream);

/*
 * Gradients of layer_norm's Y.  From dY, the stored H, gamma, mean and rstd:
 *     xhat = (h - mean) * rstd,  g = dy * gamma                     (NaN where a difference passes f32's range)
 *     dX = rstd * (g - mean(g) - xhat * mean(g * xhat)) + dH        (of x and of r alike)
 *     dgamma[j] = sum_i dy[i][j] * xhat[i][j],  dbeta[j] = sum_i dy[i][j]        (N f32 each)
 * dH: the gradient that reaches h by the residual's own way, or NULL.  dX may be dY or dH themselves.  dgamma, dbeta: NULL where one
 * is not wanted; without both no workspace is needed; M = 0 gives zeros.  The rows are summed in a fixed order
 * (two runs give the same bits) with the help of a workspace of layer_norm_grad_workspace_bytes(M, N) bytes (at most 256 rows of 2 N
 * floats), 16-byte aligned; smaller: GEMM_F16_ERR_WORKSPACE.
 */
int64_t layer_norm_grad_workspace_bytes(int64_t M, int64_t N);
int layer_norm_grad(int64_t M, int64_t N, int64_t type,
                    const void* dY, int64_t lddy, const void* H, int64_t ldh,
                    const void* gamma, const float* mean, const float* rstd,
                    const void* dH, int64_t lddh,
                    void* dX, int64_t lddx, float* dgamma, float* dbeta,
                    void* workspace, int64_t workspace_bytes, void* stream);

/*
 * Quantise the rows of X (M x N of `type`, f16 or bf16; M x 2N for SWIGLU) to 8-bit integers, a scale for each row: a token's of
 * activations, a channel's of weights.
 *     scale[i] = max(largest |x| of row i, 2^-96) * (1/127) in f32, one product with the f32 value nearest to 1/127 (127 gives 1),  element = the integer nearest to x / scale[i] (ties to even), from -127 to 127
 * act is applied first, in f32, as in quantize_e4m3_rows.  A row that holds a NaN or an infinity gets the scale NaN and elements 0, so
 * that it shows in any product; a row of zeros is zeros with the scale 2^-96 * (1/127).
 */
int quantize_i8_rows(int64_t M, int64_t N, int64_t type, int64_t act,
                     const void* X, int64_t ldx, void* Q, int64_t ldq, float* scale, void* stream);

/*
 * Product of 8-bit integer matrices with scales for each token and channel: C (M x N of c_type: f16, bf16 or f32), overwritten,
 * with A (M x K) and B (N x K: a row for each output, as weights are stored):
 *     C[i][j] = (sum_k A[i][k] B[j][k]) * a_scale[i] * b_scale[j]
 * The sum is exact, in 32-bit integers; it becomes f32 (one rounding, of sums beyond 2^24), is multiplied by the two scales in this order and
 * rounded once to c_type.  K <= 131071, so that no sum of products of any 8-bit integers (-128 to 127) leaves 32 bits; larger:
 * GEMM_F16_ERR_SIZE.  K = 0 gives zeros (a scale that is NaN or infinite gives NaN all the same).  Any alignment is
 * accepted; A and B 16-byte aligned with pitches that are multiples of 16 run the fastest kernels (K and N of any size), others take up to twice (few
 * rows) or four times (large products) as long, with pitches above 2^22 more.
 *
 * gemm_i8_grouped: the same grouped by expert as in gemm_e4m3_block_grouped: rows offsets[e] .. offsets[e+1]-1 of A (T rows) with B[e], which begins
 * b_stride * e elements behind B, and scales that begin bs_stride * e floats behind b_scale (strides from 0 on).  Rows in no group are left alone.
 *
 * gemm_i8_form: the name of the kernel that a product would run on (E < 0: gemm_i8), as gemm_ops_form; NULL for nothing to run.
 */
int gemm_i8(int64_t M, int64_t N, int64_t K,
            const void* A, int64_t lda, const float* a_scale,
            const void* B, int64_t ldb, const float* b_scale,
            void* C, int64_t ldc, int64_t c_type, void* stream);
int gemm_i8_grouped(int64_t T, int64_t N, int64_t K, int64_t E, const int32_t* offsets,
                    const void* A, int64_t lda, const float* a_scale,
                    const void* B, int64_t ldb, int64_t b_stride, const float* b_scale, int64_t bs_stride,
                    void* C, int64_t ldc, int64_t c_type, void* stream);
const char* gemm_i8_form(int64_t T, int64_t N, int64_t K, int64_t E, int64_t lda, int64_t ldb, int64_t c_type);

/*
 * Tokens to their experts.  `expert` (T x top_k, contiguous, 32- or 64-bit integers by index_type): the experts that each token
 * chose; a choice outside 0 .. E-1 is of no expert here (a padded token, an expert of another process) and dropped.  The
 * choices are sorted by expert, those of one expert in the order of the tokens (and of a token's choices):
 *     offsets   E + 1 int32: rows offsets[e] .. offsets[e+1]-1 are expert e's, as the products grouped by expert take them
 *     place     T * top_k int32: the row of choice j of token t at place[t * top_k + j], -1 for a dropped one
 *     source    T * top_k int32: the token of each row; -1 from row offsets[E] on.  May be NULL.
 * and each token's row is copied to its places:
 *     rows[place[t][j]] = X[t]                       T * top_k rows of N elements of `size` bytes (1, 2 or 4)
 *     row_scale[b][place[t][j]] = scale[b][t]        `blocks` rows of scales (e4m3: ceil(N / 128), i8: 1, none: 0), ld_scale >= T and ld_row_scale >= T * top_k
 * X NULL: only the order is formed.  Rows from offsets[E] on and their scales are left alone.  T = 0 or top_k = 0 writes zeros to offsets.
 * T * top_k <= 2^31-1, top_k and E <= 65535.  workspace: expert_dispatch_workspace_bytes(T, top_k, E) bytes (0 for few choices; at most 8 T top_k +
 * 2^22), 16-byte aligned; smaller: GEMM_F16_ERR_WORKSPACE.
 */
enum { GEMM_INDEX_I32 = 0, GEMM_INDEX_I64 = 1 };
int64_t expert_dispatch_workspace_bytes(int64_t T, int64_t top_k, int64_t E);
int expert_dispatch(int64_t T, int64_t top_k, int64_t E, int64_t index_type, const void* expert,
                    int32_t* offsets, int32_t* source, int32_t* place,
                    int64_t N, int64_t size, const void* X, int64_t ldx,
                    int64_t blocks, const float* scale, int64_t ld_scale,
                    void* rows, int64_t ld_rows, float* row_scale, int64_t ld_row_scale,
                    void* workspace, int64_t workspace_bytes, void* stream);

/*
 * And back: out[t] = add[t] + sum_j weight[t][j] * Y[place[t][j]], over the choices in their order, each product rounded to f32 and
 * then added, `add` last, rounded once to out_type (T and top_k as above).  Y: T * top_k rows of N elements of `type` (f16, bf16 or f32); weight: T x top_k f32, contiguous, NULL: 1; add (T rows of
 * `type`): NULL: 0; out_type: `type` itself or f32.  A place outside 0 .. T*top_k-1 adds nothing (a row without any is `add`, or zeros).  out may be add
 * itself where both have one type.  With weight NULL this is the gradient of expert_dispatch's rows (and add the one that reaches X by another way).
 *
 * expert_combine_grad: the gradients of that, from dOut (T rows of `type`, f16 or bf16; the one of add is dOut itself):
 *     dY[place[t][j]] = weight[t][j] * dOut[t]                of `type`; rows of no place are left alone; may be Y itself; NULL: not formed
 *     dweight[t][j] = sum_n dOut[t][n] * Y[place[t][j]][n]    T x top_k f32 in a fixed order, 0 for a choice of no place; NULL: not formed (Y is not read)
 * Places have to be different from each other.
 */
int expert_combine(int64_t T, int64_t top_k, int64_t N, int64_t type, const int32_t* place,
                   const void* Y, int64_t ldy, const float* weight, const void* add, int64_t ld_add,
                   void* out, int64_t ldo, int64_t out_type, void* stream);
int expert_combine_grad(int64_t T, int64_t top_k, int64_t N, int64_t type, const int32_t* place,
                        const void* dOut, int64_t lddo, const float* weight, const void* Y, int64_t ldy,
                        void* dY, int64_t lddy, float* dweight, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* GEMM_LAYER_H */
