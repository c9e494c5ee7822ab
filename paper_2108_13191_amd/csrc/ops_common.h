// Shared declarations of the operators of include/gemm_ops.h: parameters of the grouped and e4m3 products, launcher
// prototypes.  gfx950 only.
#pragma once
#include "gemm_common.h"

typedef __bf16 bf16_t;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int intx8 __attribute__((ext_vector_type(8)));
typedef int intx4 __attribute__((ext_vector_type(4)));

enum OpsElem { ELEM_E4M3 = 3, ELEM_I8 = 4, ELEM_F16 = 0, ELEM_BF16 = 1, ELEM_F32 = 2 };      // the 16- and 32-bit ones as GEMM_TYPE_*

// One product C = A B in groups.  What is ragged:
//   offsets == nullptr   nothing: one product of M x N x K
//   !k_ragged            rows: group e multiplies rows offsets[e] .. offsets[e+1]-1 of A (M in all) by B[e]
//   k_ragged             the sum: group e sums over k rows offsets[e] .. offsets[e+1]-1 (K in all) into C[e]
// Operands lie either with the summed index contiguous in a row ("k rows": A M x K, B N x K) or with the other one
// (A K x M, B K x N).
struct OpsGemm {
    int M, N, K, E;
    const int32_t* offsets;
    const char* A; int64_t lda;                          // pitches and strides in elements
    const char* B; int64_t ldb, b_stride;
    char* C; int64_t ldc, c_stride;
    const float* sa; int64_t ld_sa;                      // e4m3: scales of A [k block][row], of B [column block][k block]; i8: of A [row], of B [column]
    const float* sb; int64_t ld_sb, sb_stride;
    int elem, c_type;                                    // OpsElem
    bool a_kc, b_kc;                                     // summed index contiguous
    bool k_ragged;
    bool exact;                                          // e4m3: products exact whatever the result
    int num_xcd;
    hipStream_t stream;
};

// What the entry points check of their arguments
inline bool bad_size(int64_t n) { return n < 0 || n > INT32_MAX; }
inline bool bad_pitch(int64_t ld, int64_t row) { return ld < row || ld > INT32_MAX; }
inline bool unaligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) != 0; }
inline bool is_16bit(int64_t type) { return type == ELEM_F16 || type == ELEM_BF16; }
inline int type_size(int64_t type) { return type == ELEM_F32 ? 4 : 2; }

// A launch has less than 2^32 threads in a dimension of its grid.
inline bool fits_a_launch(int64_t workgroups, int threads) { return workgroups <= UINT32_MAX / threads; }
// Workgroups of a launch on bm x bn tiles, -1: more than an int counts.  k_ragged: E x (M / bm) x (N / bn); rows: as many as the groups may need, each
// of which may end in a short tile.
inline int64_t tile_grid(const OpsGemm& g, int bm, int bn)
{
    const int64_t M = g.M, tn = ((int64_t)g.N + bn - 1) / bn, tm = (M + bm - 1) / bm;
    const int64_t rows = g.k_ragged ? tm * g.E : g.offsets ? M / bm + (g.E < M ? g.E : M) : tm;
    return rows > INT32_MAX / tn ? -1 : rows * tn;
}

// ops_api.hip: a checked product on the kernel that suits it, and that kernel's name (nullptr: nothing to run, or more workgroups than a launch has)
int ops_run_product(const OpsGemm& g);
const char* ops_product_form(const OpsGemm& g);

// ops_generic.hip: any alignment, any size
int ops_launch_generic(const OpsGemm& g);

// ops_tile_*.hip: 16-byte aligned operands (TILE_128_ANY: any) with pitches up to 2^22 elements (each takes the tiles that the choice in ops_api.hip has for it)
// e4m3: TILE_256 and TILE_128_FAST on the e4m3 instructions, the others widened to f16 (_PAIR: two workgroups a compute unit, _SHORT: short groups of rows)
enum OpsTile { TILE_256, TILE_256x128, TILE_128x256, TILE_128, TILE_128_ANY, TILE_128_FAST, TILE_128_PAIR, TILE_128_SHORT, TILE_256_LONG };
int ops_launch_tiles_e4m3(const OpsGemm& g, OpsTile tile);
int ops_launch_tiles_f16(const OpsGemm& g, OpsTile tile);
int ops_launch_tiles_bf16(const OpsGemm& g, OpsTile tile);
int ops_launch_tiles_i8(const OpsGemm& g, OpsTile tile);
// ops_i8_long.hip: TILE_256_LONG, i8 on 256 x 256 tiles of four wavefronts; K >= 128
int ops_launch_long_i8(const OpsGemm& g);

// ops_skinny_e4m3.hip: few rows; fm x nb: 16 x 16 blocks of a workgroup's tile, 1 x 1, 1 x 2, 2 x 1, 2 x 2 or 2 x 4
int ops_launch_skinny_e4m3(const OpsGemm& g, int fm, int nb);
// ops_i8_few.hip: the same in i8, 1 x 1, 1 x 4, 2 x 1, 2 x 2, 2 x 4, 4 x 4 or 8 x 4
int ops_launch_few_i8(const OpsGemm& g, int fm, int nb);
// ... at any alignment, 2 x 2 or 4 x 4
int ops_launch_few_i8_any(const OpsGemm& g, int fm);

// ops_norm.hip
struct NormArgs {
    int M, N;
    const void *X, *R, *gamma; int64_t ldx, ldr;
    void *H, *Y; int64_t ldh, ldy;
    uint8_t* Q; int64_t ldq; float* scale; int64_t ld_scale;
    float* rstd; float eps;
};
struct NormGradArgs {
    int M, N;
    const void *dY, *H, *gamma, *dH; const float* rstd; int64_t lddy, ldh, lddh;
    void* dX; int64_t lddx;
    float *dgamma, *ws;
};
struct QuantArgs {
    int M, N, act;
    const void* X; int64_t ldx;
    uint8_t* Q; int64_t ldq; float* scale; int64_t ld_scale;
};
int ops_launch_norm(int type, const NormArgs& a, hipStream_t stream);
int ops_norm_grad_parts(int64_t M, int64_t N);            // rows of N floats of workspace
int ops_launch_norm_grad(int type, const NormGradArgs& a, hipStream_t stream);
int ops_launch_quant_rows(int type, const QuantArgs& a, hipStream_t stream);
int ops_launch_quant_blocks(int type, const QuantArgs& a, hipStream_t stream);

// ops_layer_norm.hip
struct LayerNormArgs {
    int M, N;
    const void *X, *R, *gamma, *beta; int64_t ldx, ldr;
    void *H, *Y; int64_t ldh, ldy;
    uint8_t* Q; int64_t ldq; float* scale;
    float *mean, *rstd; float eps;
};
struct LayerNormGradArgs {
    int M, N;
    const void *dY, *H, *gamma, *dH; const float *mean, *rstd; int64_t lddy, ldh, lddh;
    void* dX; int64_t lddx;
    float *dgamma, *dbeta, *ws;
};
int ops_launch_layer_norm(int type, const LayerNormArgs& a, hipStream_t stream);
int ops_layer_norm_grad_parts(int64_t M, int64_t N);      // rows of 2 N floats of workspace
int ops_launch_layer_norm_grad(int type, const LayerNormGradArgs& a, hipStream_t stream);
int ops_launch_quant_i8(int type, const QuantArgs& a, hipStream_t stream);

// ops_experts.hip.  T tokens with top_k choices each
struct DispatchArgs {
    int64_t T; int top_k, E;
    bool index64; const void* expert;
    int32_t *offsets, *source, *place;
    int N, size;                                         // elements of a row, bytes of one
    const void* X; int64_t ldx;
    int64_t blocks; const float* scale; int64_t ld_scale;
    void* rows; int64_t ld_rows; float* row_scale; int64_t ld_row_scale;
};
struct CombineArgs {
    int64_t T, rows; int top_k, N;                       // rows: of Y
    const int32_t* place;
    const void* Y; int64_t ldy;
    const float* weight;
    const void* add; int64_t ld_add;
    void* out; int64_t ldo;
};
struct CombineGradArgs {
    int64_t T, rows; int top_k, N;
    const int32_t* place;
    const void* dOut; int64_t lddo;
    const float* weight;
    const void* Y; int64_t ldy;
    void* dY; int64_t lddy;
    float* dweight;
};
int64_t ops_dispatch_workspace_bytes(int64_t T, int64_t top_k, int64_t E);
int ops_launch_dispatch(const DispatchArgs& a, void* workspace, hipStream_t stream);
int ops_launch_combine(int type, int out_type, const CombineArgs& a, hipStream_t stream);
int ops_launch_combine_grad(int type, const CombineGradArgs& a, hipStream_t stream);
