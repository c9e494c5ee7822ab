// The C ABI of include/gemm_ops.h: checks of arguments and the choice of kernel.
#include "ops_common.h"
#include "../../include/gemm_ops.h"
#include <math.h>

namespace {

bool bad_size(int64_t n) { return n < 0 || n > INT32_MAX; }
bool bad_pitch(int64_t ld, int64_t row) { return ld < row || ld > INT32_MAX; }
bool unaligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) != 0; }
int64_t blocks128(int64_t n) { return (n + 127) / 128; }
bool is_16bit(int64_t type) { return type == GEMM_TYPE_F16 || type == GEMM_TYPE_BF16; }
int type_size(int64_t type) { return type == GEMM_TYPE_F32 ? 4 : 2; }

// What the tiled kernels take: operands whose offsets within a tile fit 32 bits, and but for one form of the 16-bit ones 16-byte aligned ones
bool tiles_take(const OpsGemm& g)
{
    return g.lda <= (1 << 22) && g.ldb <= (1 << 22) && g.M <= INT32_MAX - 512 && g.N <= INT32_MAX - 512 && g.K <= INT32_MAX - 512;
}
bool is_aligned(const OpsGemm& g)
{
    const int64_t chunk = g.elem == ELEM_E4M3 ? 16 : 8;
    return !unaligned(g.A, 16) && !unaligned(g.B, 16) && g.lda % chunk == 0 && g.ldb % chunk == 0 && g.b_stride % chunk == 0;
}

// Tiles of bm x bn results that a launch is expected to have (how the rows are dealt is known on the device only): in groups with fewer
// rows than a tile one each, in larger ones half a tile more than their rows fill.
double expected_tiles(const OpsGemm& g, int bm, int bn)
{
    const double tn = (g.N + bn - 1) / bn;
    if (g.k_ragged) return (double)g.E * ((g.M + bm - 1) / bm) * tn;
    if (!g.offsets) return ((g.M + bm - 1) / bm) * tn;
    const double groups = g.E < g.M ? g.E : g.M, rows = g.M / groups;
    return (g.M / (double)bm + groups * (rows < bm ? 1.0 - 0.5 * rows / bm : 0.5)) * tn;
}

// The results that bm x bn tiles of an M x N matrix multiply, with the rows and columns behind its ends
double padded(int64_t M, int64_t N, int bm, int bn) { return (double)((M + bm - 1) / bm * bm) * (double)((N + bn - 1) / bn * bn); }

// What a product runs on: the kernel for any alignment, the tiled one, or the one for few rows on 16 fm x 16 nb results a workgroup.
struct Form {
    enum Kernel { ANY, TILES, FEW_ROWS } kernel;
    OpsTile tile;
    int fm, nb;
};
Form any_alignment() { return {Form::ANY, TILE_256, 0, 0}; }
Form tiles(OpsTile t) { return {Form::TILES, t, 0, 0}; }
Form few_rows(int fm, int nb) { return {Form::FEW_ROWS, TILE_256, fm, nb}; }

// Whether its workgroups are as many as one launch takes
bool fits(const OpsGemm& g, const Form& f)
{
    const bool wide = f.tile == TILE_256 || f.tile == TILE_128x256, tall = f.tile == TILE_256 || f.tile == TILE_256x128;
    const int bm = f.kernel == Form::ANY ? 64 : f.kernel == Form::FEW_ROWS ? 16 * f.fm : tall ? 256 : 128;
    const int bn = f.kernel == Form::ANY ? 64 : f.kernel == Form::FEW_ROWS ? 16 * f.nb : wide ? 256 : 128;
    const int64_t grid = tile_grid(g, bm, bn);
    return grid >= 0 && fits_a_launch(grid, f.kernel == Form::ANY ? 256 : 512);
}

// The fastest of them; us measured for the one taken | the other, groups as a random router deals them.  `rows` is the average group's: who has more is known on the device only.
// 1280 rows of 64 experts (4096,2048) in e4m3 that all go to one take 102 us on the 32-row tiles of 20 rows each, and 20 to 40 on tiles of 128; dealt evenly they take 155.
Form preferred(const OpsGemm& g, bool allow_few_rows)
{
    if (!tiles_take(g)) return any_alignment();
    // (a form that loads 8 elements at any alignment needs rows that have them)
    if (!is_aligned(g)) return g.elem == ELEM_E4M3 || g.N < 8 || (g.k_ragged ? g.M : g.K) < 8 ? any_alignment() : tiles(TILE_128_ANY);
    const int cus = chip().cus;
    const double rows = (double)g.M / g.E;                                  // of a group
    if (g.k_ragged) {
        // gradient of B, 256 x 256 | 128 x 128, from two rounds of the former on: both gradients of (16384 rows, 2048 x 1024, 32 experts) 1024 tiles 214 | 231,
        // (16384, 4096 x 2048, 8) 1024 tiles 505 | 563; below one: B's alone, (16384, 2304 x 768, 8) 216 tiles 89 | 77, (2048 x 1024, 4) 128 tiles 139 | 91.
        // Between, with many rows a group, (16384, 4096 x 2048, 3) 384 tiles 231 | 277, (2048 x 2048, 5) 320 tiles 146 | 151, with few (4000, 1408 x 2048, 8) 46 | 40; and
        // one round of a single group's, whose operands 128 x 128 tiles read too often: (16384, 4096 x 4096, 1) 380 | 602, (1000, ..) 40 | 43
        // Matrices that fill the larger tiles badly, 1.3 times and more what the smaller ones multiply: 64 experts' 640 x 640 (1.44) 50 | 41, 264 x 1032 (1.48) 52 | 40,
        // 128 x 4096 (2) 79 | 60, 128 experts' 304 x 304 (1.78) 29 | 20, 1000 experts' 48 x 72 (4) 26 | 11; below: 520 x 1032 (1.33) 69 | 66, 776 x 1032 (1.27) 97 | 97,
        // 32 experts' 1032 x 2056 (1.18) 160 | 173
        const double n = padded(g.M, g.N, 256, 256) < 1.3 * padded(g.M, g.N, 128, 128) ? expected_tiles(g, 256, 256) : 0.0;
        return tiles(n >= 2.0 * cus || (n >= 1.25 * cus && (double)g.K / g.E >= 1024.0) || n >= (double)g.E * cus ? TILE_256 : TILE_128);
    }
    // 256 x 256: groups that fill three quarters of one, and where 128 x 128 ones, two a compute unit, need a second round; 16 bits, 4 experts (2048,2048): rounds
    // of the smaller ones 1.04: 39 | 45 (gradient of A) and 55 (forward), 1.28: 41 | 47 and 55, 0.79: 39 | 30; 8 experts (2304,768) 1.15: 44 | 61, 0.96: 21 | 18.5
    const bool large = rows >= 192.0 && expected_tiles(g, 128, 128) >= 2.0 * cus;
    if (g.elem == ELEM_E4M3) {
        // few rows, by streaming B: where 64 x 32 tiles are at most some 2.6 a compute unit: 128 rows of (8192,8192) 49 | 64 (128 x 128 tiles), 256 rows
        // of (4096,4096) 27 | 34, 256 of (8192,8192) 95 | 64; groups of up to 20 rows: 16 rows each of 16 experts (4096,2048) 41 | 45, 32 each 56 | 46
        if (allow_few_rows && ((double)g.M * g.N <= 5400.0 * cus || (g.offsets && rows <= 20.0))) {
            const int fm = rows <= 16.0 ? 1 : 2;
            // the widest tiles that give every compute unit one: (16,8192,8192) 32 columns 13.6, 16 columns 17.1; (16,2048,8192) 13.1, 9.6;
            // (64,8192,8192) 64 columns 25.8, 32 columns 32; (64,4096,4096) 14.8, 10.4
            const int nb = fm == 2 && rows > 32.0 && expected_tiles(g, 32, 64) >= cus ? 4 : expected_tiles(g, 16 * fm, 32) >= cus ? 2 : 1;
            return few_rows(fm, nb);
        }
        // 16-bit results of large products, unless the caller asks for exact ones: the e4m3 matrix instructions (see ops_tile_e4m3.hip), 8192^3 441 us against 920
        // widened, (1593,7232,4552) 65 against 134, 16384 rows of 16 experts (4096,2048) 162 against 299.
        // Below 2^22 results the widened form costs little or nothing more.  256 x 256 | 128 x 128: groups of 1024 rows
        // (4096,2048) 166 | 189, (8192,8192,1024) 87 | 104; rounds of workgroups that are a quarter empty (4730,6880,272) 45 | 32, (7266,4800,1232) 75 | 70; groups
        // of 128 rows (2048,2048) 173 | 158 (widened 251); one round that is half full (4000,2304,6000) 71 | 88
        if (!g.exact && g.c_type != ELEM_F32 && (int64_t)g.M * g.N >= (1 << 22)) {
            const double rounds = expected_tiles(g, 256, 256) / cus;
            return tiles(large && rounds >= (rounds > 1.0 ? 0.75 : 0.5) * ceil(rounds) ? TILE_256 : TILE_128_FAST);
        }
        // groups that leave quarters of 128 rows empty, with | without a branch around those: 24 rows each of 16 experts (4096,2048) 39 | 46, 32 rows
        // 41 | 46, 30 rows of 64 (1408,2048) 58 | 65, 48 rows 56 | 56, 100 rows 67 | 62
        if (g.offsets && rows <= 40.0) return tiles(TILE_128_SHORT);
        // Up to a round of 128 x 128 ones, one a compute unit: those in registers for one | two, 2048^3 22 | 23, (512,8192,8192) 70 | 75.
        if (expected_tiles(g, 128, 128) <= cus) return tiles(TILE_128);
        // 256 x 128 | 128 x 128, two a compute unit: a round of the former (2048,3000,2048) 35 | 36; full rounds and long sums 4000^3 129 | 134; else (3000,3000,2048)
        // 66 | 53, (4096,8192,1024) 90 | 79, (8192,8192,256) 88 | 67, (13785,15296,400) 397 | 328, 16384 rows of 32 experts (2048,512) 66 | 56
        const double rounds = expected_tiles(g, 256, 128) / cus;
        const bool tall = rows >= 192.0 && (rounds <= 1.0 || (g.K > 2048 && rounds >= 0.9 * ceil(rounds)));
        return tiles(tall ? TILE_256x128 : TILE_128_PAIR);
    }
    // forward, groups below 192 rows, 128 x 256 | 128 x 128: (8192 rows, 2048 x 2048, 64 experts) 128 | 140, (64, 4096 x 2048, 16) 42 | 50
    // (but not where N leaves much of the last 256 columns empty: N = 264 of 8 experts of 2048 rows, K = 2048, 56 | 33, 520 of 128 of 64 rows 35 | 21, 1032 of 128 of 16 rows 42 | 39,
    // 72 of 1000 of 2 rows 58 | 30)
    const bool wide = !g.b_kc && padded(1, g.N, 1, 256) < 1.1 * padded(1, g.N, 1, 128) && expected_tiles(g, 128, 256) >= cus;
    return tiles(large ? TILE_256 : wide ? TILE_128x256 : TILE_128);
}

// ... of those that fit a launch: thousands of experts with a wide N are more small tiles than that
Form choose(const OpsGemm& g)
{
    Form f = preferred(g, true);
    if (f.kernel == Form::FEW_ROWS && !fits(g, f)) f = preferred(g, false);
    if (f.kernel == Form::TILES && f.tile != TILE_128_ANY && !fits(g, f)) f = tiles(g.elem == ELEM_E4M3 && f.tile != TILE_128_FAST ? TILE_256x128 : TILE_256);
    return f;
}

int launch(const OpsGemm& g)
{
    const Form f = choose(g);
    if (f.kernel == Form::ANY) return ops_launch_generic(g);
    if (f.kernel == Form::FEW_ROWS) return ops_launch_skinny_e4m3(g, f.fm, f.nb);
    return g.elem == ELEM_E4M3 ? ops_launch_tiles_e4m3(g, f.tile) : g.elem == ELEM_F16 ? ops_launch_tiles_f16(g, f.tile) : ops_launch_tiles_bf16(g, f.tile);
}

const char* name_of(const OpsGemm& g, const Form& f)
{
    if (f.kernel == Form::ANY) return "any_alignment_64x64";
    if (f.kernel == Form::FEW_ROWS)
        return f.fm == 1 ? (f.nb == 1 ? "few_rows_16x16" : "few_rows_16x32") : f.nb == 1 ? "few_rows_32x16" : f.nb == 2 ? "few_rows_32x32" : "few_rows_32x64";
    const bool e4m3 = g.elem == ELEM_E4M3;
    switch (f.tile) {
    case TILE_256: return e4m3 ? "e4m3_256x256" : "256x256";
    case TILE_128_FAST: return "e4m3_128x128";
    case TILE_256x128: return "widened_256x128";
    case TILE_128_PAIR: return "widened_128x128_two";
    case TILE_128_SHORT: return "widened_128x128_short_groups";
    case TILE_128x256: return "128x256";
    case TILE_128_ANY: return "any_alignment_128x128";
    case TILE_128: return e4m3 ? "widened_128x128" : "128x128";
    }
    return nullptr;
}

// The sizes of a call as the kernels have them: M x N x K, the sum over K.
OpsGemm shaped(int64_t product, int64_t T, int64_t N, int64_t K, int64_t E, const int32_t* offsets, int64_t type, int64_t c_type, void* stream)
{
    OpsGemm g = {};
    // grad A: rows of dC by rows of B[e], the sum runs over the N that both have contiguous; grad B: columns of A by columns of dC over the group's rows
    g.M = (int)(product == GEMM_OPS_GRAD_B ? K : T);
    g.N = (int)(product == GEMM_OPS_GRAD_A ? K : N);
    g.K = (int)(product == GEMM_OPS_GRAD_A ? N : product == GEMM_OPS_GRAD_B ? T : K);
    g.E = E < 0 ? 1 : (int)E;
    g.offsets = offsets;
    g.elem = product == GEMM_OPS_E4M3 ? (int)ELEM_E4M3 : (int)type;
    g.c_type = (int)(c_type & ~(int64_t)GEMM_OPS_EXACT);
    g.exact = (c_type & GEMM_OPS_EXACT) != 0;
    g.a_kc = product != GEMM_OPS_GRAD_B;
    g.b_kc = product == GEMM_OPS_E4M3 || product == GEMM_OPS_GRAD_A;
    g.k_ragged = product == GEMM_OPS_GRAD_B;
    g.num_xcd = chip().xcds;
    g.stream = (hipStream_t)stream;
    return g;
}

// The e4m3 products.  E < 0: one product, nothing grouped.
int run_e4m3(int64_t M, int64_t N, int64_t K, int64_t E, const int32_t* offsets,
             const void* A, int64_t lda, const float* sa, int64_t ld_as, const void* B, int64_t ldb, int64_t b_stride,
             const float* sb, int64_t ld_bs, int64_t bs_stride, void* C, int64_t ldc, int64_t c_type, void* stream)
{
    if (bad_size(M) || bad_size(N) || bad_size(K) || E > 65535) return GEMM_F16_ERR_SIZE;
    const int64_t type = c_type & ~(int64_t)GEMM_OPS_EXACT;
    if (!is_16bit(type) && type != GEMM_TYPE_F32) return GEMM_F16_ERR_CONFIG;
    if (M == 0 || N == 0 || E == 0) return GEMM_F16_OK;
    if (bad_pitch(lda, K) || bad_pitch(ldb, K) || bad_pitch(ldc, N) || b_stride < 0 || bs_stride < 0) return GEMM_F16_ERR_PITCH;
    if (K > 0 && (bad_pitch(ld_as, M) || bad_pitch(ld_bs, blocks128(K)))) return GEMM_F16_ERR_PITCH;
    if (!C || (E > 0 && !offsets) || (K > 0 && (!A || !B || !sa || !sb))) return GEMM_F16_ERR_NULL;
    if (unaligned(C, type_size(type)) || unaligned(sa, 4) || unaligned(sb, 4) || unaligned(offsets, 4)) return GEMM_F16_ERR_ALIGN;
    OpsGemm g = shaped(GEMM_OPS_E4M3, M, N, K, E, offsets, 0, c_type, stream);
    g.A = (const char*)A; g.lda = lda; g.B = (const char*)B; g.ldb = ldb; g.b_stride = b_stride;
    g.C = (char*)C; g.ldc = ldc;
    g.sa = sa; g.ld_sa = ld_as; g.sb = sb; g.ld_sb = ld_bs; g.sb_stride = bs_stride;
    return launch(g);
}

// What the 16-bit products grouped by expert share
int check_grouped(int64_t T, int64_t N, int64_t K, int64_t E, int64_t type, int64_t out_type)
{
    if (bad_size(T) || bad_size(N) || bad_size(K) || E < 0 || E > 65535) return GEMM_F16_ERR_SIZE;
    if (!is_16bit(type) || (out_type != type && out_type != GEMM_TYPE_F32)) return GEMM_F16_ERR_CONFIG;
    return GEMM_F16_OK;
}

}  // namespace

extern "C" {

int quantize_e4m3_rows(int64_t M, int64_t N, int64_t type, int64_t act, const void* X, int64_t ldx,
                       void* Q, int64_t ldq, float* scale, int64_t ld_scale, void* stream)
{
    if (bad_size(M) || bad_size(N)) return GEMM_F16_ERR_SIZE;
    if (!is_16bit(type) || (act != GEMM_OPS_ACT_NONE && act != GEMM_OPS_ACT_RELU && act != GEMM_OPS_ACT_SWIGLU)) return GEMM_F16_ERR_CONFIG;
    if (M == 0 || N == 0) return GEMM_F16_OK;
    if (bad_pitch(ldx, act == GEMM_OPS_ACT_SWIGLU ? 2 * N : N) || bad_pitch(ldq, N) || bad_pitch(ld_scale, M)) return GEMM_F16_ERR_PITCH;
    if (!X || !Q || !scale) return GEMM_F16_ERR_NULL;
    if (unaligned(X, 2) || unaligned(scale, 4)) return GEMM_F16_ERR_ALIGN;
    return ops_launch_quant_rows((int)type, {(int)M, (int)N, (int)act, X, ldx, (uint8_t*)Q, ldq, scale, ld_scale}, (hipStream_t)stream);
}

int quantize_e4m3_blocks(int64_t M, int64_t N, int64_t type, const void* X, int64_t ldx,
                         void* Q, int64_t ldq, float* scale, int64_t ld_scale, void* stream)
{
    if (bad_size(M) || bad_size(N)) return GEMM_F16_ERR_SIZE;
    if (!is_16bit(type)) return GEMM_F16_ERR_CONFIG;
    if (M == 0 || N == 0) return GEMM_F16_OK;
    if (bad_pitch(ldx, N) || bad_pitch(ldq, N) || bad_pitch(ld_scale, blocks128(N))) return GEMM_F16_ERR_PITCH;
    if (!X || !Q || !scale) return GEMM_F16_ERR_NULL;
    if (unaligned(X, 2) || unaligned(scale, 4)) return GEMM_F16_ERR_ALIGN;
    return ops_launch_quant_blocks((int)type, {(int)M, (int)N, GEMM_OPS_ACT_NONE, X, ldx, (uint8_t*)Q, ldq, scale, ld_scale}, (hipStream_t)stream);
}

int rms_norm(int64_t M, int64_t N, int64_t type, const void* X, int64_t ldx, const void* R, int64_t ldr,
             const void* gamma, double eps, void* H, int64_t ldh, void* Y, int64_t ldy,
             void* Q, int64_t ldq, float* scale, int64_t ld_scale, float* rstd, void* stream)
{
    if (bad_size(M) || bad_size(N)) return GEMM_F16_ERR_SIZE;
    if (!is_16bit(type) || !(eps >= 0.0)) return GEMM_F16_ERR_CONFIG;
    if (M == 0 || N == 0) return GEMM_F16_OK;
    if (bad_pitch(ldx, N) || (R && bad_pitch(ldr, N)) || (H && bad_pitch(ldh, N)) || (Y && bad_pitch(ldy, N)) ||
        (Q && (bad_pitch(ldq, N) || bad_pitch(ld_scale, M)))) return GEMM_F16_ERR_PITCH;
    if (!X || !gamma || !Q != !scale) return GEMM_F16_ERR_NULL;
    if (unaligned(X, 2) || unaligned(R, 2) || unaligned(gamma, 2) || unaligned(H, 2) || unaligned(Y, 2) || unaligned(scale, 4) || unaligned(rstd, 4)) return GEMM_F16_ERR_ALIGN;
    return ops_launch_norm((int)type, {(int)M, (int)N, X, R, gamma, ldx, ldr, H, Y, ldh, ldy, (uint8_t*)Q, ldq, scale, ld_scale, rstd, (float)eps}, (hipStream_t)stream);
}

int64_t rms_norm_grad_workspace_bytes(int64_t M, int64_t N)
{
    if (M <= 0 || N <= 0 || M > INT32_MAX || N > INT32_MAX) return 0;
    return 4 * N * ops_norm_grad_parts(M, N);
}

int rms_norm_grad(int64_t M, int64_t N, int64_t type, const void* dY, int64_t lddy, const void* H, int64_t ldh,
                  const void* gamma, const float* rstd, const void* dH, int64_t lddh, void* dX, int64_t lddx, float* dgamma,
                  void* workspace, int64_t workspace_bytes, void* stream)
{
    if (bad_size(M) || bad_size(N)) return GEMM_F16_ERR_SIZE;
    if (!is_16bit(type)) return GEMM_F16_ERR_CONFIG;
    if (N == 0 || (M == 0 && !dgamma)) return GEMM_F16_OK;
    if (M > 0) {
        if (bad_pitch(lddy, N) || bad_pitch(ldh, N) || bad_pitch(lddx, N) || (dH && bad_pitch(lddh, N))) return GEMM_F16_ERR_PITCH;
        if (!dY || !H || !gamma || !rstd || !dX || (dgamma && !workspace)) return GEMM_F16_ERR_NULL;
        if (unaligned(dY, 2) || unaligned(H, 2) || unaligned(gamma, 2) || unaligned(dH, 2) || unaligned(dX, 2) || unaligned(rstd, 4) || (dgamma && unaligned(workspace, 16))) return GEMM_F16_ERR_ALIGN;
        if (dgamma && workspace_bytes < rms_norm_grad_workspace_bytes(M, N)) return GEMM_F16_ERR_WORKSPACE;
    }
    if (unaligned(dgamma, 4)) return GEMM_F16_ERR_ALIGN;
    return ops_launch_norm_grad((int)type, {(int)M, (int)N, dY, H, gamma, dH, rstd, lddy, ldh, lddh, dX, lddx, dgamma, (float*)workspace}, (hipStream_t)stream);
}

int gemm_e4m3_block(int64_t M, int64_t N, int64_t K, const void* A, int64_t lda, const float* a_scale, int64_t ld_as,
                    const void* B, int64_t ldb, const float* b_scale, int64_t ld_bs, void* C, int64_t ldc, int64_t c_type, void* stream)
{
    return run_e4m3(M, N, K, -1, nullptr, A, lda, a_scale, ld_as, B, ldb, 0, b_scale, ld_bs, 0, C, ldc, c_type, stream);
}

int gemm_e4m3_block_grouped(int64_t T, int64_t N, int64_t K, int64_t E, const int32_t* offsets, const void* A, int64_t lda, const float* a_scale, int64_t ld_as,
                            const void* B, int64_t ldb, int64_t b_stride, const float* b_scale, int64_t ld_bs, int64_t bs_stride,
                            void* C, int64_t ldc, int64_t c_type, void* stream)
{
    if (E < 0) return GEMM_F16_ERR_SIZE;
    return run_e4m3(T, N, K, E, offsets, A, lda, a_scale, ld_as, B, ldb, b_stride, b_scale, ld_bs, bs_stride, C, ldc, c_type, stream);
}

int gemm_grouped(int64_t T, int64_t N, int64_t K, int64_t E, const int32_t* offsets, int64_t type, const void* A, int64_t lda,
                 const void* B, int64_t ldb, int64_t b_stride, void* C, int64_t ldc, int64_t c_type, void* stream)
{
    const int rc = check_grouped(T, N, K, E, type, c_type);
    if (rc != GEMM_F16_OK) return rc;
    if (T == 0 || N == 0 || E == 0) return GEMM_F16_OK;
    if (bad_pitch(lda, K) || bad_pitch(ldb, N) || bad_pitch(ldc, N) || b_stride < 0) return GEMM_F16_ERR_PITCH;
    if (!C || !offsets || (K > 0 && (!A || !B))) return GEMM_F16_ERR_NULL;
    if (unaligned(A, 2) || unaligned(B, 2) || unaligned(C, type_size(c_type)) || unaligned(offsets, 4)) return GEMM_F16_ERR_ALIGN;
    OpsGemm g = shaped(GEMM_OPS_FORWARD, T, N, K, E, offsets, type, c_type, stream);
    g.A = (const char*)A; g.lda = lda; g.B = (const char*)B; g.ldb = ldb; g.b_stride = b_stride; g.C = (char*)C; g.ldc = ldc;
    return launch(g);
}

int gemm_grouped_grad_a(int64_t T, int64_t N, int64_t K, int64_t E, const int32_t* offsets, int64_t type, const void* dC, int64_t lddc,
                        const void* B, int64_t ldb, int64_t b_stride, void* dA, int64_t ldda, int64_t a_type, void* stream)
{
    const int rc = check_grouped(T, N, K, E, type, a_type);
    if (rc != GEMM_F16_OK) return rc;
    if (T == 0 || K == 0 || E == 0) return GEMM_F16_OK;
    if (bad_pitch(lddc, N) || bad_pitch(ldb, N) || bad_pitch(ldda, K) || b_stride < 0) return GEMM_F16_ERR_PITCH;
    if (!dA || !offsets || (N > 0 && (!dC || !B))) return GEMM_F16_ERR_NULL;
    if (unaligned(dC, 2) || unaligned(B, 2) || unaligned(dA, type_size(a_type)) || unaligned(offsets, 4)) return GEMM_F16_ERR_ALIGN;
    OpsGemm g = shaped(GEMM_OPS_GRAD_A, T, N, K, E, offsets, type, a_type, stream);
    g.A = (const char*)dC; g.lda = lddc; g.B = (const char*)B; g.ldb = ldb; g.b_stride = b_stride; g.C = (char*)dA; g.ldc = ldda;
    return launch(g);
}

int gemm_grouped_grad_b(int64_t T, int64_t N, int64_t K, int64_t E, const int32_t* offsets, int64_t type, const void* A, int64_t lda,
                        const void* dC, int64_t lddc, void* dB, int64_t lddb, int64_t db_stride, int64_t b_type, void* stream)
{
    const int rc = check_grouped(T, N, K, E, type, b_type);
    if (rc != GEMM_F16_OK) return rc;
    if (N == 0 || K == 0 || E == 0) return GEMM_F16_OK;
    if (bad_pitch(lda, K) || bad_pitch(lddc, N) || bad_pitch(lddb, N) || (E > 1 && db_stride < (K - 1) * lddb + N)) return GEMM_F16_ERR_PITCH;
    if (!dB || !offsets || (T > 0 && (!A || !dC))) return GEMM_F16_ERR_NULL;
    if (unaligned(A, 2) || unaligned(dC, 2) || unaligned(dB, type_size(b_type)) || unaligned(offsets, 4)) return GEMM_F16_ERR_ALIGN;
    OpsGemm g = shaped(GEMM_OPS_GRAD_B, T, N, K, E, offsets, type, b_type, stream);
    g.A = (const char*)A; g.lda = lda; g.B = (const char*)dC; g.ldb = lddc; g.C = (char*)dB; g.ldc = lddb; g.c_stride = db_stride;
    return launch(g);
}

const char* gemm_ops_form(int64_t product, int64_t T, int64_t N, int64_t K, int64_t E, int64_t lda, int64_t ldb, int64_t c_type)
{
    if (product < GEMM_OPS_E4M3 || product > GEMM_OPS_GRAD_B || bad_size(T) || bad_size(N) || bad_size(K) || E > 65535 || (E < 0 && product != GEMM_OPS_E4M3)) return nullptr;
    const int64_t result = product == GEMM_OPS_E4M3 ? c_type & ~(int64_t)GEMM_OPS_EXACT : c_type;
    if (E == 0 || (!is_16bit(result) && result != GEMM_TYPE_F32)) return nullptr;
    static const int32_t some_offsets = 0;
    OpsGemm g = shaped(product, T, N, K, E, E < 0 ? nullptr : &some_offsets, GEMM_TYPE_F16, c_type, nullptr);
    if (g.M == 0 || g.N == 0) return nullptr;
    g.lda = lda; g.ldb = ldb;
    const Form f = choose(g);
    return fits(g, f) ? name_of(g, f) : nullptr;
}

}  // extern "C"
