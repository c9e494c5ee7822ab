// The products of include/gemm_ops.h and include/gemm_layer.h for operands of any alignment: 64 x 64 tiles, four wavefronts of 32 x 32, every element
// loaded by itself (64 consecutive ones by a wavefront), brought to f16 or bf16 (e4m3 values are exact in f16) on the way into
// LDS, and multiplied with 16 x 16 x 32 MFMAs (8-bit integers stay what they are).  e4m3: the sum over a block of 128 is formed by itself and added with its scales.
//
// Bound by the element loads (32 a lane and k step of 64 against 8 MFMAs): 40 TFLOP/s.  Takes what the other forms do not: e4m3 operands that are not 16-byte
// aligned, 16-bit ones with less than 8 elements a row, pitches beyond 2^22 elements.
#include "ops_device.h"
#include "../../include/gemm_ops.h"

namespace {

using namespace ops_dev;

constexpr int GT = 64, GK = 64, GP = GK + 8;      // tile, k step, LDS row pitch (elements): rows 16-byte aligned

__device__ __forceinline__ half_t stage_value(uint8_t v) { return (half_t)__builtin_amdgcn_cvt_f32_fp8((int)v, 0); }
__device__ __forceinline__ int8_t stage_value(int8_t v) { return v; }
__device__ __forceinline__ half_t stage_value(half_t v) { return v; }
__device__ __forceinline__ bf16_t stage_value(bf16_t v) { return v; }

__device__ __forceinline__ floatx4 mfma16(half8 a, half8 b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ floatx4 mfma16(bf16x8 a, bf16x8 b, floatx4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
typedef int8_t int8x8 __attribute__((ext_vector_type(8)));
// (half of the k of the instruction: its other half is zeros)
__device__ __forceinline__ floatx4 mfma16(int8x8 a, int8x8 b, floatx4 c)
{
    const uintx2 x = __builtin_bit_cast(uintx2, a), y = __builtin_bit_cast(uintx2, b);
    return mfma_i8(uintx4{x[0], x[1], 0u, 0u}, uintx4{y[0], y[1], 0u, 0u}, c);
}

template <int ELEM> struct Staged { typedef typename Elem<ELEM>::type type; typedef bf16x8 vec; };
template <> struct Staged<ELEM_F16> { typedef half_t type; typedef half8 vec; };
template <> struct Staged<ELEM_E4M3> { typedef half_t type; typedef half8 vec; };
template <> struct Staged<ELEM_I8> { typedef int8_t type; typedef int8x8 vec; };

// rows r0 .. of an operand (rows at or behind `rows` are zeros), k from k0 on (zeros at or behind `kend`) into LDS as [row][k]
template <int ELEM, bool KC>
__device__ __forceinline__ void stage_tile(typename Staged<ELEM>::type* lds, const char* src, int64_t ld, int64_t r0, int64_t rows, int64_t k0, int64_t kend)
{
    typedef typename Elem<ELEM>::type T;
    typedef typename Staged<ELEM>::type S;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const T* const p = (const T*)src;
    T v[GT / 4];
#pragma unroll
    for (int i = 0; i < GT / 4; i++) {
        const int row = KC ? wave + 4 * i : lane, k = KC ? lane : wave + 4 * i;
        v[i] = T(0);
        if (r0 + row < rows && k0 + k < kend) v[i] = KC ? p[(r0 + row) * ld + k0 + k] : p[(k0 + k) * ld + r0 + row];
    }
#pragma unroll
    for (int i = 0; i < GT / 4; i++) {
        const int row = KC ? wave + 4 * i : lane, k = KC ? lane : wave + 4 * i;
        lds[row * GP + k] = (S)stage_value(v[i]);
    }
}

template <int ELEM, bool AKC, bool BKC, typename CT>
__global__ __launch_bounds__(256) void ops_generic_kernel(const OpsGemm g)
{
    typedef typename Staged<ELEM>::type S;
    typedef typename Staged<ELEM>::vec V;
    __shared__ __attribute__((aligned(16))) S la[GT * GP], lb[GT * GP];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;

    // ---- the tile -----------------------------------------------------------------------------
    const int tiles_n = (int)(((int64_t)g.N + GT - 1) / GT), tile_m = (int)(blockIdx.x / (unsigned)tiles_n);
    const int64_t n0 = (int64_t)(blockIdx.x % (unsigned)tiles_n) * GT;
    int64_t row0, row_end;
    int e = 0, k_first = 0, k_end = g.K;
    if (g.k_ragged) {
        e = blockIdx.y;
        group_rows(g.offsets, e, g.K, k_first, k_end);
        row0 = (int64_t)tile_m * GT; row_end = g.M;
    } else if (g.offsets) {
        // the tile_m-th tile of all groups in order
        int want = tile_m, e0 = 0;
        GroupScan s = scan_groups<GT>(g.offsets, 0, g.E, g.M);
        while (want >= s.total()) {
            want -= s.total();
            e0 += 64;
            if (e0 >= g.E) return;
            s = scan_groups<GT>(g.offsets, e0, g.E, g.M);
        }
        const int at = s.group_of(want);
        e = e0 + at; row0 = s.lo_of(at) + (int64_t)(want - s.before(at)) * GT; row_end = s.hi_of(at);
    } else {
        row0 = (int64_t)tile_m * GT; row_end = g.M;
    }
    const char* const B = g.B + (int64_t)e * g.b_stride * Elem<ELEM>::size;
    const float* const sb = g.sb + (int64_t)e * g.sb_stride + (int64_t)(n0 / 128) * g.ld_sb;

    floatx4 acc[2][2] = {}, part[2][2] = {};
    const int wm = (wave >> 1) * 32, wn = (wave & 1) * 32, l16 = lane & 15, kq = lane >> 4;
    for (int64_t k0 = k_first; k0 < k_end; k0 += GK) {
        __syncthreads();
        stage_tile<ELEM, AKC>(la, g.A, g.lda, row0, row_end, k0, k_end);
        stage_tile<ELEM, BKC>(lb, B, g.ldb, n0, g.N, k0, k_end);
        __syncthreads();
#pragma unroll
        for (int s = 0; s < 2; s++) {
            V a[2], b[2];
#pragma unroll
            for (int i = 0; i < 2; i++) {
                a[i] = *(const V*)&la[(wm + 16 * i + l16) * GP + 32 * s + 8 * kq];
                b[i] = *(const V*)&lb[(wn + 16 * i + l16) * GP + 32 * s + 8 * kq];
            }
#pragma unroll
            for (int i = 0; i < 2; i++)
#pragma unroll
                for (int j = 0; j < 2; j++) part[i][j] = mfma16(b[j], a[i], part[i][j]);       // B first: a lane gets 4 columns of a row
        }
        if constexpr (ELEM == ELEM_E4M3) {
            if ((k0 + GK) % 128 == 0 || k0 + GK >= k_end) {
                const int64_t kb = k0 / 128;
#pragma unroll
                for (int i = 0; i < 2; i++) {
                    const int64_t row = row0 + wm + 16 * i + l16;
                    const float scale = row < row_end ? g.sa[kb * g.ld_sa + row] * sb[kb] : 0.0f;
#pragma unroll
                    for (int j = 0; j < 2; j++) {
                        acc[i][j] += part[i][j] * scale;
                        part[i][j] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
                    }
                }
            }
        }
    }
    CT* const C = (CT*)g.C + (int64_t)e * g.c_stride;
#pragma unroll
    for (int i = 0; i < 2; i++) {
        const int64_t row = row0 + wm + 16 * i + l16;
        if (row >= row_end) continue;
#pragma unroll
        for (int j = 0; j < 2; j++)
#pragma unroll
            for (int r = 0; r < 4; r++) {
                const int64_t col = n0 + wn + 16 * j + 4 * kq + r;
                if (col >= g.N) continue;
                if constexpr (ELEM == ELEM_I8) C[row * g.ldc + col] = (CT)scaled_column(scaled_sum(part[i][j][r], g.sa[row]), g.sb[(int64_t)e * g.sb_stride + col]);
                else C[row * g.ldc + col] = (CT)(ELEM == ELEM_E4M3 ? acc[i][j][r] : part[i][j][r]);
            }
    }
}

template <int ELEM, bool AKC, bool BKC>
int launch(const OpsGemm& g)
{
    const int64_t tiles = tile_grid(g, GT, GT);                 // k_ragged: a group's in x, the groups in y
    if (tiles < 0 || !fits_a_launch(tiles, 256)) return GEMM_F16_ERR_SIZE;
    const dim3 grid((unsigned)(g.k_ragged ? tiles / g.E : tiles), g.k_ragged ? (unsigned)g.E : 1u);
    switch (g.c_type) {
    case ELEM_F32: hipLaunchKernelGGL((ops_generic_kernel<ELEM, AKC, BKC, float>), grid, dim3(256), 0, g.stream, g); break;
    case ELEM_F16: hipLaunchKernelGGL((ops_generic_kernel<ELEM, AKC, BKC, half_t>), grid, dim3(256), 0, g.stream, g); break;
    default: hipLaunchKernelGGL((ops_generic_kernel<ELEM, AKC, BKC, bf16_t>), grid, dim3(256), 0, g.stream, g); break;
    }
    return hipGetLastError() == hipSuccess ? GEMM_F16_OK : GEMM_F16_ERR_LAUNCH;
}

template <int ELEM>
int launch_layout(const OpsGemm& g)
{
    if (g.a_kc) return g.b_kc ? launch<ELEM, true, true>(g) : launch<ELEM, true, false>(g);
    return launch<ELEM, false, false>(g);
}

}  // namespace

int ops_launch_generic(const OpsGemm& g)
{
    if (g.elem == ELEM_E4M3) return launch<ELEM_E4M3, true, true>(g);
    if (g.elem == ELEM_I8) return launch<ELEM_I8, true, true>(g);
    return g.elem == ELEM_F16 ? launch_layout<ELEM_F16>(g) : launch_layout<ELEM_BF16>(g);
}
