// Device-side helpers of the operators of include/gemm_ops.h: element types, reductions over lanes, and where the tiles of
// a product grouped by expert lie.
#pragma once
#include "gemm_device.h"
#include "ops_common.h"

namespace ops_dev {

template <int ELEM> struct Elem;
template <> struct Elem<ELEM_F16> { typedef half_t type; static constexpr int size = 2; };
template <> struct Elem<ELEM_BF16> { typedef bf16_t type; static constexpr int size = 2; };
template <> struct Elem<ELEM_F32> { typedef float type; static constexpr int size = 4; };
template <> struct Elem<ELEM_E4M3> { typedef uint8_t type; static constexpr int size = 1; };

// 8 elements of 16 bits at element alignment (one 16-byte access)
template <typename T> struct Vec8 { typedef T type __attribute__((ext_vector_type(8), aligned(2))); };

// magnitude as an integer: ordered as the magnitudes are, infinity above every number and NaN above infinity
__device__ __forceinline__ uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }

template <int CTRL> __device__ __forceinline__ uint32_t dpp_u32(uint32_t x) { return (uint32_t)__builtin_amdgcn_mov_dpp((int)x, CTRL, 0xf, 0xf, true); }
// the largest of 16 neighbouring lanes, in all of them (rotations within a row of 16 lanes)
__device__ __forceinline__ uint32_t max16(uint32_t x)
{
    x = max(x, dpp_u32<0x128>(x));
    x = max(x, dpp_u32<0x124>(x));
    x = max(x, dpp_u32<0x122>(x));
    return max(x, dpp_u32<0x121>(x));
}
// the sum over the 64 lanes of a wavefront, in all of them, always in the same order
__device__ __forceinline__ float sum64(float x)
{
    x += __builtin_bit_cast(float, dpp_u32<0x128>(__builtin_bit_cast(uint32_t, x)));
    x += __builtin_bit_cast(float, dpp_u32<0x124>(__builtin_bit_cast(uint32_t, x)));
    x += __builtin_bit_cast(float, dpp_u32<0x122>(__builtin_bit_cast(uint32_t, x)));
    x += __builtin_bit_cast(float, dpp_u32<0x121>(__builtin_bit_cast(uint32_t, x)));
    x += __shfl_xor(x, 16);
    x += __shfl_xor(x, 32);
    return x;
}

// The scale of a block from the largest magnitude in it (bits), and what its values are multiplied by: NaN where the block
// holds a NaN or an infinity.
constexpr float E4M3_MAX = 448.0f, SCALE_FLOOR = 0x1p-96f;
struct BlockScale { float scale, inverse; };
__device__ __forceinline__ BlockScale block_scale(uint32_t bits)
{
    if (bits >= 0x7f800000u) { const float nan = __builtin_nanf(""); return {nan, nan}; }
    const float m = fmaxf(__builtin_bit_cast(float, bits), SCALE_FLOOR);
    return {m / E4M3_MAX, E4M3_MAX / m};
}
// 8 values to e4m3, to nearest even (none is above 448 but for the last bit of the product, which rounds back)
__device__ __forceinline__ uintx2 to_e4m3(const float (&y)[8], float inverse)
{
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0] * inverse, y[1] * inverse, lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2] * inverse, y[3] * inverse, lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4] * inverse, y[5] * inverse, hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6] * inverse, y[7] * inverse, hi, true);
    return uintx2{(uint32_t)lo, (uint32_t)hi};
}

// Rows of group e, within 0 .. limit whatever the offsets hold.
__device__ __forceinline__ void group_rows(const int32_t* offsets, int e, int limit, int& lo, int& hi)
{
    lo = min(max(offsets[e], 0), limit);
    hi = min(max(offsets[e + 1], lo), limit);
}

// Tiles of `bm` rows over all groups in order: the group, first row and end of tile t, by one wavefront whose lanes look at 64
// groups at a time.  tiles_before(…) at the end of the groups is the number of tiles.
struct GroupTile { int e, row0, end, first_tile, tiles; };      // tiles `first_tile` .. + tiles - 1 are group e's
__device__ __forceinline__ int group_tile_scan(const int32_t* offsets, int E, int limit, int bm, int want, GroupTile& out)
{
    const int lane = threadIdx.x & 63;
    int base = 0;
    for (int e0 = 0; e0 < E; e0 += 64) {
        int lo = 0, hi = 0;
        if (e0 + lane < E) group_rows(offsets, e0 + lane, limit, lo, hi);
        const int n = (int)(((int64_t)(hi - lo) + bm - 1) / bm);
        int incl = n;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int v = __shfl_up(incl, d);
            if (lane >= d) incl += v;
        }
        const int total = __builtin_amdgcn_readlane(incl, 63);
        if (want >= base && want - base < total) {
            const uint64_t above = __ballot(incl > want - base);
            const int l = __builtin_ctzll(above);
            out.e = e0 + l;
            out.tiles = __builtin_amdgcn_readlane(n, l);
            out.first_tile = base + __builtin_amdgcn_readlane(incl, l) - out.tiles;
            out.row0 = __builtin_amdgcn_readlane(lo, l) + (want - out.first_tile) * bm;
            out.end = __builtin_amdgcn_readlane(hi, l);
        }
        base += total;
    }
    return base;
}
// what a launch needs at most: every group may end in a short tile
inline int64_t max_group_tiles(int64_t rows, int64_t E, int64_t bm) { return rows / bm + (E < rows ? E : rows); }

}  // namespace ops_dev
