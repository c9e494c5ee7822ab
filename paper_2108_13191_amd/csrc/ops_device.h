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

// The scale of a block from the largest magnitude in it (bits), and its reciprocal: NaN where the block holds a NaN or an infinity.
constexpr float E4M3_MAX = 448.0f, SCALE_FLOOR = 0x1p-96f;
struct BlockScale {
    float scale, inverse;
    // y / scale: the product with the reciprocal, corrected by what it leaves of y (exact in one fma).  16-bit values and their scales make ties of e4m3
    // often: the product alone rounds 1 of 1000 elements of a normal bf16 matrix the other way, 1 of 10000 in f16.  (Zeros keep their sign.)
    __device__ __forceinline__ float quotient(float y) const
    {
        const float t = y * inverse;
        return __builtin_fmaf(-__builtin_fmaf(t, scale, -y), inverse, t);
    }
};
__device__ __forceinline__ BlockScale block_scale(uint32_t bits)
{
    if (bits >= 0x7f800000u) { const float nan = __builtin_nanf(""); return {nan, nan}; }
    const float scale = fmaxf(__builtin_bit_cast(float, bits), SCALE_FLOOR) / E4M3_MAX;
    return {scale, 1.0f / scale};
}
// 8 values to e4m3, to nearest even (none is above 448 but for the last bits of the quotient, which round back)
__device__ __forceinline__ uintx2 to_e4m3(const float (&y)[8], const BlockScale& s)
{
    int lo = 0, hi = 0;
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(s.quotient(y[0]), s.quotient(y[1]), lo, false);
    lo = __builtin_amdgcn_cvt_pk_fp8_f32(s.quotient(y[2]), s.quotient(y[3]), lo, true);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(s.quotient(y[4]), s.quotient(y[5]), hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(s.quotient(y[6]), s.quotient(y[7]), hi, true);
    return uintx2{(uint32_t)lo, (uint32_t)hi};
}

// Rows of group e, within 0 .. limit whatever the offsets hold.
__device__ __forceinline__ void group_rows(const int32_t* offsets, int e, int limit, int& lo, int& hi)
{
    lo = min(max(offsets[e], 0), limit);
    hi = min(max(offsets[e + 1], lo), limit);
}

// 64 groups at a time, a lane of a wavefront each: their rows lo .. hi, the tiles of BM rows that they need, and those of all
// lanes up to and with this one.
struct GroupScan {
    int lo, hi, n, incl;
    __device__ int total() const { return __builtin_amdgcn_readlane(incl, 63); }
    __device__ int group_of(int tile) const { return __builtin_ctzll(__ballot(incl > tile) | (1ull << 63)); }    // whose tile it is
    __device__ int tiles_of(int at) const { return max(1, __builtin_amdgcn_readlane(n, at)); }
    __device__ int before(int at) const { return __builtin_amdgcn_readlane(incl, at) - __builtin_amdgcn_readlane(n, at); }
    __device__ int lo_of(int at) const { return __builtin_amdgcn_readlane(lo, at); }
    __device__ int hi_of(int at) const { return __builtin_amdgcn_readlane(hi, at); }
};
template <int BM>
__device__ __forceinline__ GroupScan scan_groups(const int32_t* offsets, int e0, int E, int limit)
{
    const int lane = threadIdx.x & 63;
    GroupScan s = {0, 0, 0, 0};
    if (e0 + lane < E) group_rows(offsets, e0 + lane, limit, s.lo, s.hi);
    s.incl = s.n = (int)(((uint32_t)(s.hi - s.lo) + BM - 1) / BM);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int v = __shfl_up(s.incl, d);
        if (lane >= d) s.incl += v;
    }
    return s;
}
// The group of the `rank`-th most rows (of equal ones the first first), of up to 64 groups.
__device__ __forceinline__ int group_by_size(const int32_t* offsets, int E, int limit, int rank)
{
    const int lane = threadIdx.x & 63;
    int lo = 0, hi = -1, before = 0;
    if (lane < E) group_rows(offsets, lane, limit, lo, hi);
    const int rows = hi - lo;                              // -1 where there is no group
    for (int i = 0; i < E; i++) {
        const int other = __builtin_amdgcn_readlane(rows, i);
        before += other > rows || (other == rows && i < lane);
    }
    return __builtin_ctzll(__ballot(lane < E && before == rank));
}
}  // namespace ops_dev
