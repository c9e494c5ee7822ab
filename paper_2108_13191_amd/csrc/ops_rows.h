// Rows of 16-bit elements in registers, 8 at a time: loads, stores and sums of the operators that go over whole rows (norms, quantisation,
// rows moved to experts and back).
#pragma once
#include "ops_device.h"

namespace ops_dev {

// ---- 8 elements of a row of which `left` are there, zeros behind its end ----------------------------------------------------
template <typename T>
__device__ __forceinline__ void load8(const T* p, int left, float (&v)[8])
{
    if (left >= 8) {
        const typename Vec8<T>::type x = *(const typename Vec8<T>::type*)p;
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = (float)x[i];
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = i < left ? (float)p[i] : 0.0f;
    }
}
template <typename T>
__device__ __forceinline__ void store8(T* p, int left, const float (&v)[8])
{
    if (left >= 8) {
        typename Vec8<T>::type x;
#pragma unroll
        for (int i = 0; i < 8; i++) x[i] = (T)v[i];
        // past the L2s, which rows on their way through would fill: norm of (16384,4096) 87.7 -> 86.0 us, of (20000,768) 24.7 -> 20.0
        __builtin_nontemporal_store(x, (typename Vec8<T>::type*)p);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) if (i < left) p[i] = (T)v[i];
    }
}
// (left above 0, and 8 or more where rows are WHOLE)
template <bool WHOLE, typename T> __device__ __forceinline__ void store8_of(T* p, int left, const float (&v)[8]) { store8(p, WHOLE ? 8 : left, v); }
typedef uintx2 uintx2_any __attribute__((aligned(1)));
template <bool WHOLE = false>
__device__ __forceinline__ void store_bytes(uint8_t* p, int left, uintx2 q)
{
    if (WHOLE || left >= 8) {
        *(uintx2_any*)p = q;
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) if (i < left) p[i] = (uint8_t)((i < 4 ? q[0] : q[1]) >> (8 * (i & 3)));
    }
}
// the same 8 elements as they are stored (4 registers), to be widened later
template <typename T> using Raw8 = T __attribute__((ext_vector_type(8)));
template <typename T>
__device__ __forceinline__ Raw8<T> load8_raw(const T* p, int left)
{
    if (left >= 8) return *(const typename Vec8<T>::type*)p;
    Raw8<T> v;
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = i < left ? p[i] : (T)0.0f;
    return v;
}
// n elements towards the first, zeros behind (8 and more: all zeros)
template <typename T>
__device__ __forceinline__ Raw8<T> moved_down(Raw8<T> v, int n)
{
    if constexpr (sizeof(T) == 2) {
        uintx4 w = __builtin_bit_cast(uintx4, v);
        const uint32_t h = (n & 1) ? 16u : 0u;
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = (uint32_t)((((uint64_t)(i < 3 ? w[i < 3 ? i + 1 : 3] : 0u) << 32) | w[i]) >> h);
        if (n & 2) w = uintx4{w[1], w[2], w[3], 0u};
        if (n & 4) w = uintx4{w[2], w[3], 0u, 0u};
        v = __builtin_bit_cast(Raw8<T>, w);
    } else {
#pragma unroll
        for (int b = 1; b < 8; b <<= 1)
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = (n & b) ? (i + b < 8 ? v[i + b < 8 ? i + b : 7] : (T)0.0f) : v[i];
    }
    return v;
}
// Elements c .. c + 7 of a row of N, zeros behind its end, in two steps: load8_of asks for them, and what would leave the row as its last 8 elements instead; settled
// moves those to their place once they are used.  So no loaded value is touched, and no branch parted, before all of a row's loads have been asked for:
// lanes behind the end that had a way of their own made their wavefront wait for each load by itself (gradients of (8191,4000) 81 us, of (8191,4096) 62).
// WHOLE: rows are whole chunks of 8, so that one is there or not: a third of the code, whose fetch is most of a small call's time (norm of 16 rows of 8192 4.5 us with all of it)
template <bool WHOLE, typename T>
__device__ __forceinline__ Raw8<T> load8_of(const T* row, int64_t c, int64_t N)
{
    if (!WHOLE && N < 8) return load8_raw(row, (int)N);
    return *(const typename Vec8<T>::type*)(row + min(c, N - 8));
}
template <typename T, bool WHOLE>
__device__ __forceinline__ Raw8<T> settled(Raw8<T> v, int64_t c, int64_t N)
{
    const int n = WHOLE ? (c < N ? 0 : 8) : (int)min(c - (N < 8 ? 0 : min(c, N - 8)), (int64_t)8);
    if (!WHOLE && (N & 7)) v = moved_down<T>(v, n);
    if constexpr (sizeof(T) == 2) {
        const uint32_t keep = n >= 8 ? 0u : ~0u;
        uintx4 w = __builtin_bit_cast(uintx4, v);
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] &= keep;
        return __builtin_bit_cast(Raw8<T>, w);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = n >= 8 ? (T)0.0f : v[i];
        return v;
    }
}
template <typename T> __device__ __forceinline__ float rounded(float x) { return (float)(T)x; }

// Sum over the W wavefronts that share a row.  `lds`: a float for each wavefront of the workgroup.
template <int W>
__device__ __forceinline__ float sum_row(float x, float* lds)
{
    x = sum64(x);
    if constexpr (W > 1) {
        const int wave = threadIdx.x >> 6;
        __syncthreads();                                 // the values of the sum before have been read
        if ((threadIdx.x & 63) == 0) lds[wave] = x;
        __syncthreads();
        x = 0.0f;
        const int first = wave / W * W;
#pragma unroll
        for (int i = 0; i < W; i++) x += lds[first + i];
    }
    return x;
}

// g / (1 + exp(-g)).  exp(-g) = 2^a 2^r: a = -g / ln 2 as f32 rounds it, r what that leaves (exact product by an fma, and the constant's own next bits),
// 2^r = 1 + r ln 2 to f32's last bit, as r is below 1e-5 where 2^a is finite.  Without r the error would grow with g, to 4e-6 at 60.  The exponential and reciprocal
// instructions are good to one unit in the last place each; a denormal reciprocal, of gates below -87.3, is 0.  Beyond +-1024, where the
// result is 0 or g itself, the exponent is that of +-1024, so that neither a nor r overflows.
__device__ __forceinline__ float silu(float g)
{
    constexpr float LOG2E = 1.4426950408889634f, LOG2E_REST = (float)(1.4426950408889634 - (double)LOG2E), LN2 = 0.6931471805599453f;
    const float x = __builtin_amdgcn_fmed3f(-g, -1024.0f, 1024.0f), a = x * LOG2E;
    const float r = __builtin_fmaf(x, LOG2E_REST, __builtin_fmaf(x, LOG2E, -a));
    return g * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(a) * __builtin_fmaf(r, LN2, 1.0f));
}
// Rows need nothing of each other: more of them than the grid of one launch has threads for (a row takes up to 1024) go in several launches.
constexpr int64_t LAUNCH_ROWS = 1 << 21;

}  // namespace ops_dev
