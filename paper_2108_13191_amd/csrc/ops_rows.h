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
typedef uintx2 uintx2_any __attribute__((aligned(1)));
__device__ __forceinline__ void store_bytes(uint8_t* p, int left, uintx2 q)
{
    if (left >= 8) {
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
