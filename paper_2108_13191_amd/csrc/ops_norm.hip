// RMS norm with the residual's addition, its gradients, and quantisation to e4m3 with a scale for each block of 128
// (include/gemm_ops.h).
//
// All of it is bound by memory: every element is read once and written once, in 16-byte accesses (8 elements of 16 bits a lane), and what a row's
// sum needs again stays in registers.  A block of 128 is 16 neighbouring lanes, so its largest magnitude takes four
// rotations within a row of lanes.  Accesses are at element alignment: rows of any pitch take the same path.
//
// Measured (a copy of 1 GiB: 5.15 TB/s): norm of (16384,4096) bf16 with residual and e4m3 output 86.4 us, 5.5 TB/s; 16 rows of 8192 4.5 us, of which a launch
// and its first load and barrier are all but little; gradients of (8191,4000) 60 us, 4.4 TB/s; SwiGLU (4096,8192) to e4m3 37.2 us, 4.5 TB/s; blocks of
// (8192,8192) 43 us, 4.7 TB/s.
#include "ops_device.h"
#include "../../include/gemm_ops.h"

namespace {

using namespace ops_dev;

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
__device__ __forceinline__ void store_e4m3(uint8_t* p, int left, uintx2 q)
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

// ---- the norm ---------------------------------------------------------------------------------------------------------------
// W wavefronts a row, each lane with P chunks of 8 columns in registers; R rows a workgroup.  LOOP: rows of any length, the chunks
// are gone through twice (the second time h comes from H, or is formed again).
template <typename T, int W, int P, int R, bool LOOP>
__global__ __launch_bounds__(64 * W * R) void rms_norm_kernel(const NormArgs a)
{
    __shared__ float lds[W * R];
    const int lane = threadIdx.x % (64 * W);
    const int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / (64 * W);
    const bool live = row < a.M;
    const T* const x = (const T*)a.X + row * a.ldx;
    const T* const r = a.R ? (const T*)a.R + row * a.ldr : nullptr;
    T* const h = a.H ? (T*)a.H + row * a.ldh : nullptr;

    float v[P][8];
    Raw8<T> gamma[P];                                     // asked for ahead of the sum
    float sum = 0.0f;
    auto form = [&](int64_t c, float (&o)[8]) {
        load8(x + c, (int)(a.N - c), o);
        if (r) {
            float s[8];
            load8(r + c, (int)(a.N - c), s);
#pragma unroll
            for (int i = 0; i < 8; i++) o[i] = rounded<T>(o[i] + s[i]);      // h as it is stored is what is normed
        }
    };
    auto finish = [&](int64_t c, const float (&o)[8], const Raw8<T>& gm, float rstd) {
        const int left = (int)(a.N - c);
        float y[8];
#pragma unroll
        for (int i = 0; i < 8; i++) y[i] = o[i] * rstd * (float)gm[i];
        if (a.Y) store8((T*)a.Y + row * a.ldy + c, left, y);
        if (a.Q) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; i++) m = max(m, magnitude(y[i]));
            const BlockScale s = block_scale(max16(m));
            store_e4m3(a.Q + row * a.ldq + c, left, to_e4m3(y, s));
            if ((lane & 15) == 0) a.scale[c / 128 * a.ld_scale + row] = s.scale;
        }
    };
    if (live) {
        const int passes = LOOP ? (int)(((int64_t)a.N + 512 * W - 1) / (512 * W)) : P;
        for (int p0 = 0; p0 < passes; p0 += P)
#pragma unroll
            for (int p = 0; p < P; p++) {
                const int64_t c = 8 * ((int64_t)lane + 64 * W * (p0 + p));
                if (c < a.N) {
                    form(c, v[p]);
                    if constexpr (!LOOP) gamma[p] = load8_raw((const T*)a.gamma + c, (int)(a.N - c));
                    if (h) store8(h + c, (int)(a.N - c), v[p]);
                } else {
#pragma unroll
                    for (int i = 0; i < 8; i++) { v[p][i] = 0.0f; gamma[p][i] = (T)0.0f; }
                }
#pragma unroll
                for (int i = 0; i < 8; i++) sum += v[p][i] * v[p][i];
            }
    }
    const float rstd = 1.0f / sqrtf(sum_row<W>(sum, lds) / (float)a.N + a.eps);
    if (!live) return;
    if (a.rstd && lane == 0) a.rstd[row] = rstd;
    if (!a.Y && !a.Q) return;
    if constexpr (LOOP) {
        // whole blocks of 16 lanes take part in a block's scale: a chunk behind the row's end is zeros
        for (int64_t c = 8 * (int64_t)lane; c < ((int64_t)a.N + 127) / 128 * 128; c += 512 * W) {
            float o[8] = {};
            if (c < a.N) { if (h) load8((const T*)h + c, (int)(a.N - c), o); else form(c, o); }
            finish(c, o, load8_raw((const T*)a.gamma + c, (int)min((int64_t)8, a.N - c)), rstd);
        }
    } else {
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int c = 8 * (lane + 64 * W * p);
            if (c < (a.N + 127) / 128 * 128) finish(c, v[p], gamma[p], rstd);
        }
    }
}

template <typename T, int W, int P, int R, bool LOOP = false>
int launch_norm(const NormArgs& a, hipStream_t stream)
{
    const unsigned grid = (unsigned)(((int64_t)a.M + R - 1) / R);
    hipLaunchKernelGGL((rms_norm_kernel<T, W, P, R, LOOP>), dim3(grid), dim3(64 * W * R), 0, stream, a);
    return hipGetLastError() == hipSuccess ? GEMM_F16_OK : GEMM_F16_ERR_LAUNCH;
}

template <typename T>
int norm_of_type(const NormArgs& a, hipStream_t stream)
{
    // few rows: as many wavefronts a row as it has chunks of 512 columns, (16,8192) f16 4.5 us against 5.9 with 4
    if (a.M <= 2 * chip().cus && a.N > 2048 && a.N <= 8192) return launch_norm<T, 16, 1, 1>(a, stream);
    if (a.N <= 512) return launch_norm<T, 1, 1, 4>(a, stream);
    if (a.N <= 1024) return launch_norm<T, 1, 2, 4>(a, stream);
    if (a.N <= 2048) return launch_norm<T, 1, 4, 4>(a, stream);
    if (a.N <= 4096) return launch_norm<T, 4, 2, 1>(a, stream);
    if (a.N <= 8192) return launch_norm<T, 4, 4, 1>(a, stream);
    if (a.N <= 16384) return launch_norm<T, 8, 4, 1>(a, stream);
    return launch_norm<T, 16, 1, 1, true>(a, stream);
}

// ---- its gradients ------------------------------------------------------------------------------------------------------------
// dX row by row; the columns' sums of dy xhat stay in registers over all rows of a workgroup, which writes them as one row of the workspace;
// a second kernel adds those.  Every sum has a fixed order.
// 16 wavefronts a workgroup with two chunks a lane: (8191,4000) bf16 with dH 60 us, 4.4 TB/s (rows of 8192 bytes 4.9); one chunk a lane and the next row's loads
// ahead 68, four chunks a lane in 8 wavefronts 64 (against 62 then).
template <typename T, int W, int P, int R>
__global__ __launch_bounds__(64 * W * R) void rms_norm_grad_kernel(const NormGradArgs a)
{
    extern __shared__ float dyn[];                        // 2 * W * R floats (32), then R * 512 * W of sums (32 KB)
    const int lane = threadIdx.x % (64 * W), sub = threadIdx.x / (64 * W), wave = threadIdx.x >> 6;
    float dg[P][8] = {};
    Raw8<T> gamma[P];
#pragma unroll
    for (int p = 0; p < P; p++) gamma[p] = load8_raw((const T*)a.gamma + 8 * (lane + 64 * W * p), a.N - 8 * (lane + 64 * W * p));

    const int64_t step = (int64_t)gridDim.x * R;
    int slot = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * R; row0 < a.M; row0 += step) {      // the same number of trips for the whole workgroup
        const int64_t row = row0 + sub;
        const bool live = row < a.M;
        Raw8<T> dyr[P], hr[P], dhr[P];
        const float rstd = live ? a.rstd[row] : 0.0f;
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int c = 8 * (lane + 64 * W * p), left = live ? a.N - c : 0;      // not above 0: nothing is read
            dyr[p] = load8_raw((const T*)a.dY + row * a.lddy + c, left);
            hr[p] = load8_raw((const T*)a.H + row * a.ldh + c, left);
        }
        if (a.dH) {
#pragma unroll
            for (int p = 0; p < P; p++) dhr[p] = load8_raw((const T*)a.dH + row * a.lddh + 8 * (lane + 64 * W * p), live ? a.N - 8 * (lane + 64 * W * p) : 0);
        }
        float dot = 0.0f;
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float xhat = (float)hr[p][i] * rstd, dy = (float)dyr[p][i];
                dg[p][i] += dy * xhat;
                dot += dy * (float)gamma[p][i] * xhat;
            }
        dot = sum64(dot);
        if constexpr (W > 1) {                            // two sets of partial sums in turn: one barrier a row
            if ((threadIdx.x & 63) == 0) dyn[slot * W * R + wave] = dot;
            __syncthreads();
            dot = 0.0f;
#pragma unroll
            for (int i = 0; i < W; i++) dot += dyn[slot * W * R + wave / W * W + i];
            slot ^= 1;
        }
        const float mean = dot / (float)a.N;
        if (!live) continue;
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int c = 8 * (lane + 64 * W * p);
            if (c >= a.N) continue;
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                o[i] = rstd * ((float)dyr[p][i] * (float)gamma[p][i] - (float)hr[p][i] * rstd * mean);
                if (a.dH) o[i] += (float)dhr[p][i];
            }
            store8((T*)a.dX + row * a.lddx + c, a.N - c, o);
        }
    }
    if (!a.dgamma) return;
    // sums of the workgroup's row slots, in their order, 512 W columns at a time
    float* const sums = dyn + 2 * W * R;
    float* const out = gridDim.x == 1 ? a.dgamma : a.ws + (int64_t)blockIdx.x * a.N;       // one workgroup's sums are the result
#pragma unroll
    for (int p = 0; p < P; p++) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; i += 4) *(floatx4*)&sums[sub * 512 * W + 8 * lane + i] = floatx4{dg[p][i], dg[p][i + 1], dg[p][i + 2], dg[p][i + 3]};
        __syncthreads();
        for (int j = threadIdx.x; j < 512 * W; j += 64 * W * R) {
            const int c = 512 * W * p + j;
            float s = sums[j];
#pragma unroll
            for (int r = 1; r < R; r++) s += sums[r * 512 * W + j];
            if (c < a.N) out[c] = s;
        }
    }
}

// Rows longer than the registers hold: dX in two passes over a row ...
template <typename T>
__global__ __launch_bounds__(1024) void rms_norm_grad_long_kernel(const NormGradArgs a)
{
    __shared__ float lds[16];
    const int64_t row = blockIdx.x;
    const T *const dyr = (const T*)a.dY + row * a.lddy, *const hr = (const T*)a.H + row * a.ldh, *const gr = (const T*)a.gamma;
    const float rstd = a.rstd[row];
    float dy[8], hv[8], gm[8], dot = 0.0f;
    for (int64_t c = 8 * (int64_t)threadIdx.x; c < a.N; c += 8192) {
        load8(dyr + c, (int)(a.N - c), dy); load8(hr + c, (int)(a.N - c), hv); load8(gr + c, (int)(a.N - c), gm);
#pragma unroll
        for (int i = 0; i < 8; i++) dot += dy[i] * gm[i] * (hv[i] * rstd);
    }
    const float mean = sum_row<16>(dot, lds) / (float)a.N;
    for (int64_t c = 8 * (int64_t)threadIdx.x; c < a.N; c += 8192) {
        float up[8] = {}, o[8];
        load8(dyr + c, (int)(a.N - c), dy); load8(hr + c, (int)(a.N - c), hv); load8(gr + c, (int)(a.N - c), gm);
        if (a.dH) load8((const T*)a.dH + row * a.lddh + c, (int)(a.N - c), up);
#pragma unroll
        for (int i = 0; i < 8; i++) o[i] = rstd * (dy[i] * gm[i] - hv[i] * rstd * mean) + up[i];
        store8((T*)a.dX + row * a.lddx + c, (int)(a.N - c), o);
    }
}
// ... and the columns' sums before it (dX may be dY): a workgroup takes 2048 columns and every gridDim.y-th row
template <typename T>
__global__ __launch_bounds__(256) void rms_norm_dgamma_long_kernel(const NormGradArgs a)
{
    const int64_t c = 8 * ((int64_t)blockIdx.x * 256 + threadIdx.x);
    if (c >= a.N) return;
    float dg[8] = {}, dy[8], hv[8];
    for (int64_t row = blockIdx.y; row < a.M; row += gridDim.y) {
        load8((const T*)a.dY + row * a.lddy + c, (int)(a.N - c), dy);
        load8((const T*)a.H + row * a.ldh + c, (int)(a.N - c), hv);
        const float rstd = a.rstd[row];
#pragma unroll
        for (int i = 0; i < 8; i++) dg[i] += dy[i] * (hv[i] * rstd);
    }
    for (int i = 0; i < 8; i++) if (c + i < a.N) a.ws[(int64_t)blockIdx.y * a.N + c + i] = dg[i];
}

// dgamma[j] = sum of `parts` rows of the workspace: 64 columns a workgroup, wavefront w takes rows w, w + 16, ...
__global__ __launch_bounds__(1024) void column_sum_kernel(const float* __restrict__ ws, int parts, int N, float* __restrict__ out)
{
    __shared__ float lds[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
    float s = 0.0f;
    if (c < N) {
#pragma unroll 4
        for (int r = wave; r < parts; r += 16) s += ws[(int64_t)r * N + c];
    }
    lds[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < N) {
#pragma unroll
        for (int w = 1; w < 16; w++) s += lds[w][lane];
        out[c] = s;
    }
}

// rows a workgroup of the gradient takes at a time
inline int grad_rows(int N) { return N <= 1024 ? 16 : N <= 2048 ? 8 : N <= 4096 ? 4 : N <= 8192 ? 2 : 1; }

template <typename T, int W, int P, int R>
int launch_norm_grad(const NormGradArgs& a, int parts, hipStream_t stream)
{
    hipLaunchKernelGGL((rms_norm_grad_kernel<T, W, P, R>), dim3((unsigned)parts), dim3(64 * W * R), (2 * W * R + R * 512 * W) * sizeof(float), stream, a);
    return hipGetLastError() == hipSuccess ? GEMM_F16_OK : GEMM_F16_ERR_LAUNCH;
}
template <typename T>
int norm_grad_of_type(const NormGradArgs& a, hipStream_t stream)
{
    const int parts = ops_norm_grad_parts(a.M, a.N);
    int rc = GEMM_F16_OK;
    if (a.M > 0) {
        if (a.N <= 512) rc = launch_norm_grad<T, 1, 1, 16>(a, parts, stream);
        else if (a.N <= 1024) rc = launch_norm_grad<T, 1, 2, 16>(a, parts, stream);
        else if (a.N <= 2048) rc = launch_norm_grad<T, 2, 2, 8>(a, parts, stream);
        else if (a.N <= 4096) rc = launch_norm_grad<T, 4, 2, 4>(a, parts, stream);
        else if (a.N <= 8192) rc = launch_norm_grad<T, 8, 2, 2>(a, parts, stream);
        else if (a.N <= 16384) rc = launch_norm_grad<T, 16, 2, 1>(a, parts, stream);
        else {
            if (!fits_a_launch(a.M, 1024)) return GEMM_F16_ERR_SIZE;
            if (a.dgamma) hipLaunchKernelGGL(rms_norm_dgamma_long_kernel<T>, dim3((unsigned)(((int64_t)a.N + 2047) / 2048), (unsigned)parts), dim3(256), 0, stream, a);
            hipLaunchKernelGGL(rms_norm_grad_long_kernel<T>, dim3((unsigned)a.M), dim3(1024), 0, stream, a);
            rc = hipGetLastError() == hipSuccess ? GEMM_F16_OK : GEMM_F16_ERR_LAUNCH;
        }
        if (rc != GEMM_F16_OK) return rc;
    }
    if (!a.dgamma || (parts == 1 && a.N <= 16384)) return rc;
    hipLaunchKernelGGL(column_sum_kernel, dim3((unsigned)(((int64_t)a.N + 63) / 64)), dim3(1024), 0, stream, a.ws, parts, a.N, a.dgamma);
    return hipGetLastError() == hipSuccess ? GEMM_F16_OK : GEMM_F16_ERR_LAUNCH;
}

// ---- quantisation in rows: a wavefront takes 2048 columns of a row, 512 at a time, 16 lanes a block of 128; a workgroup's four rows'
// scales are stored together ---------------------------------------------------------------------------------------------------
constexpr int ROW_PASSES = 4;
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
template <typename T, int ACT>
__global__ __launch_bounds__(256) void quantize_rows_kernel(const QuantArgs a)
{
    __shared__ float scales[4 * ROW_PASSES][4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t row = (int64_t)blockIdx.x * 4 + wave, first = (int64_t)blockIdx.y * (512 * ROW_PASSES) + 8 * lane;
    const bool live = row < a.M;
    const T* const x = (const T*)a.X + row * a.ldx + first;
    Raw8<T> v[ROW_PASSES], u[ROW_PASSES];
    auto left_at = [&](int p) { const int64_t n = live ? a.N - (first + 512 * p) : 0; return n > 8 ? 8 : (int)max(n, (int64_t)0); };
#pragma unroll
    for (int p = 0; p < ROW_PASSES; p++) {
        v[p] = load8_raw(x + 512 * p, left_at(p));
        if constexpr (ACT == GEMM_OPS_ACT_SWIGLU) u[p] = load8_raw(x + a.N + 512 * p, left_at(p));
    }
#pragma unroll
    for (int p = 0; p < ROW_PASSES; p++) {
        float y[8];
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            y[i] = (float)v[p][i];
            if constexpr (ACT == GEMM_OPS_ACT_RELU) y[i] = y[i] < 0.0f ? 0.0f : y[i];
            else if constexpr (ACT == GEMM_OPS_ACT_SWIGLU) y[i] = silu(y[i]) * (float)u[p][i];
            m = max(m, magnitude(y[i]));
        }
        const BlockScale s = block_scale(max16(m));
        if (left_at(p) > 0) store_e4m3(a.Q + row * a.ldq + first + 512 * p, left_at(p), to_e4m3(y, s));
        if ((lane & 15) == 0) scales[4 * p + lane / 16][wave] = s.scale;
    }
    __syncthreads();
    if (threadIdx.x < 16 * ROW_PASSES) {
        const int64_t kb = (int64_t)blockIdx.y * (4 * ROW_PASSES) + threadIdx.x / 4, r = (int64_t)blockIdx.x * 4 + threadIdx.x % 4;
        if (128 * kb < a.N && r < a.M) a.scale[kb * a.ld_scale + r] = scales[threadIdx.x / 4][threadIdx.x % 4];
    }
}

// ---- quantisation in blocks: a workgroup takes 128 x 128, 16 rows at a time, and keeps them in registers -----------------------------
template <typename T>
__global__ __launch_bounds__(256) void quantize_blocks_kernel(const QuantArgs a)
{
    __shared__ uint32_t most[4];
    const int blocks_n = (int)(((int64_t)a.N + 127) / 128);
    const int64_t bm = blockIdx.x / blocks_n, bn = blockIdx.x % blocks_n;
    const int64_t c = 128 * bn + 8 * (threadIdx.x & 15);
    float y[8][8];
    uint32_t m = 0;
#pragma unroll
    for (int p = 0; p < 8; p++) {
        const int64_t row = 128 * bm + 16 * p + threadIdx.x / 16;
        if (row < a.M && c < a.N) {
            load8((const T*)a.X + row * a.ldx + c, (int)(a.N - c), y[p]);
        } else {
#pragma unroll
            for (int i = 0; i < 8; i++) y[p][i] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 8; i++) m = max(m, magnitude(y[p][i]));
    }
    m = max16(m);
    m = max(m, (uint32_t)__shfl_xor((int)m, 16));
    m = max(m, (uint32_t)__shfl_xor((int)m, 32));
    if ((threadIdx.x & 63) == 0) most[threadIdx.x >> 6] = m;
    __syncthreads();
    const BlockScale s = block_scale(max(max(most[0], most[1]), max(most[2], most[3])));
    if (threadIdx.x == 0) a.scale[bm * a.ld_scale + bn] = s.scale;
#pragma unroll
    for (int p = 0; p < 8; p++) {
        const int64_t row = 128 * bm + 16 * p + threadIdx.x / 16;
        if (row < a.M && c < a.N) store_e4m3(a.Q + row * a.ldq + c, (int)(a.N - c), to_e4m3(y[p], s));
    }
}

template <typename T>
int quant_rows_of_type(const QuantArgs& a, hipStream_t stream)
{
    const int64_t nb = ((int64_t)a.N + 127) / 128, gy = (nb + 4 * ROW_PASSES - 1) / (4 * ROW_PASSES);
    // y takes 65535 workgroups: 134 million columns
    if (gy > 65535) return GEMM_F16_ERR_SIZE;
    const dim3 grid((unsigned)(((int64_t)a.M + 3) / 4), (unsigned)gy);
    switch (a.act) {
    case GEMM_OPS_ACT_NONE: hipLaunchKernelGGL((quantize_rows_kernel<T, GEMM_OPS_ACT_NONE>), grid, dim3(256), 0, stream, a); break;
    case GEMM_OPS_ACT_RELU: hipLaunchKernelGGL((quantize_rows_kernel<T, GEMM_OPS_ACT_RELU>), grid, dim3(256), 0, stream, a); break;
    default: hipLaunchKernelGGL((quantize_rows_kernel<T, GEMM_OPS_ACT_SWIGLU>), grid, dim3(256), 0, stream, a); break;
    }
    return hipGetLastError() == hipSuccess ? GEMM_F16_OK : GEMM_F16_ERR_LAUNCH;
}
template <typename T>
int quant_blocks_of_type(const QuantArgs& a, hipStream_t stream)
{
    const int64_t tiles = (((int64_t)a.M + 127) / 128) * (((int64_t)a.N + 127) / 128);
    if (!fits_a_launch(tiles, 256)) return GEMM_F16_ERR_SIZE;
    hipLaunchKernelGGL(quantize_blocks_kernel<T>, dim3((unsigned)tiles), dim3(256), 0, stream, a);
    return hipGetLastError() == hipSuccess ? GEMM_F16_OK : GEMM_F16_ERR_LAUNCH;
}

}  // namespace

int ops_norm_grad_parts(int64_t M, int64_t N)
{
    const int64_t rows = grad_rows((int)(N < INT32_MAX ? N : INT32_MAX)), g = (M + rows - 1) / rows;
    return (int)(g < 256 ? g : 256);
}
// Rows need nothing of each other: more of them than the grid of one launch has threads for (a row takes up to 1024) go in several launches.
constexpr int64_t LAUNCH_ROWS = 1 << 21;
int ops_launch_norm(int type, const NormArgs& all, hipStream_t stream)
{
    int rc = GEMM_F16_OK;
    for (int64_t i = 0; i < all.M && rc == GEMM_F16_OK; i += LAUNCH_ROWS) {
        NormArgs a = all;
        a.M = (int)(all.M - i < LAUNCH_ROWS ? all.M - i : LAUNCH_ROWS);
        a.X = (const half_t*)all.X + i * all.ldx;                          // both types have 2 bytes
        if (a.R) a.R = (const half_t*)all.R + i * all.ldr;
        if (a.H) a.H = (half_t*)all.H + i * all.ldh;
        if (a.Y) a.Y = (half_t*)all.Y + i * all.ldy;
        if (a.Q) { a.Q += i * all.ldq; a.scale += i; }
        if (a.rstd) a.rstd += i;
        rc = type == GEMM_TYPE_F16 ? norm_of_type<half_t>(a, stream) : norm_of_type<bf16_t>(a, stream);
    }
    return rc;
}
int ops_launch_norm_grad(int type, const NormGradArgs& a, hipStream_t stream) { return type == GEMM_TYPE_F16 ? norm_grad_of_type<half_t>(a, stream) : norm_grad_of_type<bf16_t>(a, stream); }
int ops_launch_quant_rows(int type, const QuantArgs& all, hipStream_t stream)
{
    int rc = GEMM_F16_OK;
    for (int64_t i = 0; i < all.M && rc == GEMM_F16_OK; i += LAUNCH_ROWS) {
        QuantArgs a = all;
        a.M = (int)(all.M - i < LAUNCH_ROWS ? all.M - i : LAUNCH_ROWS);
        a.X = (const half_t*)all.X + i * all.ldx;
        a.Q += i * all.ldq; a.scale += i;
        rc = type == GEMM_TYPE_F16 ? quant_rows_of_type<half_t>(a, stream) : quant_rows_of_type<bf16_t>(a, stream);
    }
    return rc;
}
int ops_launch_quant_blocks(int type, const QuantArgs& a, hipStream_t stream) { return type == GEMM_TYPE_F16 ? quant_blocks_of_type<half_t>(a, stream) : quant_blocks_of_type<bf16_t>(a, stream); }
