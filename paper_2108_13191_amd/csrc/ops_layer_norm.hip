// Layer norm with the residual's addition, its gradients, and quantisation of rows to 8-bit integers (include/gemm_layer.h).
//
// Bound by memory: a row is read once, 8 elements of 16 bits a lane and access, and stays in registers for its mean, its squares about the mean and its
// largest magnitude.
#include <type_traits>
#include "ops_rows.h"
#include "../../include/gemm_layer.h"

namespace {

using namespace ops_dev;

int launched() { return hipGetLastError() == hipSuccess ? GEMM_F16_OK : GEMM_F16_ERR_LAUNCH; }

// ---- statistics of a row -----------------------------------------------------------------------------------------------------
// the sum of the L neighbouring threads that share a row, of a wavefront's where those are more than one
template <int L>
__device__ __forceinline__ float sum_lanes(float x)
{
    if constexpr (L >= 64) return sum64(x);
#pragma unroll
    for (int d = 1; d < L; d <<= 1) x += __shfl_xor(x, d);
    return x;
}
// the sum of W values, lane i of a wavefront having the i % W-th: of 16 neighbouring lanes, which have each 16 / W times
template <int W>
__device__ __forceinline__ float sum_waves(float x)
{
    static_assert(W <= 16 && (W & (W - 1)) == 0);
    auto add = [&](uint32_t y) { x += __builtin_bit_cast(float, y); };
    if constexpr (W >= 16) add(dpp_u32<0x128>(__builtin_bit_cast(uint32_t, x)));
    if constexpr (W >= 8) add(dpp_u32<0x124>(__builtin_bit_cast(uint32_t, x)));
    if constexpr (W >= 4) add(dpp_u32<0x122>(__builtin_bit_cast(uint32_t, x)));
    if constexpr (W >= 2) add(dpp_u32<0x121>(__builtin_bit_cast(uint32_t, x)));
    return x;
}
// Mean and sum of squares about it, of which each wavefront has those of its own elements: the row's mean is that of the wavefronts' by their elements, and
// squares about it are those about the wavefront's mean + n (its mean - the row's)^2.  So one exchange serves both.
struct Moments { float mean, squares; };
// n_of(w): elements of the row's w-th wavefront; lds: 2 floats for each wavefront of the workgroup
template <int L, typename F>
__device__ __forceinline__ Moments row_moments(float own_mean, float squares, int N, float* lds, F n_of)
{
    if constexpr (L <= 64) return {own_mean, squares};
    constexpr int W = L > 64 ? L / 64 : 1;
    const int wave = threadIdx.x >> 6, w = threadIdx.x & (W - 1);
    if ((threadIdx.x & 63) == 0) { lds[2 * wave] = own_mean; lds[2 * wave + 1] = squares; }
    __syncthreads();
    const float* const pair = &lds[2 * (wave / W * W + w)];
    const float at = pair[0], n = (float)n_of(w);
    const float mean = sum_waves<W>(n * at) / (float)N, d = at - mean;
    return {mean, sum_waves<W>(pair[1] + (n > 0.0f ? n * d * d : 0.0f))};
}

// The moments of a bf16 row whose squares, as they were summed, are not finite (f16 has no values whose sums could leave f32's range).  Its elements may be infinite or NaN, or sums of
// parts, squares or differences from the mean have passed f32's range; which of them do depends on how the row is dealt to threads, what the row gives must not.  `scaled`: this thread's sum
// of elements times 2^-31, which never passes it, of 2^31 elements.  Where the whole sum does not either, the squares do (so does any part's sum if the row's does not, where the elements
// are not all alike), and rstd is 0; else the row is NaN.
constexpr float DOWN = 0x1p-31f;
template <int L>
__device__ __forceinline__ Moments moments_beyond(float scaled, int N, float* lds)
{
    if constexpr (L > 64) scaled = sum_row<L / 64>(scaled, lds);
    else scaled = sum_lanes<L>(scaled);
    const float sum = scaled / DOWN;
    if (!(__builtin_fabsf(sum) < __builtin_inff())) return {__builtin_nanf(""), __builtin_nanf("")};
    return {sum / (float)N, __builtin_inff()};
}

// the largest of a row's magnitudes over its L threads; lds: a word for each wavefront of the workgroup, used for nothing else
template <int L>
__device__ __forceinline__ uint32_t max_row(uint32_t m, uint32_t* lds)
{
    if constexpr (L >= 16) m = max16(m);
    else {
#pragma unroll
        for (int d = 1; d < L; d <<= 1) m = max(m, (uint32_t)__shfl_xor((int)m, d));
    }
    if constexpr (L >= 32) m = max(m, (uint32_t)__shfl_xor((int)m, 16));
    if constexpr (L >= 64) m = max(m, (uint32_t)__shfl_xor((int)m, 32));
    if constexpr (L > 64) {
        const int wave = threadIdx.x >> 6, first = wave / (L / 64) * (L / 64);
        if ((threadIdx.x & 63) == 0) lds[wave] = m;
        __syncthreads();
        m = max16(lds[first + (threadIdx.x & (L / 64 - 1))]);
    }
    return m;
}

// ---- a row in 8-bit integers ---------------------------------------------------------------------------------------------------
struct RowScale {
    float scale, inverse;
    bool finite;
    // The integer nearest to y / scale, ties to even, in the low byte.  The product with the reciprocal is off by its last bits, enough to miss at borders (bf16
    // values come near one once in 3000); what the integer leaves of y is exact in one fma, and tells.  (Adding 1.5 2^23 leaves the rounded integer in the low bits.)
    __device__ __forceinline__ int nearest(float y) const
    {
        const float u = y * inverse + 0x1.8p23f, n = u - 0x1.8p23f;
        const float r = __builtin_fmaf(-n, scale, y), border = 0.5f * scale;
        int i = (int)__builtin_bit_cast(uint32_t, u);
        const bool over = __builtin_fabsf(r) > border || (__builtin_fabsf(r) == border && (i & 1));
        i += over ? (r > 0.0f ? 1 : -1) : 0;
        return i;
    }
};
__device__ __forceinline__ RowScale row_scale(uint32_t bits)
{
    if (bits >= 0x7f800000u) return {__builtin_nanf(""), 0.0f, false};
    const float scale = fmaxf(__builtin_bit_cast(float, bits), SCALE_FLOOR) * (1.0f / 127.0f);
    return {scale, 1.0f / scale, true};
}
__device__ __forceinline__ uintx2 to_i8(const float (&y)[8], const RowScale& s)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; i++) w[i] = __builtin_amdgcn_perm((uint32_t)s.nearest(y[2 * i + 1]), (uint32_t)s.nearest(y[2 * i]), 0x0c0c0400u);
    const uintx2 q = {w[0] | (w[1] << 16), w[2] | (w[3] << 16)};
    return s.finite ? q : uintx2{0u, 0u};
}

// ---- the norm --------------------------------------------------------------------------------------------------------------------
// L threads a row, each with P chunks of 8 columns in registers; R rows a workgroup.  (16384,4096) bf16, all of x, r, h and y, 93 us, 5.7 TB/s; 16 rows of 8192, a chunk a thread, 3.9 in a graph.
template <typename T, bool WHOLE, int L, int P, int R>
__global__ __launch_bounds__(L * R) void layer_norm_kernel(const LayerNormArgs a)
{
    __shared__ float lds[L * R / 64 * 3];
    const int lane = threadIdx.x % L;
    const int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / L, there = min(row, (int64_t)a.M - 1);
    const bool live = row < a.M;
    const T* const x = (const T*)a.X + there * a.ldx;
    const T* const r = a.R ? (const T*)a.R + there * a.ldr : nullptr;

    Raw8<T> raw[P], res[P], gamma[P], beta[P];            // all asked for ahead of the sums
#pragma unroll
    for (int p = 0; p < P; p++) {
        const int c = 8 * (lane + L * p);
        raw[p] = load8_of<WHOLE>(x, c, a.N);
        if (r) res[p] = load8_of<WHOLE>(r, c, a.N);
        gamma[p] = load8_of<WHOLE>((const T*)a.gamma, c, a.N);
        if (a.beta) beta[p] = load8_of<WHOLE>((const T*)a.beta, c, a.N);
    }
    float v[P][8], sum = 0.0f, squares = 0.0f;
#pragma unroll
    for (int p = 0; p < P; p++) {
        const int c = 8 * (lane + L * p);
        raw[p] = settled<T, WHOLE>(raw[p], c, a.N);
        if (r) res[p] = settled<T, WHOLE>(res[p], c, a.N);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            v[p][i] = (float)raw[p][i];
            if (r) v[p][i] = rounded<T>(v[p][i] + (float)res[p][i]);         // h as it is stored is what is normed
            sum += v[p][i];
        }
        if (a.H && live && c < a.N) store8_of<WHOLE>((T*)a.H + row * a.ldh + c, a.N - c, v[p]);
    }
    auto n_of = [&](int w) {                              // elements of the row's w-th wavefront
        int n = 0;
#pragma unroll
        for (int p = 0; p < P; p++) n += min(max(a.N - 8 * (64 * w + L * p), 0), 512);
        return n;
    };
    sum = sum_lanes<L>(sum);
    const int own = L <= 64 ? a.N : n_of((threadIdx.x >> 6) % (L >= 64 ? L / 64 : 1));
    const float centre = own ? sum / (float)own : 0.0f;
#pragma unroll
    for (int p = 0; p < P; p++) {
        const int left = a.N - 8 * (lane + L * p);
#pragma unroll
        for (int i = 0; i < 8; i++) { const float d = (WHOLE ? left > 0 : i < left) ? v[p][i] - centre : 0.0f; squares += d * d; }
    }
    Moments m = row_moments<L>(centre, sum_lanes<L>(squares), a.N, lds, n_of);
    if constexpr (std::is_same_v<T, bf16_t>) {
        if (__builtin_expect(!(m.squares < __builtin_inff()), false)) {      // (the same for all threads of a row)
            float scaled = 0.0f;
#pragma unroll
            for (int p = 0; p < P; p++)
#pragma unroll
                for (int i = 0; i < 8; i++) scaled += v[p][i] * DOWN;
            m = moments_beyond<L>(scaled, a.N, lds);
#pragma unroll
            for (int p = 0; p < P; p++)
#pragma unroll
                for (int i = 0; i < 8; i++) v[p][i] = m.mean;                // differences, which rstd makes 0, may pass the range
        }
    }
    const float rstd = 1.0f / sqrtf(m.squares / (float)a.N + a.eps);
    if (live && lane == 0) {
        if (a.mean) a.mean[row] = m.mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    if (!a.Y && !a.Q) return;
    uint32_t big = 0;
#pragma unroll
    for (int p = 0; p < P; p++) {
        const int c = 8 * (lane + L * p), left = a.N - c;
        gamma[p] = settled<T, WHOLE>(gamma[p], c, a.N);
        if (a.beta) beta[p] = settled<T, WHOLE>(beta[p], c, a.N);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            float y = (v[p][i] - m.mean) * rstd * (float)gamma[p][i];
            if (a.beta) y += (float)beta[p][i];
            v[p][i] = (WHOLE ? left > 0 : i < left) ? y : 0.0f;
            big = max(big, magnitude(v[p][i]));
        }
        if (a.Y && live && left > 0) store8_of<WHOLE>((T*)a.Y + row * a.ldy + c, left, v[p]);
    }
    if (!a.Q) return;
    const RowScale s = row_scale(max_row<L>(big, (uint32_t*)&lds[L * R / 64 * 2]));
    if (!live) return;
    if (lane == 0) a.scale[row] = s.scale;
#pragma unroll
    for (int p = 0; p < P; p++) {
        const int c = 8 * (lane + L * p);
        if (c < a.N) store_bytes<WHOLE>(a.Q + row * a.ldq + c, a.N - c, to_i8(v[p], s));
    }
}

// Rows of any length, a workgroup each: its chunks are gone through once for each of the mean, the squares, the largest magnitude, the outputs.
constexpr int LONG = 1024;
template <typename T>
__global__ __launch_bounds__(LONG) void layer_norm_long_kernel(const LayerNormArgs a)
{
    __shared__ float lds[LONG / 64 * 3];
    const int lane = threadIdx.x;
    const int64_t row = blockIdx.x, first = 8 * (int64_t)lane, step = 8 * LONG;
    const T* const x = (const T*)a.X + row * a.ldx;
    const T* const r = a.R ? (const T*)a.R + row * a.ldr : nullptr;
    T* const h = a.H ? (T*)a.H + row * a.ldh : nullptr;
    float sum = 0.0f, squares = 0.0f, o[8];
    auto form = [&](int64_t c) {
        load8(x + c, (int)(a.N - c), o);
        if (r) {
            float s[8];
            load8(r + c, (int)(a.N - c), s);
#pragma unroll
            for (int i = 0; i < 8; i++) o[i] = rounded<T>(o[i] + s[i]);
        }
    };
    auto again = [&](int64_t c) { if (h) load8((const T*)h + c, (int)(a.N - c), o); else form(c); };
    for (int64_t c = first; c < a.N; c += step) {
        form(c);
        if (h) store8(h + c, (int)(a.N - c), o);
#pragma unroll
        for (int i = 0; i < 8; i++) sum += o[i];
    }
    sum = sum64(sum);
    auto n_of = [&](int w) {                              // whole rounds of the workgroup, and what the last one leaves
        const int rounds = a.N / (8 * LONG), rest = a.N - rounds * (8 * LONG);
        return 512 * rounds + min(max(rest - 512 * w, 0), 512);
    };
    const int own = n_of(threadIdx.x >> 6);
    const float centre = own ? sum / (float)own : 0.0f;
    for (int64_t c = first; c < a.N; c += step) {
        again(c);
#pragma unroll
        for (int i = 0; i < 8; i++) { const float d = c + i < a.N ? o[i] - centre : 0.0f; squares += d * d; }
    }
    Moments m = row_moments<LONG>(centre, sum64(squares), a.N, lds, n_of);
    bool beyond = false;
    if constexpr (std::is_same_v<T, bf16_t>) {
        beyond = !(m.squares < __builtin_inff());
        if (beyond) {
            float scaled = 0.0f;
            for (int64_t c = first; c < a.N; c += step) {
                again(c);
#pragma unroll
                for (int i = 0; i < 8; i++) scaled += o[i] * DOWN;
            }
            m = moments_beyond<LONG>(scaled, a.N, lds);
        }
    }
    const float rstd = 1.0f / sqrtf(m.squares / (float)a.N + a.eps);
    if (lane == 0) {
        if (a.mean) a.mean[row] = m.mean;
        if (a.rstd) a.rstd[row] = rstd;
    }
    if (!a.Y && !a.Q) return;
    uint32_t big = 0;
    auto output = [&](int64_t c) {
        const int left = (int)min((int64_t)8, a.N - c);
        again(c);
        const Raw8<T> gm = load8_raw((const T*)a.gamma + c, left), bt = load8_raw((const T*)a.beta + c, a.beta ? left : 0);
#pragma unroll
        for (int i = 0; i < 8; i++) { const float y = ((beyond ? m.mean : o[i]) - m.mean) * rstd * (float)gm[i] + (float)bt[i]; o[i] = i < left ? y : 0.0f; }
    };
    for (int64_t c = first; c < a.N; c += step) {
        output(c);
        if (a.Y) store8((T*)a.Y + row * a.ldy + c, (int)(a.N - c), o);
#pragma unroll
        for (int i = 0; i < 8; i++) big = max(big, magnitude(o[i]));
    }
    if (!a.Q) return;
    const RowScale s = row_scale(max_row<LONG>(big, (uint32_t*)&lds[LONG / 64 * 2]));
    if (lane == 0) a.scale[row] = s.scale;
    for (int64_t c = first; c < a.N; c += step) {
        output(c);
        store_bytes(a.Q + row * a.ldq + c, (int)(a.N - c), to_i8(o, s));
    }
}

template <typename T, int L, int P, int R>
int launch_norm(const LayerNormArgs& a, hipStream_t stream)
{
    const dim3 grid((unsigned)(((int64_t)a.M + R - 1) / R));
    if (a.N % 8 == 0) hipLaunchKernelGGL((layer_norm_kernel<T, true, L, P, R>), grid, dim3(L * R), 0, stream, a);
    else hipLaunchKernelGGL((layer_norm_kernel<T, false, L, P, R>), grid, dim3(L * R), 0, stream, a);
    return launched();
}
template <typename T>
int norm_of_type(const LayerNormArgs& a, hipStream_t stream)
{
    if (a.M <= 2 * chip().cus && a.N > 2048 && a.N <= 8192) return launch_norm<T, 1024, 1, 1>(a, stream);
    if (a.N <= 64) return launch_norm<T, 8, 1, 32>(a, stream);
    if (a.N <= 128) return launch_norm<T, 16, 1, 16>(a, stream);
    if (a.N <= 256) return launch_norm<T, 32, 1, 8>(a, stream);
    if (a.N <= 512) return launch_norm<T, 64, 1, 4>(a, stream);
    if (a.N <= 1024) return launch_norm<T, 64, 2, 4>(a, stream);
    if (a.N <= 2048) return launch_norm<T, 64, 4, 4>(a, stream);
    if (a.N <= 4096) return launch_norm<T, 256, 2, 1>(a, stream);
    if (a.N <= 8192) return launch_norm<T, 256, 4, 1>(a, stream);
    if (a.N <= 16384) return launch_norm<T, 512, 4, 1>(a, stream);
    hipLaunchKernelGGL(layer_norm_long_kernel<T>, dim3((unsigned)a.M), dim3(LONG), 0, stream, a);
    return launched();
}

// ---- its gradients -----------------------------------------------------------------------------------------------------------------
// A row of dY, H and dH, chunks of 8 columns of one of its L threads; rows behind the last one are that one, with nothing in dy
template <typename T, bool WHOLE, int L, int P>
struct GradRow {
    Raw8<T> dy[P], h[P], dh[P];
    float mean, rstd;
    __device__ __forceinline__ void load(const LayerNormGradArgs& a, int lane, int64_t row)
    {
        row = min(row, (int64_t)a.M - 1);
        rstd = a.rstd[row];
        mean = a.mean[row];
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int c = 8 * (lane + L * p);
            dy[p] = load8_of<WHOLE>((const T*)a.dY + row * a.lddy, c, a.N);
            h[p] = load8_of<WHOLE>((const T*)a.H + row * a.ldh, c, a.N);
            if (a.dH) dh[p] = load8_of<WHOLE>((const T*)a.dH + row * a.lddh, c, a.N);
        }
    }
    __device__ __forceinline__ void settle(const LayerNormGradArgs& a, int lane, bool live)
    {
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int c = 8 * (lane + L * p);
            dy[p] = settled<T, WHOLE>(dy[p], live ? c : (int64_t)a.N + 8, a.N);
            h[p] = settled<T, WHOLE>(h[p], c, a.N);
            if (a.dH) dh[p] = settled<T, WHOLE>(dh[p], c, a.N);
        }
    }
    // from the sums of g and g xhat
    __device__ __forceinline__ void store(const LayerNormGradArgs& a, int lane, int64_t row, const Raw8<T> (&gamma)[P], float s1, float s2) const
    {
        const float m1 = s1 / (float)a.N, m2 = s2 / (float)a.N;
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int c = 8 * (lane + L * p);
            if (c >= a.N) continue;
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                o[i] = rstd * ((float)dy[p][i] * (float)gamma[p][i] - m1 - ((float)h[p][i] - mean) * rstd * m2);
                if (a.dH) o[i] += (float)dh[p][i];
            }
            store8_of<WHOLE>((T*)a.dX + row * a.lddx + c, a.N - c, o);
        }
    }
};
// two sums over the L threads that share a row; set: 2 floats for each wavefront of the workgroup
template <int L>
__device__ __forceinline__ void sum_pair(float& x, float& y, float* set)
{
    if constexpr (L < 64) {
#pragma unroll
        for (int d = 1; d < L; d <<= 1) { x += __shfl_xor(x, d); y += __shfl_xor(y, d); }
    } else {
        x = sum64(x);
        y = sum64(y);
    }
    if constexpr (L > 64) {
        const int wave = threadIdx.x >> 6, first = wave / (L / 64) * (L / 64);
        if ((threadIdx.x & 63) == 0) { set[2 * wave] = x; set[2 * wave + 1] = y; }
        __syncthreads();
        const float* const pair = &set[2 * (first + (threadIdx.x & (L / 64 - 1)))];
        x = sum_waves<L / 64>(pair[0]);
        y = sum_waves<L / 64>(pair[1]);
    }
}

// dX row by row; the columns' sums of dy xhat and dy stay in registers over all rows of a workgroup, which writes them as one row of the
// workspace; a second kernel adds those.  Every sum has a fixed order.  L threads a row, R rows a workgroup, P chunks of 8 columns a thread.  (8191,4000) bf16 with dH 52 us, 5 TB/s, and 4 for the
// second launch.
template <typename T, bool WHOLE, int L, int P, int R>
__global__ __launch_bounds__(L * R) void layer_norm_grad_kernel(const LayerNormGradArgs a)
{
    extern __shared__ float dyn[];                        // 4 floats for each wavefront, then R * 8 L of sums
    const int lane = threadIdx.x % L, sub = threadIdx.x / L;
    constexpr int WAVES = L * R / 64;
    float dg[P][8] = {}, db[P][8] = {};
    Raw8<T> gamma[P];
#pragma unroll
    for (int p = 0; p < P; p++) gamma[p] = settled<T, WHOLE>(load8_of<WHOLE>((const T*)a.gamma, 8 * (lane + L * p), a.N), 8 * (lane + L * p), a.N);
    // the values as they were loaded, to be widened again: kept widened over the sums they would take twice the registers
    auto again = [](Raw8<T>& x) { uintx4 r = __builtin_bit_cast(uintx4, x); asm volatile("" : "+v"(r)); x = __builtin_bit_cast(Raw8<T>, r); };

    const int64_t step = (int64_t)gridDim.x * R;
    int slot = 0;
    constexpr bool AHEAD = L * R <= 512;                  // the next row's loads ahead: registers for it where a workgroup has 512 threads
    GradRow<T, WHOLE, L, P> next;
    if constexpr (AHEAD) next.load(a, lane, (int64_t)blockIdx.x * R + sub);
    for (int64_t row0 = (int64_t)blockIdx.x * R; row0 < a.M; row0 += step) {      // the same number of trips for the whole workgroup
        const int64_t row = row0 + sub;
        const bool live = row < a.M;
        if constexpr (!AHEAD) next.load(a, lane, row);
        GradRow<T, WHOLE, L, P> x = next;
        x.settle(a, lane, live);
        float s1 = 0.0f, s2 = 0.0f;                       // of g and g xhat; dy is zero behind the row's end
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float dy = (float)x.dy[p][i], xhat = ((float)x.h[p][i] - x.mean) * x.rstd, g = dy * (float)gamma[p][i];
                dg[p][i] += dy * xhat;
                db[p][i] += dy;
                s1 += g;
                s2 += g * xhat;
            }
        if constexpr (AHEAD) next.load(a, lane, row + step);      // while this row's sums are exchanged and its gradient is formed
#pragma unroll
        for (int p = 0; p < P; p++) { again(x.dy[p]); again(x.h[p]); again(gamma[p]); }
        sum_pair<L>(s1, s2, dyn + slot * 2 * WAVES);      // two sets of partial sums in turn: one barrier a row
        slot ^= 1;
        if (live) x.store(a, lane, row, gamma, s1, s2);
    }
    if (!a.dgamma && !a.dbeta) return;
    // sums of the workgroup's row slots, in their order, 8 L columns at a time
    float* const sums = dyn + 4 * WAVES;
    const bool only = gridDim.x == 1;                     // one workgroup's sums are the result
    auto put = [&](const float (&d)[P][8], float* out) {
#pragma unroll
        for (int p = 0; p < P; p++) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; i += 4) *(floatx4*)&sums[sub * 8 * L + 8 * lane + i] = floatx4{d[p][i], d[p][i + 1], d[p][i + 2], d[p][i + 3]};
            __syncthreads();
            for (int j = threadIdx.x; j < 8 * L; j += L * R) {
                const int c = 8 * L * p + j;
                float s = sums[j];
#pragma unroll
                for (int r = 1; r < R; r++) s += sums[r * 8 * L + j];
                if (c < a.N) out[c] = s;
            }
        }
    };
    if (a.dgamma) put(dg, only ? a.dgamma : a.ws + (int64_t)blockIdx.x * 2 * a.N);
    if (a.dbeta) put(db, only ? a.dbeta : a.ws + ((int64_t)blockIdx.x * 2 + 1) * a.N);
}

// Few rows: one launch, (512,768) 5.0 us in a graph.  The columns' sums need nothing of the rows' sums, so some workgroups form dX and others read the rows once more for 64 columns of dgamma and dbeta: 8
// threads of 8 columns, 64 rows at a time.
template <typename T, bool WHOLE, int L, int P>
__global__ __launch_bounds__(512) void layer_norm_grad_few_kernel(const LayerNormGradArgs a, int row_groups)
{
    __shared__ float lds[2][64][65];
    if ((int)blockIdx.x < row_groups) {
        const int lane = threadIdx.x % L;
        const int64_t row = (int64_t)blockIdx.x * (512 / L) + threadIdx.x / L;
        const bool live = row < a.M;
        GradRow<T, WHOLE, L, P> x;
        Raw8<T> gamma[P];
        x.load(a, lane, row);
#pragma unroll
        for (int p = 0; p < P; p++) gamma[p] = load8_of<WHOLE>((const T*)a.gamma, 8 * (lane + L * p), a.N);
        x.settle(a, lane, live);
        float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
        for (int p = 0; p < P; p++) {
            gamma[p] = settled<T, WHOLE>(gamma[p], 8 * (lane + L * p), a.N);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float g = (float)x.dy[p][i] * (float)gamma[p][i];
                s1 += g;
                s2 += g * (((float)x.h[p][i] - x.mean) * x.rstd);
            }
        }
        sum_pair<L>(s1, s2, &lds[0][0][0]);
        if (live) x.store(a, lane, row, gamma, s1, s2);
        return;
    }
    const int lane = threadIdx.x & 7, sub = threadIdx.x >> 3;
    const int64_t c = ((int64_t)blockIdx.x - row_groups) * 64 + 8 * lane;
    // Many rows (the widest form has up to 2^21 that are no whole chunks, the others 2047 at most): sums are put aside every 2048, so that 32 and M / 2048 additions follow one another, not M / 64
    constexpr bool MANY = !WHOLE && 8 * L * P > 8192;
    float dg[8] = {}, db[8] = {}, dg_all[8] = {}, db_all[8] = {};
    auto add = [&](Raw8<T> dy, Raw8<T> h, float mean, float rstd, bool live) {
        dy = settled<T, WHOLE>(dy, live ? c : (int64_t)a.N + 8, a.N);
        h = settled<T, WHOLE>(h, c, a.N);
#pragma unroll
        for (int i = 0; i < 8; i++) { dg[i] += (float)dy[i] * (((float)h[i] - mean) * rstd); db[i] += (float)dy[i]; }
    };
    constexpr int AT_ONCE = 4, ASIDE = 2048;
    for (int64_t row0 = sub; row0 - sub < a.M; row0 += 64 * AT_ONCE) {
        Raw8<T> dy[AT_ONCE], h[AT_ONCE];
        float mean[AT_ONCE], rstd[AT_ONCE];
#pragma unroll
        for (int u = 0; u < AT_ONCE; u++) {
            const int64_t row = min(row0 + 64 * u, (int64_t)a.M - 1);
            dy[u] = load8_of<WHOLE>((const T*)a.dY + row * a.lddy, c, a.N);
            h[u] = load8_of<WHOLE>((const T*)a.H + row * a.ldh, c, a.N);
            mean[u] = a.mean[row];
            rstd[u] = a.rstd[row];
        }
#pragma unroll
        for (int u = 0; u < AT_ONCE; u++) add(dy[u], h[u], mean[u], rstd[u], row0 + 64 * u < a.M);
        if (MANY && ((row0 - sub) & (ASIDE - 1)) == ASIDE - 64 * AT_ONCE) {
#pragma unroll
            for (int i = 0; i < 8; i++) { dg_all[i] += dg[i]; db_all[i] += db[i]; dg[i] = db[i] = 0.0f; }
        }
    }
    if constexpr (MANY) {
#pragma unroll
        for (int i = 0; i < 8; i++) { dg[i] += dg_all[i]; db[i] += db_all[i]; }
    }
#pragma unroll
    for (int i = 0; i < 8; i++) { lds[0][8 * lane + i][sub] = dg[i]; lds[1][8 * lane + i][sub] = db[i]; }
    __syncthreads();
    // a wavefront adds the 64 rows' slots of a column: 8 of each kind
    const int wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const int64_t col = ((int64_t)blockIdx.x - row_groups) * 64 + 8 * wave + i;
        const float g = sum64(lds[0][8 * wave + i][threadIdx.x & 63]), b = sum64(lds[1][8 * wave + i][threadIdx.x & 63]);
        if ((threadIdx.x & 63) == 0 && col < a.N) {
            if (a.dgamma) a.dgamma[col] = g;
            if (a.dbeta) a.dbeta[col] = b;
        }
    }
}

// Rows longer than the registers hold: dX in two passes over a row ...
template <typename T>
__global__ __launch_bounds__(1024) void layer_norm_grad_long_kernel(const LayerNormGradArgs a)
{
    __shared__ float lds[16];
    const int64_t row = blockIdx.x;
    const T *const dyr = (const T*)a.dY + row * a.lddy, *const hr = (const T*)a.H + row * a.ldh, *const gr = (const T*)a.gamma;
    const float rstd = a.rstd[row], mean = a.mean[row];
    float dy[8], hv[8], gm[8], s1 = 0.0f, s2 = 0.0f;
    for (int64_t c = 8 * (int64_t)threadIdx.x; c < a.N; c += 8192) {
        load8(dyr + c, (int)(a.N - c), dy); load8(hr + c, (int)(a.N - c), hv); load8(gr + c, (int)(a.N - c), gm);
#pragma unroll
        for (int i = 0; i < 8; i++) { s1 += dy[i] * gm[i]; s2 += dy[i] * gm[i] * ((hv[i] - mean) * rstd); }
    }
    const float m1 = sum_row<16>(s1, lds) / (float)a.N, m2 = sum_row<16>(s2, lds) / (float)a.N;
    for (int64_t c = 8 * (int64_t)threadIdx.x; c < a.N; c += 8192) {
        float up[8] = {}, o[8];
        load8(dyr + c, (int)(a.N - c), dy); load8(hr + c, (int)(a.N - c), hv); load8(gr + c, (int)(a.N - c), gm);
        if (a.dH) load8((const T*)a.dH + row * a.lddh + c, (int)(a.N - c), up);
#pragma unroll
        for (int i = 0; i < 8; i++) o[i] = rstd * (dy[i] * gm[i] - m1 - (hv[i] - mean) * rstd * m2) + up[i];
        store8((T*)a.dX + row * a.lddx + c, (int)(a.N - c), o);
    }
}
// ... and the columns' sums before it (dX may be dY): a workgroup takes 2048 columns and every gridDim.y-th row
template <typename T>
__global__ __launch_bounds__(256) void layer_norm_columns_long_kernel(const LayerNormGradArgs a)
{
    const int64_t c = 8 * ((int64_t)blockIdx.x * 256 + threadIdx.x);
    if (c >= a.N) return;
    float dg[8] = {}, db[8] = {}, dy[8], hv[8];
    for (int64_t row = blockIdx.y; row < a.M; row += gridDim.y) {
        load8((const T*)a.dY + row * a.lddy + c, (int)(a.N - c), dy);
        load8((const T*)a.H + row * a.ldh + c, (int)(a.N - c), hv);
        const float rstd = a.rstd[row], mean = a.mean[row];
#pragma unroll
        for (int i = 0; i < 8; i++) { dg[i] += dy[i] * ((hv[i] - mean) * rstd); db[i] += dy[i]; }
    }
    float* const out = a.ws + (int64_t)blockIdx.y * 2 * a.N + c;
    for (int i = 0; i < 8; i++) if (c + i < a.N) { out[i] = dg[i]; out[a.N + i] = db[i]; }
}

// dgamma[j] and dbeta[j]: sums of `parts` rows of 2 N floats of the workspace, from column `first` on, 64 columns a workgroup, wavefront w takes rows w, w + 16, ...
__global__ __launch_bounds__(1024) void column_sums_kernel(const float* __restrict__ ws, int parts, int N, int64_t first, float* __restrict__ dgamma, float* __restrict__ dbeta)
{
    __shared__ float lds[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = first + (int64_t)blockIdx.x * 64 + lane;
    float* const out = blockIdx.y ? dbeta : dgamma;
    if (!out) return;
    float s = 0.0f;
    if (c < N) {
#pragma unroll 4
        for (int r = wave; r < parts; r += 16) s += ws[((int64_t)r * 2 + blockIdx.y) * N + c];
    }
    lds[wave][lane] = s;
    __syncthreads();
    if (wave == 0 && c < N) {
#pragma unroll
        for (int w = 1; w < 16; w++) s += lds[w][lane];
        out[c] = s;
    }
}

constexpr int64_t LAUNCH_COLUMNS = 1 << 27;              // 16 threads each: 2^31 of the 2^32 of a launch

// threads that share a row in the gradient, and rows that a workgroup takes at a time
inline int grad_rows(int64_t N) { return N <= 64 ? 64 : N <= 128 ? 32 : N <= 512 ? 16 : N <= 1024 ? 8 : N <= 2048 ? 4 : N <= 4096 ? 2 : 1; }
// Whether one launch forms everything, us | two launches.  Up to 512 rows, 768 of more than 512 columns: (512,768) 6.0 | 7.7, (512,4096) 8.5 | 12.8, (768,8192) 15.6 | 18.2, (512,64) 5.7 | 5.9; more:
// (700,64) 7.0 | 6.1, (1024,768) 9.2 | 8.4, (2048,4096) 28 | 20.  Rows of more than 8192, whose columns' sums leave no registers for the next row, up to 2047 of them: (800,16384) 28 | 36,
// (1024,9000) 23 | 26; more: (2048,9000) 44 | 43, (2048,16384) 71 | 67, (6000,10000) 150 | 108, (20000,9000) 459 | 295; any number where they are no whole chunks of 8, whose shifts take more registers:
// (1500,12001) 57 | 80, (2048,16383) 93 | 117, (20000,9001) 564 | 716.
// Not where dX takes dY's place, which is read twice.
inline bool grad_few(const LayerNormGradArgs& a)
{
    if (a.N > 16384 || a.M > LAUNCH_ROWS) return false;
    if (!a.dgamma && !a.dbeta) return true;
    return a.dX != a.dY && (a.M <= 512 || (a.N > 512 && a.M <= 768) || (a.N > 8192 && (a.M < 2048 || a.N % 8 != 0)));
}

template <typename T, int L, int P, int R>
int launch_norm_grad(const LayerNormGradArgs& a, int parts, hipStream_t stream)
{
    constexpr size_t lds = (L * R / 16 + R * 8 * L) * sizeof(float);
    if (a.N % 8 == 0) hipLaunchKernelGGL((layer_norm_grad_kernel<T, true, L, P, R>), dim3((unsigned)parts), dim3(L * R), lds, stream, a);
    else hipLaunchKernelGGL((layer_norm_grad_kernel<T, false, L, P, R>), dim3((unsigned)parts), dim3(L * R), lds, stream, a);
    return launched();
}
template <typename T, int L, int P>
int launch_norm_grad_few(const LayerNormGradArgs& a, hipStream_t stream)
{
    const int row_groups = (a.M + 512 / L - 1) / (512 / L), columns = a.dgamma || a.dbeta ? (a.N + 63) / 64 : 0;
    const dim3 grid((unsigned)(row_groups + columns));
    if (a.N % 8 == 0) hipLaunchKernelGGL((layer_norm_grad_few_kernel<T, true, L, P>), grid, dim3(512), 0, stream, a, row_groups);
    else hipLaunchKernelGGL((layer_norm_grad_few_kernel<T, false, L, P>), grid, dim3(512), 0, stream, a, row_groups);
    return launched();
}
template <typename T>
int norm_grad_of_type(const LayerNormGradArgs& a, hipStream_t stream)
{
    const bool columns = a.dgamma || a.dbeta;
    if (a.M > 0 && grad_few(a)) {
        if (a.N <= 64) return launch_norm_grad_few<T, 8, 1>(a, stream);
        if (a.N <= 256) return launch_norm_grad_few<T, 32, 1>(a, stream);
        if (a.N <= 512) return launch_norm_grad_few<T, 64, 1>(a, stream);
        if (a.N <= 1024) return launch_norm_grad_few<T, 128, 1>(a, stream);
        if (a.N <= 2048) return launch_norm_grad_few<T, 256, 1>(a, stream);
        if (a.N <= 4096) return launch_norm_grad_few<T, 512, 1>(a, stream);
        return a.N <= 8192 ? launch_norm_grad_few<T, 512, 2>(a, stream) : launch_norm_grad_few<T, 512, 4>(a, stream);
    }
    const int parts = ops_layer_norm_grad_parts(a.M, a.N);
    int rc = GEMM_F16_OK;
    if (a.M > 0) {
        if (a.N <= 64) rc = launch_norm_grad<T, 8, 1, 64>(a, parts, stream);
        else if (a.N <= 128) rc = launch_norm_grad<T, 16, 1, 32>(a, parts, stream);
        else if (a.N <= 256) rc = launch_norm_grad<T, 32, 1, 16>(a, parts, stream);
        else if (a.N <= 512) rc = launch_norm_grad<T, 64, 1, 16>(a, parts, stream);
        else if (a.N <= 1024) rc = launch_norm_grad<T, 64, 2, 8>(a, parts, stream);
        else if (a.N <= 2048) rc = launch_norm_grad<T, 128, 2, 4>(a, parts, stream);
        else if (a.N <= 4096) rc = launch_norm_grad<T, 256, 2, 2>(a, parts, stream);
        else if (a.N <= 8192) rc = launch_norm_grad<T, 512, 2, 1>(a, parts, stream);
        else if (a.N <= 16384) rc = launch_norm_grad<T, 1024, 2, 1>(a, parts, stream);
        else {
            if (!fits_a_launch(a.M, 1024)) return GEMM_F16_ERR_SIZE;
            if (columns) hipLaunchKernelGGL(layer_norm_columns_long_kernel<T>, dim3((unsigned)(((int64_t)a.N + 2047) / 2048), (unsigned)parts), dim3(256), 0, stream, a);
            hipLaunchKernelGGL(layer_norm_grad_long_kernel<T>, dim3((unsigned)a.M), dim3(1024), 0, stream, a);
            rc = launched();
        }
        if (rc != GEMM_F16_OK) return rc;
    }
    if (!columns || (parts == 1 && a.N <= 16384)) return rc;
    for (int64_t first = 0; first < a.N && rc == GEMM_F16_OK; first += LAUNCH_COLUMNS) {
        const int64_t left = a.N - first;
        hipLaunchKernelGGL(column_sums_kernel, dim3((unsigned)(((left < LAUNCH_COLUMNS ? left : LAUNCH_COLUMNS) + 63) / 64), 2), dim3(1024), 0, stream, a.ws, parts, a.N, first, a.dgamma, a.dbeta);
        rc = launched();
    }
    return rc;
}

// ---- rows to 8-bit integers ----------------------------------------------------------------------------------------------------------
// values of x (and u, of SWIGLU) after the activation
template <typename T, int ACT>
__device__ __forceinline__ void activated8(const Raw8<T>& x, const Raw8<T>& u, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; i++) {
        v[i] = (float)x[i];
        if constexpr (ACT == GEMM_OPS_ACT_RELU) v[i] = v[i] < 0.0f ? 0.0f : v[i];
        else if constexpr (ACT == GEMM_OPS_ACT_SWIGLU) v[i] = silu(v[i]) * (float)u[i];
    }
}
// L threads a row, P chunks of 8 columns a thread, R rows a workgroup.  (8192,8192) bf16 39 us, 5.2 TB/s; (4000,4000) 11.3
template <typename T, int ACT, bool WHOLE, int L, int P, int R>
__global__ __launch_bounds__(L * R) void quantize_i8_kernel(const QuantArgs a)
{
    __shared__ uint32_t most[L * R / 64];
    const int lane = threadIdx.x % L;
    const int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / L;
    const T* const x = (const T*)a.X + min(row, (int64_t)a.M - 1) * a.ldx;
    Raw8<T> xr[P], ur[P];
#pragma unroll
    for (int p = 0; p < P; p++) {
        xr[p] = load8_of<WHOLE>(x, 8 * (lane + L * p), a.N);
        if constexpr (ACT == GEMM_OPS_ACT_SWIGLU) ur[p] = load8_of<WHOLE>(x + a.N, 8 * (lane + L * p), a.N);
    }
    float v[P][8];
    uint32_t big = 0;
#pragma unroll
    for (int p = 0; p < P; p++) {
        const int c = 8 * (lane + L * p);
        xr[p] = settled<T, WHOLE>(xr[p], c, a.N);
        if constexpr (ACT == GEMM_OPS_ACT_SWIGLU) ur[p] = settled<T, WHOLE>(ur[p], c, a.N);
        activated8<T, ACT>(xr[p], ur[p], v[p]);
#pragma unroll
        for (int i = 0; i < 8; i++) big = max(big, magnitude(v[p][i]));
    }
    const RowScale s = row_scale(max_row<L>(big, most));
    if (row >= a.M) return;
    if (lane == 0) a.scale[row] = s.scale;
#pragma unroll
    for (int p = 0; p < P; p++) {
        const int c = 8 * (lane + L * p);
        if (c < a.N) store_bytes<WHOLE>(a.Q + row * a.ldq + c, a.N - c, to_i8(v[p], s));
    }
}
// rows of any length, a workgroup each, in two passes
template <typename T, int ACT>
__global__ __launch_bounds__(LONG) void quantize_i8_long_kernel(const QuantArgs a)
{
    __shared__ uint32_t most[LONG / 64];
    const int64_t row = blockIdx.x;
    const T* const x = (const T*)a.X + row * a.ldx;
    float v[8];
    auto at = [&](int64_t c) {
        const int left = (int)min((int64_t)8, a.N - c);
        const Raw8<T> xr = load8_raw(x + c, left), ur = ACT == GEMM_OPS_ACT_SWIGLU ? load8_raw(x + a.N + c, left) : xr;
        activated8<T, ACT>(xr, ur, v);
    };
    uint32_t big = 0;
    for (int64_t c = 8 * (int64_t)threadIdx.x; c < a.N; c += 8 * LONG) {
        at(c);
#pragma unroll
        for (int i = 0; i < 8; i++) big = max(big, magnitude(v[i]));
    }
    const RowScale s = row_scale(max_row<LONG>(big, most));
    if (threadIdx.x == 0) a.scale[row] = s.scale;
    for (int64_t c = 8 * (int64_t)threadIdx.x; c < a.N; c += 8 * LONG) {
        at(c);
        store_bytes(a.Q + row * a.ldq + c, (int)(a.N - c), to_i8(v, s));
    }
}
template <typename T, int ACT, int L, int P, int R>
int launch_quant(const QuantArgs& a, hipStream_t stream)
{
    const dim3 grid((unsigned)(((int64_t)a.M + R - 1) / R));
    if (a.N % 8 == 0) hipLaunchKernelGGL((quantize_i8_kernel<T, ACT, true, L, P, R>), grid, dim3(L * R), 0, stream, a);
    else hipLaunchKernelGGL((quantize_i8_kernel<T, ACT, false, L, P, R>), grid, dim3(L * R), 0, stream, a);
    return launched();
}
template <typename T, int ACT>
int quant_of_act(const QuantArgs& a, hipStream_t stream)
{
    if (a.M <= 2 * chip().cus && a.N > 2048 && a.N <= 8192) return launch_quant<T, ACT, 1024, 1, 1>(a, stream);
    if (a.N <= 64) return launch_quant<T, ACT, 8, 1, 32>(a, stream);
    if (a.N <= 128) return launch_quant<T, ACT, 16, 1, 16>(a, stream);
    if (a.N <= 256) return launch_quant<T, ACT, 32, 1, 8>(a, stream);
    if (a.N <= 512) return launch_quant<T, ACT, 64, 1, 4>(a, stream);
    if (a.N <= 1024) return launch_quant<T, ACT, 64, 2, 4>(a, stream);
    if (a.N <= 2048) return launch_quant<T, ACT, 64, 4, 4>(a, stream);
    if (a.N <= 4096) return launch_quant<T, ACT, 256, 2, 1>(a, stream);
    if (a.N <= 8192) return launch_quant<T, ACT, 256, 4, 1>(a, stream);
    if (a.N <= 16384) return launch_quant<T, ACT, 512, 4, 1>(a, stream);
    hipLaunchKernelGGL((quantize_i8_long_kernel<T, ACT>), dim3((unsigned)a.M), dim3(LONG), 0, stream, a);
    return launched();
}
template <typename T>
int quant_of_type(const QuantArgs& a, hipStream_t stream)
{
    return a.act == GEMM_OPS_ACT_NONE ? quant_of_act<T, GEMM_OPS_ACT_NONE>(a, stream) :
           a.act == GEMM_OPS_ACT_RELU ? quant_of_act<T, GEMM_OPS_ACT_RELU>(a, stream) : quant_of_act<T, GEMM_OPS_ACT_SWIGLU>(a, stream);
}

}  // namespace

int ops_layer_norm_grad_parts(int64_t M, int64_t N)
{
    const int64_t rows = grad_rows(N), g = (M + rows - 1) / rows;
    return (int)(g < 256 ? g : 256);
}
int ops_launch_layer_norm(int type, const LayerNormArgs& all, hipStream_t stream)
{
    int rc = GEMM_F16_OK;
    for (int64_t i = 0; i < all.M && rc == GEMM_F16_OK; i += LAUNCH_ROWS) {
        LayerNormArgs a = all;
        a.M = (int)(all.M - i < LAUNCH_ROWS ? all.M - i : LAUNCH_ROWS);
        a.X = (const half_t*)all.X + i * all.ldx;                          // both types have 2 bytes
        if (a.R) a.R = (const half_t*)all.R + i * all.ldr;
        if (a.H) a.H = (half_t*)all.H + i * all.ldh;
        if (a.Y) a.Y = (half_t*)all.Y + i * all.ldy;
        if (a.Q) { a.Q += i * all.ldq; a.scale += i; }
        if (a.mean) a.mean += i;
        if (a.rstd) a.rstd += i;
        rc = type == GEMM_TYPE_F16 ? norm_of_type<half_t>(a, stream) : norm_of_type<bf16_t>(a, stream);
    }
    return rc;
}
int ops_launch_layer_norm_grad(int type, const LayerNormGradArgs& a, hipStream_t stream) { return type == GEMM_TYPE_F16 ? norm_grad_of_type<half_t>(a, stream) : norm_grad_of_type<bf16_t>(a, stream); }
int ops_launch_quant_i8(int type, const QuantArgs& all, hipStream_t stream)
{
    int rc = GEMM_F16_OK;
    for (int64_t i = 0; i < all.M && rc == GEMM_F16_OK; i += LAUNCH_ROWS) {
        QuantArgs a = all;
        a.M = (int)(all.M - i < LAUNCH_ROWS ? all.M - i : LAUNCH_ROWS);
        a.X = (const half_t*)all.X + i * all.ldx;
        a.Q += i * all.ldq;
        a.scale += i;
        rc = type == GEMM_TYPE_F16 ? quant_of_type<half_t>(a, stream) : quant_of_type<bf16_t>(a, stream);
    }
    return rc;
}
