// Layer norm with the residual's addition, its gradients, and quantisation of rows to 8-bit integers (include/gemm_layer.h).
//
// Bound by memory: a row is read once, 8 elements of 16 bits a lane and access, and stays in registers for its mean, its squares about the mean and its
// largest magnitude.
#include "ops_rows.h"
#include "../../include/gemm_layer.h"

namespace {

using namespace ops_dev;

// ---- statistics of a row -----------------------------------------------------------------------------------------------------
// Mean and sum of squares about it, of which each wavefront has those of its own elements: mean = sum of sums / N, and
// squares about the row's mean = squares about the wavefront's own + n (its mean - the row's)^2.  So one exchange serves both.
struct Moments { float mean, squares; };
// W wavefronts a row; n_of(w): elements of the row's w-th wavefront; lds: 2 floats for each wavefront of the workgroup
template <int W, typename F>
__device__ __forceinline__ Moments row_moments(float sum, float squares, int N, float* lds, F n_of)
{
    if constexpr (W == 1) return {sum / (float)N, squares};
    const int wave = threadIdx.x >> 6, first = wave / W * W;
    if ((threadIdx.x & 63) == 0) { lds[2 * wave] = sum; lds[2 * wave + 1] = squares; }
    __syncthreads();
    float total = 0.0f, out = 0.0f;
#pragma unroll
    for (int w = 0; w < W; w++) total += lds[2 * (first + w)];
    const float mean = total / (float)N;
#pragma unroll
    for (int w = 0; w < W; w++) {
        const int n = n_of(w);
        const float d = n ? lds[2 * (first + w)] / (float)n - mean : 0.0f;
        out += lds[2 * (first + w) + 1] + (float)n * d * d;
    }
    return {mean, out};
}

// the largest of a row's magnitudes over its W wavefronts; lds: a word for each wavefront of the workgroup, used for nothing else
template <int W>
__device__ __forceinline__ uint32_t max_row(uint32_t m, uint32_t* lds)
{
    m = max16(m);
    m = max(m, (uint32_t)__shfl_xor((int)m, 16));
    m = max(m, (uint32_t)__shfl_xor((int)m, 32));
    if constexpr (W > 1) {
        const int wave = threadIdx.x >> 6, first = wave / W * W;
        if ((threadIdx.x & 63) == 0) lds[wave] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < W; w++) m = max(m, lds[first + w]);
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
// W wavefronts a row, each lane with P chunks of 8 columns in registers; R rows a workgroup.  LOOP: rows of any length, whose chunks are gone
// through once for each of: the mean, the squares, the largest magnitude, the outputs.
template <typename T, int W, int P, int R, bool LOOP>
__global__ __launch_bounds__(64 * W * R) void layer_norm_kernel(const LayerNormArgs a)
{
    __shared__ float lds[3 * W * R];
    const int lane = threadIdx.x % (64 * W);
    const int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / (64 * W);
    const bool live = row < a.M;
    const T* const x = (const T*)a.X + row * a.ldx;
    const T* const r = a.R ? (const T*)a.R + row * a.ldr : nullptr;
    T* const h = a.H ? (T*)a.H + row * a.ldh : nullptr;
    auto form = [&](int64_t c, float (&o)[8]) {
        load8(x + c, (int)(a.N - c), o);
        if (r) {
            float s[8];
            load8(r + c, (int)(a.N - c), s);
#pragma unroll
            for (int i = 0; i < 8; i++) o[i] = rounded<T>(o[i] + s[i]);      // h as it is stored is what is normed
        }
    };
    // y from h, zeros behind the row's end
    auto normed = [&](float (&o)[8], int left, float mean, float rstd, const Raw8<T>& gm, const Raw8<T>& bt) {
#pragma unroll
        for (int i = 0; i < 8; i++) { const float y = (o[i] - mean) * rstd * (float)gm[i] + (float)bt[i]; o[i] = i < left ? y : 0.0f; }
    };
    auto beta_at = [&](int64_t c) { return load8_raw((const T*)a.beta + c, a.beta ? (int)(a.N - c) : 0); };
    uint32_t* const most = (uint32_t*)&lds[2 * W * R];

    if constexpr (!LOOP) {
        float v[P][8], sum = 0.0f, squares = 0.0f;
        Raw8<T> gamma[P], beta[P];                        // asked for ahead of the sums
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int c = 8 * (lane + 64 * W * p);
            if (live && c < a.N) {
                form(c, v[p]);
                gamma[p] = load8_raw((const T*)a.gamma + c, a.N - c);
                beta[p] = beta_at(c);
            } else {
#pragma unroll
                for (int i = 0; i < 8; i++) { v[p][i] = 0.0f; gamma[p][i] = beta[p][i] = (T)0.0f; }
            }
        }
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int c = 8 * (lane + 64 * W * p);
            if (h && live && c < a.N) store8(h + c, a.N - c, v[p]);
#pragma unroll
            for (int i = 0; i < 8; i++) sum += v[p][i];
        }
        auto n_of = [&](int w) {
            int n = 0;
#pragma unroll
            for (int p = 0; p < P; p++) n += min(max(a.N - 512 * (w + W * p), 0), 512);
            return n;
        };
        sum = sum64(sum);
        const int own = n_of((threadIdx.x >> 6) % W);
        const float centre = own ? sum / (float)own : 0.0f;
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int left = a.N - 8 * (lane + 64 * W * p);
#pragma unroll
            for (int i = 0; i < 8; i++) { const float d = i < left ? v[p][i] - centre : 0.0f; squares += d * d; }
        }
        const Moments m = row_moments<W>(sum, sum64(squares), a.N, lds, n_of);
        const float rstd = 1.0f / sqrtf(m.squares / (float)a.N + a.eps);
        if (live && lane == 0) {
            if (a.mean) a.mean[row] = m.mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        if (!a.Y && !a.Q) return;
        uint32_t big = 0;
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int c = 8 * (lane + 64 * W * p);
            normed(v[p], a.N - c, m.mean, rstd, gamma[p], beta[p]);
            if (a.Y && live && c < a.N) store8((T*)a.Y + row * a.ldy + c, a.N - c, v[p]);
#pragma unroll
            for (int i = 0; i < 8; i++) big = max(big, magnitude(v[p][i]));
        }
        if (!a.Q) return;
        const RowScale s = row_scale(max_row<W>(big, most));
        if (!live) return;
        if (lane == 0) a.scale[row] = s.scale;
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int c = 8 * (lane + 64 * W * p);
            if (c < a.N) store_bytes(a.Q + row * a.ldq + c, a.N - c, to_i8(v[p], s));
        }
    } else {
        static_assert(R == 1, "a workgroup has one row, which is there");
        float sum = 0.0f, squares = 0.0f, o[8];
        int own = 0;
        auto again = [&](int64_t c) { if (h) load8((const T*)h + c, (int)(a.N - c), o); else form(c, o); };
        const int64_t first = 8 * (int64_t)lane, step = 512 * W;
        for (int64_t c = first; c < a.N; c += step) {
            form(c, o);
            if (h) store8(h + c, (int)(a.N - c), o);
#pragma unroll
            for (int i = 0; i < 8; i++) sum += o[i];
        }
        sum = sum64(sum);
        auto n_of = [&](int w) {                          // whole rounds of 512 W columns, and what the last one leaves
            const int rounds = a.N / (512 * W), rest = a.N - rounds * (512 * W);
            return 512 * rounds + min(max(rest - 512 * w, 0), 512);
        };
        own = n_of(threadIdx.x >> 6);
        const float centre = own ? sum / (float)own : 0.0f;
        for (int64_t c = first; c < a.N; c += step) {
            again(c);
#pragma unroll
            for (int i = 0; i < 8; i++) { const float d = c + i < a.N ? o[i] - centre : 0.0f; squares += d * d; }
        }
        const Moments m = row_moments<W>(sum, sum64(squares), a.N, lds, n_of);
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
            normed(o, left, m.mean, rstd, load8_raw((const T*)a.gamma + c, left), beta_at(c));
        };
        for (int64_t c = first; c < a.N; c += step) {
            output(c);
            if (a.Y) store8((T*)a.Y + row * a.ldy + c, (int)(a.N - c), o);
#pragma unroll
            for (int i = 0; i < 8; i++) big = max(big, magnitude(o[i]));
        }
        if (!a.Q) return;
        const RowScale s = row_scale(max_row<W>(big, most));
        if (lane == 0) a.scale[row] = s.scale;
        for (int64_t c = first; c < a.N; c += step) {
            output(c);
            store_bytes(a.Q + row * a.ldq + c, (int)(a.N - c), to_i8(o, s));
        }
    }
}

template <typename T, int W, int P, int R, bool LOOP = false>
int launch_norm(const LayerNormArgs& a, hipStream_t stream)
{
    const unsigned grid = (unsigned)(((int64_t)a.M + R - 1) / R);
    hipLaunchKernelGGL((layer_norm_kernel<T, W, P, R, LOOP>), dim3(grid), dim3(64 * W * R), 0, stream, a);
    return hipGetLastError() == hipSuccess ? GEMM_F16_OK : GEMM_F16_ERR_LAUNCH;
}
template <typename T>
int norm_of_type(const LayerNormArgs& a, hipStream_t stream)
{
    if (a.M <= 2 * chip().cus && a.N > 2048 && a.N <= 8192) return launch_norm<T, 16, 1, 1>(a, stream);
    if (a.N <= 512) return launch_norm<T, 1, 1, 4>(a, stream);
    if (a.N <= 1024) return launch_norm<T, 1, 2, 4>(a, stream);
    if (a.N <= 2048) return launch_norm<T, 1, 4, 4>(a, stream);
    if (a.N <= 4096) return launch_norm<T, 4, 2, 1>(a, stream);
    if (a.N <= 8192) return launch_norm<T, 4, 4, 1>(a, stream);
    if (a.N <= 16384) return launch_norm<T, 8, 4, 1>(a, stream);
    return launch_norm<T, 16, 1, 1, true>(a, stream);
}

// ---- its gradients -----------------------------------------------------------------------------------------------------------------
// dX row by row; the columns' sums of dy xhat and dy stay in registers over all rows of a workgroup, which writes them as one row of the
// workspace; a second kernel adds those.  Every sum has a fixed order.
template <typename T, int W, int P, int R>
__global__ __launch_bounds__(64 * W * R) void layer_norm_grad_kernel(const LayerNormGradArgs a)
{
    extern __shared__ float dyn[];                        // 4 W R floats, then R * 512 W of sums
    const int lane = threadIdx.x % (64 * W), sub = threadIdx.x / (64 * W), wave = threadIdx.x >> 6;
    float dg[P][8] = {}, db[P][8] = {};
    Raw8<T> gamma[P];
#pragma unroll
    for (int p = 0; p < P; p++) gamma[p] = load8_raw((const T*)a.gamma + 8 * (lane + 64 * W * p), a.N - 8 * (lane + 64 * W * p));

    const int64_t step = (int64_t)gridDim.x * R;
    int slot = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * R; row0 < a.M; row0 += step) {      // the same number of trips for the whole workgroup
        const int64_t row = row0 + sub;
        const bool live = row < a.M;
        Raw8<T> dyr[P], hr[P], dhr[P];
        const float rstd = live ? a.rstd[row] : 0.0f, mean = live ? a.mean[row] : 0.0f;
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
        float s1 = 0.0f, s2 = 0.0f;                       // of g and g xhat; dy is zero behind the row's end
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float dy = (float)dyr[p][i], xhat = ((float)hr[p][i] - mean) * rstd, g = dy * (float)gamma[p][i];
                dg[p][i] += dy * xhat;
                db[p][i] += dy;
                s1 += g;
                s2 += g * xhat;
            }
        s1 = sum64(s1);
        s2 = sum64(s2);
        if constexpr (W > 1) {                            // two sets of partial sums in turn: one barrier a row
            float* const set = dyn + slot * 2 * W * R;
            if ((threadIdx.x & 63) == 0) { set[2 * wave] = s1; set[2 * wave + 1] = s2; }
            __syncthreads();
            s1 = s2 = 0.0f;
#pragma unroll
            for (int i = 0; i < W; i++) { s1 += set[2 * (wave / W * W + i)]; s2 += set[2 * (wave / W * W + i) + 1]; }
            slot ^= 1;
        }
        const float m1 = s1 / (float)a.N, m2 = s2 / (float)a.N;
        if (!live) continue;
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int c = 8 * (lane + 64 * W * p);
            if (c >= a.N) continue;
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; i++) {
                o[i] = rstd * ((float)dyr[p][i] * (float)gamma[p][i] - m1 - ((float)hr[p][i] - mean) * rstd * m2);
                if (a.dH) o[i] += (float)dhr[p][i];
            }
            store8((T*)a.dX + row * a.lddx + c, a.N - c, o);
        }
    }
    if (!a.dgamma && !a.dbeta) return;
    // sums of the workgroup's row slots, in their order, 512 W columns at a time
    float* const sums = dyn + 4 * W * R;
    const bool only = gridDim.x == 1;                     // one workgroup's sums are the result
    auto put = [&](const float (&d)[P][8], float* out) {
#pragma unroll
        for (int p = 0; p < P; p++) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < 8; i += 4) *(floatx4*)&sums[sub * 512 * W + 8 * lane + i] = floatx4{d[p][i], d[p][i + 1], d[p][i + 2], d[p][i + 3]};
            __syncthreads();
            for (int j = threadIdx.x; j < 512 * W; j += 64 * W * R) {
                const int c = 512 * W * p + j;
                float s = sums[j];
#pragma unroll
                for (int r = 1; r < R; r++) s += sums[r * 512 * W + j];
                if (c < a.N) out[c] = s;
            }
        }
    };
    if (a.dgamma) put(dg, only ? a.dgamma : a.ws + (int64_t)blockIdx.x * 2 * a.N);
    if (a.dbeta) put(db, only ? a.dbeta : a.ws + ((int64_t)blockIdx.x * 2 + 1) * a.N);
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

// dgamma[j] and dbeta[j]: sums of `parts` rows of 2 N floats of the workspace, 64 columns a workgroup, wavefront w takes rows w, w + 16, ...
__global__ __launch_bounds__(1024) void column_sums_kernel(const float* __restrict__ ws, int parts, int N, float* __restrict__ dgamma, float* __restrict__ dbeta)
{
    __shared__ float lds[16][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t c = (int64_t)blockIdx.x * 64 + lane;
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

// rows a workgroup of the gradient takes at a time
inline int grad_rows(int64_t N) { return N <= 1024 ? 16 : N <= 2048 ? 8 : N <= 4096 ? 4 : N <= 8192 ? 2 : 1; }

template <typename T, int W, int P, int R>
int launch_norm_grad(const LayerNormGradArgs& a, int parts, hipStream_t stream)
{
    hipLaunchKernelGGL((layer_norm_grad_kernel<T, W, P, R>), dim3((unsigned)parts), dim3(64 * W * R), (4 * W * R + R * 512 * W) * sizeof(float), stream, a);
    return hipGetLastError() == hipSuccess ? GEMM_F16_OK : GEMM_F16_ERR_LAUNCH;
}
template <typename T>
int norm_grad_of_type(const LayerNormGradArgs& a, hipStream_t stream)
{
    const int parts = ops_layer_norm_grad_parts(a.M, a.N);
    const bool columns = a.dgamma || a.dbeta;
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
            if (columns) hipLaunchKernelGGL(layer_norm_columns_long_kernel<T>, dim3((unsigned)(((int64_t)a.N + 2047) / 2048), (unsigned)parts), dim3(256), 0, stream, a);
            hipLaunchKernelGGL(layer_norm_grad_long_kernel<T>, dim3((unsigned)a.M), dim3(1024), 0, stream, a);
            rc = hipGetLastError() == hipSuccess ? GEMM_F16_OK : GEMM_F16_ERR_LAUNCH;
        }
        if (rc != GEMM_F16_OK) return rc;
    }
    if (!columns || (parts == 1 && a.N <= 16384)) return rc;
    hipLaunchKernelGGL(column_sums_kernel, dim3((unsigned)(((int64_t)a.N + 63) / 64), 2), dim3(1024), 0, stream, a.ws, parts, a.N, a.dgamma, a.dbeta);
    return hipGetLastError() == hipSuccess ? GEMM_F16_OK : GEMM_F16_ERR_LAUNCH;
}

// ---- rows to 8-bit integers ----------------------------------------------------------------------------------------------------------
template <typename T, int ACT>
__device__ __forceinline__ void activated8(const T* x, int64_t N, int64_t c, float (&v)[8])
{
    load8(x + c, (int)(N - c), v);
    if constexpr (ACT == GEMM_OPS_ACT_RELU) {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = v[i] < 0.0f ? 0.0f : v[i];
    } else if constexpr (ACT == GEMM_OPS_ACT_SWIGLU) {
        float u[8];
        load8(x + N + c, (int)(N - c), u);
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = silu(v[i]) * u[i];
    }
}
// W wavefronts a row, P chunks of 8 columns a lane, R rows a workgroup; LOOP: two passes over a row of any length
template <typename T, int ACT, int W, int P, int R, bool LOOP>
__global__ __launch_bounds__(64 * W * R) void quantize_i8_kernel(const QuantArgs a)
{
    __shared__ uint32_t most[W * R];
    const int lane = threadIdx.x % (64 * W);
    const int64_t row = (int64_t)blockIdx.x * R + threadIdx.x / (64 * W);
    const bool live = row < a.M;
    const T* const x = (const T*)a.X + row * a.ldx;
    uint32_t big = 0;
    if constexpr (!LOOP) {
        float v[P][8];
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int c = 8 * (lane + 64 * W * p);
            if (live && c < a.N) activated8<T, ACT>(x, a.N, c, v[p]);
            else {
#pragma unroll
                for (int i = 0; i < 8; i++) v[p][i] = 0.0f;
            }
        }
#pragma unroll
        for (int p = 0; p < P; p++)
#pragma unroll
            for (int i = 0; i < 8; i++) big = max(big, magnitude(v[p][i]));
        const RowScale s = row_scale(max_row<W>(big, most));
        if (!live) return;
        if (lane == 0) a.scale[row] = s.scale;
#pragma unroll
        for (int p = 0; p < P; p++) {
            const int c = 8 * (lane + 64 * W * p);
            if (c < a.N) store_bytes(a.Q + row * a.ldq + c, a.N - c, to_i8(v[p], s));
        }
    } else {
        static_assert(R == 1, "a workgroup has one row, which is there");
        float v[8];
        for (int64_t c = 8 * (int64_t)lane; c < a.N; c += 512 * W) {
            activated8<T, ACT>(x, a.N, c, v);
#pragma unroll
            for (int i = 0; i < 8; i++) big = max(big, magnitude(v[i]));
        }
        const RowScale s = row_scale(max_row<W>(big, most));
        if (lane == 0) a.scale[row] = s.scale;
        for (int64_t c = 8 * (int64_t)lane; c < a.N; c += 512 * W) {
            activated8<T, ACT>(x, a.N, c, v);
            store_bytes(a.Q + row * a.ldq + c, (int)(a.N - c), to_i8(v, s));
        }
    }
}
template <typename T, int ACT, int W, int P, int R, bool LOOP = false>
int launch_quant(const QuantArgs& a, hipStream_t stream)
{
    hipLaunchKernelGGL((quantize_i8_kernel<T, ACT, W, P, R, LOOP>), dim3((unsigned)(((int64_t)a.M + R - 1) / R)), dim3(64 * W * R), 0, stream, a);
    return hipGetLastError() == hipSuccess ? GEMM_F16_OK : GEMM_F16_ERR_LAUNCH;
}
template <typename T, int ACT>
int quant_of_act(const QuantArgs& a, hipStream_t stream)
{
    if (a.M <= 2 * chip().cus && a.N > 2048 && a.N <= 8192) return launch_quant<T, ACT, 16, 1, 1>(a, stream);
    if (a.N <= 512) return launch_quant<T, ACT, 1, 1, 4>(a, stream);
    if (a.N <= 1024) return launch_quant<T, ACT, 1, 2, 4>(a, stream);
    if (a.N <= 2048) return launch_quant<T, ACT, 1, 4, 4>(a, stream);
    if (a.N <= 4096) return launch_quant<T, ACT, 4, 2, 1>(a, stream);
    if (a.N <= 8192) return launch_quant<T, ACT, 4, 4, 1>(a, stream);
    if (a.N <= 16384) return launch_quant<T, ACT, 8, 4, 1>(a, stream);
    return launch_quant<T, ACT, 16, 1, 1, true>(a, stream);
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
