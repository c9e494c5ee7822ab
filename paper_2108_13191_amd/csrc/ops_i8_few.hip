// Products of 8-bit integers (include/gemm_layer.h) whose tiles of 128 x 128 would leave compute units idle: 16 FM x 16 NB results a workgroup, whose wavefronts take the k steps
// of 128 bytes in turn, each through S stages of its own in LDS, and add their sums there at the end.  No barrier before that.
//
// Bound by what a compute unit loads, (FM + NB) * 16 rows of K bytes a tile.  Loaded straight into registers, as fragments have them, neighbouring lanes read different rows, and a
// load of 1 KB takes the 64 cycles of 64 requests: 16 bytes a cycle whatever is asked for ahead (16 to 64 k steps).  Copied to LDS eight lanes read one row's 128 bytes, and
// fragments come from there: twice to three times that.  us, here | by registers: (16,8192,8192) 12.2 | 14.4, (16,1000,16384) 7.9 | 16.8, (64,8192,8192) 14.0 | 25.5 (from memory 13.5),
// (256,4096,16384) 26 | 88, (700,1000,16384) 25 | 88, (300,300,300) 3.2 | 3.2.  128 x 64 in one stage, as a wavefront's products (64 MFMAs) are as long as the copies of its next
// step: (400,4096,16384) 39 to 42 us by the card, 64 x 64 in two rounds 48, 128 x 128 of the tiled kernel 60.  Tried: three and four stages, twice or half the wavefronts, 32 x 128, 64 x 128 and 128 x 128 tiles: no faster.
#include "ops_tile.h"

namespace {

using namespace ops_tile;

typedef uintx4 uintx4_any __attribute__((aligned(1)));

template <int N> __device__ __forceinline__ void wait_copies() { asm volatile("s_waitcnt vmcnt(%0)" :: "n"(N) : "memory"); }

// S = 0: operands of any alignment, a k step ahead in registers and one stage in LDS.  us, here | the kernel for any alignment of ops_generic.hip: 16 rows of (8192,8190) 15.0 | 541,
// (300,700,1100) 5.6 | 70, (2000,2000,2001) 35 | 365, (4000,4000,4001) 208 | 3165
template <int FM, int NB, int WAVES, int S, typename CT>
__global__ __launch_bounds__(64 * WAVES) void ops_i8_few_kernel(const OpsGemm g)
{
    constexpr bool ANY = S == 0;
    constexpr int BM = 16 * FM, BN = 16 * NB, COPIES = 2 * (FM + NB), STAGE = COPIES * 1024, RING = (ANY ? 1 : S) * STAGE;
    constexpr int PASS = FM * NB * 1024 <= RING ? FM * NB : FM * NB / 2;       // blocks of sums that a ring holds
    static_assert(PASS * 1024 <= RING && FM * NB % PASS == 0 && WAVES * RING <= 160 * 1024 && S <= 2);
    __shared__ __attribute__((aligned(1024))) char smem[WAVES * RING];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, q = lane >> 4;
    const uint32_t smem_base = (uint32_t)(uintptr_t)(lds_ptr_t)smem, ring = smem_base + wave * RING;

    const TileAt t = find_tile<BM, BN>(g);
    if (!t.valid) return;
    const int K = g.K, k_full = K / STEP, left = K % STEP;
    const char* const a_tile = g.A + (int64_t)t.row0 * g.lda;
    const char* const b_tile = g.B + ((int64_t)t.e * g.b_stride + (int64_t)t.n0 * g.ldb);
    const int a_last = t.row_end - t.row0 - 1, b_last = g.N - t.n0 - 1;

    // a copy is 8 rows of 128 bytes; lane l's 16 bytes are chunk (l % 8) ^ (row / 2) % 8 of row l / 8, so that the reads of 16 rows' chunks below meet no bank twice
    uint32_t off[COPIES];
#pragma unroll
    for (int i = 0; i < COPIES; i++) {
        const int r = 8 * (i < 2 * FM ? i : i - 2 * FM) + (lane >> 3);
        off[i] = (uint32_t)min(r, i < 2 * FM ? a_last : b_last) * (uint32_t)(i < 2 * FM ? g.lda : g.ldb) + 16u * ((lane & 7) ^ ((r >> 1) & 7));
    }
    auto copy = [&](int k, uint32_t stage) {
        const char *const ap = a_tile + (int64_t)k * STEP, *const bp = b_tile + (int64_t)k * STEP;
#pragma unroll
        for (int i = 0; i < COPIES; i++) async_copy16(i < 2 * FM ? ap : bp, off[i], stage + 1024 * i);
    };
    floatx4 acc[FM][NB];
#pragma unroll
    for (int m = 0; m < FM; m++)
#pragma unroll
        for (int n = 0; n < NB; n++) acc[m][n] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};
    Frag a[FM], b[NB];
    auto multiply = [&] {
#pragma unroll
        for (int m = 0; m < FM; m++)
#pragma unroll
            for (int n = 0; n < NB; n++) acc[m][n] = mfma_step<ELEM_I8>(b[n], a[m], acc[m][n]);
    };
    const uint32_t rd0 = l16 * STEP + 16 * (q ^ (l16 >> 1)), rd1 = l16 * STEP + 16 * ((4 + q) ^ (l16 >> 1));
    auto get = [&](uint32_t at) { return *(__attribute__((address_space(3))) const uintx4*)(uintptr_t)at; };
    auto read = [&](uint32_t stage) {
#pragma unroll
        for (int m = 0; m < FM; m++) { a[m].lo = get(stage + m * 2048 + rd0); a[m].hi = get(stage + m * 2048 + rd1); }
#pragma unroll
        for (int n = 0; n < NB; n++) { b[n].lo = get(stage + (FM + n) * 2048 + rd0); b[n].hi = get(stage + (FM + n) * 2048 + rd1); }
    };

    if constexpr (ANY) {
        uintx4 v[COPIES];                                                     // the next step
        auto fetch = [&](int k) {
            const char *const ap = a_tile + (int64_t)k * STEP, *const bp = b_tile + (int64_t)k * STEP;
#pragma unroll
            for (int i = 0; i < COPIES; i++) v[i] = *(const uintx4_any*)((i < 2 * FM ? ap : bp) + off[i]);
        };
        if (wave < k_full) fetch(wave);
        for (int k = wave; k < k_full; k += WAVES) {
#pragma unroll
            for (int i = 0; i < COPIES; i++) *(__attribute__((address_space(3))) uintx4*)(uintptr_t)(ring + 1024 * i + 16 * lane) = v[i];
            wave_exchange();
            if (k + WAVES < k_full) fetch(k + WAVES);
            read(ring);
            wave_exchange();
            multiply();
        }
    } else {
        uint32_t stage = ring, other = ring + (S - 1) * STAGE;
        if (wave < k_full) copy(wave, stage);
        if (S > 1 && wave + WAVES < k_full) copy(wave + WAVES, other);
        for (int k = wave; k < k_full; k += WAVES) {
            if (S > 1 && k + WAVES < k_full) wait_copies<COPIES>();           // the next step's may be on their way
            else                             wait_copies<0>();
            read(stage);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");                // before the stage is written again
            if (k + S * WAVES < k_full) copy(k + S * WAVES, stage);
            const uint32_t s = stage;
            stage = other;
            other = s;
            multiply();
        }
    }
    if (left > 0 && k_full % WAVES == wave) {                                 // the short last step, straight into registers: zeros behind K
        auto chunk = [&](const char* p, int n) {
            uintx4 v = {0u, 0u, 0u, 0u};
            if constexpr (ANY) {                                              // nothing behind the row's end is read: its last 16 bytes, moved down, or byte by byte
                if (n >= 16) v = *(const uintx4_any*)p;
                else if (n > 0 && K >= 16) {
                    typedef uint64_t pair __attribute__((ext_vector_type(2)));
                    const pair x = __builtin_bit_cast(pair, *(const uintx4_any*)(p - (16 - n)));
                    const int s = 8 * (16 - n);
                    v = __builtin_bit_cast(uintx4, s >= 64 ? pair{x[1] >> (s - 64), 0ull} : pair{(x[0] >> s) | (x[1] << (64 - s)), x[1] >> s});
                } else
                    for (int i = 0; i < n; i++) v[i >> 2] |= (uint32_t)(uint8_t)p[i] << (8 * (i & 3));
                return v;
            }
            if (n > 0) {
                v = *(const uintx4*)p;
#pragma unroll
                for (int w = 0; w < 4; w++) { const int m = n - 4 * w; v[w] = m >= 4 ? v[w] : m <= 0 ? 0u : v[w] & ((1u << (8 * m)) - 1u); }
            }
            return v;
        };
        const int64_t at = (int64_t)k_full * STEP + 16 * q;
#pragma unroll
        for (int n = 0; n < NB; n++) { const char* const p = b_tile + (int64_t)min(16 * n + l16, b_last) * g.ldb + at; b[n].lo = chunk(p, left - 16 * q); b[n].hi = chunk(p + 64, left - 16 * q - 64); }
#pragma unroll
        for (int m = 0; m < FM; m++) { const char* const p = a_tile + (int64_t)min(16 * m + l16, a_last) * g.lda + at; a[m].lo = chunk(p, left - 16 * q); a[m].hi = chunk(p + 64, left - 16 * q - 64); }
        multiply();
    }

    // ---- the wavefronts' sums: each into its ring, then each adds some of the 16 x 16 blocks -----------------------------------
    auto sums = [&](int w, int block) { return (__attribute__((address_space(3))) floatx4*)(uintptr_t)(smem_base + w * RING + block * 1024 + 16 * lane); };
#pragma unroll
    for (int p0 = 0; p0 < FM * NB; p0 += PASS) {
        if (p0) __syncthreads();
#pragma unroll
        for (int i = 0; i < PASS; i++) *sums(wave, i) = acc[(p0 + i) / NB][(p0 + i) % NB];
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PASS; i += WAVES) {
            const int block = p0 + i + wave;
            if (i + wave >= PASS) break;
            intx4 sum = __builtin_bit_cast(intx4, *sums(0, i + wave));
#pragma unroll
            for (int w = 1; w < WAVES; w++) sum += __builtin_bit_cast(intx4, *sums(w, i + wave));
            const int row = t.row0 + 16 * (block / NB) + l16, col = t.n0 + 16 * (block % NB) + 4 * q;
            if (row >= t.row_end) continue;
            const float rs = g.sa[row];
            const float* const cs = g.sb + (int64_t)t.e * g.sb_stride;
            floatx4 v;
#pragma unroll
            for (int e = 0; e < 4; e++) v[e] = scaled_column((float)sum[e] * rs, cs[min(col + e, g.N - 1)]);
            CT* const dst = (CT*)g.C + (int64_t)row * g.ldc + col;
            if (col + 4 <= g.N) {
                typename CVec4<CT>::type o;
#pragma unroll
                for (int e = 0; e < 4; e++) o[e] = (CT)v[e];
                *(typename CVec4<CT>::type*)dst = o;
            } else {
#pragma unroll
                for (int e = 0; e < 4; e++) if (col + e < g.N) dst[e] = (CT)v[e];
            }
        }
    }
}

template <int FM, int NB, int WAVES, int S = 2>
int launch_few(const OpsGemm& g)
{
    const int64_t grid = tile_grid(g, 16 * FM, 16 * NB);
    if (grid < 0 || !fits_a_launch(grid, 64 * WAVES)) return GEMM_F16_ERR_SIZE;
    if (g.c_type == ELEM_F32)      hipLaunchKernelGGL((ops_i8_few_kernel<FM, NB, WAVES, S, float>), dim3((unsigned)grid), dim3(64 * WAVES), 0, g.stream, g);
    else if (g.c_type == ELEM_F16) hipLaunchKernelGGL((ops_i8_few_kernel<FM, NB, WAVES, S, half_t>), dim3((unsigned)grid), dim3(64 * WAVES), 0, g.stream, g);
    else                           hipLaunchKernelGGL((ops_i8_few_kernel<FM, NB, WAVES, S, bf16_t>), dim3((unsigned)grid), dim3(64 * WAVES), 0, g.stream, g);
    return hipGetLastError() == hipSuccess ? GEMM_F16_OK : GEMM_F16_ERR_LAUNCH;
}

}  // namespace

int ops_launch_few_i8_any(const OpsGemm& g, int fm) { return fm == 2 ? launch_few<2, 2, 4, 0>(g) : launch_few<4, 4, 4, 0>(g); }
int ops_launch_few_i8(const OpsGemm& g, int fm, int nb)
{
    if (fm == 1) return nb == 1 ? launch_few<1, 1, 8>(g) : launch_few<1, 4, 4>(g);
    if (fm == 2) return nb == 1 ? launch_few<2, 1, 8>(g) : nb == 2 ? launch_few<2, 2, 4>(g) : launch_few<2, 4, 4>(g);
    return fm == 4 ? launch_few<4, 4, 4>(g) : launch_few<8, 4, 4, 1>(g);
}
