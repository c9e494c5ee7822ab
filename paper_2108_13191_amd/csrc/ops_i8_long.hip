// Large products of 8-bit integers (include/gemm_layer.h): 256 x 256 results a workgroup of FOUR wavefronts, each of which owns 128 x 128 of them -- 8 x 8 accumulators of
// 16 x 16, the whole AccVGPR file -- with the k loop in assembly (ops_i8_loop.inc, written by gen_i8_loop.py, which documents the schedule).
//
// Why this shape: 8-bit MFMAs are twice as fast as 16-bit ones on the same bytes, so that with eight wavefronts of 128 x 64 (ops_tile.h) the reads of fragments from
// LDS take as long as the MFMAs; here A is read by two wavefronts instead of four, which leaves LDS a quarter of its time.  Measured: a k step (128 k) of a tile 1.35 us against 1.53;
// 8192^3 to bf16 366 to 396 us by the card, 2.8 to 3.0 POPS; on one of them 394, with f32 results 391 (436 and 425 there).  MFMAs alone run at 3.9 POPS on such operands, at 4.8 on zeros: the chip's power.  What a tile takes around its
// loop, 10 to 11 us, is stores of all compute units at once and latency that one wavefront a SIMD does not hide.  Tried: results straight from the registers, 64 bytes of a row a
// store (8192^3 f32 460, (8192,8192,1024) 114 against 93 through LDS).
#include "ops_tile.h"
#include "ops_i8_loop.inc"

namespace {

using namespace ops_tile;

constexpr int BT = 256, NCOPY = 8;                         // tile; copies of 1 KB of a wavefront, buffer and k step
constexpr int A_BUF = BT * STEP, B_REGION = 2 * A_BUF, LDS_BYTES = 5 * A_BUF;      // 2 A and 3 B buffers of 32 KB

__device__ __forceinline__ uint32_t uniform(uint32_t x) { return __builtin_amdgcn_readfirstlane(x); }

template <typename CT, int W> struct StoreOf { typedef CT type __attribute__((ext_vector_type(W), aligned(sizeof(CT)))); };

template <typename CT>
__global__ __launch_bounds__(256) void ops_i8_long_kernel(const OpsGemm g)
{
    __shared__ __attribute__((aligned(1024))) char smem[LDS_BYTES];
    const uint32_t smem_base = (uint32_t)(uintptr_t)(lds_ptr_t)smem;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = (wave >> 1) * 128, wn = (wave & 1) * 128, l16 = lane & 15, q = lane >> 4;

    const TileAt t = find_tile<BT, BT>(g);
    if (!t.valid) return;
    const int left = g.K % STEP;                           // of the sum, behind its last whole k step (there is one at least)
    const uint32_t kt = uniform((uint32_t)(g.K / STEP + (left > 0)));

    // copies: the LDS image of ops_tile.h.  Copy c = wave + 4 i is 8 rows of 128 bytes; lane l writes row 8 c + l / 8, chunk l % 8, which holds chunk (l % 8) ^ (row / 2) % 8.
    // Rows behind the end of the group or of B are loaded from the last one and never stored.
    const int a_rows = t.row_end - t.row0, b_rows = g.N - t.n0;
    const int chunk = (lane & 7) ^ (4 * (wave & 1) + (lane >> 4));
    uint32_t a_off[NCOPY], b_off[NCOPY];
#pragma unroll
    for (int i = 0; i < NCOPY; i++) {
        const int row = 8 * (wave + 4 * i) + (lane >> 3);
        a_off[i] = (uint32_t)min(row, a_rows - 1) * (uint32_t)g.lda + 16u * chunk;
        b_off[i] = (uint32_t)min(row, b_rows - 1) * (uint32_t)g.ldb + 16u * chunk;
    }
    const char* const a_tile = g.A + (int64_t)t.row0 * g.lda;
    const char* const b_tile = g.B + ((int64_t)t.e * g.b_stride + (int64_t)t.n0 * g.ldb);
    const uint32_t lds_wave = smem_base + 1024 * wave;

    uint32_t a_rd[2], b_rd[2];
#pragma unroll
    for (int s = 0; s < 2; s++) {
        const uint32_t at = l16 * STEP + 16 * ((4 * s + q) ^ (l16 >> 1));
        a_rd[s] = smem_base + wm * STEP + at;
        b_rd[s] = smem_base + B_REGION + wn * STEP + at;
    }

    // C goes through LDS, a lane's four columns and their scales, asked for in front of the loop
    const int col = t.n0 + wn + 4 * (lane & 31);
    const float* const cs = g.sb + (int64_t)t.e * g.sb_stride;
    floatx4 col_scale;
#pragma unroll
    for (int e = 0; e < 4; e++) col_scale[e] = cs[min(col + e, g.N - 1)];
    const int row_first = t.row0 + wm;
    float row_scale[8];                                    // of row 16 m + l16
#pragma unroll
    for (int m = 0; m < 8; m++) row_scale[m] = g.sa[min(row_first + 16 * m + l16, t.row_end - 1)];

    // K steps in any order, as sums of integers are exact: the short one, if there is one, is the second, through registers with zeros behind the end of the sum.  The first two
    // are brought here, the loop copies from then on.
    auto stage = [&](int s) {                              // whole k step s into the s-th buffers
#pragma unroll
        for (int i = 0; i < NCOPY; i++) {
            async_copy16(a_tile + s * STEP, a_off[i], lds_wave + s * A_BUF + 4096 * i);
            async_copy16(b_tile + s * STEP, b_off[i], lds_wave + B_REGION + s * A_BUF + 4096 * i);
        }
    };
    if (left > 0) {
        const int64_t at = (int64_t)(g.K / STEP) * STEP;
        const int mine = left - 16 * chunk;                // bytes of this lane's chunks within the sum
        uintx4 a[NCOPY], b[NCOPY];
#pragma unroll
        for (int i = 0; i < NCOPY; i++) {
            a[i] = b[i] = uintx4{0u, 0u, 0u, 0u};
            if (mine > 0) { a[i] = *(const uintx4*)(a_tile + at + a_off[i]); b[i] = *(const uintx4*)(b_tile + at + b_off[i]); }
        }
        stage(0);
        auto put = [&](uint32_t dst, uintx4 v) {
#pragma unroll
            for (int w = 0; w < 4; w++) { const int n = mine - 4 * w; v[w] = n >= 4 ? v[w] : n <= 0 ? 0u : v[w] & ((1u << (8 * n)) - 1u); }
            *(__attribute__((address_space(3))) uintx4*)(uintptr_t)(dst + 16 * lane) = v;
        };
#pragma unroll
        for (int i = 0; i < NCOPY; i++) { put(lds_wave + A_BUF + 4096 * i, a[i]); put(lds_wave + B_REGION + A_BUF + 4096 * i, b[i]); }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (the loop leaves 16 copies of a second k step out)
    } else {
        stage(0);
        if (kt > 1) stage(1);
    }
    const int skipped = left > 0 ? 1 : 0;
    const uint64_t a_base = (uint64_t)(uintptr_t)a_tile, b_base = (uint64_t)(uintptr_t)b_tile, a_ptr = a_base + (2 - skipped) * STEP, b_ptr = b_base + (2 - skipped) * STEP;
    const uint32_t a_base_lo = uniform((uint32_t)a_base), a_base_hi = uniform((uint32_t)(a_base >> 32)), b_base_lo = uniform((uint32_t)b_base), b_base_hi = uniform((uint32_t)(b_base >> 32));
    const uint32_t a_ptr_lo = uniform((uint32_t)a_ptr), a_ptr_hi = uniform((uint32_t)(a_ptr >> 32)), b_ptr_lo = uniform((uint32_t)b_ptr), b_ptr_hi = uniform((uint32_t)(b_ptr >> 32));
    floatx4 acc[8][8];                                     // 32-bit integers
    asm volatile(I8_LOOP_ASM : I8_LOOP_OUTPUTS(acc) : I8_LOOP_INPUTS : I8_LOOP_CLOBBERS);

    // ---- to C: 32 rows of a wavefront at a time through LDS, so that whole row segments are stored
    __builtin_amdgcn_s_barrier();                          // no wavefront's copies are on their way into LDS
    asm volatile("" ::: "memory");
    constexpr int PITCH = 128 * 4 + 16;
    const uint32_t buf = smem_base + wave * (32 * PITCH);
    CT* const C = (CT*)g.C + (int64_t)(row_first + (lane >> 5)) * g.ldc + col;
    const int rows = t.row_end - row_first - (lane >> 5);  // of this lane's, every second one
    typedef typename CVec4<CT>::type ctx4;
#pragma unroll
    for (int m2 = 0; m2 < 4; m2++) {
#pragma unroll
        for (int r = 0; r < 2; r++)
#pragma unroll
            for (int n = 0; n < 8; n++) {
                floatx4 v;
#pragma unroll
                for (int e = 0; e < 4; e++) v[e] = scaled_sum(acc[2 * m2 + r][n][e], row_scale[2 * m2 + r]);
                *(__attribute__((address_space(3))) floatx4*)(uintptr_t)(buf + (16 * r + l16) * PITCH + (16 * n + 4 * q) * 4) = v;
            }
        wave_exchange();
#pragma unroll
        for (int p = 0; p < 16; p++) {
            floatx4 v = *(__attribute__((address_space(3))) const floatx4*)(uintptr_t)(buf + (2 * p + (lane >> 5)) * PITCH + 16 * (lane & 31));
#pragma unroll
            for (int e = 0; e < 4; e++) v[e] = scaled_column(v[e], col_scale[e]);
            const int r = 32 * m2 + 2 * p;
            if (r >= rows) continue;
            CT* const dst = C + (int64_t)r * g.ldc;
            if (col + 4 <= g.N) {
                ctx4 o;
#pragma unroll
                for (int e = 0; e < 4; e++) o[e] = (CT)v[e];
                __builtin_nontemporal_store(o, (ctx4*)dst);
            } else {
#pragma unroll
                for (int e = 0; e < 4; e++) if (col + e < g.N) dst[e] = (CT)v[e];
            }
        }
        wave_exchange();
    }
}

}  // namespace

int ops_launch_long_i8(const OpsGemm& g)
{
    const int64_t grid = tile_grid(g, BT, BT);
    if (grid < 0 || !fits_a_launch(grid, 512)) return GEMM_F16_ERR_SIZE;
    if (g.c_type == ELEM_F32)      hipLaunchKernelGGL(ops_i8_long_kernel<float>, dim3((unsigned)grid), dim3(256), 0, g.stream, g);
    else if (g.c_type == ELEM_F16) hipLaunchKernelGGL(ops_i8_long_kernel<half_t>, dim3((unsigned)grid), dim3(256), 0, g.stream, g);
    else                           hipLaunchKernelGGL(ops_i8_long_kernel<bf16_t>, dim3((unsigned)grid), dim3(256), 0, g.stream, g);
    return hipGetLastError() == hipSuccess ? GEMM_F16_OK : GEMM_F16_ERR_LAUNCH;
}
