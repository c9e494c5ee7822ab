// Few rows against large e4m3 matrices (include/gemm_ops.h): 16 FM x 16 NB results a
// workgroup, whose eight wavefronts take the k steps of 128 bytes in turn and add their sums in LDS at the end.
//
// Such products are bound by streaming B once: each lane loads its fragments of a k step straight into registers (4 lanes cover the 128
// bytes of a row) and multiplies them.  No LDS, no barrier before the end; what keeps the memory busy is that 16 to 32 wavefronts
// a compute unit do so.  (A ring of 2 to 6 steps in registers ahead of the multiplication, with fewer wavefronts: (16,8192,8192) e4m3
// 13.9 to 19.9 us against 13.7, 64 rows of 16 experts (4096,2048) 29.5 to 57 against 26.3.)  e4m3 values are widened to f16: the matrix
// rate does not matter here.  Measured: (16,8192,8192) 16.2 us from memory, 4.2 TB/s, 13.5 where B (67 MB) is still in the 256 MB memory-side cache; 64 rows of 16
// experts (4096,2048) 26 to 29 us, 4.6 to 5.1 TB/s.  More rows a workgroup
// than 32 make A's reads, once for each 32 columns, the bound: 32 rows each of 16 experts 75 us with 64, 56 with 32.
#include "ops_tile.h"

namespace {

using namespace ops_tile;

constexpr int WAVES = 8;      // (16 for the fewest workgroups: no faster)

// OCC: wavefronts a SIMD that the registers leave room for
template <int FM, int NB, int OCC, typename CT>
__global__ __launch_bounds__(64 * WAVES, OCC) void ops_skinny_kernel(const OpsGemm g)
{
    constexpr int BM = 16 * FM, BN = 16 * NB;
    __shared__ floatx4 sums[WAVES][FM * NB][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, q = lane >> 4;

    const TileAt t = find_tile<BM, BN>(g);
    if (!t.valid) return;
    const int K = g.K, KT = (K + STEP - 1) / STEP, k_full = K / STEP;

    // rows behind the end of the group or of B are read from the last one and never stored
    const char* const a_tile = g.A + (int64_t)t.row0 * g.lda;
    const char* const b_tile = g.B + ((int64_t)t.e * g.b_stride + (int64_t)t.n0 * g.ldb);
    uint32_t a_off[FM], b_off[NB], s_off[FM];
#pragma unroll
    for (int m = 0; m < FM; m++) {
        const int row = min(16 * m + l16, t.row_end - t.row0 - 1);
        a_off[m] = (uint32_t)row * (uint32_t)g.lda + 16u * q;
        s_off[m] = (uint32_t)row;
    }
#pragma unroll
    for (int n = 0; n < NB; n++) b_off[n] = (uint32_t)min(16 * n + l16, g.N - t.n0 - 1) * (uint32_t)g.ldb + 16u * q;
    const float* const sa = g.sa + t.row0;
    const float* const sb = g.sb + (int64_t)t.e * g.sb_stride + (int64_t)(t.n0 / 128) * g.ld_sb;

    floatx4 acc[FM][NB];
#pragma unroll
    for (int m = 0; m < FM; m++)
#pragma unroll
        for (int n = 0; n < NB; n++) acc[m][n] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};

    struct Step { Frag a[FM], b[NB]; float sa[FM], sb; };
    auto load = [&](Step& x, int k) {
        const char *const ap = a_tile + (int64_t)k * STEP, *const bp = b_tile + (int64_t)k * STEP;
#pragma unroll
        for (int n = 0; n < NB; n++) { x.b[n].lo = *(const uintx4*)(bp + b_off[n]); x.b[n].hi = *(const uintx4*)(bp + b_off[n] + 64); }
#pragma unroll
        for (int m = 0; m < FM; m++) { x.a[m].lo = *(const uintx4*)(ap + a_off[m]); x.a[m].hi = *(const uintx4*)(ap + a_off[m] + 64); }
        x.sb = sb[k];
#pragma unroll
        for (int m = 0; m < FM; m++) x.sa[m] = sa[(int64_t)k * g.ld_sa + s_off[m]];
    };
    auto load_tail = [&](Step& x, int k) {                                   // the short last step: zeros behind K
        const char *const ap = a_tile + (int64_t)k * STEP, *const bp = b_tile + (int64_t)k * STEP;
        auto chunk = [&](const char* p, int left) {
            uintx4 v = {0u, 0u, 0u, 0u};
            if (left > 0) {
                v = *(const uintx4*)p;
#pragma unroll
                for (int w = 0; w < 4; w++) { const int n = left - 4 * w; v[w] = n >= 4 ? v[w] : n <= 0 ? 0u : v[w] & ((1u << (8 * n)) - 1u); }
            }
            return v;
        };
        const int left = K - k * STEP - 16 * q;
#pragma unroll
        for (int n = 0; n < NB; n++) { x.b[n].lo = chunk(bp + b_off[n], left); x.b[n].hi = chunk(bp + b_off[n] + 64, left - 64); }
#pragma unroll
        for (int m = 0; m < FM; m++) { x.a[m].lo = chunk(ap + a_off[m], left); x.a[m].hi = chunk(ap + a_off[m] + 64, left - 64); }
        x.sb = sb[k];
#pragma unroll
        for (int m = 0; m < FM; m++) x.sa[m] = sa[(int64_t)k * g.ld_sa + s_off[m]];
    };
    auto multiply = [&](const Step& x) {
#pragma unroll
        for (int m = 0; m < FM; m++)
#pragma unroll
            for (int n = 0; n < NB; n++) {
                const floatx4 p = mfma_step(widened(x.b[n]), widened(x.a[m]));
#pragma unroll
                for (int e = 0; e < 4; e++) acc[m][n][e] = __builtin_fmaf(p[e], x.sa[m] * x.sb, acc[m][n][e]);
            }
    };

    Step x;
    for (int k = wave; k < k_full; k += WAVES) { load(x, k); multiply(x); }
    if (k_full < KT && k_full % WAVES == wave) { load_tail(x, k_full); multiply(x); }

    // ---- the wavefronts' sums, in their order -----------------------------------------------------------------------------
#pragma unroll
    for (int m = 0; m < FM; m++)
#pragma unroll
        for (int n = 0; n < NB; n++) sums[wave][m * NB + n][lane] = acc[m][n];
    __syncthreads();
    const int block = wave;                                                  // wavefront w adds block w of 16 x 16
    if (block >= FM * NB) return;
    floatx4 v = sums[0][block][lane];
#pragma unroll
    for (int w = 1; w < WAVES; w++) v += sums[w][block][lane];
    const int row = t.row0 + 16 * (block / NB) + l16, col = t.n0 + 16 * (block % NB) + 4 * q;
    if (row >= t.row_end) return;
    CT* const dst = (CT*)g.C + (int64_t)t.e * g.c_stride + (int64_t)row * g.ldc + col;
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

template <int FM, int NB, int OCC>
int launch_skinny(const OpsGemm& g)
{
    static_assert(FM * NB <= WAVES, "a wavefront adds one block");
    const int64_t grid = tile_grid(g, 16 * FM, 16 * NB);
    if (grid < 0 || !fits_a_launch(grid, 64 * WAVES)) return GEMM_F16_ERR_SIZE;
    if (g.c_type == ELEM_F32)      hipLaunchKernelGGL((ops_skinny_kernel<FM, NB, OCC, float>), dim3((unsigned)grid), dim3(64 * WAVES), 0, g.stream, g);
    else if (g.c_type == ELEM_F16) hipLaunchKernelGGL((ops_skinny_kernel<FM, NB, OCC, half_t>), dim3((unsigned)grid), dim3(64 * WAVES), 0, g.stream, g);
    else                           hipLaunchKernelGGL((ops_skinny_kernel<FM, NB, OCC, bf16_t>), dim3((unsigned)grid), dim3(64 * WAVES), 0, g.stream, g);
    return hipGetLastError() == hipSuccess ? GEMM_F16_OK : GEMM_F16_ERR_LAUNCH;
}

}  // namespace

int ops_launch_skinny_e4m3(const OpsGemm& g, int fm, int nb)
{
    if (fm == 1) return nb == 1 ? launch_skinny<1, 1, 8>(g) : launch_skinny<1, 2, 4>(g);
    return nb == 1 ? launch_skinny<2, 1, 6>(g) : nb == 2 ? launch_skinny<2, 2, 4>(g) : launch_skinny<2, 4, 3>(g);
}
