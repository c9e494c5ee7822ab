// The tiled kernel of the products of include/gemm_ops.h for 16-byte aligned operands: BM x BN results a workgroup, eight wavefronts,
// k steps of 128 bytes a row (128 e4m3 values, 64 of 16 bits), f32 accumulators in registers.
//
// Operands with the summed index contiguous ("k rows") are staged as rows of 128 bytes and read 16 bytes a lane; those with the
// other index contiguous as 64 k rows, read through transposing LDS reads.  Either way a fragment is 8 registers for 16 rows and a
// whole k step: one 16 x 16 x 128 MFMA in e4m3, two 16 x 16 x 32 ones in 16 bits.  (e4m3: lanes 16 q .. of an operand hold
// 16-byte chunks q and q + 4 of their row.  Which k a lane holds does not matter as long as A and B agree.)
//
// Schedule: wavefronts 0-3 (X) own the top half of the tile's rows, 4-7 (Y) the bottom half, each a quarter of the columns;
// wavefronts w and w + 4 share a SIMD.  Time is cut into phases by workgroup barriers; in a phase one group reads fragments while
// the other multiplies with every operand in registers and issues global -> LDS copies for two k steps ahead.  A k step is two
// pairs of phases: the first half of the wavefront's rows with all of its columns, then the second half.
//   X: phase 4k     reads A rows 1st half, B         Y: one phase later
//      phase 4k+1   multiplies; copies A 1st half (k+2)         (Y: and B; X may not: Y is reading B)
//      phase 4k+2   reads A rows 2nd half
//      phase 4k+3   multiplies; copies A 2nd half, B (k+2)      (Y: A 2nd half)
// Each copy overwrites what every reader read in an earlier phase, so two stages are enough: 128 KB of LDS for 256 x 256 and room
// for scales (S stages, copies S k steps ahead, for smaller tiles).  X waits for k+1 at the end of its last multiplying phase of k (the copies for
// later k steps may be on their way),
// Y, whose B rows X reads a phase earlier than Y itself, at the end of both.
//
// e4m3: each MFMA starts from zero and its 4 results are added to the accumulators times a_scale * b_scale, in f32.  With the B
// fragment first a lane holds 4 columns of one row, so the factor is one register for a block of 16 x 16; the columns of a
// wavefront lie in one block of 128, whose scale is a scalar.  The scales of the tile's rows come into LDS with the operands.
//
// Measured.  256 x 256 x 8192^2 in e4m3: 437 us, 2.5 PFLOP/s, MFMAs busy 63 % at 1.87 GHz: the chip's power (zero operands: 354 us).  Shorter sums are bound by
// what a tile does around its loop -- its group, the first copies, its stores, which all compute units do at once -- and by the last round of tiles: f16
// (16384,2304,768) of 8 experts 68 us, 24 us a round of which 11 are MFMAs; gradients (16384 rows, 2048 x 1024, 32 experts) 95 and 117 us.  Tried for those: a
// workgroup a compute unit that goes from tile to tile and requests the next one's operands before its stores, half of the workgroups
// later than the others: no faster.
#pragma once
#include <type_traits>
#include "ops_device.h"
#include "../../include/gemm_ops.h"

namespace ops_tile {

using namespace gemm_dev;
using namespace ops_dev;

typedef uintx4 frag_half;
struct Frag { uintx4 lo, hi; };                     // 8 registers: 16 rows x 128 bytes over a wavefront

__device__ __forceinline__ void copy_dword(const void* base, uint32_t byte_off, uint32_t lds_byte_addr)
{
    asm volatile("s_mov_b32 m0, %2\n\t"
                 "s_nop 0\n\t"
                 "global_load_lds_dword %0, %1"
                 :: "v"(byte_off), "s"(base), "s"(lds_byte_addr) : "memory", "m0");
}

// The same values of a fragment of e4m3 in f16 (exact): 4 slices of 8
struct Wide { half8 s[4]; };
__device__ __forceinline__ Wide widened(const Frag& f)
{
    Wide w;
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int x = (int)(i < 2 ? f.lo : f.hi)[2 * (i & 1)], y = (int)(i < 2 ? f.lo : f.hi)[2 * (i & 1) + 1];
        const half2v a = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.0f, true);
        const half2v c = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(y, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(y, 1.0f, true);
        w.s[i] = half8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
    }
    return w;
}
__device__ __forceinline__ floatx4 mfma_step(const Wide& a, const Wide& b)
{
    floatx4 c = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < 4; i++) c = __builtin_amdgcn_mfma_f32_16x16x32_f16(a.s[i], b.s[i], c, 0, 0, 0);
    return c;
}

template <int ELEM> __device__ __forceinline__ floatx4 mfma_step(const Frag& a, const Frag& b, floatx4 c)
{
    if constexpr (ELEM == ELEM_E4M3) {
        typedef uint32_t uintx8 __attribute__((ext_vector_type(8)));
        const intx8 x = __builtin_bit_cast(intx8, (uintx8)__builtin_shufflevector(a.lo, a.hi, 0, 1, 2, 3, 4, 5, 6, 7));
        const intx8 y = __builtin_bit_cast(intx8, (uintx8)__builtin_shufflevector(b.lo, b.hi, 0, 1, 2, 3, 4, 5, 6, 7));
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 0, 0, 0, 0, 0, 0);
    } else if constexpr (ELEM == ELEM_F16) {
        c = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a.lo), __builtin_bit_cast(half8, b.lo), c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a.hi), __builtin_bit_cast(half8, b.hi), c, 0, 0, 0);
    } else {
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.lo), __builtin_bit_cast(bf16x8, b.lo), c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a.hi), __builtin_bit_cast(bf16x8, b.hi), c, 0, 0, 0);
    }
}

// Where a workgroup's tile lies (uniform); valid: whether there is one for this workgroup.
struct TileAt { int e, row0, row_end, k0, k_end, n0; bool valid; };

// The l-th of tm x tn tiles, `group` rows of tiles at a time
__device__ __forceinline__ void in_order(int l, int tm, int tn, int group, int& m, int& n)
{
    group = min(group, tm);
    const int per = group * tn, g = l / per, first = g * group, rows = min(group, tm - first), r = l - g * per;
    m = first + r % rows;
    n = r / rows;
}

template <int BM, int BN>
__device__ __forceinline__ TileAt find_tile(const OpsGemm& g)
{
    const int tn = (g.N + BN - 1) / BN, pid = blockIdx.x;
    int e = 0, row0 = 0, row_end = g.M, k0 = 0, k_end = g.K, m = 0, n = 0;
    bool valid = true;
    if (g.k_ragged) {
        // Experts one after another, each dealt to all XCDs: (16384 rows, 4096 x 2048, 8 uneven experts) 425 us with an eighth of all tiles, one
        // expert's, on each XCD.  Up to 32 of them the one with the most rows first (249 us against 261, (2304 x 768) 79 against 91); with more
        // they even out, and finding out who has most costs more: (4404, 496 x 2048, 128) 144 against 118.
        const int tm = (g.M + BM - 1) / BM, per = tm * tn;
        e = g.E <= 32 ? group_by_size(g.offsets, g.E, g.K, pid / per) : pid / per;
        in_order(xcd_slice(per, g.num_xcd, pid % per), tm, tn, 8, m, n);
        group_rows(g.offsets, e, g.K, k0, k_end);
    } else if (g.offsets) {
        GroupScan s = scan_groups<BM>(g.offsets, 0, g.E, g.M);
        int total = s.total();
        for (int e0 = 64; e0 < g.E; e0 += 64) total += scan_groups<BM>(g.offsets, e0, g.E, g.M).total();
        valid = pid < total * tn;
        const int l = valid ? xcd_slice(total * tn, g.num_xcd, pid) : 0;
        int want = l / tn, e0 = 0;                                // the want-th tile of rows is one of the group's
        while (valid && want >= s.total()) {
            want -= s.total();
            e0 += 64;
            valid = e0 < g.E;                                     // (false only for offsets that overlap beyond what an int counts)
            if (valid) s = scan_groups<BM>(g.offsets, e0, g.E, g.M);
        }
        const int at = valid ? s.group_of(want) : 0;
        e = e0 + at;
        const int tiles = valid ? s.tiles_of(at) : 1;
        in_order(l - (l / tn - (want - s.before(at))) * tn, tiles, tn, 8, m, n);
        row0 = s.lo_of(at);
        row_end = s.hi_of(at);
    } else {
        const int tm = (g.M + BM - 1) / BM;
        in_order(xcd_slice(tm * tn, g.num_xcd, pid), tm, tn, 8, m, n);
    }
    auto uniform = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
    return {uniform(e), uniform(row0 + m * BM), uniform(row_end), uniform(k0), uniform(k_end), uniform(n * BN), valid};
}

// Where chunk `chunk` of k row `krow` lies in its row of CPR chunks.  Rows of 256 and 512 bytes all begin at bank 0, so the 4 k rows of a
// transposing read, and k and k + 8, are told apart in bits 1 to 3; rows of 128 bytes begin at banks 0 and 32 in turn, so k and k + 2, and
// k and k + 8, in bits 1 and 2.  Always an even change, the same for k rows 4, 16 and 32 apart.
template <int CPR> __device__ __forceinline__ int mc_chunk(int chunk, int krow)
{
    if constexpr (CPR == 8) return chunk ^ ((((krow >> 1) & 1) << 1) | (((krow >> 3) & 1) << 2));
    else                    return chunk ^ (((krow & 3) << 2) | (((krow >> 3) & 1) << 1));
}

constexpr int STEP = 128;                                  // bytes of a k row a step; 64 k rows a step in the other layout
template <int BM, int BN, int S, bool SCALED> constexpr int lds_bytes()
{
    const int stages = S * ((BM + BN) * STEP + (SCALED ? BM * 4 : 0)), out = 8 * 32 * (BN + 16);
    return stages > out ? stages : out;
}

// Forms of the kernel
enum Form {
    PLAIN,
    WIDENED,            // e4m3 values are widened to f16 and multiplied by f16 MFMAs
    WIDENED_PAIR,       // in registers for two workgroups a compute unit, of 128 x 128
    WIDENED_SHORT,      // quarters of the tile without rows are left out
    // operands of any alignment, in 16 bits, with rows of 8 elements or more: copies go through registers, a 16-byte load at element alignment and
    // a k step later, where the copy into LDS would be asked for, a write to LDS.  A chunk that would leave its row is loaded as the row's
    // last 8 elements and shifted, so that no load lies in a branch: behind one the compiler waits for every load in flight.
    ANY_ALIGNMENT
};

template <int ELEM, bool AKC, bool BKC, int BM, int BN, int S, Form FORM, typename CT>
// (128 x 128 tiles: registers for two workgroups a compute unit, also where some are spilled: 16-bit (16384,2047,1023) of any alignment 131 us against 175)
__global__ __launch_bounds__(512, BM == 128 && BN == 128 && FORM != WIDENED && FORM != WIDENED_SHORT ? 4 : 2) void ops_tile_kernel(const OpsGemm g)
{
    constexpr bool SCALED = ELEM == ELEM_E4M3, EXACT = FORM == WIDENED || FORM == WIDENED_PAIR || FORM == WIDENED_SHORT, ANY = FORM == ANY_ALIGNMENT, SHORT = FORM == WIDENED_SHORT;
    constexpr int ES = Elem<ELEM>::size, KE = STEP / ES;   // elements of a k step
    constexpr int HM = BM / 2, WN = BN / 4;                // rows of a group, columns of a wavefront
    constexpr int FM = HM / 16, FN = WN / 16, FH = FM / 2; // blocks of 16 x 16; rows of blocks of a half
    constexpr int A_STAGE = BM * STEP, B_STAGE = BN * STEP, A_HALF = A_STAGE / 2, B_HALF = B_STAGE / 2;
    constexpr int TA = HM / 32, TB = BN / 64;              // copies of 1 KB of a wavefront and k step
    constexpr int NC = TA + TB + (SCALED ? 1 : 0);
    constexpr uint32_t A0 = 0, B0 = S * A_STAGE, S0 = B0 + S * B_STAGE;
    static_assert(S * NC <= 63, "copies in flight are counted in 6 bits");
    static_assert(TA >= 2 && (AKC || TA == 4 || TA == 2), "copies of a group's rows come in two halves");

    __shared__ __attribute__((aligned(1024))) char smem[lds_bytes<BM, BN, S, SCALED>()];
    const uint32_t smem_base = (uint32_t)(uintptr_t)(lds_ptr_t)smem;
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int grp = wave >> 2, wn = wave & 3;

    const TileAt t = find_tile<BM, BN>(g);
    if (!t.valid) return;
    const int K = t.k_end - t.k0, k_full = K / KE, KT = (K + KE - 1) / KE;

    // ---- copies ---------------------------------------------------------------------------------------------------
    // k rows: copy q = 8 rows of 128 bytes; lane i writes row 8q + i/8, chunk position i%8, which holds chunk position ^ (row/2)%8.
    // Other layout: copy q = 1 KB of a block of k rows of R * 2 bytes; the position of a chunk in its row is chunk_position().
    // A: each group brings in its own half of the rows (a block of HM columns in the other layout); B: half of the rows, or of the k rows.
    auto kc_offset = [&](int row, int limit, int64_t ld) -> uint32_t {       // row within the tile, clamped: loaded, never stored
        const int chunk = (lane & 7) ^ ((row >> 1) & 7);
        return (uint32_t)min(row, limit - 1) * (uint32_t)(ld * ES) + 16u * chunk;
    };
    uint32_t a_off[TA], b_off[TB];
    int a_shift[TA], b_shift[TB];                          // ANY: elements that a chunk begins before its place
    constexpr int A_CPR = HM / 8, B_CPR = BN / 8;                            // chunks of a k row (other layout)
    const int a_cols = t.row_end - t.row0, b_cols = g.N - t.n0;
#pragma unroll
    for (int i = 0; i < TA; i++) {
        if constexpr (AKC) {
            a_off[i] = kc_offset(grp * HM + 8 * (wn + 4 * i) + (lane >> 3), a_cols, g.lda);
        } else {
            const int c = 64 * (wn + 4 * i) + lane, krow = c / A_CPR;
            int col = grp * HM + 8 * mc_chunk<A_CPR>(c % A_CPR, krow);
            if constexpr (ANY) { a_shift[i] = max(0, col + 8 - a_cols); col -= a_shift[i]; }
            else if (col >= a_cols) col = 0;
            a_off[i] = ((uint32_t)krow * (uint32_t)g.lda + (uint32_t)col) * ES;
        }
    }
#pragma unroll
    for (int i = 0; i < TB; i++) {
        if constexpr (BKC) {
            b_off[i] = kc_offset(grp * (BN / 2) + 8 * (wn + 4 * i) + (lane >> 3), b_cols, g.ldb);
        } else {
            const int c = 64 * (wn + 4 * i) + lane, krow = c / B_CPR + 32 * grp;
            int col = 8 * mc_chunk<B_CPR>(c % B_CPR, krow);
            if constexpr (ANY) { b_shift[i] = max(0, col + 8 - b_cols); col -= b_shift[i]; }
            else if (col >= b_cols) col = 0;
            b_off[i] = ((uint32_t)krow * (uint32_t)g.ldb + (uint32_t)col) * ES;
        }
    }
    const char* const a_tile = AKC ? g.A + ((int64_t)t.row0 * g.lda + t.k0) * ES : g.A + ((int64_t)t.k0 * g.lda + t.row0) * ES;
    const char* const b_mat = g.B + (int64_t)t.e * g.b_stride * ES;
    const char* const b_tile = BKC ? b_mat + ((int64_t)t.n0 * g.ldb + t.k0) * ES : b_mat + ((int64_t)t.k0 * g.ldb + t.n0) * ES;
    const int64_t a_step = AKC ? STEP : 64 * g.lda * ES, b_step = BKC ? STEP : 64 * g.ldb * ES;
    // scales of A: wavefronts wn and wn + 2 of a group bring in the same 64 rows (the same count of copies for all)
    uint32_t s_off = SCALED ? 4u * (uint32_t)min(grp * HM + (HM >= 128 ? 64 * (wn & 1) : 0) + lane, a_cols - 1) : 0u;
    const float* const s_tile = SCALED ? g.sa + t.row0 : nullptr;
    typedef const __attribute__((address_space(4))) float* const_f32;
    const const_f32 sb = SCALED ? (const_f32)(uintptr_t)(g.sb + (int64_t)t.e * g.sb_stride + (int64_t)((t.n0 + wn * WN) / 128 < (g.N + 127) / 128 ? (t.n0 + wn * WN) / 128 : 0) * g.ld_sb) : nullptr;

    auto a_dst = [&](int st, int i) -> uint32_t { return smem_base + A0 + st * A_STAGE + grp * A_HALF + 1024 * (wn + 4 * i); };
    auto b_dst = [&](int st, int i) -> uint32_t { return smem_base + B0 + st * B_STAGE + grp * B_HALF + 1024 * (wn + 4 * i); };
    // a chunk of the last, short k step goes through registers with zeros behind the end of the sum
    auto tail_chunk = [&](const char* src, int left_bytes) -> uintx4 {       // left_bytes: of the chunk within the sum
        uintx4 v = {0u, 0u, 0u, 0u};
        if (left_bytes > 0) {
            v = *(const uintx4*)src;
#pragma unroll
            for (int w = 0; w < 4; w++) {
                const int n = left_bytes - 4 * w;
                v[w] = n >= 4 ? v[w] : n <= 0 ? 0u : v[w] & ((1u << (8 * n)) - 1u);
            }
        }
        return v;
    };
    auto put = [&](uint32_t dst, uintx4 v) { *(__attribute__((address_space(3))) uintx4*)(uintptr_t)(dst + 16 * lane) = v; };
    // ANY: chunk i of k step s; in the short last step its k rows behind the sum are any, its chunks of a k row end with the sum
    typedef uintx4 uintx4_any __attribute__((aligned(2)));
    auto fetch = [&](const char* tile, uint32_t off, int64_t step, int64_t ld, int k_at, int s, bool kc, auto whole) -> uintx4 {      // k_at: of the chunk in its k step
        int64_t back = 0;
        if constexpr (!decltype(whole)::value)
            back = kc ? ES * (int64_t)max(0, s * KE + k_at + 8 - K) : (int64_t)max(0, s * KE + k_at + 1 - K) * ld * ES;
        return *(const uintx4_any*)(tile + s * step + (int64_t)(int32_t)off - back);      // (a chunk may begin before its tile)
    };
    auto shifted = [](uintx4 v, int n) -> uintx4 {                           // by n elements towards the first, zeros behind
        const uint32_t h = (n & 1) ? 16u : 0u;
        uintx4 w;
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const uint32_t lo = v[i], hi = i < 3 ? v[i < 3 ? i + 1 : 3] : 0u;
            w[i] = (uint32_t)((((uint64_t)hi << 32) | lo) >> h);
        }
        if (n & 2) w = uintx4{w[1], w[2], w[3], 0u};
        if (n & 4) w = uintx4{w[2], w[3], 0u, 0u};
        if (n >= 8) w = uintx4{0u, 0u, 0u, 0u};
        return w;
    };
    const bool edge_a = !AKC && t.row0 + BM > t.row_end, edge_b = !BKC && t.n0 + BN > g.N;
    auto a_k = [&](int i) { if constexpr (AKC) return 8 * ((lane & 7) ^ (((grp * HM + 8 * (wn + 4 * i) + (lane >> 3)) >> 1) & 7)); else return (64 * (wn + 4 * i) + lane) / A_CPR; };
    auto b_k = [&](int i) { if constexpr (BKC) return 8 * ((lane & 7) ^ (((grp * (BN / 2) + 8 * (wn + 4 * i) + (lane >> 3)) >> 1) & 7)); else return (64 * (wn + 4 * i) + lane) / B_CPR + 32 * grp; };
    uintx4 held_a[ANY ? TA : 1], held_b[ANY ? TB : 1];                       // the chunks of the k step to be written next
    auto fetch_a = [&](int s, int i, auto whole) { held_a[i] = fetch(a_tile, a_off[i], a_step, g.lda, a_k(i), s, AKC, whole); };
    auto fetch_b = [&](int s, int i, auto whole) { held_b[i] = fetch(b_tile, b_off[i], b_step, g.ldb, b_k(i), s, BKC, whole); };
    auto finished = [&](uintx4 v, int shift, bool edge, int k_at, int s, bool kc, auto whole) -> uintx4 {
        if (edge) v = shifted(v, shift);
        if (!decltype(whole)::value && s >= k_full) {                        // the short step
            if (kc) v = shifted(v, max(0, s * KE + k_at + 8 - K));
            else if (s * KE + k_at >= K) v = uintx4{0u, 0u, 0u, 0u};
        }
        return v;
    };
    // k step s into stage st
    auto copy_a = [&](int s, int st, int i, auto whole) {
        if constexpr (ANY) { put(a_dst(st, i), finished(held_a[i], AKC ? 0 : a_shift[i], edge_a, a_k(i), s, AKC, whole)); if (whole || s + 1 < KT) fetch_a(s + 1, i, whole); }
        else if constexpr (decltype(whole)::value) { async_copy16(a_tile + s * a_step, a_off[i], a_dst(st, i)); }
        else if constexpr (AKC) {
            const int row = grp * HM + 8 * (wn + 4 * i) + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
            put(a_dst(st, i), tail_chunk(a_tile + s * a_step + a_off[i], (K - s * KE) * ES - 16 * chunk));
        } else {
            const int krow = (64 * (wn + 4 * i) + lane) / A_CPR;
            put(a_dst(st, i), tail_chunk(a_tile + s * a_step + a_off[i], krow < K - s * KE ? 16 : 0));
        }
    };
    auto copy_b = [&](int s, int st, int i, auto whole) {
        if constexpr (ANY) { put(b_dst(st, i), finished(held_b[i], BKC ? 0 : b_shift[i], edge_b, b_k(i), s, BKC, whole)); if (whole || s + 1 < KT) fetch_b(s + 1, i, whole); }
        else if constexpr (decltype(whole)::value) { async_copy16(b_tile + s * b_step, b_off[i], b_dst(st, i)); }
        else if constexpr (BKC) {
            const int row = grp * (BN / 2) + 8 * (wn + 4 * i) + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
            put(b_dst(st, i), tail_chunk(b_tile + s * b_step + b_off[i], (K - s * KE) * ES - 16 * chunk));
        } else {
            const int krow = (64 * (wn + 4 * i) + lane) / B_CPR + 32 * grp;
            put(b_dst(st, i), tail_chunk(b_tile + s * b_step + b_off[i], krow < K - s * KE ? 16 : 0));
        }
    };
    auto copy_s = [&](int s, int st) {
        if constexpr (SCALED) copy_dword(s_tile + s * g.ld_sa, s_off, smem_base + S0 + st * (BM * 4) + grp * (HM * 4) + (HM >= 128 ? 256 * (wn & 1) : 0));
    };
    typedef std::true_type Whole;
    typedef std::false_type Tail;

    floatx4 acc[FM][FN];
#pragma unroll
    for (int m = 0; m < FM; m++)
#pragma unroll
        for (int n = 0; n < FN; n++) acc[m][n] = floatx4{0.0f, 0.0f, 0.0f, 0.0f};

    if (KT > 0) {
        // k step s into stage s, in the order that the loop issues copies in: Y waits for its B rows, which X reads first, while its
        // second half of A may still be on its way
        auto issue_in_order = [&](int s, auto whole) {
#pragma unroll
            for (int i = 0; i < (AKC ? TA / 2 : 0); i++) copy_a(s, s, i, whole);
#pragma unroll
            for (int i = 0; i < TB; i++) copy_b(s, s, i, whole);
#pragma unroll
            for (int i = AKC ? TA / 2 : 0; i < TA; i++) copy_a(s, s, i, whole);
            copy_s(s, s);
        };
        auto issue = [&](int s) {
            if (s >= KT) return;
            if (!ANY && s < k_full) issue_in_order(s, Whole{});
            else                    issue_in_order(s, Tail{});
        };
        if constexpr (ANY) {
#pragma unroll
            for (int i = 0; i < TA; i++) fetch_a(0, i, Tail{});
#pragma unroll
            for (int i = 0; i < TB; i++) fetch_b(0, i, Tail{});
        }
#pragma unroll
        for (int s = 0; s < S; s++) issue(s);

        // ---- fragment addresses -----------------------------------------------------------------------------------
        const int l16 = lane & 15, q = lane >> 4;
        uint32_t a_rd[AKC ? 2 : FM], b_rd[BKC ? 2 : FN];
        if constexpr (AKC) {
#pragma unroll
            for (int h = 0; h < 2; h++) a_rd[h] = smem_base + A0 + grp * A_HALF + l16 * STEP + 16 * ((4 * h + q) ^ ((l16 >> 1) & 7));
        } else {
            const int krow = 8 * q + (l16 >> 2);
#pragma unroll
            for (int m = 0; m < FM; m++) { const int col = 16 * m + 4 * (l16 & 3); a_rd[m] = smem_base + A0 + grp * A_HALF + krow * (HM * 2) + 16 * mc_chunk<A_CPR>(col >> 3, krow) + 2 * (col & 7); }
        }
        if constexpr (BKC) {
#pragma unroll
            for (int h = 0; h < 2; h++) b_rd[h] = smem_base + B0 + (wn * WN + l16) * STEP + 16 * ((4 * h + q) ^ ((l16 >> 1) & 7));
        } else {
            const int krow = 8 * q + (l16 >> 2);
#pragma unroll
            for (int n = 0; n < FN; n++) { const int col = wn * WN + 16 * n + 4 * (l16 & 3); b_rd[n] = smem_base + B0 + krow * (BN * 2) + 16 * mc_chunk<B_CPR>(col >> 3, krow) + 2 * (col & 7); }
        }
        uint32_t s_rd = smem_base + S0 + (grp * HM + l16) * 4;

        // SHORT: quarters of the tile without rows are neither read nor multiplied, by a branch in each phase (the copies stay, as the waits count them)
        const int live = SHORT ? min(max((t.row_end - t.row0 - grp * HM + HM / 2 - 1) / (HM / 2), 0), 2) : 2;

        Frag fa[FH], fb[FN];
        Wide wa[EXACT ? FH : 1], wb[EXACT ? FN : 1];
        float scale[FH];
        float sbk = 0.0f;
        auto read_tr = [&](uint32_t at, int row_bytes) -> Frag {             // 8 k rows of slice 0 and of slice 1
            Frag f;
#pragma unroll
            for (int h = 0; h < 2; h++) {
                const uintx2 lo = __builtin_bit_cast(uintx2, lds_read_tr16(at + h * 32 * row_bytes)), hi = __builtin_bit_cast(uintx2, lds_read_tr16(at + (h * 32 + 4) * row_bytes));
                (h ? f.hi : f.lo) = uintx4{lo[0], lo[1], hi[0], hi[1]};
            }
            return f;
        };
        auto read16 = [&](uint32_t at) -> uintx4 { return *(__attribute__((address_space(3))) const uintx4*)(uintptr_t)at; };
        auto read_phase = [&](int k, int st, int h) {
            const uint32_t as = st * A_STAGE, bs = st * B_STAGE;
            if (h == 0) {
                if constexpr (BKC) {
                    uint32_t b0 = b_rd[0] + bs, b1 = b_rd[1] + bs;
                    asm volatile("" : "+v"(b0), "+v"(b1));
#pragma unroll
                    for (int n = 0; n < FN; n++) { fb[n].lo = read16(b0 + n * 16 * STEP); fb[n].hi = read16(b1 + n * 16 * STEP); }
                } else {
#pragma unroll
                    for (int n = 0; n < FN; n++) { uint32_t b0 = b_rd[n] + bs; asm volatile("" : "+v"(b0)); fb[n] = read_tr(b0, BN * 2); }
                }
                if constexpr (SCALED) sbk = sb[k];
                if constexpr (FORM == WIDENED_PAIR) {                        // before A is read: fewer registers at a time
#pragma unroll
                    for (int n = 0; n < FN; n++) wb[n] = widened(fb[n]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            if constexpr (AKC) {
                uint32_t a0 = a_rd[0] + as, a1 = a_rd[1] + as;
                asm volatile("" : "+v"(a0), "+v"(a1));
#pragma unroll
                for (int m = 0; m < FH; m++) { fa[m].lo = read16(a0 + (h * FH + m) * 16 * STEP); fa[m].hi = read16(a1 + (h * FH + m) * 16 * STEP); }
            } else {
#pragma unroll
                for (int m = 0; m < FH; m++) { uint32_t a0 = a_rd[h * FH + m] + as; asm volatile("" : "+v"(a0)); fa[m] = read_tr(a0, HM * 2); }
            }
            if constexpr (SCALED) {
#pragma unroll
                for (int m = 0; m < FH; m++)
                    scale[m] = *(__attribute__((address_space(3))) const float*)(uintptr_t)(s_rd + st * (BM * 4) + (h * FH + m) * 64);
            }
            if constexpr (EXACT) {
                if (h == 0 && FORM != WIDENED_PAIR) {
#pragma unroll
                    for (int n = 0; n < FN; n++) wb[n] = widened(fb[n]);
                }
#pragma unroll
                for (int m = 0; m < FH; m++) wa[m] = widened(fa[m]);
            }
        };
        // COPY: 1 of a whole k step, 2 of the short one, both into the stage that this k step has been read from; 0 and below: none, this is
        // the last k step but -COPY
        // GRP: the group, as a constant (both have their own code, without branches in a phase)
        auto multiply_phase = [&](int k, int st, auto half, auto copy, auto group) {
            constexpr int COPY = decltype(copy)::value, h = decltype(half)::value, GRP = decltype(group)::value;
            constexpr int NM = FH * FN;
            // copies of this phase behind MFMA i: A's half in k rows (all of A in the second phase otherwise), B in X's second and Y's first phase
            auto copies = [&](int i) {
                if constexpr (COPY > 0) {
                    typedef typename std::conditional<COPY == 1, Whole, Tail>::type W;
                    constexpr int SLOTS = 8;                                  // places of copies among the MFMAs
                    constexpr int EVERY = NM >= SLOTS ? NM / SLOTS : 1, PER = NM >= SLOTS ? 1 : SLOTS / NM;
                    if (i % EVERY == 0) {
                        const int slot = i / EVERY;
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int j = 0; j < PER; j++) {
                            const int c = slot * PER + j;                     // 0 .. 7
                            const int na = AKC ? TA / 2 : (h == 0 ? 0 : TA), a_first = AKC ? h * (TA / 2) : 0;
                            if (c < na) copy_a(k + S, st, a_first + c, W{});
                            else if (c < na + TB && GRP == 1 - h) copy_b(k + S, st, c - na, W{});
                            if (SCALED && h == 1 && c == 7) copy_s(k + S, st);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
            };
            if (!(h < live)) {
#pragma unroll
                for (int i = 0; i < NM; i++) copies(i);
                return;
            }
            if constexpr (SCALED) {
#pragma unroll
                for (int m = 0; m < FH; m++) scale[m] *= sbk;
            }
            // e4m3: the results of MFMA i are added while MFMAs i + 1 and i + 2 run
            constexpr int BEHIND = 2;
            floatx4 part[BEHIND + 1];
            auto block_m = [](int i) { return i / FN; };
            auto block_n = [](int i) { return (i / FN & 1) ? FN - 1 - i % FN : i % FN; };
            auto add = [&](int i) {
                const int m = block_m(i), n = block_n(i);
#pragma unroll
                for (int e = 0; e < 4; e++) acc[h * FH + m][n][e] = __builtin_fmaf(part[i % (BEHIND + 1)][e], scale[m], acc[h * FH + m][n][e]);
                asm volatile("" : "+v"(acc[h * FH + m][n]));                 // added here and not in a later block
            };
#pragma unroll
            for (int i = 0; i < NM; i++) {
                const int m = block_m(i), n = block_n(i);
                if constexpr (SCALED) {
                    if constexpr (EXACT) part[i % (BEHIND + 1)] = mfma_step(wb[n], wa[m]);
                    else                 part[i % (BEHIND + 1)] = mfma_step<ELEM>(fb[n], fa[m], floatx4{0.0f, 0.0f, 0.0f, 0.0f});
                    __builtin_amdgcn_sched_barrier(0);
                    if (i >= BEHIND) { add(i - BEHIND); __builtin_amdgcn_sched_barrier(0); }
                } else {
                    acc[h * FH + m][n] = mfma_step<ELEM>(fb[n], fa[m], acc[h * FH + m][n]);
                }
                copies(i);
            }
            if constexpr (SCALED) {
#pragma unroll
                for (int i = NM - BEHIND; i < NM; i++) add(i);
            }
        };
        auto half_step = [&](int k, int st, auto half, auto copy, auto group) {
            constexpr int h = decltype(half)::value, GRP = decltype(group)::value, COPY = decltype(copy)::value;
            if (h < live) read_phase(k, st, h);
            __builtin_amdgcn_s_waitcnt(0xC07F);                              // lgkmcnt(0)
            asm volatile("" ::: "memory");
            phase_barrier();
            multiply_phase(k, st, half, copy, group);
            if constexpr (h == 1 || GRP == 1) {
                __builtin_amdgcn_sched_barrier(0);
                // copies for later k steps than the next may be on their way
                if constexpr (ANY)           asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                else if constexpr (COPY == 1) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(NC * (S - 1)) : "memory");
                else if constexpr (COPY == 2) asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
                else                          asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(COPY <= -1 ? NC * (-COPY - 1) : 0) : "memory");
            }
            // Y began one barrier later and leaves out the last one
            if constexpr (COPY != 0 || GRP == 0 || h == 0) phase_barrier();
        };
        auto run_loop = [&](auto group) {
            int k = 0, st = 0;                                               // the k step and its stage
            auto k_step = [&](auto copy) {
                half_step(k, st, std::integral_constant<int, 0>{}, copy, group);
                half_step(k, st, std::integral_constant<int, 1>{}, copy, group);
                k++;
                st = st + 1 == S ? 0 : st + 1;
            };
            // what the loop uses is in registers before it begins: a spilled offset reloaded behind the loop's head would be
            // waited for in every k step, and every copy in flight with it
            auto pin = [](uint32_t& x) { asm volatile("" : "+v"(x)); };
#pragma unroll
            for (int i = 0; i < TA; i++) pin(a_off[i]);
#pragma unroll
            for (int i = 0; i < TB; i++) pin(b_off[i]);
#pragma unroll
            for (uint32_t& x : a_rd) pin(x);
#pragma unroll
            for (uint32_t& x : b_rd) pin(x);
            if constexpr (SCALED) { pin(s_off); pin(s_rd); }
            // (ANY: a k step also loads the one behind the one that it writes)
            while (k + S + (ANY ? 1 : 0) < k_full) k_step(std::integral_constant<int, 1>{});
            if constexpr (ANY) { while (k + S < KT) k_step(std::integral_constant<int, 2>{}); }
            else if (k + S < KT) k_step(std::integral_constant<int, 2>{});
            auto last = [&](auto left) { if (KT - k == 1 - decltype(left)::value) k_step(left); };     // left = 0: the last one
            if constexpr (S >= 4) last(std::integral_constant<int, -3>{});
            if constexpr (S >= 3) last(std::integral_constant<int, -2>{});
            last(std::integral_constant<int, -1>{});
            last(std::integral_constant<int, 0>{});
        };
        // k step 0 has landed, those behind it may be on their way
        if (ANY)              asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        else if (S <= k_full) asm volatile("s_waitcnt vmcnt(%0)" :: "n"(NC * (S - 1)) : "memory");
        else                  asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        phase_barrier();
        if (grp == 0) {
            run_loop(std::integral_constant<int, 0>{});
        } else {
            phase_barrier();
            run_loop(std::integral_constant<int, 1>{});
        }
    }

    // ---- to C: 32 rows of a wavefront at a time through LDS, so that whole row segments are stored ------------------------
    constexpr int PITCH = WN * 4 + 16, LPR = WN / 4, RPP = 64 / LPR;          // lanes of a row, rows of a pass
    const uint32_t buf = smem_base + wave * (32 * PITCH);
    const int l16 = lane & 15, q = lane >> 4;
    const int orow = lane / LPR, ocol = 4 * (lane % LPR);
    const int col = t.n0 + wn * WN + ocol, row_first = t.row0 + grp * HM + orow;
    CT* const C = (CT*)g.C + (int64_t)t.e * g.c_stride + (int64_t)row_first * g.ldc + col;
    typedef typename CVec4<CT>::type ctx4;
#pragma unroll
    for (int m2 = 0; m2 < FM / 2; m2++) {
#pragma unroll
        for (int r = 0; r < 2; r++)
#pragma unroll
            for (int n = 0; n < FN; n++)
                *(__attribute__((address_space(3))) floatx4*)(uintptr_t)(buf + (16 * r + l16) * PITCH + (16 * n + 4 * q) * 4) = acc[2 * m2 + r][n];
#pragma unroll
        for (int ps = 0; ps < 32 / RPP; ps++) {
            const floatx4 v = *(__attribute__((address_space(3))) const floatx4*)(uintptr_t)(buf + (RPP * ps + orow) * PITCH + ocol * 4);
            const int r = 32 * m2 + RPP * ps;
            if (row_first + r < t.row_end) {
                CT* const dst = C + (int64_t)r * g.ldc;
                if (col + 4 <= g.N) {
                    ctx4 o;
#pragma unroll
                    for (int e = 0; e < 4; e++) o[e] = (CT)v[e];
                    __builtin_nontemporal_store(o, (ctx4*)dst);      // past the L2s, which hold what other tiles read: 16-bit (16384,2304,768) 76 -> 68 us
                } else {
#pragma unroll
                    for (int e = 0; e < 4; e++) if (col + e < g.N) dst[e] = (CT)v[e];
                }
            }
        }
    }
}

template <int ELEM, bool AKC, bool BKC, int BM, int BN, int S, Form FORM = PLAIN>
int launch_tiles(const OpsGemm& g)
{
    const int64_t grid = tile_grid(g, BM, BN);
    if (grid < 0 || !fits_a_launch(grid, 512)) return GEMM_F16_ERR_SIZE;
    if (g.c_type == ELEM_F32) hipLaunchKernelGGL((ops_tile_kernel<ELEM, AKC, BKC, BM, BN, S, FORM, float>), dim3((unsigned)grid), dim3(512), 0, g.stream, g);
    else if (ELEM != ELEM_BF16 && g.c_type == ELEM_F16) { if constexpr (ELEM != ELEM_BF16) hipLaunchKernelGGL((ops_tile_kernel<ELEM, AKC, BKC, BM, BN, S, FORM, half_t>), dim3((unsigned)grid), dim3(512), 0, g.stream, g); }
    else if constexpr (ELEM != ELEM_F16) hipLaunchKernelGGL((ops_tile_kernel<ELEM, AKC, BKC, BM, BN, S, FORM, bf16_t>), dim3((unsigned)grid), dim3(512), 0, g.stream, g);
    return hipGetLastError() == hipSuccess ? GEMM_F16_OK : GEMM_F16_ERR_LAUNCH;
}

}  // namespace ops_tile
