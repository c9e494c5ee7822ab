// Tokens sorted by expert, their rows moved there and back with weights applied, and the gradients of that (include/gemm_layer.h).
//
// The order is a counting sort: how many choices of each expert lie before a choice's own, and how many of its own.  Nothing atomic
// decides a place, so the order is always the same.  Rows move by token: a token's row is read once and stored to its places,
// and on the way back a lane adds the elements of a token's rows in their order.  Both are bound by memory.
#include <type_traits>
#include "ops_rows.h"
#include "../../include/gemm_layer.h"

namespace {

using namespace ops_dev;

// The expert of choice i, E for one of no expert here
__device__ __forceinline__ int key_of(const DispatchArgs& a, int64_t i)
{
    const int64_t e = a.index64 ? ((const int64_t*)a.expert)[i] : (int64_t)((const int32_t*)a.expert)[i];
    return e < 0 || e >= a.E ? a.E : (int)e;
}

// ---- rows to their places ------------------------------------------------------------------------------------------------------
typedef uintx4 uintx4_any __attribute__((aligned(1)));
constexpr int ROW_CHUNKS = 4;                              // 16-byte chunks of a lane: a wavefront takes 4 KB of a token's row

// Bytes first .. of token t's row, in registers of a wavefront.  The last chunk of a row of 16 bytes and more ends with the row, so that two lanes may store the
// same bytes twice; shorter rows go byte by byte.
struct RowPiece {
    uintx4 v[ROW_CHUNKS];
    int64_t at[ROW_CHUNKS];                                // byte of the row, -1: none
    __device__ __forceinline__ void load(const char* row, int64_t first, int64_t bytes)
    {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int i = 0; i < ROW_CHUNKS; i++) {
            const int64_t c = first + 16 * (lane + 64 * i);
            at[i] = c >= bytes ? -1 : bytes < 16 ? c : min(c, bytes - 16);
            if (at[i] >= 0 && bytes >= 16) v[i] = *(const uintx4_any*)(row + at[i]);
        }
        if (bytes < 16 && at[0] >= 0) {
            v[0] = uintx4{0u, 0u, 0u, 0u};
            for (int b = 0; b < bytes; b++) v[0][b >> 2] |= (uint32_t)(uint8_t)row[b] << (8 * (b & 3));
        }
    }
    // PAST: past the caches
    template <bool PAST = false>
    __device__ __forceinline__ void store(char* row, int64_t bytes) const
    {
#pragma unroll
        for (int i = 0; i < ROW_CHUNKS; i++)
            if (at[i] >= 0 && bytes >= 16) {
                if constexpr (PAST) __builtin_nontemporal_store(v[i], (uintx4_any*)(row + at[i]));
                else                *(uintx4_any*)(row + at[i]) = v[i];
            }
        if (bytes < 16 && at[0] >= 0)
            for (int b = 0; b < bytes; b++) row[b] = (char)(v[0][b >> 2] >> (8 * (b & 3)));
    }
};
constexpr int64_t PIECE = 16 * 64 * ROW_CHUNKS;

// the scales of token t to a place
__device__ __forceinline__ void move_scales(const DispatchArgs& a, int64_t t, int64_t place)
{
    for (int64_t b = threadIdx.x & 63; b < a.blocks; b += 64) a.row_scale[b * a.ld_row_scale + place] = a.scale[b * a.ld_scale + t];
}

__global__ __launch_bounds__(256) void move_rows_kernel(const DispatchArgs a, int64_t pieces, int64_t items)
{
    const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= items) return;
    const int64_t t = item / pieces, piece = item % pieces, bytes = (int64_t)a.N * a.size;
    RowPiece row;
    row.load((const char*)a.X + t * a.ldx * a.size, piece * PIECE, bytes);
    for (int j = 0; j < a.top_k; j++) {
        const int place = __builtin_amdgcn_readfirstlane(a.place[t * a.top_k + j]);
        if (place < 0) continue;
        row.store((char*)a.rows + (int64_t)place * a.ld_rows * a.size, bytes);
        if (piece == 0) move_scales(a, t, place);
    }
}

// ---- few choices: one launch -----------------------------------------------------------------------------------------------------
// Every wavefront holds all choices (64 NR at most) in registers as expert << 10 | number, so that a choice's row is the number
// of smaller ones: NR comparisons of a wavefront.  A wavefront for each piece of a token's row, and one for each 8 experts' offsets.  32 tokens to 2 of 16 experts, rows of 2048 bytes 3.4 us, a launch.
template <int NR>
__global__ __launch_bounds__(256) void dispatch_few_kernel(const DispatchArgs a, int64_t pieces, int64_t items)
{
    const int lane = threadIdx.x & 63, n = (int)a.T * a.top_k;
    const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t key[NR];
#pragma unroll
    for (int i = 0; i < NR; i++) {
        const int c = 64 * i + lane;
        key[i] = c < n ? ((uint32_t)key_of(a, c) << 10) | (uint32_t)c : ~0u;
    }
    auto below = [&](uint32_t limit) {
        int s = 0;
#pragma unroll
        for (int i = 0; i < NR; i++) s += __popcll(__ballot(key[i] < limit));
        return s;
    };
    if (item >= items) {
        const int64_t first = (item - items) * 8;
        int mine = 0;
        for (int j = 0; j < 8; j++) { const int s = below((uint32_t)min((int64_t)a.E, first + j) << 10); if (lane == j) mine = s; }
        if (lane < 8 && first + lane <= a.E) a.offsets[first + lane] = mine;
        return;
    }
    const int64_t t = item / pieces, piece = item % pieces, bytes = (int64_t)a.N * a.size;
    RowPiece row;
    if (a.X) row.load((const char*)a.X + t * a.ldx * a.size, piece * PIECE, bytes);
    for (int j = 0; j < a.top_k; j++) {
        const int c = (int)t * a.top_k + j;
        uint32_t own = 0;
#pragma unroll
        for (int i = 0; i < NR; i++) if (c / 64 == i) own = (uint32_t)__builtin_amdgcn_readlane((int)key[i], c % 64);
        const int at = below(own);
        const bool valid = (int)(own >> 10) < a.E;
        if (piece == 0 && lane == 0) {
            a.place[c] = valid ? at : -1;
            if (a.source) a.source[at] = valid ? (int)t : -1;
        }
        if (!valid || !a.X) continue;
        row.store((char*)a.rows + (int64_t)at * a.ld_rows * a.size, bytes);
        if (piece == 0) move_scales(a, t, at);
    }
}

// sums of all lanes up to and with this one: within rows of 16 lanes, then the last lane of a row to the next, then of the first two rows to the others
__device__ __forceinline__ int scan64(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}

// ---- some choices: still one launch ----------------------------------------------------------------------------------------------------
// Every workgroup counts all choices in LDS, those in front of its tokens' by themselves, so that a choice's row is what lies before its expert, what of its expert lies in front, and
// the equal ones of its own 64.  `tokens` tokens a workgroup, 64 choices at most.
__global__ __launch_bounds__(256) void dispatch_some_kernel(const DispatchArgs a, int tokens, int64_t pieces)
{
    extern __shared__ int counts[];                        // [expert]: in front, then the others
    __shared__ int wave_sums[2][4], places[64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), bins = a.E + 1, n = (int)a.T * a.top_k;
    const int t0 = (int)blockIdx.x * tokens, own = min((int)a.T - t0, tokens), first = t0 * a.top_k, mine = own * a.top_k;
    const int64_t bytes = (int64_t)a.N * a.size;
    // pieces of rows, a wavefront each; where those are few `shared` wavefronts take a piece, each to some of its places
    const int rows = own * (int)pieces, shared = rows >= 4 ? 1 : rows >= 2 ? 2 : 4, items = rows * shared;
    RowPiece row;
    auto load = [&](int item) { row.load((const char*)a.X + (t0 + item / shared / (int)pieces) * a.ldx * a.size, item / shared % (int)pieces * PIECE, bytes); };
    if (a.X && wave < items) load(wave);                   // the first while choices are counted
    for (int b = threadIdx.x; b < 2 * bins; b += 256) counts[b] = 0;
    __syncthreads();
    constexpr int U = 4;
    for (int i0 = threadIdx.x; i0 < n; i0 += 256 * U) {
        int key[U];
#pragma unroll
        for (int u = 0; u < U; u++) key[u] = i0 + 256 * u < n ? key_of(a, i0 + 256 * u) : -1;
#pragma unroll
        for (int u = 0; u < U; u++) if (key[u] >= 0) atomicAdd(&counts[key[u] + (i0 + 256 * u < first ? 0 : bins)], 1);
    }
    __syncthreads();
    // where each expert begins, and the part's choices of it
    int run = 0;
    for (int b0 = 0, slot = 0; b0 < bins; b0 += 256, slot ^= 1) {
        const int b = b0 + threadIdx.x, front = b < bins ? counts[b] : 0, sum = b < bins ? front + counts[bins + b] : 0, incl = scan64(sum);
        if (lane == 63) wave_sums[slot][wave] = incl;
        __syncthreads();
        int before = run;
        for (int w = 0; w < 4; w++) { const int s = wave_sums[slot][w]; before += w < wave ? s : 0; run += s; }
        if (b < bins) {
            counts[b] = before + incl - sum + front;
            if (blockIdx.x == 0) a.offsets[b] = before + incl - sum;
        }
    }
    __syncthreads();
    if (wave == 0) {
        const int key = lane < mine ? key_of(a, first + lane) : a.E + 1;
        uint64_t same = mine < 64 ? (1ull << mine) - 1 : ~0ull;
        const int bits = 32 - __builtin_clz(a.E | 1);
        for (int b = 0; b < bits; b++) {
            const bool set = (key >> b) & 1;
            const uint64_t m = __ballot(set);
            same &= set ? m : ~m;
        }
        if (lane < mine) {
            const int at = counts[key] + __popcll(same & ((1ull << lane) - 1));
            places[lane] = key < a.E ? at : -1;
            a.place[first + lane] = key < a.E ? at : -1;
            if (a.source) a.source[at] = key < a.E ? t0 + lane / a.top_k : -1;
        }
    }
    if (!a.X) return;
    __syncthreads();
    for (int64_t i = threadIdx.x; i < mine * a.blocks; i += 256) {
        const int c = (int)(i % mine), at = places[c];
        if (at >= 0) a.row_scale[i / mine * a.ld_row_scale + at] = a.scale[i / mine * a.ld_scale + t0 + c / a.top_k];
    }
    for (int item = wave; item < items; item += 4) {
        if (item != wave) load(item);
        const int at = places[item / shared / (int)pieces * a.top_k + min(lane, a.top_k - 1)];
        for (int j = item % shared; j < a.top_k; j += shared) {
            const int place = __builtin_amdgcn_readlane(at, j);
            if (place >= 0) row.store((char*)a.rows + (int64_t)place * a.ld_rows * a.size, bytes);
        }
    }
}

// ---- more choices or experts: counting sorts by two digits ------------------------------------------------------------------------------------
// `parts` workgroups of part_rows choices each count their digits; a second launch makes of each digit's counts the sums of those before;
// a third one finds each choice's place.  The choices are sorted by the experts' low 8 bits and then by the rest.
struct SortPass {
    DispatchArgs a;
    const int32_t* seq;                                    // the choices in the order that this pass goes by; NULL: as they are
    int shift, bins, part_rows, parts;
    int32_t *counts, *totals;                              // [digit][part], [digit]; the former become the sums of those in front
    int32_t* out;                                          // the choices as this pass orders them; NULL: the places and sources are written
    int32_t* keys;                                         // the experts in order, of the last pass
};
__device__ __forceinline__ int digit_of(const SortPass& s, int key) { return s.shift < 0 ? key & 255 : key >> s.shift; }

__global__ __launch_bounds__(256) void sort_count_kernel(const SortPass s)
{
    extern __shared__ int hist[];
    for (int b = threadIdx.x; b < s.bins; b += 256) hist[b] = 0;
    __syncthreads();
    const int64_t n = s.a.T * s.a.top_k, first = (int64_t)blockIdx.x * s.part_rows, end = min(n, first + s.part_rows);
    for (int64_t i = first + threadIdx.x; i < end; i += 256) atomicAdd(&hist[digit_of(s, key_of(s.a, s.seq ? s.seq[i] : i))], 1);
    __syncthreads();
    for (int b = threadIdx.x; b < s.bins; b += 256) s.counts[(int64_t)b * s.parts + blockIdx.x] = hist[b];
}

// a workgroup for each digit
__global__ __launch_bounds__(1024) void sort_scan_kernel(int32_t* counts, int32_t* totals, int parts)
{
    __shared__ int sums[2][16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x / 64;
    int32_t* const c = counts + (int64_t)blockIdx.x * parts;
    int before = 0, slot = 0;
    for (int p0 = 0; p0 < parts; p0 += blockDim.x) {
        const int p = p0 + threadIdx.x, v = p < parts ? c[p] : 0, incl = scan64(v);
        if (lane == 63) sums[slot][wave] = incl;
        __syncthreads();                                   // (two sets of sums in turn)
        int front = 0, all = 0;
        for (int w = 0; w < waves; w++) { const int n = sums[slot][w]; all += n; front += w < wave ? n : 0; }
        if (p < parts) c[p] = before + front + incl - v;
        before += all;
        slot ^= 1;
    }
    if (threadIdx.x == 0) totals[blockIdx.x] = before;
}

__global__ __launch_bounds__(256) void sort_place_kernel(const SortPass s)
{
    extern __shared__ int base[];                          // [wavefront][digit]
    __shared__ int wave_sums[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int* const own = base + wave * s.bins;
    for (int b = threadIdx.x; b < 4 * s.bins; b += 256) base[b] = 0;
    __syncthreads();
    const int64_t n = s.a.T * s.a.top_k;
    const int64_t first = (int64_t)blockIdx.x * s.part_rows + (int64_t)wave * (s.part_rows / 4);
    const int64_t end = min(n, first + s.part_rows / 4);
    for (int64_t i = first + lane; i < end; i += 64) atomicAdd(&own[digit_of(s, key_of(s.a, s.seq ? s.seq[i] : i))], 1);
    __syncthreads();
    // where each digit begins: sums over the digits before, a thread each (there are 256 at most)
    const int b = threadIdx.x, sum = b < s.bins ? s.totals[b] : 0, incl = scan64(sum);
    if (lane == 63) wave_sums[wave] = incl;
    __syncthreads();
    if (b < s.bins) {
        int at = incl - sum + s.counts[(int64_t)b * s.parts + blockIdx.x];
        for (int w = 0; w < wave; w++) at += wave_sums[w];
        for (int w = 0; w < 4; w++) { const int c = base[w * s.bins + b]; base[w * s.bins + b] = at; at += c; }
    }
    __syncthreads();
    // 64 choices at a time: lanes of one digit find each other, the first of them moves the digit's place on
    const int bits = 32 - __builtin_clz(s.bins - 1 | 1);
    for (int64_t i0 = first; i0 < end; i0 += 64) {
        const int64_t i = i0 + lane;
        const bool there = i < end;
        const int64_t choice = there ? (s.seq ? s.seq[i] : i) : 0;
        const int key = there ? key_of(s.a, choice) : 0, digit = digit_of(s, key);
        uint64_t same = __ballot(there);
        for (int b = 0; b < bits; b++) {
            const bool set = (digit >> b) & 1;
            const uint64_t m = __ballot(set);
            same &= set ? m : ~m;
        }
        int at = 0;
        const int leader = there ? __builtin_ctzll(same) : lane;
        if (there && lane == leader) at = atomicAdd(&own[digit], __popcll(same));
        at = __shfl(at, leader) + __popcll(same & ((1ull << lane) - 1));
        if (!there) continue;
        if (s.out) { s.out[at] = (int32_t)choice; continue; }
        const bool valid = key < s.a.E;
        s.a.place[choice] = valid ? at : -1;
        if (s.a.source) s.a.source[at] = valid ? (int32_t)(choice / s.a.top_k) : -1;
        s.keys[at] = key;
    }
}

// ---- up to 2047 experts and 2^19 choices, 256 a token: places and rows in one launch, behind two short ones -----------------------------------------
// The tokens go in `parts` parts of 64 choices, or more where the counts would pass 4 MB.  One launch counts the experts of each part, a second one adds the counts of
// the parts in front (sort_scan_kernel).  In the third each wavefront finds its token's places by itself, from the counts and the choices of its part in front of its own, while
// the piece of the token's row that it copies is on its way.  8192 tokens to 2 of 16, bf16 rows of 4096: 36.6 us, of which 31 are the third launch's (6.2 TB/s).
struct Parts {
    DispatchArgs a;
    int tokens, parts;                                     // tokens of a part
    int32_t *counts, *totals;                              // [expert][part], [expert]
};
__global__ __launch_bounds__(256) void part_count_kernel(const Parts s)
{
    extern __shared__ int hist[];
    const int lane = threadIdx.x & 63, bins = s.a.E + 1;
    const int64_t part = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    int* const own = hist + (threadIdx.x >> 6) * bins;
    for (int b = lane; b < bins; b += 64) own[b] = 0;
    wave_exchange();
    if (part >= s.parts) return;
    const int64_t rows = (int64_t)s.tokens * s.a.top_k, first = part * rows, end = min(s.a.T * s.a.top_k, first + rows);
    for (int64_t i = first + lane; i < end; i += 64) atomicAdd(&own[key_of(s.a, i)], 1);
    wave_exchange();
    for (int b = lane; b < bins; b += 64) s.counts[(int64_t)b * s.parts + part] = own[b];
}

// Sums of the totals of the experts in front of each lane's.  (e: E + 1 where a lane has none)
__device__ __forceinline__ int rows_before(const Parts& s, int e)
{
    const int lane = threadIdx.x & 63, bins = s.a.E + 1;
    int run = 0, start = 0;
    for (int b0 = 0; b0 < bins; b0 += 64) {
        const int v = b0 + lane < bins ? s.totals[b0 + lane] : 0, incl = scan64(v);
        const int at = __shfl(incl - v, e & 63);
        if (e >> 6 == b0 >> 6) start = run + at;
        run += __builtin_amdgcn_readlane(incl, 63);
    }
    return start;
}
template <bool PAST>
__global__ __launch_bounds__(256) void part_move_kernel(const Parts s, int64_t pieces, int64_t items)
{
    const DispatchArgs& a = s.a;
    const int lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= items) {                                   // offsets, 64 a wavefront
        const int64_t e = (item - items) * 64 + lane;
        if ((item - items) * 64 > a.E) return;
        const int start = rows_before(s, (int)e);
        if (e <= a.E) a.offsets[e] = start;
        return;
    }
    const int64_t t = item / pieces, piece = item % pieces, bytes = (int64_t)a.N * a.size, part = t / s.tokens, n = a.T * a.top_k;
    RowPiece row;
    if (a.X) row.load((const char*)a.X + t * a.ldx * a.size, piece * PIECE, bytes);
    for (int j0 = 0; j0 < a.top_k; j0 += 64) {             // 64 of the token's choices at a time, a lane each
        const int64_t first = t * a.top_k + j0;
        const int mine = min(a.top_k - j0, 64), own = lane < mine ? key_of(a, first + lane) : a.E + 1;
        const int front = lane < mine ? s.counts[(int64_t)own * s.parts + part] : 0;
        const int base = rows_before(s, own) + front;
        int at = base;                                     // and the equal ones of the part in front of it
        for (int64_t i0 = part * s.tokens * a.top_k; i0 < first + mine - 1; i0 += 64) {
            const int64_t i = i0 + lane;
            const int key = i < n ? key_of(a, i) : a.E + 1;
            const int64_t in_front = first - i0;           // lanes in front of the token's choice 0 here; below 0: the token began in the 64 choices before these
            for (int j = 0; j < mine; j++) {
                const uint64_t front_of_j = in_front + j >= 64 ? ~0ull : in_front + j <= 0 ? 0ull : (1ull << (in_front + j)) - 1;
                const int c = __popcll(__ballot(key == __builtin_amdgcn_readlane(own, j)) & front_of_j);
                if (lane == j) at += c;
            }
        }
        if (piece == 0 && lane < mine) {
            a.place[first + lane] = own < a.E ? at : -1;
            if (a.source) a.source[at] = own < a.E ? (int32_t)t : -1;
        }
        if (!a.X) continue;
        for (int j = 0; j < mine; j++) {
            if (__builtin_amdgcn_readlane(own, j) >= a.E) continue;
            const int64_t place = __builtin_amdgcn_readlane(at, j);
            row.store<PAST>((char*)a.rows + place * a.ld_rows * a.size, bytes);
            if (piece == 0) move_scales(a, t, place);
        }
    }
}

// The same for rows of up to 256 bytes in parts of 64 choices and less: a wavefront for a part, whose lanes of one expert find each other; R lanes a row, 64 / R rows at a time.
__global__ __launch_bounds__(256) void part_move_narrow_kernel(const Parts s, int R)
{
    const DispatchArgs& a = s.a;
    const int lane = threadIdx.x & 63;
    const int64_t part = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (part >= s.parts) {                                 // offsets, 64 a wavefront
        const int64_t e = (part - s.parts) * 64 + lane;
        if (e - lane > a.E) return;
        const int start = rows_before(s, (int)e);
        if (e <= a.E) a.offsets[e] = start;
        return;
    }
    const int64_t t0 = part * s.tokens, first = t0 * a.top_k, bytes = (int64_t)a.N * a.size;
    const int mine = (int)(min(a.T - t0, (int64_t)s.tokens) * a.top_k);
    const int key = lane < mine ? key_of(a, first + lane) : a.E + 1;
    const int front = lane < mine ? s.counts[(int64_t)key * s.parts + part] : 0;
    uint64_t same = mine < 64 ? (1ull << mine) - 1 : ~0ull;
    const int bits = 32 - __builtin_clz(a.E | 1);
    for (int b = 0; b < bits; b++) {
        const bool set = (key >> b) & 1;
        const uint64_t m = __ballot(set);
        same &= set ? m : ~m;
    }
    const int rank = rows_before(s, key) + front + __popcll(same & ((1ull << lane) - 1));
    const int at = key < a.E ? rank : -1, token = lane / a.top_k;
    if (lane < mine) {
        a.place[first + lane] = at;
        if (a.source) a.source[rank] = key < a.E ? (int32_t)(t0 + token) : -1;
    }
    if (!a.X) return;
    if (at >= 0)
        for (int64_t b = 0; b < a.blocks; b++) a.row_scale[b * a.ld_row_scale + at] = a.scale[b * a.ld_scale + t0 + token];
    const int rows = 64 / R, sub = lane / R;
    const int64_t byte = bytes < 16 ? 0 : min((int64_t)16 * (lane % R), bytes - 16);
    constexpr int U = 4;
    for (int c0 = 0; c0 < mine; c0 += U * rows) {
        uintx4 v[U];
        int to[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int c = c0 + u * rows + sub;
            to[u] = __shfl(at, c & 63);
            if (c >= mine) to[u] = -1;
            if (bytes >= 16) v[u] = *(const uintx4_any*)((const char*)a.X + (t0 + __shfl(token, min(c, mine - 1))) * a.ldx * a.size + byte);
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            if (to[u] < 0) continue;
            char* const out = (char*)a.rows + (int64_t)to[u] * a.ld_rows * a.size + byte;
            if (bytes >= 16) { *(uintx4_any*)out = v[u]; continue; }
            const char* const in = (const char*)a.X + (t0 + (c0 + u * rows + sub) / a.top_k) * a.ldx * a.size;
            for (int b = 0; b < bytes; b++) out[b] = in[b];
        }
    }
}

// offsets of sorted experts: the first row of each that is not below it
__global__ __launch_bounds__(256) void sort_offsets_kernel(const int32_t* __restrict__ keys, int64_t n, int E, int32_t* __restrict__ offsets)
{
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e > E) return;
    int64_t lo = 0, hi = n;
    while (lo < hi) {
        const int64_t mid = (lo + hi) / 2;
        if (keys[mid] < e) lo = mid + 1; else hi = mid;
    }
    offsets[e] = (int32_t)lo;
}

__global__ __launch_bounds__(256) void zero_offsets_kernel(int32_t* offsets, int E)
{
    const int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (e <= E) offsets[e] = 0;
}

constexpr int FEW = 1024, ONE_DIGIT = 2047;                // choices of one launch; experts of one pass
constexpr int MOST_PARTS = 256;
// bytes of a row that is copied by part: 20000 tokens to 8 of 64, rows of 128 bytes 16.9 us, by token 31.5; of 256 20.6 | 31.9; of 512 38.9 | 35.1
constexpr int64_t NARROW = 256;
constexpr int64_t SOME = 1 << 19;                          // choices that are placed by part
// Choices that every workgroup counts, us | a wavefront for each choice's comparisons up to 1024, or three launches; calls in a row, in a graph: 32 tokens to 2 of 16 experts, rows of 2048 bytes 5.2, 3.9 | 5.1, 3.3
// (which costs less up to some 256 comparisons of a token's choices), 125 to 8 of 64 5.3, 4.7 | 10.9, 11.0, 600 to 2 of 16, rows of 8192 bytes 6.4, 6.2 | 11.9, 9.4, 2000 13.9, 14.3 | 14.6, 14.6, 4000 to 1 of 8, rows of 2048
// bytes 8.4, 8.5 | 11.7, 9.5; more: 3000 to 2 of 16, 8192 bytes 20 | 18, 8000 to 2 of 32, 512 bytes 18 | 13
constexpr int64_t COUNTED = 4096, COMPARED = 256;
bool at_once(int64_t n, int64_t top_k, int64_t E) { return n <= COUNTED && n * top_k > COMPARED && E <= ONE_DIGIT && top_k <= 64; }
constexpr int64_t SHORT_LIST = 256;                        // ... of a token: those in front of each are gone through for each, so that the work grows with their square
bool by_part(int64_t n, int64_t top_k, int64_t E) { return E <= ONE_DIGIT && n <= SOME && top_k <= SHORT_LIST; }
int64_t most_parts(int64_t E) { return (1 << 20) / (E + 1); }      // 4 MB of counts

int parts_of(int64_t n, int& part_rows)
{
    const int64_t rows = (n + MOST_PARTS - 1) / MOST_PARTS;
    part_rows = (int)((rows + 255) / 256 * 256);           // 64 of each of four wavefronts, or a multiple
    return (int)((n + part_rows - 1) / part_rows);
}

int64_t up16(int64_t bytes) { return (bytes + 15) / 16 * 16; }

int launched() { return hipGetLastError() == hipSuccess ? GEMM_F16_OK : GEMM_F16_ERR_LAUNCH; }

void launch_scan(int bins, int32_t* counts, int32_t* totals, int parts, hipStream_t stream)
{
    hipLaunchKernelGGL(sort_scan_kernel, dim3(bins), dim3(parts <= 256 ? 256 : 1024), 0, stream, counts, totals, parts);
}

int sort_pass(SortPass s, hipStream_t stream)
{
    hipLaunchKernelGGL(sort_count_kernel, dim3(s.parts), dim3(256), s.bins * sizeof(int), stream, s);
    launch_scan(s.bins, s.counts, s.totals, s.parts, stream);
    hipLaunchKernelGGL(sort_place_kernel, dim3(s.parts), dim3(256), 4 * s.bins * sizeof(int), stream, s);
    return launched();
}

// ---- and back ------------------------------------------------------------------------------------------------------------------------
// L threads for 8 L columns of a token, 8 each.  Rows of up to four choices are asked for together; products are rounded before they are added, in the
// order of the choices.  5001 tokens of 6 rows of 2304 in f16, and one more added: 32.6 us, 5.2 TB/s.
template <typename T, typename OT, bool WHOLE, int L>
__global__ __launch_bounds__(256) void combine_kernel(const CombineArgs a, int64_t pieces, int64_t items)
{
#pragma clang fp contract(off)
    int64_t item = (int64_t)blockIdx.x * (256 / L) + threadIdx.x / L;
    if constexpr (L == 64) item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= items) return;
    const int64_t t = item / pieces, c = (item % pieces * L + threadIdx.x % L) * 8;
    if (c >= a.N) return;
    float sum[8] = {};
    auto choices = [&](int j, auto number) {
        constexpr int U = decltype(number)::value;
        Raw8<T> v[U] = {};
        float w[U];
        bool there[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int place = a.place[t * a.top_k + j + u];
            there[u] = place >= 0 && place < a.rows;
            w[u] = a.weight ? a.weight[t * a.top_k + j + u] : 1.0f;
            if (there[u]) v[u] = load8_of<WHOLE>((const T*)a.Y + (int64_t)place * a.ldy, c, a.N);
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
            v[u] = settled<T, WHOLE>(v[u], c, a.N);
#pragma unroll
            for (int i = 0; i < 8; i++) { const float next = sum[i] + w[u] * (float)v[u][i]; sum[i] = there[u] ? next : sum[i]; }
        }
    };
    int j = 0;
    for (; j + 4 <= a.top_k; j += 4) choices(j, std::integral_constant<int, 4>{});
    if (j + 2 <= a.top_k) { choices(j, std::integral_constant<int, 2>{}); j += 2; }
    if (j < a.top_k) choices(j, std::integral_constant<int, 1>{});
    if (a.add) {
        const Raw8<T> v = settled<T, WHOLE>(load8_of<WHOLE>((const T*)a.add + t * a.ld_add, c, a.N), c, a.N);
#pragma unroll
        for (int i = 0; i < 8; i++) sum[i] += (float)v[i];
    }
    store8_of<WHOLE>((OT*)a.out + t * a.ldo + c, (int)min((int64_t)8, a.N - c), sum);
}

// ---- the gradients of that -----------------------------------------------------------------------------------------------------------
// L threads a token, R tokens a workgroup, P chunks of 8 columns a thread, U choices at a time.  8192 tokens of 2 rows of 2048 in bf16: 30.7 us, 5.5 TB/s.
template <typename T, bool WHOLE, int L, int P, int R, int U>
__global__ __launch_bounds__(L * R) void combine_grad_kernel(const CombineGradArgs a)
{
    constexpr int WAVES = L * R / 64, W = L > 64 ? L / 64 : 1;
    __shared__ float lds[2][U][WAVES];
    const int lane = threadIdx.x % L, wave = threadIdx.x >> 6;
    int64_t t = (int64_t)blockIdx.x * R + threadIdx.x / L;
    if constexpr (L == 64) t = (int64_t)blockIdx.x * R + __builtin_amdgcn_readfirstlane(wave);
    const bool live = t < a.T;
    t = min(t, a.T - 1);
    Raw8<T> dout[P];
#pragma unroll
    for (int p = 0; p < P; p++) dout[p] = load8_of<WHOLE>((const T*)a.dOut + t * a.lddo, 8 * (lane + L * p), a.N);
    int slot = 0;
    for (int j0 = 0; j0 < a.top_k; j0 += U) {
        Raw8<T> y[U][P] = {};
        float w[U], dot[U] = {};
        int place[U];
#pragma unroll
        for (int u = 0; u < U; u++) {
            const int64_t at = t * a.top_k + min(j0 + u, a.top_k - 1);
            place[u] = a.place[at];
            if (!live || j0 + u >= a.top_k || place[u] >= a.rows) place[u] = -1;
            w[u] = a.weight ? a.weight[at] : 1.0f;
            if (a.dweight && place[u] >= 0) {
#pragma unroll
                for (int p = 0; p < P; p++) y[u][p] = load8_of<WHOLE>((const T*)a.Y + (int64_t)place[u] * a.ldy, 8 * (lane + L * p), a.N);
            }
        }
        if (j0 == 0) {
#pragma unroll
            for (int p = 0; p < P; p++) dout[p] = settled<T, WHOLE>(dout[p], 8 * (lane + L * p), a.N);
        }
#pragma unroll
        for (int u = 0; u < U; u++) {
#pragma unroll
            for (int p = 0; p < P; p++) {
                const int c = 8 * (lane + L * p);
                y[u][p] = settled<T, WHOLE>(y[u][p], c, a.N);
#pragma unroll
                for (int i = 0; i < 8; i++) dot[u] += (float)dout[p][i] * (float)y[u][p][i];
                if (a.dY && place[u] >= 0 && c < a.N) {
                    float o[8];
#pragma unroll
                    for (int i = 0; i < 8; i++) o[i] = w[u] * (float)dout[p][i];
                    store8_of<WHOLE>((T*)a.dY + (int64_t)place[u] * a.lddy + c, a.N - c, o);
                }
            }
        }
        if (!a.dweight) continue;
#pragma unroll
        for (int u = 0; u < U; u++) {
            if constexpr (L >= 64) dot[u] = sum64(dot[u]);
            else {
#pragma unroll
                for (int d = 1; d < L; d <<= 1) dot[u] += __shfl_xor(dot[u], d);
            }
        }
        if constexpr (L > 64) {                            // two sets in turn: one barrier for U choices
#pragma unroll
            for (int u = 0; u < U; u++) if ((threadIdx.x & 63) == 0) lds[slot][u][wave] = dot[u];
            __syncthreads();
#pragma unroll
            for (int u = 0; u < U; u++) {
                dot[u] = 0.0f;
#pragma unroll
                for (int i = 0; i < W; i++) dot[u] += lds[slot][u][wave / W * W + i];
            }
            slot ^= 1;
        }
#pragma unroll
        for (int u = 0; u < U; u++) if (live && lane == 0 && j0 + u < a.top_k) a.dweight[t * a.top_k + j0 + u] = place[u] >= 0 ? dot[u] : 0.0f;
    }
}
// rows of any length, a workgroup a token, gone through again for each choice
template <typename T>
__global__ __launch_bounds__(512) void combine_grad_long_kernel(const CombineGradArgs a)
{
    __shared__ float lds[8];
    const int64_t t = blockIdx.x;
    const T* const d = (const T*)a.dOut + t * a.lddo;
    for (int j = 0; j < a.top_k; j++) {
        const int place = a.place[t * a.top_k + j];
        const bool there = place >= 0 && place < a.rows;
        const float w = a.weight ? a.weight[t * a.top_k + j] : 1.0f;
        float dot = 0.0f;
        for (int64_t c = 8 * (int64_t)threadIdx.x; there && c < a.N; c += 4096) {
            const int left = (int)min((int64_t)8, a.N - c);
            float g[8], v[8], o[8];
            load8(d + c, left, g);
            if (a.dweight) {
                load8((const T*)a.Y + (int64_t)place * a.ldy + c, left, v);
#pragma unroll
                for (int i = 0; i < 8; i++) dot += g[i] * v[i];
            }
#pragma unroll
            for (int i = 0; i < 8; i++) o[i] = w * g[i];
            if (a.dY) store8((T*)a.dY + (int64_t)place * a.lddy + c, left, o);
        }
        if (a.dweight) {
            dot = sum_row<8>(dot, lds);
            if (threadIdx.x == 0) a.dweight[t * a.top_k + j] = dot;
        }
    }
}

template <typename T, int L, int P, int R, int U>
int launch_combine_grad(const CombineGradArgs& a, hipStream_t stream)
{
    const dim3 grid((unsigned)((a.T + R - 1) / R));
    if (a.N % 8 == 0) hipLaunchKernelGGL((combine_grad_kernel<T, true, L, P, R, U>), grid, dim3(L * R), 0, stream, a);
    else hipLaunchKernelGGL((combine_grad_kernel<T, false, L, P, R, U>), grid, dim3(L * R), 0, stream, a);
    return launched();
}
template <typename T>
int launch_combine_grad_long(const CombineGradArgs& a, hipStream_t stream)
{
    hipLaunchKernelGGL(combine_grad_long_kernel<T>, dim3((unsigned)a.T), dim3(512), 0, stream, a);
    return launched();
}
template <typename T>
int combine_grad_of_type(const CombineGradArgs& a, hipStream_t stream)
{
    if (a.N == 0) return launch_combine_grad_long<T>(a, stream);             // zeros to dweight: the others read a row's last 8 elements in place of what it has not
    if (a.T <= 2 * chip().cus && a.N > 1024 && a.N <= 8192) return a.N <= 4096 ? launch_combine_grad<T, 512, 1, 1, 4>(a, stream) : launch_combine_grad<T, 1024, 1, 1, 4>(a, stream);
    if (a.N <= 64) return launch_combine_grad<T, 8, 1, 32, 4>(a, stream);
    if (a.N <= 128) return launch_combine_grad<T, 16, 1, 16, 4>(a, stream);
    if (a.N <= 256) return launch_combine_grad<T, 32, 1, 8, 4>(a, stream);
    if (a.N <= 512) return launch_combine_grad<T, 64, 1, 4, 4>(a, stream);
    if (a.N <= 1024) return launch_combine_grad<T, 64, 2, 4, 2>(a, stream);
    if (a.N <= 2048) return launch_combine_grad<T, 64, 4, 4, 2>(a, stream);
    if (a.N <= 4096) return launch_combine_grad<T, 256, 2, 1, 2>(a, stream);
    return a.N <= 8192 ? launch_combine_grad<T, 256, 4, 1, 2>(a, stream) : launch_combine_grad_long<T>(a, stream);
}

template <typename T, typename OT, int L>
int launch_combine(const CombineArgs& a, hipStream_t stream)
{
    const int64_t pieces = ((int64_t)a.N + 8 * L - 1) / (8 * L), items = a.T * pieces;
    const dim3 grid((unsigned)((items + 256 / L - 1) / (256 / L)));
    if (a.N % 8 == 0) hipLaunchKernelGGL((combine_kernel<T, OT, true, L>), grid, dim3(256), 0, stream, a, pieces, items);
    else hipLaunchKernelGGL((combine_kernel<T, OT, false, L>), grid, dim3(256), 0, stream, a, pieces, items);
    return launched();
}
template <typename T, typename OT>
int combine_of_type(const CombineArgs& a, hipStream_t stream)
{
    return a.N <= 64 ? launch_combine<T, OT, 8>(a, stream) : a.N <= 128 ? launch_combine<T, OT, 16>(a, stream) : a.N <= 256 ? launch_combine<T, OT, 32>(a, stream) : launch_combine<T, OT, 64>(a, stream);
}

// Tokens need nothing of each other: more than the grid of one launch has wavefronts for (pieces of a token each) go in several.
int64_t tokens_of_a_launch(int64_t pieces) { return pieces >= (1 << 24) ? 1 : (1 << 24) / pieces; }
template <typename F>
int by_tokens(int64_t T, int64_t pieces, F launch)
{
    const int64_t most = tokens_of_a_launch(pieces);
    int rc = GEMM_F16_OK;
    for (int64_t t = 0; t < T && rc == GEMM_F16_OK; t += most) rc = launch(t, T - t < most ? T - t : most);
    return rc;
}
const char* ahead(const void* p, int64_t bytes) { return p ? (const char*)p + bytes : nullptr; }

}  // namespace

int64_t ops_dispatch_workspace_bytes(int64_t T, int64_t top_k, int64_t E)
{
    const int64_t n = T * top_k;
    if (n <= FEW || at_once(n, top_k, E)) return 0;
    if (by_part(n, top_k, E)) return up16(4 * (E + 1) * (most_parts(E) + 1));
    int part_rows;
    return up16(4 * 256 * ((int64_t)parts_of(n, part_rows) + 1)) + 2 * up16(4 * n);
}

int ops_launch_dispatch(const DispatchArgs& a, void* workspace, hipStream_t stream)
{
    const int64_t n = a.T * a.top_k;
    if (n == 0) {
        hipLaunchKernelGGL(zero_offsets_kernel, dim3((unsigned)(((int64_t)a.E + 256) / 256)), dim3(256), 0, stream, a.offsets, a.E);
        return launched();
    }
    const int64_t bytes = (int64_t)a.N * a.size, pieces = a.X && bytes > PIECE ? (bytes + PIECE - 1) / PIECE : 1, items = a.T * pieces;
    if (at_once(n, a.top_k, a.E)) {
        const int64_t most = 64 / a.top_k, each = (a.T + 511) / 512;         // 512 workgroups: two a compute unit count at the same time
        const int tokens = (int)(each < most ? each : most);
        hipLaunchKernelGGL(dispatch_some_kernel, dim3((unsigned)((a.T + tokens - 1) / tokens)), dim3(256), 2 * (a.E + 1) * sizeof(int), stream, a, tokens, pieces);
        return launched();
    }
    if (n <= FEW) {
        if (!fits_a_launch((items + 3) / 4 + ((int64_t)a.E + 8) / 8, 256)) return GEMM_F16_ERR_SIZE;
        const dim3 grid((unsigned)((items + ((int64_t)a.E + 8) / 8 + 3) / 4));
        if (n <= 64) hipLaunchKernelGGL(dispatch_few_kernel<1>, grid, dim3(256), 0, stream, a, pieces, items);
        else if (n <= 256) hipLaunchKernelGGL(dispatch_few_kernel<4>, grid, dim3(256), 0, stream, a, pieces, items);
        else hipLaunchKernelGGL(dispatch_few_kernel<16>, grid, dim3(256), 0, stream, a, pieces, items);
        return launched();
    }
    if (by_part(n, a.top_k, a.E)) {
        Parts s = {};
        s.a = a;
        const int bins = a.E + 1;
        const int64_t some = a.top_k < 64 ? 64 / a.top_k : 1, enough = (a.T + most_parts(a.E) - 1) / most_parts(a.E);
        s.tokens = (int)(some > enough ? some : enough);
        s.parts = (int)((a.T + s.tokens - 1) / s.tokens);
        s.totals = (int32_t*)workspace;
        s.counts = s.totals + bins;
        const bool narrow = bytes <= NARROW && (int64_t)s.tokens * a.top_k <= 64;
        const int64_t waves = (narrow ? s.parts : items) + (bins + 63) / 64;
        if (!fits_a_launch((waves + 3) / 4, 256)) return GEMM_F16_ERR_SIZE;
        hipLaunchKernelGGL(part_count_kernel, dim3((s.parts + 3) / 4), dim3(256), 4 * bins * sizeof(int), stream, s);
        launch_scan(bins, s.counts, s.totals, s.parts, stream);
        // From half of the 256 MB cache on rows go past it.  That pays for the call by itself, and neither pays nor costs for it and what reads the rows next: us past | through the cache, 8192 tokens
        // to 2 of 16, bf16 rows of 4096 (134 MB) 37 | 46, with a copy of the rows behind it 97 | 97, with a product of 768 columns 137 | 140, of 1024 209 | 201, of 4096 499 | 496; 16384 tokens (268 MB)
        // 80 | 84, 188 | 183, 261 | 269, 288 | 290, 877 | 874; 16384 to 8 of 64, rows of 1024 63 | 70, 173 | 184, 267 | 269, 328 | 331, 1053 | 1048.  Below, a reader finds them in the cache:
        // 4096 tokens (67 MB) 22 | 26, with a copy 50 | 46
        if (narrow) {
            int R = 1;
            while (16 * R < bytes) R *= 2;
            hipLaunchKernelGGL(part_move_narrow_kernel, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, stream, s, R);
        } else if (n * bytes >= 128e6) hipLaunchKernelGGL(part_move_kernel<true>, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, stream, s, pieces, items);
        else hipLaunchKernelGGL(part_move_kernel<false>, dim3((unsigned)((waves + 3) / 4)), dim3(256), 0, stream, s, pieces, items);
        return launched();
    }
    SortPass s = {};
    s.a = a;
    s.parts = parts_of(n, s.part_rows);
    s.totals = (int32_t*)workspace;
    s.counts = s.totals + 256;
    int32_t* const order = (int32_t*)((char*)workspace + up16(4 * 256 * ((int64_t)s.parts + 1)));
    int32_t* const keys = (int32_t*)((char*)order + up16(4 * n));
    s.shift = -1; s.bins = 256; s.out = order;
    int rc = sort_pass(s, stream);
    s.seq = order; s.shift = 8; s.bins = (a.E >> 8) + 1; s.out = nullptr; s.keys = keys;
    if (rc == GEMM_F16_OK) rc = sort_pass(s, stream);
    if (rc == GEMM_F16_OK) hipLaunchKernelGGL(sort_offsets_kernel, dim3((unsigned)(((int64_t)a.E + 256) / 256)), dim3(256), 0, stream, keys, n, a.E, a.offsets);
    if (rc == GEMM_F16_OK) rc = launched();
    if (rc != GEMM_F16_OK || !a.X) return rc;
    return by_tokens(a.T, pieces, [&](int64_t t, int64_t tokens) {
        DispatchArgs m = a;
        m.T = tokens;
        m.X = ahead(a.X, t * a.ldx * a.size);
        m.place = a.place + t * a.top_k;
        m.scale = (const float*)ahead(a.scale, 4 * t);
        hipLaunchKernelGGL(move_rows_kernel, dim3((unsigned)((tokens * pieces + 3) / 4)), dim3(256), 0, stream, m, pieces, tokens * pieces);
        return launched();
    });
}

int ops_launch_combine(int type, int out_type, const CombineArgs& all, hipStream_t stream)
{
    const int64_t size = type == GEMM_TYPE_F32 ? 4 : 2, out_size = out_type == GEMM_TYPE_F32 ? 4 : 2;
    return by_tokens(all.T, ((int64_t)all.N + 511) / 512, [&](int64_t t, int64_t tokens) {
        CombineArgs a = all;
        a.T = tokens;
        a.place = all.place + t * all.top_k;
        a.weight = (const float*)ahead(all.weight, 4 * t * all.top_k);
        a.add = ahead(all.add, t * all.ld_add * size);
        a.out = (char*)all.out + t * all.ldo * out_size;
        if (type == GEMM_TYPE_F32) return combine_of_type<float, float>(a, stream);
        if (type == GEMM_TYPE_F16) return out_type == GEMM_TYPE_F32 ? combine_of_type<half_t, float>(a, stream) : combine_of_type<half_t, half_t>(a, stream);
        return out_type == GEMM_TYPE_F32 ? combine_of_type<bf16_t, float>(a, stream) : combine_of_type<bf16_t, bf16_t>(a, stream);
    });
}
int ops_launch_combine_grad(int type, const CombineGradArgs& all, hipStream_t stream)
{
    return by_tokens(all.T, 8, [&](int64_t t, int64_t tokens) {
        CombineGradArgs a = all;
        a.T = tokens;
        a.place = all.place + t * all.top_k;
        a.dOut = ahead(all.dOut, t * all.lddo * 2);
        a.weight = (const float*)ahead(all.weight, 4 * t * all.top_k);
        a.dweight = (float*)ahead(all.dweight, 4 * t * all.top_k);
        return type == GEMM_TYPE_F16 ? combine_grad_of_type<half_t>(a, stream) : combine_grad_of_type<bf16_t>(a, stream);
    });
}
