// Tokens sorted by expert, their rows moved there and back with weights applied, and the gradients of that (include/gemm_layer.h).
//
// The order is a counting sort: how many choices of each expert lie before a choice's own, and how many of its own.  Nothing atomic
// decides a place, so the order is always the same.  Rows move by token: a token's row is read once and stored to its places,
// and on the way back a lane adds the elements of a token's rows in their order.  Both are bound by memory.
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
    __device__ __forceinline__ void store(char* row, int64_t bytes) const
    {
#pragma unroll
        for (int i = 0; i < ROW_CHUNKS; i++)
            if (at[i] >= 0 && bytes >= 16) *(uintx4_any*)(row + at[i]) = v[i];
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
// of smaller ones: NR comparisons of a wavefront.  A wavefront for each piece of a token's row, and one for each 8 experts' offsets.
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

// ---- many choices: a counting sort by one digit ------------------------------------------------------------------------------------
// `parts` workgroups of part_rows choices each count their digits; a second launch makes of each digit's counts the sums of those before;
// a third one finds each choice's place.  Up to 2047 experts are one digit; more are sorted by the low 8 bits and then by the rest.
struct SortPass {
    DispatchArgs a;
    const int32_t* seq;                                    // the choices in the order that this pass goes by; NULL: as they are
    int shift, bins, part_rows, parts;
    int32_t *counts, *totals;                              // [digit][part], [digit]
    int32_t* out;                                          // the choices as this pass orders them; NULL: the places and sources are written
    int32_t* keys;                                         // the experts in order, of the last of two passes; NULL: there is one pass, which writes offsets
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

__device__ __forceinline__ int scan64(int x)               // sums of all lanes up to and with this one
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const int v = __shfl_up(x, d);
        if (lane >= d) x += v;
    }
    return x;
}

__global__ __launch_bounds__(256) void sort_scan_kernel(const SortPass s)
{
    const int lane = threadIdx.x & 63, b = blockIdx.x * 4 + (threadIdx.x >> 6);
    if (b >= s.bins) return;
    int32_t* const c = s.counts + (int64_t)b * s.parts;
    int before = 0;
    for (int p = 0; p < s.parts; p += 64) {
        const int v = p + lane < s.parts ? c[p + lane] : 0, incl = scan64(v);
        if (p + lane < s.parts) c[p + lane] = before + incl - v;
        before += __shfl(incl, 63);
    }
    if (lane == 0) s.totals[b] = before;
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
    // where each digit begins: sums over the digits before, 8 of them a thread
    int sum = 0;
    for (int i = 0; i < 8; i++) { const int b = threadIdx.x * 8 + i; if (b < s.bins) sum += s.totals[b]; }
    const int incl = scan64(sum);
    if (lane == 63) wave_sums[wave] = incl;
    __syncthreads();
    int start = incl - sum;
    for (int w = 0; w < wave; w++) start += wave_sums[w];
    for (int i = 0; i < 8; i++) {
        const int b = threadIdx.x * 8 + i;
        if (b >= s.bins) break;
        if (blockIdx.x == 0 && !s.out && !s.keys) s.a.offsets[b] = start;
        int at = start + s.counts[(int64_t)b * s.parts + blockIdx.x];
        for (int w = 0; w < 4; w++) { const int c = base[w * s.bins + b]; base[w * s.bins + b] = at; at += c; }
        start += s.totals[b];
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
        if (s.keys) s.keys[at] = key;
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

int parts_of(int64_t n, int& part_rows)
{
    const int64_t rows = (n + MOST_PARTS - 1) / MOST_PARTS;
    part_rows = (int)((rows + 255) / 256 * 256);           // 64 of each of four wavefronts, or a multiple
    return (int)((n + part_rows - 1) / part_rows);
}

int64_t up16(int64_t bytes) { return (bytes + 15) / 16 * 16; }

int launched() { return hipGetLastError() == hipSuccess ? GEMM_F16_OK : GEMM_F16_ERR_LAUNCH; }

int sort_pass(SortPass s, hipStream_t stream)
{
    hipLaunchKernelGGL(sort_count_kernel, dim3(s.parts), dim3(256), s.bins * sizeof(int), stream, s);
    hipLaunchKernelGGL(sort_scan_kernel, dim3((s.bins + 3) / 4), dim3(256), 0, stream, s);
    hipLaunchKernelGGL(sort_place_kernel, dim3(s.parts), dim3(256), 4 * s.bins * sizeof(int), stream, s);
    return launched();
}

// ---- and back ------------------------------------------------------------------------------------------------------------------------
// 8 elements a lane, a wavefront for 512 columns of a token.  Products are rounded before they are added, in the order of the choices.
template <typename T, typename OT>
__global__ __launch_bounds__(256) void combine_kernel(const CombineArgs a, int64_t pieces, int64_t items)
{
#pragma clang fp contract(off)
    const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (item >= items) return;
    const int64_t t = item / pieces, c = item % pieces * 512 + 8 * (threadIdx.x & 63);
    if (c >= a.N) return;
    const int left = (int)min((int64_t)8, a.N - c);
    float sum[8] = {};
    for (int j = 0; j < a.top_k; j++) {
        const int place = __builtin_amdgcn_readfirstlane(a.place[t * a.top_k + j]);
        if (place < 0 || place >= a.rows) continue;
        const float w = a.weight ? a.weight[t * a.top_k + j] : 1.0f;
        float v[8];
        load8((const T*)a.Y + (int64_t)place * a.ldy + c, left, v);
#pragma unroll
        for (int i = 0; i < 8; i++) sum[i] += w * v[i];
    }
    if (a.add) {
        float v[8];
        load8((const T*)a.add + t * a.ld_add + c, left, v);
#pragma unroll
        for (int i = 0; i < 8; i++) sum[i] += v[i];
    }
    store8((OT*)a.out + t * a.ldo + c, left, sum);
}

// ---- the gradients of that -----------------------------------------------------------------------------------------------------------
// W wavefronts a token, R tokens a workgroup, P chunks of 8 columns a lane in registers; LOOP: rows of any length, gone through again for each choice
template <typename T, int W, int P, int R, bool LOOP>
__global__ __launch_bounds__(64 * W * R) void combine_grad_kernel(const CombineGradArgs a)
{
    __shared__ float lds[W * R];
    const int lane = threadIdx.x % (64 * W);
    const int64_t t = (int64_t)blockIdx.x * R + threadIdx.x / (64 * W);
    const bool live = t < a.T;
    const T* const d = (const T*)a.dOut + t * a.lddo;
    Raw8<T> dout[P];
    if constexpr (!LOOP) {
#pragma unroll
        for (int p = 0; p < P; p++) dout[p] = load8_raw(d + 8 * (lane + 64 * W * p), live ? a.N - 8 * (lane + 64 * W * p) : 0);
    }
    for (int j = 0; j < a.top_k; j++) {
        const int place = live ? a.place[t * a.top_k + j] : -1;
        const bool there = place >= 0 && place < a.rows;
        const float w = there && a.weight ? a.weight[t * a.top_k + j] : 1.0f;
        const T* const y = (const T*)a.Y + (int64_t)place * a.ldy;
        T* const dy = (T*)a.dY + (int64_t)place * a.lddy;
        float dot = 0.0f;
        auto chunk = [&](int64_t c, const Raw8<T>& g) {
            const int left = (int)min((int64_t)8, a.N - c);
            if (a.dweight) {
                float v[8];
                load8(y + c, left, v);
#pragma unroll
                for (int i = 0; i < 8; i++) dot += (float)g[i] * v[i];
            }
            if (a.dY) {
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; i++) o[i] = w * (float)g[i];
                store8(dy + c, left, o);
            }
        };
        if (there) {
            if constexpr (LOOP) {
                for (int64_t c = 8 * (int64_t)lane; c < a.N; c += 512 * W) chunk(c, load8_raw(d + c, (int)min((int64_t)8, a.N - c)));
            } else {
#pragma unroll
                for (int p = 0; p < P; p++) if (8 * (lane + 64 * W * p) < a.N) chunk(8 * (lane + 64 * W * p), dout[p]);
            }
        }
        if (a.dweight) {
            dot = sum_row<W>(dot, lds);
            if (live && lane == 0) a.dweight[t * a.top_k + j] = dot;
        }
    }
}

template <typename T, int W, int P, int R, bool LOOP = false>
int launch_combine_grad(const CombineGradArgs& a, hipStream_t stream)
{
    hipLaunchKernelGGL((combine_grad_kernel<T, W, P, R, LOOP>), dim3((unsigned)((a.T + R - 1) / R)), dim3(64 * W * R), 0, stream, a);
    return launched();
}
template <typename T>
int combine_grad_of_type(const CombineGradArgs& a, hipStream_t stream)
{
    if (a.N <= 512) return launch_combine_grad<T, 1, 1, 4>(a, stream);
    if (a.N <= 1024) return launch_combine_grad<T, 1, 2, 4>(a, stream);
    if (a.N <= 2048) return launch_combine_grad<T, 1, 4, 4>(a, stream);
    if (a.N <= 4096) return launch_combine_grad<T, 4, 2, 1>(a, stream);
    if (a.N <= 8192) return launch_combine_grad<T, 4, 4, 1>(a, stream);
    return launch_combine_grad<T, 8, 1, 1, true>(a, stream);
}

template <typename T, typename OT>
int launch_combine(const CombineArgs& a, hipStream_t stream)
{
    const int64_t pieces = ((int64_t)a.N + 511) / 512, items = a.T * pieces;
    hipLaunchKernelGGL((combine_kernel<T, OT>), dim3((unsigned)((items + 3) / 4)), dim3(256), 0, stream, a, pieces, items);
    return launched();
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

int64_t ops_dispatch_workspace_bytes(int64_t n, int64_t E)
{
    if (n <= FEW) return 0;
    int part_rows;
    const int64_t parts = parts_of(n, part_rows), bins = E <= ONE_DIGIT ? E + 1 : 256;
    return up16(4 * bins * (parts + 1)) + (E <= ONE_DIGIT ? 0 : 2 * up16(4 * n));
}

int ops_launch_dispatch(const DispatchArgs& a, void* workspace, hipStream_t stream)
{
    const int64_t n = a.T * a.top_k;
    if (n == 0) {
        hipLaunchKernelGGL(zero_offsets_kernel, dim3((unsigned)(((int64_t)a.E + 256) / 256)), dim3(256), 0, stream, a.offsets, a.E);
        return launched();
    }
    const int64_t bytes = (int64_t)a.N * a.size, pieces = a.X && bytes > PIECE ? (bytes + PIECE - 1) / PIECE : 1, items = a.T * pieces;
    if (n <= FEW) {
        if (!fits_a_launch((items + 3) / 4 + ((int64_t)a.E + 8) / 8, 256)) return GEMM_F16_ERR_SIZE;
        const dim3 grid((unsigned)((items + ((int64_t)a.E + 8) / 8 + 3) / 4));
        if (n <= 64) hipLaunchKernelGGL(dispatch_few_kernel<1>, grid, dim3(256), 0, stream, a, pieces, items);
        else if (n <= 256) hipLaunchKernelGGL(dispatch_few_kernel<4>, grid, dim3(256), 0, stream, a, pieces, items);
        else hipLaunchKernelGGL(dispatch_few_kernel<16>, grid, dim3(256), 0, stream, a, pieces, items);
        return launched();
    }
    SortPass s = {};
    s.a = a;
    s.parts = parts_of(n, s.part_rows);
    int rc;
    if (a.E <= ONE_DIGIT) {
        s.shift = 0;
        s.bins = a.E + 1;
        s.totals = (int32_t*)workspace;
        s.counts = s.totals + s.bins;
        rc = sort_pass(s, stream);
    } else {
        s.totals = (int32_t*)workspace;
        s.counts = s.totals + 256;
        int32_t* const order = (int32_t*)((char*)workspace + up16(4 * 256 * ((int64_t)s.parts + 1)));
        int32_t* const keys = (int32_t*)((char*)order + up16(4 * n));
        s.shift = -1; s.bins = 256; s.out = order;
        rc = sort_pass(s, stream);
        s.seq = order; s.shift = 8; s.bins = (a.E >> 8) + 1; s.out = nullptr; s.keys = keys;
        if (rc == GEMM_F16_OK) rc = sort_pass(s, stream);
        if (rc == GEMM_F16_OK) hipLaunchKernelGGL(sort_offsets_kernel, dim3((unsigned)(((int64_t)a.E + 256) / 256)), dim3(256), 0, stream, keys, n, a.E, a.offsets);
    }
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
        if (type == GEMM_TYPE_F32) return launch_combine<float, float>(a, stream);
        if (type == GEMM_TYPE_F16) return out_type == GEMM_TYPE_F32 ? launch_combine<half_t, float>(a, stream) : launch_combine<half_t, half_t>(a, stream);
        return out_type == GEMM_TYPE_F32 ? launch_combine<bf16_t, float>(a, stream) : launch_combine<bf16_t, bf16_t>(a, stream);
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
