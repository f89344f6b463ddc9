// Products with a weight held in its compressed form: y = act(x W^T + b) + r, and the gradients.
//
// Numbers: the matrix cores multiply fp16 numbers (11 bits) exactly into fp32 sums.  A row of an operand is scaled by a
// power of two that brings its largest magnitude into [2^14, 2^15), so that everything above 2^-29 of that magnitude is a
// normal fp16 number and nothing is off by more than 2^-39 of it; a second plane of fp16 numbers takes what the first one
// leaves over (22 bits together).  With h and l for the planes of either side a product takes
//   1 pass   h h                for bfloat16 results: a factor rounded to 11 bits is off by 2^-11 at most, an eighth of
//                               the result's own 2^-8 (a quarter where both are rounded, as in the gradient below an
//                               activation), and bfloat16 activations (8 bits) are exact in h
//   2 passes h h + h l          for fp16 results: fp16 activations are exact in h, the weight is off by 2^-23
//   3 passes h h + h l + l h    for fp32 results: what is left out, l l, is 2^-22 of the product, and each factor off by 2^-23
// (two passes for bfloat16 would double what bounds the large products, for a tenth of the results one step of 2^-8 nearer.)
// (three planes of bfloat16 would need six passes for fp32, and two for bfloat16 results).
//
// What bounds it, measured: 2048 rows through 4096 x 11008 bf16 226 to 251 us from card to card, of which the product takes 224 to 231 (0.8 PFLOP/s, the matrix
// cores at work in 48 % of the busy cycles; its floor at the rate of the library's largest products is 133) and the
// weight's planes 38 (34 MB of symbols to 90 MB of planes, 3.3 TB/s).  Small products and the gradients are three to six launches
// one after the other: 512 rows through 768 x 768 fp32 24 us, the gradients of 1024 x 1024 x 4096 bf16 66, of 515 x 1000 x 1537 fp32 51.
#include "inshr_table.h"

#include <algorithm>

namespace inshr {

// ------------------------------------------------------------------------------------------
// planes of an operand whose reduction runs along its rows
// ------------------------------------------------------------------------------------------
constexpr u32 KT = 64; // planes are padded to it along the reduction, with zeros
constexpr u32 KS = 32; // reduction per step of the product
constexpr u32 GROUP = 4;
inline u64 up(u64 v, u64 to) { return (v + to - 1) / to * to; }

// Planes lie in blocks of 16 rows x 32 numbers, 1024 bytes that one load of the product takes to LDS as they are: a row's
// four pieces of eight numbers in an order of the row's own (piece c at c ^ turn_of(row)), so that the lanes whose reads of LDS
// are served together meet in different banks: the 16 rows of a piece, and also rows 0-3 and 12-15 of one piece with 4-11
// of the next (with c ^ (row / 4 % 4) every read took four cycles more, of twelve).  (Rows of a row-major plane gave the loads pieces of 64 bytes, at 60 % of
// what a CU takes from L2 in whole lines.)  Place of number c of row r, for planes of ld numbers a row:
__device__ __forceinline__ u32 turn_of(u32 r) { return (0u - (r >> 2)) & 3u; }
__device__ __forceinline__ u64 plane_at(u64 r, u64 c, u64 ld)
{
    return ((r >> 4) * (ld / KS) + c / KS) * (16u * KS) + (r & 15u) * KS + ((c / 8u & 3u) ^ turn_of((u32)r)) * 8u + (c & 7u);
}

struct PlaneSrc { // a matrix of elements; act != ACT_NONE: multiplied by the slope at the values of `pre`
    const void *p, *pre;
    u64 stride, pre_stride;
    u32 rows, cols, act, pad;
};

// The largest magnitudes of the centres and of parts of the protected list, to be joined by whoever needs the scale.
constexpr u32 WMAX_PARTS = 64;
__device__ __forceinline__ void weight_max_part(const WDesc &w, u32 which, u32 *part)
{
    u32 m = 0u;
    if (which == 0 && threadIdx.x < w.K) m = finite_mag(gptr(w.codebook)[threadIdx.x]);
    for (u64 j = which * 256ull + threadIdx.x; j < w.n_outlier; j += 256ull * WMAX_PARTS) m = max(m, finite_mag(protected_value(w, j)));
    __shared__ u32 red[4];
    m = wave_max_u(m);
    if ((threadIdx.x & 63u) == 0u) red[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x == 0) part[which] = max(max(red[0], red[1]), max(red[2], red[3]));
}
__device__ __forceinline__ void weight_scale(const u32 *part, float &s, float &inv) // by every wave
{
    scale_of(wave_max_u(gptr(part)[threadIdx.x & 63u]), s, inv);
}

// Eight scaled values as one or two planes.
template <int P>
__device__ __forceinline__ void put_planes(const float (&v)[8], float s, _Float16 *at, u64 plane)
{
    h8 hi, lo;
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const float x = v[i] * s;
        hi[i] = (_Float16)x;
        lo[i] = (_Float16)(x - (float)hi[i]);
    }
    *(h8 *)at = hi;
    if (P > 1) *(h8 *)(at + plane) = lo;
}

struct RowPlanes {
    PlaneSrc src;
    _Float16 *dst;
    u64 plane;
    float *inv;
    u32 ld, type;
};

// Row r, by a workgroup of 256, which reads it twice.
template <u32 TY, int P>
__device__ __forceinline__ void row_planes(const RowPlanes &j, u64 r)
{
    typedef typename Elem<TY>::type T;
    const GLOBAL_AS T *p = (const GLOBAL_AS T *)j.src.p + r * j.src.stride;
    __shared__ u32 red[4];
    u32 m = 0u;
    for (u32 c = threadIdx.x * 8u; c < j.src.cols; c += 2048u) {
        const Raw8<TY> x = load_raw8<TY>(p + c, j.src.cols - c);
#pragma unroll
        for (int i = 0; i < 8; i++) m = max(m, finite_mag(x[i]));
    }
    m = wave_max_u(m);
    if ((threadIdx.x & 63u) == 0u) red[threadIdx.x >> 6] = m;
    __syncthreads();
    float s, inv;
    scale_of(max(max(red[0], red[1]), max(red[2], red[3])), s, inv);
    if (threadIdx.x == 0) j.inv[r] = inv;
    for (u32 c = threadIdx.x * 8u; c < j.ld; c += 2048u) {
        float v[8];
        load8<TY>(p + c, c < j.src.cols ? j.src.cols - c : 0u, v);
        put_planes<P>(v, s, j.dst + plane_at(r, c, j.ld), j.plane);
    }
}

// The rows, and in the first WMAX_PARTS workgroups the weight's largest values.
template <u32 TY, int P>
__global__ __launch_bounds__(256) void k_row_planes(RowPlanes j, WDesc w, u32 *__restrict__ part)
{
    if (blockIdx.x < WMAX_PARTS)
        weight_max_part(w, blockIdx.x, part);
    else
        row_planes<TY, P>(j, blockIdx.x - WMAX_PARTS);
}

// ------------------------------------------------------------------------------------------
// the gradient below the activation, and the activations turned round
// ------------------------------------------------------------------------------------------
// Both are cut into tiles of 64 x 64.  k_tile_stats takes each tile's largest magnitudes per row and per column and its
// sums per column; k_scales (or the launch of the weight's planes) joins them, in a fixed order; k_tile_planes works the values
// out again (they come from the caches, and two planes of them would be as much to write and read) and stores the
// planes, the turned ones through LDS.  Memory and the slopes bound both: 8.4 and 10 us at 1024 x 1024 x 4096 bf16 gelu_tanh
// (19 MB read each, 19 MB of planes written; 4 us of it a launch).
struct TileJob {
    PlaneSrc src;
    u32 col_tiles, row_tiles;
    u32 *row_max, *col_max;  // [col_tiles][rows], [row_tiles][cols]; NULL: not wanted
    float *col_sum;          // [row_tiles][cols]
    float *inv_row, *inv_col, *sum; // joined
    _Float16 *by_row, *by_col;      // planes of the rows, of the columns
    u64 plane_row, plane_col, ld_row, ld_col;
};
struct TileJobs {
    TileJob job[2];
    u32 tiles0, tiles; // of the first, of both
};

// Rows i / 8 and i / 8 + 32 of the tile, eight columns from i % 8 * 8 on, for thread i.
template <u32 TY>
__device__ __forceinline__ void tile_values(const PlaneSrc &src, u64 r0, u32 c0, float (&v)[2][8])
{
    typedef typename Elem<TY>::type T;
    const u32 c = c0 + (threadIdx.x & 7u) * 8u;
#pragma unroll
    for (u32 h = 0; h < 2u; h++) {
        const u64 r = r0 + (threadIdx.x >> 3) + 32u * h;
        const u32 left = r < src.rows && c < src.cols ? src.cols - c : 0u;
        load8<TY>((const GLOBAL_AS T *)src.p + r * src.stride + c, left, v[h]);
        if (src.act != ACT_NONE) {
            float a[8];
            load8<TY>((const GLOBAL_AS T *)src.pre + r * src.pre_stride + c, left, a);
            act_grad(v[h], a, src.act); // (0 where nothing is: 0 times a slope at 0)
        }
    }
}

template <u32 TY>
__global__ __launch_bounds__(256) void k_tile_stats(TileJobs jobs, WDesc w, u32 *__restrict__ part)
{
    if (blockIdx.x >= jobs.tiles) {
        weight_max_part(w, blockIdx.x - jobs.tiles, part);
        return;
    }
    const bool second = blockIdx.x >= jobs.tiles0;
    const TileJob &j = jobs.job[second];
    const u32 tile = blockIdx.x - (second ? jobs.tiles0 : 0u), rt = tile / j.col_tiles, ct = tile - rt * j.col_tiles;
    const u64 r0 = rt * 64ull;
    const u32 c0 = ct * 64u, i = threadIdx.x;
    float v[2][8];
    tile_values<TY>(j.src, r0, c0, v);
    __shared__ u32 mags[4][64];
    __shared__ float sums[4][64];
    u32 cm[8];
    float cs[8];
#pragma unroll
    for (int q = 0; q < 8; q++) {
        cm[q] = max(finite_mag(v[0][q]), finite_mag(v[1][q]));
        cs[q] = v[0][q] + v[1][q];
    }
    if (j.row_max) {
#pragma unroll
        for (u32 h = 0; h < 2u; h++) {
            u32 m = 0u;
#pragma unroll
            for (int q = 0; q < 8; q++) m = max(m, finite_mag(v[h][q]));
#pragma unroll
            for (int d = 4; d; d >>= 1) m = max(m, __shfl_xor(m, d));
            const u64 r = r0 + (i >> 3) + 32u * h;
            if ((i & 7u) == 0u && r < j.src.rows) j.row_max[(u64)ct * j.src.rows + r] = m;
        }
    }
    // lanes 8, 16 and 32 apart hold the same columns
#pragma unroll
    for (int d = 8; d < 64; d <<= 1)
#pragma unroll
        for (int q = 0; q < 8; q++) {
            cm[q] = max(cm[q], __shfl_xor(cm[q], d));
            cs[q] += __shfl_xor(cs[q], d);
        }
    if ((i & 63u) < 8u) {
#pragma unroll
        for (int q = 0; q < 8; q++) {
            mags[i >> 6][(i & 7u) * 8u + q] = cm[q];
            sums[i >> 6][(i & 7u) * 8u + q] = cs[q];
        }
    }
    __syncthreads();
    if (i < 64u && c0 + i < j.src.cols) {
        if (j.col_max) j.col_max[(u64)rt * j.src.cols + c0 + i] = max(max(mags[0][i], mags[1][i]), max(mags[2][i], mags[3][i]));
        if (j.col_sum) j.col_sum[(u64)rt * j.src.cols + c0 + i] = (sums[0][i] + sums[1][i]) + (sums[2][i] + sums[3][i]);
    }
}

// Lines (the rows and columns of both jobs) in blocks of 16, by a workgroup of 256: the tiles of a line are dealt to 16
// threads, whose results are joined in order (one thread a line read its tiles in 12 us at 1024 x 4096, most of it waiting).
constexpr u32 LINES = 16;
__device__ __forceinline__ u32 line_blocks(const TileJobs &jobs, u32 which) // rows and columns of the first, then of the second
{
    const TileJob &j = jobs.job[which >> 1];
    return j.src.p ? ((which & 1u ? j.src.cols : j.src.rows) + LINES - 1u) / LINES : 0u;
}
__device__ __forceinline__ void join_lines(const TileJobs &jobs, u32 block)
{
    __shared__ u32 mags[16][LINES];
    __shared__ float sums[16][LINES];
    const u32 lane = threadIdx.x % LINES, part = threadIdx.x / LINES;
    u32 which = 0u;
    for (; which < 3u && block >= line_blocks(jobs, which); which++) block -= line_blocks(jobs, which);
    const TileJob &j = jobs.job[which >> 1];
    const bool by_col = which & 1u;
    const u32 lines = by_col ? j.src.cols : j.src.rows, tiles = by_col ? j.row_tiles : j.col_tiles, line = block * LINES + lane;
    const u32 *max_of = by_col ? j.col_max : j.row_max;
    const float *sum_of = by_col ? j.col_sum : nullptr;
    u32 m = 0u;
    float sum = 0.0f;
    if (line < lines) {
#pragma unroll 4
        for (u32 t = part; t < tiles; t += 16u) {
            if (max_of) m = max(m, gptr(max_of)[(u64)t * lines + line]);
            if (sum_of) sum += gptr(sum_of)[(u64)t * lines + line];
        }
    }
    mags[part][lane] = m;
    sums[part][lane] = sum;
    __syncthreads();
    if (part == 0u && line < lines) {
        for (u32 t = 1; t < 16u; t++) {
            m = max(m, mags[t][lane]);
            sum += sums[t][lane];
        }
        float s;
        if (max_of) scale_of(m, s, (by_col ? j.inv_col : j.inv_row)[line]);
        if (sum_of) j.sum[line] = sum;
    }
}
__global__ __launch_bounds__(256) void k_scales(TileJobs jobs) { join_lines(jobs, blockIdx.x); }

// P1, P2: planes by row and by column (of both jobs)
template <u32 TY, int PR, int PC0, int PC1>
__global__ __launch_bounds__(256) void k_tile_planes(TileJobs jobs)
{
    const bool second = blockIdx.x >= jobs.tiles0;
    const TileJob &j = jobs.job[second];
    const u32 tile = blockIdx.x - (second ? jobs.tiles0 : 0u), rt = tile / j.col_tiles, ct = tile - rt * j.col_tiles;
    const u64 r0 = rt * 64ull;
    const u32 c0 = ct * 64u, i = threadIdx.x;
    float v[2][8];
    tile_values<TY>(j.src, r0, c0, v);
    if (j.by_row) {
#pragma unroll
        for (u32 h = 0; h < 2u; h++) {
            const u64 r = r0 + (i >> 3) + 32u * h;
            if (r < j.src.rows) put_planes<PR>(v[h], 1.0f / gptr(j.inv_row)[r], j.by_row + plane_at(r, c0 + (i & 7u) * 8u, j.ld_row), j.plane_row);
        }
    }
    if (j.by_col) {
        __shared__ float lds[64][65];
#pragma unroll
        for (u32 h = 0; h < 2u; h++)
#pragma unroll
            for (u32 q = 0; q < 8u; q++) lds[(i >> 3) + 32u * h][(i & 7u) * 8u + q] = v[h][q];
        __syncthreads();
#pragma unroll
        for (u32 h = 0; h < 2u; h++) {
            const u32 c = (i >> 3) + 32u * h, r = (i & 7u) * 8u;
            if (c0 + c >= j.src.cols) continue;
            float x[8];
#pragma unroll
            for (u32 q = 0; q < 8u; q++) x[q] = lds[r + q][c];
            const float s = 1.0f / gptr(j.inv_col)[c0 + c]; // (a power of two)
            _Float16 *at = j.by_col + plane_at(c0 + c, r0 + r, j.ld_col);
            if (second)
                put_planes<PC1>(x, s, at, j.plane_col);
            else
                put_planes<PC0>(x, s, at, j.plane_col);
        }
    }
}

// ------------------------------------------------------------------------------------------
// the weight
// ------------------------------------------------------------------------------------------
constexpr u32 ONE_MARK = 0xFC00FC00u; // (minus infinity twice: no entry has a high part that is infinite and one that is left over)

// Eight entries of the table into the planes, the marked ones left out.
template <int P>
__device__ __forceinline__ void store_entries(const u32 (&e)[8][2], _Float16 *at, u64 plane)
{
    u4_16 hi, lo;
    u32 least = ~0u; // 0: one is marked
#pragma unroll
    for (int q = 0; q < 8; q++) least = min(least, e[q][0] ^ ONE_MARK);
#pragma unroll
    for (int q = 0; q < 4; q++) {
        hi[q] = low_halves(e[2 * q][0], e[2 * q + 1][0]);
        lo[q] = high_halves(e[2 * q][0], e[2 * q + 1][0]);
    }
    if (least != 0u) {
        *(u4_16 *)at = hi;
        if (P > 1) *(u4_16 *)(at + plane) = lo;
    } else {
#pragma unroll
        for (int q = 0; q < 8; q++) {
            if (e[q][0] == ONE_MARK) continue;
            ((u16 *)at)[q] = (u16)(hi[q / 2] >> (16 * (q & 1)));
            if (P > 1) ((u16 *)(at + plane))[q] = (u16)(lo[q / 2] >> (16 * (q & 1)));
        }
    }
}
// What shares the launch with the weight: rows of activations, or the lines of a gradient's scales.
struct Beside {
    RowPlanes rows;
    TileJobs jobs;
    u32 n_rows, n_lines; // workgroups
};
constexpr u32 SHORT_LIST = 4096; // protected values that every workgroup looks through by itself

// The largest magnitude of those that this thread of 256 looks at, of a short list.
template <u32 TY>
__device__ __forceinline__ u32 listed_max(const WDesc &w)
{
    const u32 n = (u32)w.n_outlier;
    Raw8<TY> x[SHORT_LIST / 2048];
#pragma unroll
    for (u32 h = 0; h < SHORT_LIST / 2048; h++) {
        const u32 j = h * 2048u + threadIdx.x * 8u;
        x[h] = load_raw8<TY>((const GLOBAL_AS typename Elem<TY>::type *)w.out_val + j, j < n ? n - j : 0u);
    }
    u32 m = 0u;
#pragma unroll
    for (u32 h = 0; h < SHORT_LIST / 2048; h++)
#pragma unroll
        for (int i = 0; i < 8; i++) m = max(m, finite_mag(x[h][i]));
    return m;
}

// Planes of the rows (T == false) or, turned, of the columns; padding of the reduction is zero.  A thread decodes runs of eight
// symbols; protected places are left to the workgroups behind the tiles, which take them from the list (indices outside the
// weight are left out).  The largest values are there (`part`), or with a short list every workgroup finds them and the
// first tile's leaves them there: 512 rows through 768 x 768, fp32, 26.3 -> 24.5 us for a launch less;
// the lines of a gradient's scales, 1024 x 1024 x 4096 bf16, 73.7 -> 70.8 us.
template <int W, int P, bool T>
__global__ __launch_bounds__(256) void k_weight_planes(WDesc w, u32 tiles, u32 *__restrict__ part, bool looks, _Float16 *__restrict__ dst, u64 plane, u64 ld, Beside beside)
{
    const u32 others = beside.n_rows + beside.n_lines;
    if (blockIdx.x < others) {
        if (beside.n_lines)
            join_lines(beside.jobs, blockIdx.x);
        else if (P == 1) // (the types and their planes: planes_x, planes_w)
            row_planes<TY_BF16, 1>(beside.rows, blockIdx.x);
        else if (beside.rows.type == TY_F32)
            row_planes<TY_F32, 2>(beside.rows, blockIdx.x);
        else
            row_planes<TY_F16, 1>(beside.rows, blockIdx.x);
        return;
    }
    const u32 block = blockIdx.x - others;
    typedef Table<TY_F16, W> Tab;
    constexpr int ND = (8 * W + 31) / 32;
    __shared__ __attribute__((aligned(16))) u32 table[Tab::BYTES / 4];
    // a tile of 64 rows x 128 columns (64 for turned planes): four runs a thread (two), asked for before anything else
    constexpr u32 TILE_C = T ? 64u : 128u, RUNS = TILE_C / 32u, DOWN = 2048u / TILE_C; // rows from a thread's run to its next
    const u32 col_tiles = (w.cols + TILE_C - 1u) / TILE_C;
    const u64 r0 = block / col_tiles * 64ull;
    const u32 c0 = block % col_tiles * TILE_C;
    const bool is_tile = block < tiles;
    const u32 run = threadIdx.x % (TILE_C / 8u) * 8u, down = threadIdx.x / (TILE_C / 8u), c = c0 + run;
    const u64 bit0 = ((r0 + down) * w.cols + c) * W, next_bits = (u64)w.cols * (DOWN * W); // (of its first run)
    u32 raw[RUNS][ND + 1];
#pragma unroll
    for (u32 h = 0; h < RUNS; h++)
        load_words<ND + 1>(w.packed, (bit0 + h * next_bits) >> 5, is_tile && r0 + down + h * DOWN < w.rows && c < w.cols ? w.n_words : 0, raw[h]);
    float s, inv;
    if (looks) {
        __shared__ u32 red[4];
        u32 m = threadIdx.x < w.K ? finite_mag(gptr(w.codebook)[threadIdx.x]) : 0u;
        m = max(m, w.val_bf16 ? listed_max<TY_BF16>(w) : listed_max<TY_F32>(w));
        m = wave_max_u(m);
        if ((threadIdx.x & 63u) == 0u) red[threadIdx.x >> 6] = m;
        __syncthreads();
        m = max(max(red[0], red[1]), max(red[2], red[3]));
        scale_of(m, s, inv);
        if (block == 0 && threadIdx.x < WMAX_PARTS) part[threadIdx.x] = m;
    } else {
        weight_scale(part, s, inv);
    }
    if (!is_tile) {
        for (u64 j = (block - tiles) * 256ull + threadIdx.x; j < w.n_outlier; j += (u64)((gridDim.x - others) - tiles) * 256u) {
            const u32 i = gptr(w.out_idx)[j], r = i / w.cols, c = i - r * w.cols;
            if (r >= w.rows) continue;
            const float x = protected_value(w, j) * s;
            const _Float16 hi = (_Float16)x;
            _Float16 *at = dst + (T ? plane_at(c, r, ld) : plane_at(r, c, ld));
            at[0] = hi;
            if (P > 1) at[plane] = (_Float16)(x - (float)hi);
        }
        return;
    }
    fill_table<TY_F16, W>(w, table, s);
    // (this thread's entry; without a list nobody would write the places that are left out)
    if (w.n_outlier && threadIdx.x >= Tab::COPIES && threadIdx.x < 2u * Tab::COPIES) table[threadIdx.x] = ONE_MARK;
    __syncthreads();
    const u32 mine = lane_copy<TY_F16, W>();
    __shared__ u32 turned[T ? 64 : 1][65];
    _Float16 *const at = dst + (T ? plane_at(c0 + (threadIdx.x >> 3), r0 + (threadIdx.x & 7u) * 8u, ld) : plane_at(r0 + down, c, ld));
#pragma unroll
    for (u32 h = 0; h < RUNS; h++) {
        const u64 r = r0 + down + h * DOWN;
        const u32 left = r < w.rows && c < w.cols ? w.cols - c : 0u;
        u32 d[ND + 1];
        const u32 shift = (u32)(bit0 + h * next_bits) & 31u;
#pragma unroll
        for (int q = 0; q < ND; q++) d[q] = __builtin_amdgcn_alignbit(raw[h][q + 1], raw[h][q], shift);
        d[ND] = 0u;
        u32 e[8][2];
#pragma unroll
        for (int q = 0; q < 8; q++) look_up<TY_F16, W>((const char *)table, mine, d, q, e[q]);
        if (left < 8u) {
#pragma unroll
            for (u32 q = 0; q < 8u; q++)
                if (q >= left) e[q][0] = 0u;
        }
        if (T) {
#pragma unroll
            for (int q = 0; q < 8; q++) turned[down + h * DOWN][run + q] = e[q][0];
        } else if (r < w.rows && c < (u32)ld) {
            store_entries<P>(e, at + h * DOWN * ld, plane); // (blocks of 16 rows follow each other)
        }
    }
    if (T) {
        __syncthreads();
#pragma unroll
        for (u32 h = 0; h < 2u; h++) {
            const u32 col = (threadIdx.x >> 3) + 32u * h, r = (threadIdx.x & 7u) * 8u;
            if (c0 + col >= w.cols) continue;
            u32 e[8][2];
#pragma unroll
            for (u32 q = 0; q < 8u; q++) e[q][0] = turned[r + q][col];
            store_entries<P>(e, at + h * 32u * ld, plane);
        }
    }
}

// ------------------------------------------------------------------------------------------
// the product: C[m][n] = sum_k A[m][k] B[n][k], over pairs of planes
// ------------------------------------------------------------------------------------------
struct Gemm {
    const _Float16 *a, *b;   // planes of M and of N rows
    u64 plane_a, plane_b;
    u32 M, N, ld;            // ld: the padded reduction, of both
    u32 n_tiles, m_tiles;
    u32 pairs;               // number of passes
    u32 pa, pb;              // plane of pass i: bit i
    const float *inv_a, *inv_b; // per row; inv_b NULL: the weight's
    const u32 *wpart;
    Finish end;
    u32 type;                // of the results
    u32 splits, steps;       // the reduction is dealt to `splits` workgroups, `steps` steps of KS each
    float *partial;          // [splits][M][n8] their sums; NULL: one workgroup has the whole reduction
    u32 n8;                  // N rounded up to 8
};
struct Gemms { // one product, or two that share a launch (the other's type is fp32, or the same)
    Gemm g[2];
    u32 first;      // workgroups of the first
    u32 join_first; // workgroups of k_join for the first
};

// A block of 1024 bytes from device memory to LDS without registers in between.
__device__ __forceinline__ void to_lds(const _Float16 *from, u32 lane, _Float16 *to)
{
    __builtin_amdgcn_global_load_lds((const GLOBAL_AS u32 *)from + lane * 4u, (LDS_AS u32 *)to, 16, 0, 0);
}

// The scaled sums of row m, columns n .. n + 7, to where they belong, as elements of TY or of fp32.  (The scales are powers of two, and the exponents are
// added first: a row near the upper end of fp32 times a small weight would overflow with one of them alone.)
template <u32 TY>
__device__ __forceinline__ void scaled8(const Gemm &g, u32 m, u32 n, float (&v)[8], float inv_w)
{
    const int e = exponent_of(gptr(g.inv_a)[m]);
    float b[8];
    if (g.inv_b) load8<TY_F32>(gptr(g.inv_b) + n, min(g.N - n, 8u), b);
#pragma unroll
    for (int t = 0; t < 8; t++) v[t] = __builtin_ldexpf(v[t], e + exponent_of(g.inv_b ? b[t] : inv_w));
    if (TY == TY_F32 || g.type == TY)
        finish8<TY>(g.end, m, n, v);
    else
        store8<TY_F32>((GLOBAL_AS float *)g.end.out.p + (u64)m * g.end.out.stride + n, min(g.N - n, 8u), v);
}

// Waits until at most N loads to LDS of this wave are on their way and all its reads of LDS have come, then for the others.
template <int N>
__device__ __forceinline__ void wait_and_meet()
{
    static_assert(N < 64, "");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// A tile of BM x BN, by waves of WM x WN.  A step takes 32 of the reduction: a block of the planes for 16 rows.  LDS holds D
// steps.  While the matrix cores work on step t, the operands of step t + 1 are read from LDS into a second set of
// registers, and the blocks of the steps up to t + D are on their way.
template <u32 TY, int BM, int BN, int WM, int WN, int D>
// (Eight waves: with four, one a SIMD, the compiler keeps the sums in accumulation registers and moves them to and fro
// around every product, 0.5 us a step of 128 x 128.)
__global__ __launch_bounds__(BM / WM * (BN / WN) * 64) void k_product(Gemms both)
{
    const bool second = blockIdx.x >= both.first;
    const Gemm g = both.g[second];
    const u32 block = blockIdx.x - (second ? both.first : 0u);
    constexpr int WAVES_M = BM / WM, WAVES = WAVES_M * (BN / WN), TM = WM / 16, TN = WN / 16;
    constexpr int LOADS = (BM + BN) / 16 / WAVES; // of 16 rows each, per wave and step
    constexpr u32 SLOT = (BM + BN) * KS;
    __shared__ __attribute__((aligned(1024))) _Float16 lds[D * SLOT];
    // (the wave's number in a scalar register, and with it all addresses but the lane's 16 bytes)
    const u32 wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63u;
    // Workgroups go to the eight XCDs in turn; each XCD gets a run of them, of one split first, whose blocks it finds in its
    // own L2 ...
    const u32 tiles = g.m_tiles * g.n_tiles, all = tiles * g.splits, per = (all + 7u) / 8u;
    const u32 full = all - (per - 1u) * 8u, xcd = block & 7u, at = block >> 3; // the first `full` XCDs have `per`
    u32 id = xcd < full ? xcd * per + at : full * per + (xcd - full) * (per - 1u) + at;
    const u32 split = id / tiles;
    id -= split * tiles;
    // ... in strips of GROUP rows of tiles, so that a run is as high as it is wide
    const u32 strip = id / (GROUP * g.n_tiles), in = id - strip * (GROUP * g.n_tiles), high = min(GROUP, g.m_tiles - strip * GROUP);
    const u32 m0 = (strip * GROUP + in % high) * BM, n0 = in / high * BN;
    const u32 wm = wave % WAVES_M * WM, wn = wave / WAVES_M * WN;
    // this wave's blocks of a step (a's, then b's)
    u64 from[LOADS];
    bool is_b[LOADS];
#pragma unroll
    for (int j = 0; j < LOADS; j++) {
        const u32 r = (wave * LOADS + j) * 16u;
        is_b[j] = r >= (u32)BM;
        // (blocks past the last are the last: their results are not stored)
        const u32 sixteen = is_b[j] ? min(n0 + r - BM, g.N - 1u) / 16u : min(m0 + r, g.M - 1u) / 16u;
        from[j] = (u64)sixteen * 16u * g.ld;
    }
    const u32 step0 = split * g.steps, n_steps = min(g.steps, g.ld / KS - step0) * g.pairs;
    u64 k = (u64)step0 * (16u * KS); // blocks of a row follow each other
    u32 pass = 0, asked = 0;
    auto fetch = [&](u32 slot) { // the next step's rows; past the last step once more the last one's, which nobody reads
        const _Float16 *a = g.a + ((g.pa >> pass) & 1u) * g.plane_a + k, *b = g.b + ((g.pb >> pass) & 1u) * g.plane_b + k;
#pragma unroll
        for (int j = 0; j < LOADS; j++) to_lds((is_b[j] ? b : a) + from[j], lane, lds + slot * SLOT + (wave * LOADS + j) * (16u * KS));
        if (++asked < n_steps && ++pass == g.pairs) {
            pass = 0;
            k += 16u * KS;
        }
    };
    struct Operands {
        h8 a[TM], b[TN];
    } even, odd;
    const u32 r16 = lane & 15u, piece = ((lane >> 4) ^ turn_of(r16)) * 8u;
    auto read = [&](Operands &o, u32 slot) {
        const _Float16 *as = lds + slot * SLOT + (wm + r16) * KS + piece, *bs = lds + slot * SLOT + (BM + wn + r16) * KS + piece;
#pragma unroll
        for (int j = 0; j < TN; j++) o.b[j] = *(const h8 *)(bs + j * 16 * KS);
#pragma unroll
        for (int i = 0; i < TM; i++) o.a[i] = *(const h8 *)(as + i * 16 * KS);
    };
    f4 acc[TM][TN] = {};
    auto step = [&](const Operands &now, Operands &next, u32 t) {
        wait_and_meet<LOADS *(D - 2)>(); // step t + 1 is there for all waves, and nobody reads step t any more
        fetch(t % D);
        read(next, (t + 1u) % D);
        // (the columns of C are the rows of the instruction's result: a lane gets four consecutive ones)
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
            for (int j = 0; j < TN; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(now.b[j], now.a[i], acc[i][j], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < TM + TN; i++) { // a few products, then a read
            __builtin_amdgcn_sched_group_barrier(0x008, (TM * TN + TM + TN - 1) / (TM + TN), 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
    };
#pragma unroll
    for (u32 q = 0; q < (u32)D; q++) fetch(q);
    wait_and_meet<LOADS *(D - 1)>();
    read(even, 0);
    for (u32 t = 0; t < n_steps; t += 2u) { // (an even number: see cuts_of)
        step(even, odd, t);
        step(odd, even, t + 1u);
    }
    wait_and_meet<0>(); // (the last step's loads once more are still on their way, of all waves, to where the sums go next)
    // The sums go through LDS, 32 or 64 rows of a wave at a time, so that eight lanes hold a row's 64 columns.
    constexpr int MOST = (int)(D * SLOT / (WAVES * 128)), ROWS = WM <= MOST && WM <= 64 ? WM : MOST >= 64 ? 64 : 32; // (64 floats a row)
    static_assert(WN % 64 == 0 && WM % ROWS == 0 && ROWS <= MOST, "every wave has its rows in LDS");
    float s, inv_w = 1.0f;
    if (!g.inv_b && !g.partial) weight_scale(g.wpart, s, inv_w);
    float *const mine = (float *)lds + wave * (ROWS * 64u); // [ROWS][64], the pieces of 4 of a row in an order of its own
#pragma unroll
    for (int part = 0; part < WM / ROWS * (WN / 64); part++) {
        const int down = part % (WM / ROWS), across = part / (WM / ROWS);
        const u32 n = n0 + wn + across * 64u + (lane & 7u) * 8u;
        __syncthreads();
#pragma unroll
        for (u32 i = 0; i < ROWS / 16u; i++)
#pragma unroll
            for (u32 j = 0; j < 4u; j++)
                *(f4 *)(mine + (i * 16u + r16) * 64u + ((j * 4u + (lane >> 4)) ^ r16) * 4u) = acc[down * (ROWS / 16) + i][across * 4 + j];
        __syncthreads();
#pragma unroll 1
        for (u32 q = 0; q < ROWS / 8u; q++) {
            const u32 r = q * 8u + (lane >> 3), m = m0 + wm + down * ROWS + r, c = (lane & 7u) * 2u;
            if (m >= g.M || n >= g.N) continue;
            const f4 x = *(const f4 *)(mine + r * 64u + (c ^ (r & 15u)) * 4u), y = *(const f4 *)(mine + r * 64u + ((c + 1u) ^ (r & 15u)) * 4u);
            if (g.partial) {
                float *to = g.partial + ((u64)split * g.M + m) * g.n8 + n;
                *(f4 *)to = x;
                *(f4 *)(to + 4) = y;
            } else {
                float v[8] = {x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
                scaled8<TY>(g, m, n, v, inv_w);
            }
        }
    }
}

// The sums of the splits, in their order: eight results a thread.  A launch and the traffic of the sums: 5 us for 9 MB.
template <u32 TY>
__global__ __launch_bounds__(256) void k_join(Gemms both)
{
    const bool second = blockIdx.x >= both.join_first;
    const Gemm g = both.g[second];
    const u64 i = (blockIdx.x - (second ? both.join_first : 0u)) * 256ull + threadIdx.x;
    float s, inv_w = 1.0f;
    if (!g.inv_b) weight_scale(g.wpart, s, inv_w);
    const u32 parts = g.n8 / 8u, m = (u32)(i / parts), n = (u32)(i - (u64)m * parts) * 8u;
    if (m >= g.M) return;
    float v[8] = {};
#pragma unroll 4
    for (u32 q = 0; q < g.splits; q++) {
        const GLOBAL_AS f4 *p = (const GLOBAL_AS f4 *)(gptr(g.partial) + ((u64)q * g.M + m) * g.n8 + n);
        const f4 x = p[0], y = p[1];
#pragma unroll
        for (int t = 0; t < 4; t++) {
            v[t] += x[t];
            v[t + 4] += y[t];
        }
    }
    scaled8<TY>(g, m, n, v, inv_w);
}

// ------------------------------------------------------------------------------------------
// calls
// ------------------------------------------------------------------------------------------
namespace {

struct Room { // the parts of a workspace
    u64 at = 0;
    u64 take(u64 bytes)
    {
        const u64 here = at;
        at += up(bytes, 256);
        return here;
    }
};

struct Planes {
    u64 off, inv; // of the planes and of the rows' scales
    u64 plane, ld;
    u32 count;
};
Planes planes_for(Room &r, u64 rows, u64 reduction, u32 count)
{
    Planes p;
    p.ld = up(reduction, KT);
    p.plane = up(rows, 16) * p.ld;
    p.count = count;
    p.off = r.take(p.plane * count * 2u);
    p.inv = r.take(rows * 4u);
    return p;
}

// x's planes and the parts of the weight's largest magnitude
void start_rows(const RowPlanes &x, const WDesc &w, u32 *part, hipStream_t s)
{
    const u32 grid = x.src.rows + WMAX_PARTS;
    switch (x.type) {
    case TY_F32: PROF("k_row_planes", s, k_row_planes<TY_F32, 2><<<grid, 256, 0, s>>>(x, w, part)); break;
    case TY_BF16: PROF("k_row_planes", s, k_row_planes<TY_BF16, 1><<<grid, 256, 0, s>>>(x, w, part)); break;
    default: PROF("k_row_planes", s, k_row_planes<TY_F16, 1><<<grid, 256, 0, s>>>(x, w, part)); break;
    }
}

// along: the reduction runs along the stored rows; looks: the largest values are not there yet
void weight_planes(const WDesc &w, bool along, const Planes &p, char *ws, u64 part, bool looks, const Beside &beside, hipStream_t s)
{
    u32 *pm = (u32 *)(ws + part);
    _Float16 *dst = (_Float16 *)(ws + p.off);
    // (the padding along the reduction belongs to the tiles: it is written as zeros)
    const u32 tile_c = along ? 128u : 64u, tiles = (w.cols + tile_c - 1u) / tile_c * ((w.rows + 63u) / 64u);
    const u32 grid = beside.n_rows + beside.n_lines + tiles + (u32)std::min<u64>((w.n_outlier + 255) / 256, 512);
    with_width(w.w, [&](auto width) {
        constexpr int W = decltype(width)::value;
        auto start = [&](auto planes, auto turned) {
            PROF("k_weight_planes", s, k_weight_planes<W, decltype(planes)::value, decltype(turned)::value><<<grid, 256, 0, s>>>(w, tiles, pm, looks, dst, p.plane, p.ld, beside));
        };
        typedef std::integral_constant<int, 1> One;
        typedef std::integral_constant<int, 2> Two;
        if (p.count > 1)
            along ? start(Two(), std::false_type()) : start(Two(), std::true_type());
        else
            along ? start(One(), std::false_type()) : start(One(), std::true_type());
    });
}

// How products that share a launch are cut: tiles of 256 x 256, 128 x 256 or 128 x 128, one size for both, and where the
// tiles are too few for the chip the reduction of a tile among several workgroups.
struct Shape { // M == 0: no such product
    u64 M = 0, N = 0, ld = 0;
    u32 pairs = 1;
};
struct Cut {
    u32 m_tiles, n_tiles, splits, steps;
    u64 partial; // bytes
};
struct Cuts {
    int kind;
    Cut c[2];
};
constexpr u32 CUS = 256;
constexpr u32 KIND_M[3] = {256, 128, 128}, KIND_N[3] = {256, 256, 128};
// Measured, in 0.01 us: a step of a tile on a full chip; what a workgroup takes beside its steps (the first loads, the
// results), and a launch of k_join; and 4 bytes of fp32 sums written and read again, in 2^-20 of it
constexpr u32 KIND_TIME[3] = {91, 52, 35}, KIND_FIXED[3] = {900, 500, 300}, JOIN_TIME = 350, SUM_TIME = 210;

// The time until all workgroups are done, the ones that take longer first: n0 that take t0 each and n1 that take t1.
u64 time_of(u32 n0, u32 t0, u32 n1, u32 t1)
{
    if (t0 < t1) {
        std::swap(n0, n1);
        std::swap(t0, t1);
    }
    const u32 busy = n0 % CUS, free = CUS - busy; // `busy` CUs have longer ones `until`, the others until `full`
    const u64 full = (u64)(n0 / CUS) * t0, until = full + (busy ? t0 : 0);
    const u32 beside = busy ? t0 / t1 : 0; // shorter ones that end beside a last longer one
    if ((u64)n1 <= (u64)beside * free) return std::max(until, full + (u64)((n1 + free - 1) / free) * t1);
    n1 -= beside * free;
    const u32 rounds = n1 / CUS, left = n1 % CUS;
    const u64 end = until + (u64)rounds * t1;
    if (left == 0) return end;
    return left > free ? end + t1 : std::max(end, full + (u64)(beside + rounds + 1) * t1);
}

// Numbers of workgroups for a tile that are looked at.
constexpr u32 MOST_SPLITS = 16, SPLITS[] = {1, 2, 3, 4, 5, 6, 8, 10, 12, MOST_SPLITS};
struct Choice {
    u32 groups, time, extra;
    Cut c;
};
// Those of a product, `MOST_SPLITS` at most; returns how many.
u32 choices_of(const Shape &x, int kind, Choice *to)
{
    Choice o = {};
    o.c.splits = 1;
    o.time = 1; // (no such product: no workgroups)
    if (x.M == 0) {
        to[0] = o;
        return 1;
    }
    o.c.m_tiles = (u32)(up(x.M, KIND_M[kind]) / KIND_M[kind]);
    o.c.n_tiles = (u32)(up(x.N, KIND_N[kind]) / KIND_N[kind]);
    const u32 tiles = o.c.m_tiles * o.c.n_tiles, steps = (u32)(x.ld / KS);
    u32 n = 0;
    for (u32 want : SPLITS) {
        if (want > 1 && (tiles * want > 2 * CUS || steps * x.pairs < 8 * want)) break; // (eight steps each)
        // (two sets of operands take turns: an even number of steps and passes; `steps` is even, as KT / KS is)
        o.c.steps = (u32)up((steps + want - 1) / want, x.pairs & 1u ? 2 : 1);
        o.c.splits = (steps + o.c.steps - 1) / o.c.steps;
        o.c.partial = o.c.splits > 1 ? up(x.N, 8) * x.M * o.c.splits * 4u : 0;
        o.groups = tiles * o.c.splits;
        o.time = KIND_FIXED[kind] + o.c.steps * x.pairs * KIND_TIME[kind];
        o.extra = (u32)(o.c.partial / 4u * SUM_TIME >> 20) + (o.c.partial ? JOIN_TIME : 0u);
        if (n == 0 || o.c.steps < to[n - 1].c.steps) to[n++] = o;
    }
    return n;
}

Cuts cuts_of(const Shape &a, const Shape &b)
{
    Cuts best = {};
    u64 least = ~0ull;
    for (int kind = 0; kind < 3; kind++) {
        Choice x[MOST_SPLITS], y[MOST_SPLITS];
        const u32 nx = choices_of(a, kind, x), ny = choices_of(b, kind, y);
        for (u32 i = 0; i < nx; i++)
            for (u32 j = 0; j < ny; j++) {
                const u64 extra = x[i].extra + y[j].extra - (x[i].extra && y[j].extra ? JOIN_TIME : 0u); // (one launch)
                if (((u64)x[i].groups * x[i].time + (u64)y[j].groups * y[j].time) / CUS + extra >= least) continue;
                const u64 time = time_of(x[i].groups, x[i].time, y[j].groups, y[j].time) + extra;
                if (time >= least) continue;
                least = time;
                best = {kind, {x[i].c, y[j].c}};
            }
    }
    return best;
}

template <u32 TY>
void products_of(const Gemms &g, int kind, u32 grid, u32 join, hipStream_t s)
{
    switch (kind) {
    case 0: PROF("k_product", s, k_product<TY, 256, 256, 128, 64, 4><<<grid, 512, 0, s>>>(g)); break;
    case 1: PROF("k_product", s, k_product<TY, 128, 256, 64, 64, 4><<<grid, 512, 0, s>>>(g)); break;
    default: PROF("k_product", s, k_product<TY, 128, 128, 32, 64, 8><<<grid, 512, 0, s>>>(g)); break;
    }
    if (join) PROF("k_join", s, k_join<TY><<<join, 256, 0, s>>>(g));
}

// Where a product's operands and sums are.
void lay_out(Gemm &g, const Planes &a, const Planes &b, const Cut &c, u64 partial, char *ws)
{
    g.a = (const _Float16 *)(ws + a.off);
    g.b = (const _Float16 *)(ws + b.off);
    g.plane_a = a.plane;
    g.plane_b = b.plane;
    g.ld = (u32)a.ld;
    g.inv_a = (const float *)(ws + a.inv);
    // (smallest terms first) l h, h l, h h
    if (a.count > 1) g.pa |= 1u << g.pairs++;
    if (b.count > 1) g.pb |= 1u << g.pairs++;
    g.pairs++;
    g.m_tiles = c.m_tiles;
    g.n_tiles = c.n_tiles;
    g.splits = c.splits;
    g.steps = c.steps;
    g.n8 = (u32)up(g.N, 8);
    g.partial = c.partial ? (float *)(ws + partial) : nullptr;
}
// One product (b NULL) or two, whose results have this type or, the second's, fp32.  The one whose workgroups take longer
// goes first.
void products(const Gemm &a, const Gemm *b, u32 type, int kind, hipStream_t s)
{
    Gemms g = {};
    const bool turn = b && (u64)b->steps * b->pairs > (u64)a.steps * a.pairs;
    g.g[0] = turn ? *b : a;
    if (b) g.g[1] = turn ? a : *b;
    u32 grid = 0, join = 0;
    for (int j = 0; j < (b ? 2 : 1); j++) {
        const Gemm &x = g.g[j];
        grid += x.m_tiles * x.n_tiles * x.splits;
        join += x.partial ? (u32)(((u64)x.M * (x.n8 / 8u) + 255u) / 256u) : 0u;
        if (j == 0) {
            g.first = grid;
            g.join_first = join;
        }
    }
    switch (type) {
    case TY_F32: products_of<TY_F32>(g, kind, grid, join, s); break;
    case TY_BF16: products_of<TY_BF16>(g, kind, grid, join, s); break;
    default: products_of<TY_F16>(g, kind, grid, join, s); break;
    }
}

// planes of the sides of a product whose result has this type
u32 planes_x(u32 type) { return type == TY_F32 ? 2u : 1u; }  // activations: bf16 and fp16 are exact in one
u32 planes_w(u32 type) { return type == TY_BF16 ? 1u : 2u; }

struct LinearRoom {
    Planes x, w;
    u64 part, partial, bytes;
    Cuts cuts;
    LinearRoom(u64 rows, u32 n_in, u32 n_out, u32 type)
    {
        Room r;
        x = planes_for(r, rows, n_in, planes_x(type));
        w = planes_for(r, n_out, n_in, planes_w(type));
        part = r.take(WMAX_PARTS * 4u);
        cuts = cuts_of({rows, n_out, x.ld, x.count + w.count - 1}, {});
        partial = r.take(cuts.c[0].partial);
        bytes = r.at;
    }
};
struct GradRoom {
    u64 part = 0, partial[2] = {0, 0}, bytes = 0;
    u64 row_max = 0, col_max = 0, col_sum = 0, x_max = 0;
    Planes dr = {}, w = {}, dc = {}, xc = {};
    Cuts cuts;
    GradRoom(u64 rows, u32 n_in, u32 n_out, u32 in_out, u32 type, u32 act, bool dx, bool dw)
    {
        Room r;
        const u64 row_tiles = up(rows, 64) / 64, col_tiles = up(n_out, 64) / 64;
        // d is what it is in its type, or, below an activation, an fp32 number
        const u32 dt = act != ACT_NONE ? TY_F32 : type;
        col_sum = r.take(row_tiles * n_out * 4u);
        const u32 d_count = type == TY_BF16 ? 1u : planes_x(dt), w_count = planes_w(type), dc_count = planes_x(dt), x_count = planes_x(type);
        // (cut as if both were wanted, so that a result does not depend on whether the other one is)
        const u64 of_rows = up(rows, KT), m = in_out ? n_in : n_out, n = in_out ? n_out : n_in;
        cuts = cuts_of({rows, n_in, up(n_out, KT), d_count + w_count - 1}, {m, n, of_rows, dc_count + x_count - 1});
        if (dx) {
            dr = planes_for(r, rows, n_out, d_count);
            w = planes_for(r, n_in, n_out, w_count);
            part = r.take(WMAX_PARTS * 4u);
            row_max = r.take(col_tiles * rows * 4u);
            partial[0] = r.take(cuts.c[0].partial);
        }
        if (dw) { // (fp32 results)
            dc = planes_for(r, n_out, rows, dc_count);
            xc = planes_for(r, n_in, rows, x_count);
            col_max = r.take(row_tiles * n_out * 4u);
            x_max = r.take(row_tiles * n_in * 4u);
            partial[1] = r.take(cuts.c[1].partial);
        }
        bytes = r.at;
    }
};

template <u32 TY>
void tile_planes(const TileJobs &t, u32 dr, u32 dc, hipStream_t s)
{
    constexpr int PX = TY == TY_F32 ? 2 : 1;
    if (dr > 1)
        PROF("k_tile_planes", s, k_tile_planes<TY, 2, 2, PX><<<t.tiles, 256, 0, s>>>(t));
    else if (dc > 1)
        PROF("k_tile_planes", s, k_tile_planes<TY, 1, 2, PX><<<t.tiles, 256, 0, s>>>(t));
    else
        PROF("k_tile_planes", s, k_tile_planes<TY, 1, 1, PX><<<t.tiles, 256, 0, s>>>(t));
}

} // namespace

u64 linear_space(u64 rows, u32 n_in, u32 n_out, u32 in_out, u32 type, u32 w, bool listed)
{
    return is_few(rows, n_out, in_out, type, w) ? few_space(rows, n_in, n_out, in_out, type, w, listed) : LinearRoom(rows, n_in, n_out, type).bytes;
}
u64 linear_grad_space(u64 rows, u32 n_in, u32 n_out, u32 in_out, u32 type, u32 act, bool dx, bool dw)
{
    return rows ? GradRoom(rows, n_in, n_out, in_out, type, act, dx, dw).bytes : 0;
}

hipError_t launch_linear(const LinearCall &c, hipStream_t s)
{
    if (is_few(c.rows, c.n_out, c.in_out, c.type, c.w.w)) return launch_few(c, s);
    const LinearRoom r(c.rows, c.n_in, c.n_out, c.type);
    const bool looks = c.w.n_outlier <= SHORT_LIST;
    Beside beside = {};
    beside.rows = {{c.x.p, nullptr, c.x.stride, 0, (u32)c.rows, c.n_in, ACT_NONE, 0}, (_Float16 *)(c.ws + r.x.off), r.x.plane, (float *)(c.ws + r.x.inv), (u32)r.x.ld, c.type};
    if (looks)
        beside.n_rows = (u32)c.rows;
    else
        start_rows(beside.rows, c.w, (u32 *)(c.ws + r.part), s);
    weight_planes(c.w, !c.in_out, r.w, c.ws, r.part, looks, beside, s);
    Gemm g = {};
    g.M = (u32)c.rows;
    g.N = c.n_out;
    g.wpart = (const u32 *)(c.ws + r.part);
    g.end = {c.bias, c.residual, c.y, c.pre, c.n_out, c.act};
    g.type = c.type;
    lay_out(g, r.x, r.w, r.cuts.c[0], r.partial, c.ws);
    products(g, nullptr, c.type, r.cuts.kind, s);
    return hipGetLastError();
}

__global__ __launch_bounds__(256) void k_zero(float *p, u64 n)
{
    for (u64 i = blockIdx.x * 256ull + threadIdx.x; i < n; i += gridDim.x * 256ull) p[i] = 0.0f;
}

hipError_t launch_linear_grad(const LinearGradCall &c, hipStream_t s)
{
    if (c.rows == 0) { // sums over no rows
        if (c.dw) PROF("k_zero", s, k_zero<<<1024, 256, 0, s>>>(c.dw, (u64)c.n_in * c.n_out));
        if (c.db) PROF("k_zero", s, k_zero<<<64, 256, 0, s>>>(c.db, c.n_out));
        return hipGetLastError();
    }
    const GradRoom r(c.rows, c.n_in, c.n_out, c.in_out, c.type, c.act, c.dx.p != nullptr, c.dw != nullptr);
    const bool dx = c.dx.p != nullptr, dw = c.dw != nullptr;
    TileJobs t = {};
    TileJob &d = t.job[0], &x = t.job[1];
    d.src = {c.dy.p, c.pre.p, c.dy.stride, c.pre.stride, (u32)c.rows, c.n_out, c.act, 0};
    d.col_tiles = (c.n_out + 63u) / 64u;
    d.row_tiles = ((u32)c.rows + 63u) / 64u;
    d.sum = c.db;
    if (c.db) d.col_sum = (float *)(c.ws + r.col_sum);
    if (dx) {
        d.row_max = (u32 *)(c.ws + r.row_max);
        d.inv_row = (float *)(c.ws + r.dr.inv);
        d.by_row = (_Float16 *)(c.ws + r.dr.off);
        d.plane_row = r.dr.plane;
        d.ld_row = r.dr.ld;
    }
    t.tiles0 = t.tiles = d.col_tiles * d.row_tiles;
    if (dw) {
        d.col_max = (u32 *)(c.ws + r.col_max);
        d.inv_col = (float *)(c.ws + r.dc.inv);
        d.by_col = (_Float16 *)(c.ws + r.dc.off);
        d.plane_col = r.dc.plane;
        d.ld_col = r.dc.ld;
        x.src = {c.x.p, nullptr, c.x.stride, 0, (u32)c.rows, c.n_in, ACT_NONE, 0};
        x.col_tiles = (c.n_in + 63u) / 64u;
        x.row_tiles = d.row_tiles;
        x.col_max = (u32 *)(c.ws + r.x_max);
        x.inv_col = (float *)(c.ws + r.xc.inv);
        x.by_col = (_Float16 *)(c.ws + r.xc.off);
        x.plane_col = r.xc.plane;
        x.ld_col = r.xc.ld;
        t.tiles += x.col_tiles * x.row_tiles;
    }
    u32 *part = dx ? (u32 *)(c.ws + r.part) : nullptr;
    const u32 grid = t.tiles + (dx ? WMAX_PARTS : 0u);
    auto blocks = [](u64 lines) { return (u32)((lines + LINES - 1u) / LINES); };
    const u32 lines = blocks(c.rows) + blocks(c.n_out) + (dw ? blocks(c.rows) + blocks(c.n_in) : 0u);
    switch (c.type) {
    case TY_F32: PROF("k_tile_stats", s, k_tile_stats<TY_F32><<<grid, 256, 0, s>>>(t, c.w, part)); break;
    case TY_BF16: PROF("k_tile_stats", s, k_tile_stats<TY_BF16><<<grid, 256, 0, s>>>(t, c.w, part)); break;
    default: PROF("k_tile_stats", s, k_tile_stats<TY_F16><<<grid, 256, 0, s>>>(t, c.w, part)); break;
    }
    if (dx) {
        Beside beside = {};
        beside.jobs = t;
        beside.n_lines = lines;
        weight_planes(c.w, c.in_out, r.w, c.ws, r.part, false, beside, s);
    } else {
        PROF("k_scales", s, k_scales<<<lines, 256, 0, s>>>(t));
    }
    if (dx || dw) switch (c.type) {
    case TY_F32: tile_planes<TY_F32>(t, r.dr.count, r.dc.count, s); break;
    case TY_BF16: tile_planes<TY_BF16>(t, r.dr.count, r.dc.count, s); break;
    default: tile_planes<TY_F16>(t, r.dr.count, r.dc.count, s); break;
    }
    Gemm gx = {}, gw = {};
    if (dx) {
        gx.M = (u32)c.rows;
        gx.N = c.n_in;
        gx.wpart = (const u32 *)(c.ws + r.part);
        gx.end = {nullptr, {}, c.dx, {}, c.n_in, ACT_NONE};
        gx.type = c.type;
        lay_out(gx, r.dr, r.w, r.cuts.c[0], r.partial[0], c.ws);
    }
    if (dw) {
        const Planes &a = c.in_out ? r.xc : r.dc, &b = c.in_out ? r.dc : r.xc;
        gw.M = c.in_out ? c.n_in : c.n_out;
        gw.N = c.in_out ? c.n_out : c.n_in;
        gw.inv_b = (const float *)(c.ws + b.inv);
        gw.end = {nullptr, {}, {c.dw, gw.N}, {}, gw.N, ACT_NONE};
        gw.type = TY_F32;
        lay_out(gw, a, b, r.cuts.c[1], r.partial[1], c.ws);
    }
    if (dx)
        products(gx, dw ? &gw : nullptr, c.type, r.cuts.kind, s);
    else if (dw)
        products(gw, nullptr, TY_F32, r.cuts.kind, s);
    return hipGetLastError();
}

} // namespace inshr
