// Products with a weight held in its compressed form: y = act(x W^T + b) + r, and the gradients.
//
// Numbers: the matrix cores multiply fp16 numbers (11 bits) exactly into fp32 sums.  A row of an operand is scaled by a
// power of two that brings its largest magnitude into [2^14, 2^15), so that everything above 2^-29 of that magnitude is a
// normal fp16 number and nothing is off by more than 2^-40 of it; a second plane of fp16 numbers takes what the first one
// leaves over (22 bits together).  With h and l for the planes of either side a product takes
//   1 pass   h h                for bfloat16 results: a factor rounded to 11 bits is off by 2^-11 at most, an eighth of
//                               the result's own 2^-8, and bfloat16 activations (8 bits) are exact in h
//   2 passes h h + h l          for fp16 results: fp16 activations are exact in h, the weight keeps 22 bits
//   3 passes h h + h l + l h    for fp32 results: what is left out, l l, is 2^-22 of the product
// (three planes of bfloat16 would need six passes for fp32, and two for bfloat16 results).
#include "inshr_product.h"

#include <algorithm>

namespace inshr {

// ------------------------------------------------------------------------------------------
// planes of an operand whose reduction runs along its rows
// ------------------------------------------------------------------------------------------
constexpr u32 KT = 64;  // reduction per step of the product: planes are padded to it with zeros
inline u64 up(u64 v, u64 to) { return (v + to - 1) / to * to; }

struct PlaneSrc { // a matrix of elements; act != ACT_NONE: multiplied by the slope at the values of `pre`
    const void *p, *pre;
    u64 stride, pre_stride;
    u32 rows, cols, act;
};

// One workgroup per row.
template <u32 TY, int P>
__global__ __launch_bounds__(256) void k_row_planes(PlaneSrc src, _Float16 *__restrict__ dst, u64 plane, u32 Cp, float *__restrict__ inv_out)
{
    typedef typename Elem<TY>::type T;
    const u64 r = blockIdx.x;
    const GLOBAL_AS T *p = (const GLOBAL_AS T *)src.p + r * src.stride;
    __shared__ u32 red[4];
    u32 m = 0u;
    for (u32 c = threadIdx.x * 8u; c < src.cols; c += 2048u) {
        float v[8];
        load8<TY>(p + c, src.cols - c, v);
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const u32 f = finite_mag(v[i]);
            m = m > f ? m : f;
        }
    }
    m = wave_max_u(m);
    if ((threadIdx.x & 63u) == 0u) red[threadIdx.x >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; i++) m = m > red[i] ? m : red[i];
    float s, inv;
    scale_of(m, s, inv);
    if (threadIdx.x == 0) inv_out[r] = inv;
    for (u32 c = threadIdx.x * 8u; c < Cp; c += 2048u) {
        float v[8];
        load8<TY>(p + c, c < src.cols ? src.cols - c : 0u, v);
        h8 hi, lo;
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float x = v[i] * s;
            hi[i] = (_Float16)x;
            lo[i] = (_Float16)(x - (float)hi[i]);
        }
        *(h8 *)(dst + r * Cp + c) = hi;
        if (P > 1) *(h8 *)(dst + plane + r * Cp + c) = lo;
    }
}

// ------------------------------------------------------------------------------------------
// columns: largest magnitudes, sums, and the slope applied
// ------------------------------------------------------------------------------------------
// A workgroup takes 64 columns and all rows: the sums are in a fixed order.
template <u32 TY>
__global__ __launch_bounds__(256) void k_col_stats(PlaneSrc src, float *__restrict__ d_out, float *__restrict__ inv_out,
                                                   float *__restrict__ sum_out)
{
    typedef typename Elem<TY>::type T;
    const u32 c = blockIdx.x * 64u + (threadIdx.x & 63u), part = threadIdx.x >> 6;
    __shared__ float sums[4][64];
    __shared__ u32 mags[4][64];
    float sum = 0.0f;
    u32 m = 0u;
    if (c < src.cols)
        for (u64 r = part; r < src.rows; r += 4u) {
            float v = Elem<TY>::get(((const GLOBAL_AS T *)src.p)[r * src.stride + c]);
            if (src.act != ACT_NONE) v *= act_grad(Elem<TY>::get(((const GLOBAL_AS T *)src.pre)[r * src.pre_stride + c]), src.act);
            if (d_out) d_out[r * src.cols + c] = v;
            sum += v;
            const u32 f = finite_mag(v);
            m = m > f ? m : f;
        }
    sums[part][threadIdx.x & 63u] = sum;
    mags[part][threadIdx.x & 63u] = m;
    __syncthreads();
    if (part == 0u && c < src.cols) {
        const u32 l = threadIdx.x;
        if (sum_out) sum_out[c] = (sums[0][l] + sums[1][l]) + (sums[2][l] + sums[3][l]);
        u32 all = 0u;
        for (int i = 0; i < 4; i++) all = all > mags[i][l] ? all : mags[i][l];
        float s, inv;
        scale_of(all, s, inv);
        if (inv_out) inv_out[c] = inv;
    }
}

// The planes of the transposed matrix, [cols][Rp]: tiles of 64 x 64 through LDS.
template <u32 TY, int P>
__global__ __launch_bounds__(256) void k_col_planes(PlaneSrc src, const float *__restrict__ inv, _Float16 *__restrict__ dst, u64 plane, u64 Rp)
{
    typedef typename Elem<TY>::type T;
    __shared__ float tile[64][65];
    const u32 row_tiles = (src.rows + 63u) / 64u;
    const u64 r0 = blockIdx.x % row_tiles * 64ull;
    const u32 c0 = blockIdx.x / row_tiles * 64u;
    for (u32 i = threadIdx.x; i < 4096u; i += 256u) {
        const u64 r = r0 + (i >> 6);
        const u32 c = c0 + (i & 63u);
        tile[i >> 6][i & 63u] = r < src.rows && c < src.cols ? Elem<TY>::get(((const GLOBAL_AS T *)src.p)[r * src.stride + c]) : 0.0f;
    }
    __syncthreads();
    for (u32 i = threadIdx.x; i < 512u; i += 256u) {
        const u32 c = i >> 3, r = (i & 7u) * 8u;
        if (c0 + c >= src.cols) continue;
        const float s = 1.0f / inv[c0 + c]; // (a power of two)
        h8 hi, lo;
#pragma unroll
        for (int j = 0; j < 8; j++) {
            const float x = tile[r + j][c] * s;
            hi[j] = (_Float16)x;
            lo[j] = (_Float16)(x - (float)hi[j]);
        }
        _Float16 *at = dst + (u64)(c0 + c) * Rp + r0 + r;
        *(h8 *)at = hi;
        if (P > 1) *(h8 *)(at + plane) = lo;
    }
}

// ------------------------------------------------------------------------------------------
// the weight
// ------------------------------------------------------------------------------------------
constexpr u32 WMAX_PARTS = 64;

// largest magnitudes of the centres and of parts of the protected list
__global__ __launch_bounds__(256) void k_weight_max(WDesc w, u32 *__restrict__ part)
{
    u32 m = 0u;
    if (blockIdx.x == 0 && threadIdx.x < w.K) m = finite_mag(gptr(w.codebook)[threadIdx.x]);
    for (u64 j = blockIdx.x * 256ull + threadIdx.x; j < w.n_outlier; j += 256ull * WMAX_PARTS) {
        const u32 f = finite_mag(protected_value(w, j));
        m = m > f ? m : f;
    }
    __shared__ u32 red[4];
    m = wave_max_u(m);
    if ((threadIdx.x & 63u) == 0u) red[threadIdx.x >> 6] = m;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 1; i < 4; i++) m = m > red[i] ? m : red[i];
        part[blockIdx.x] = m;
    }
}
// the whole of k_weight_max's parts, by every wave
__device__ __forceinline__ void weight_scale(const u32 *part, float &s, float &inv)
{
    scale_of(wave_max_u(gptr(part)[threadIdx.x & 63u]), s, inv);
}

// Symbol i of the stream; words past its end are not read.
__device__ __forceinline__ u32 symbol_at(const WDesc &w, u64 i)
{
    const u64 bit = i * w.w, at = bit >> 5;
    const u32 lo = gptr(w.packed)[at], hi = at + 1 < w.n_words ? gptr(w.packed)[at + 1] : 0u;
    return __builtin_amdgcn_alignbit(hi, lo, (u32)bit & 31u) & ((1u << w.w) - 1u);
}

// Planes [rows][Cp] (T == false) or, transposed, [cols][Rp]; padding of the reduction is zero.
template <int P, bool T>
__global__ __launch_bounds__(256) void k_weight_planes(WDesc w, const u32 *__restrict__ part, _Float16 *__restrict__ dst, u64 plane, u64 ld)
{
    __shared__ _Float16 hi[512], lo[512];
    __shared__ u16 sym[64][66];
    float s, inv;
    weight_scale(part, s, inv);
    for (u32 i = threadIdx.x; i < 512u; i += 256u) {
        const float x = symbol_value(w, i) * s;
        hi[i] = (_Float16)x;
        lo[i] = (_Float16)(x - (float)hi[i]);
    }
    const u32 col_tiles = (w.cols + 63u) / 64u;
    const u64 r0 = blockIdx.x / col_tiles * 64ull;
    const u32 c0 = blockIdx.x % col_tiles * 64u;
    for (u32 i = threadIdx.x; i < 4096u; i += 256u) {
        const u64 r = r0 + (i >> 6);
        const u32 c = c0 + (i & 63u);
        sym[i >> 6][i & 63u] = r < w.rows && c < w.cols ? (u16)symbol_at(w, r * w.cols + c) : (u16)0;
    }
    __syncthreads();
    for (u32 i = threadIdx.x; i < 512u; i += 256u) {
        const u32 a = i >> 3, b = (i & 7u) * 8u; // a: row of the planes, b: along the reduction
        const u64 row = (T ? c0 : r0) + a;
        if (row >= (T ? w.cols : w.rows)) continue;
        h8 vh, vl;
#pragma unroll
        for (u32 j = 0; j < 8u; j++) {
            const u32 q = T ? sym[b + j][a] : sym[a][b + j];
            vh[j] = hi[q];
            vl[j] = lo[q];
        }
        _Float16 *at = dst + row * ld + (T ? r0 : c0) + b;
        *(h8 *)at = vh;
        if (P > 1) *(h8 *)(at + plane) = vl;
    }
}

// The protected values into the planes (indices outside the weight are left out).
template <int P, bool T>
__global__ __launch_bounds__(256) void k_weight_protected(WDesc w, const u32 *__restrict__ part, _Float16 *__restrict__ dst, u64 plane, u64 ld)
{
    float s, inv;
    weight_scale(part, s, inv);
    for (u64 j = blockIdx.x * 256ull + threadIdx.x; j < w.n_outlier; j += (u64)gridDim.x * 256u) {
        const u32 i = gptr(w.out_idx)[j], r = i / w.cols, c = i - r * w.cols;
        if (r >= w.rows) continue;
        const float x = protected_value(w, j) * s;
        const _Float16 hi = (_Float16)x;
        _Float16 *at = dst + (T ? (u64)c * ld + r : (u64)r * ld + c);
        at[0] = hi;
        if (P > 1) at[plane] = (_Float16)(x - (float)hi);
    }
}

// ------------------------------------------------------------------------------------------
// the product: C[m][n] = sum_k A[m][k] B[n][k], over pairs of planes
// ------------------------------------------------------------------------------------------
struct Gemm {
    const _Float16 *a, *b;   // planes [M][ld], [N][ld]
    u64 plane_a, plane_b;
    u32 M, N, ld;            // ld: the padded reduction, of both
    u32 n_tiles, m_tiles;
    u32 pairs;               // number of passes
    u32 pa, pb;              // plane of pass i: bit i
    const float *inv_a, *inv_b; // per row; inv_b NULL: the weight's
    const u32 *wpart;
    Finish end;
    u32 type;                // of the results
    u32 splits, steps;       // the reduction is dealt to `splits` workgroups, `steps` steps of KT each
    float *partial;          // [splits][M][n8] their sums; NULL: one workgroup has the whole reduction
    u32 n8;                  // N rounded up to 8
};

// 16 bytes per lane from device memory to LDS without registers in between: lane l's go to `to` + 16 l.
__device__ __forceinline__ void to_lds(const _Float16 *from, _Float16 *to)
{
    __builtin_amdgcn_global_load_lds((const GLOBAL_AS u32 *)from, (LDS_AS u32 *)to, 16, 0, 0);
}

// The scaled sums of row m, columns n .. n + 7, to where they belong.
template <u32 TY>
__device__ __forceinline__ void scaled8(const Gemm &g, u32 m, u32 n, float (&v)[8], float inv_w)
{
    const float inv_a = gptr(g.inv_a)[m];
    float b[8];
    if (g.inv_b) load8<TY_F32>(gptr(g.inv_b) + n, min(g.N - n, 8u), b);
#pragma unroll
    for (int t = 0; t < 8; t++) v[t] = v[t] * inv_a * (g.inv_b ? b[t] : inv_w);
    finish8<TY>(g.end, m, n, v);
}

// A tile of BM x BN, by waves of WM x WN.  A step takes 64 of the reduction: rows of 128 bytes in LDS, whose eight pieces
// of 16 bytes lie in an order of the row's own (piece c at c ^ (row / 2 % 8)), so that the 16 rows that a read touches
// fall into different banks.  The next step's rows are on their way while one is worked on.
template <u32 TY, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(BM / WM * (BN / WN) * 64) void k_product(Gemm g)
{
    constexpr int WAVES_M = BM / WM, WAVES = WAVES_M * (BN / WN), TM = WM / 16, TN = WN / 16;
    constexpr int LOADS = (BM + BN) / 8 / WAVES; // of 8 rows each, per wave and step
    __shared__ __attribute__((aligned(1024))) _Float16 lds[2][(BM + BN) * KT];
    const u32 wave = threadIdx.x >> 6, lane = threadIdx.x & 63u;
    // Workgroups go to the eight XCDs in turn; each XCD gets a run of tiles whose rows it finds in its own L2.
    u32 id = blockIdx.x;
    const u32 tiles = g.m_tiles * g.n_tiles, split = id / tiles;
    id -= split * tiles;
    const u32 per = (tiles + 7u) / 8u, full = tiles - (per - 1u) * 8u; // the first `full` XCDs have `per` tiles
    const u32 xcd = id & 7u, at = id >> 3;
    id = xcd < full ? xcd * per + at : full * per + (xcd - full) * (per - 1u) + at;
    const u32 m0 = id % g.m_tiles * BM, n0 = id / g.m_tiles * BN;
    const u32 wm = wave % WAVES_M * WM, wn = wave / WAVES_M * WN;
    // this lane's pieces of a step: row r of the tile's rows (a's, then b's)
    u64 from[LOADS];
    bool is_b[LOADS];
#pragma unroll
    for (int j = 0; j < LOADS; j++) {
        const u32 r = (wave * LOADS + j) * 8u + (lane >> 3), c = (lane & 7u) ^ ((r >> 1) & 7u);
        is_b[j] = (wave * LOADS + j) * 8u >= (u32)BM;
        // (rows past the last are the last: their results are not stored)
        const u32 row = is_b[j] ? min(n0 + r - BM, g.N - 1u) : min(m0 + r, g.M - 1u);
        from[j] = (u64)row * g.ld + c * 8u;
    }
    const u32 step0 = split * g.steps, n_steps = min(g.steps, g.ld / KT - step0) * g.pairs;
    u32 k = step0 * KT, pass = 0;
    auto fetch = [&](int buf) {
        const _Float16 *a = g.a + ((g.pa >> pass) & 1u) * g.plane_a + k, *b = g.b + ((g.pb >> pass) & 1u) * g.plane_b + k;
#pragma unroll
        for (int j = 0; j < LOADS; j++) to_lds((is_b[j] ? b : a) + from[j], lds[buf] + (wave * LOADS + j) * 8u * KT);
        if (++pass == g.pairs) {
            pass = 0;
            k += KT;
        }
    };
    f4 acc[TM][TN] = {};
    fetch(0);
    for (u32 t = 0; t < n_steps; t++) {
        __syncthreads(); // this step's rows have come, and the other buffer has been read
        if (t + 1 < n_steps) fetch((t + 1) & 1);
        const _Float16 *as = lds[t & 1], *bs = as + BM * KT;
#pragma unroll
        for (u32 kk = 0; kk < 2u; kk++) {
            h8 fa[TM], fb[TN];
            const u32 r = lane & 15u, c = ((kk * 4u + (lane >> 4)) ^ (r >> 1)) * 8u;
#pragma unroll
            for (u32 i = 0; i < TM; i++) fa[i] = *(const h8 *)(as + (wm + i * 16u + r) * KT + c);
#pragma unroll
            for (u32 j = 0; j < TN; j++) fb[j] = *(const h8 *)(bs + (wn + j * 16u + r) * KT + c);
            // (the columns of C are the rows of the instruction's result: a lane gets four consecutive ones)
#pragma unroll
            for (u32 i = 0; i < TM; i++)
#pragma unroll
                for (u32 j = 0; j < TN; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fb[j], fa[i], acc[i][j], 0, 0, 0);
        }
    }
    // The sums go through LDS, 64 rows of a wave at a time, so that eight lanes hold a row's 64 columns.
    static_assert(WM % 64 == 0 && WN == 64, "");
    float s, inv_w = 1.0f;
    if (!g.inv_b && !g.partial) weight_scale(g.wpart, s, inv_w);
    float *const mine = (float *)lds + wave * 4096u; // [64][64], the pieces of 4 of a row in an order of its own
#pragma unroll
    for (int half = 0; half < WM / 64; half++) {
        __syncthreads();
#pragma unroll
        for (u32 i = 0; i < 4u; i++)
#pragma unroll
            for (u32 j = 0; j < 4u; j++) {
                const u32 r = lane & 15u, c = j * 4u + (lane >> 4);
                *(f4 *)(mine + (i * 16u + r) * 64u + ((c ^ r) * 4u)) = acc[half * 4 + i][j];
            }
        __syncthreads();
        const u32 n = n0 + wn + (lane & 7u) * 8u;
#pragma unroll 1
        for (u32 q = 0; q < 8u; q++) {
            const u32 r = q * 8u + (lane >> 3), m = m0 + wm + half * 64u + r, c = (lane & 7u) * 2u;
            if (m >= g.M || n >= g.N) continue;
            float v[8];
            *(f4 *)v = *(const f4 *)(mine + r * 64u + (c ^ (r & 15u)) * 4u);
            *(f4 *)(v + 4) = *(const f4 *)(mine + r * 64u + ((c + 1u) ^ (r & 15u)) * 4u);
            if (g.partial) {
                float *to = g.partial + ((u64)split * g.M + m) * g.n8 + n;
                *(f4 *)to = *(const f4 *)v;
                *(f4 *)(to + 4) = *(const f4 *)(v + 4);
            } else {
                scaled8<TY>(g, m, n, v, inv_w);
            }
        }
    }
}

// The sums of the splits, in their order.
template <u32 TY>
__global__ __launch_bounds__(256) void k_join(Gemm g)
{
    float s, inv_w = 1.0f;
    if (!g.inv_b) weight_scale(g.wpart, s, inv_w);
    const u32 parts = g.n8 / 8u;
    const u64 all = (u64)g.M * parts;
    for (u64 i = blockIdx.x * 256ull + threadIdx.x; i < all; i += (u64)gridDim.x * 256u) {
        const u32 m = (u32)(i / parts), n = (u32)(i - (u64)m * parts) * 8u;
        float v[8] = {};
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
    p.plane = rows * p.ld;
    p.count = count;
    p.off = r.take(p.plane * count * 2u);
    p.inv = r.take(rows * 4u);
    return p;
}

template <int P>
void row_planes(const PlaneSrc &src, u32 type, const Planes &p, char *ws, hipStream_t s)
{
    _Float16 *dst = (_Float16 *)(ws + p.off);
    float *inv = (float *)(ws + p.inv);
    switch (type) {
    case TY_F32: PROF("k_row_planes", s, k_row_planes<TY_F32, P><<<src.rows, 256, 0, s>>>(src, dst, p.plane, (u32)p.ld, inv)); break;
    case TY_BF16: PROF("k_row_planes", s, k_row_planes<TY_BF16, P><<<src.rows, 256, 0, s>>>(src, dst, p.plane, (u32)p.ld, inv)); break;
    default: PROF("k_row_planes", s, k_row_planes<TY_F16, P><<<src.rows, 256, 0, s>>>(src, dst, p.plane, (u32)p.ld, inv)); break;
    }
}
void row_planes(const PlaneSrc &src, u32 type, const Planes &p, char *ws, hipStream_t s)
{
    if (p.count > 1)
        row_planes<2>(src, type, p, ws, s);
    else
        row_planes<1>(src, type, p, ws, s);
}

template <u32 TY>
void col_planes_of(const PlaneSrc &src, const Planes &p, char *ws, hipStream_t s)
{
    const u32 grid = (src.rows + 63u) / 64u * ((src.cols + 63u) / 64u);
    _Float16 *dst = (_Float16 *)(ws + p.off);
    const float *inv = (const float *)(ws + p.inv);
    if (p.count > 1)
        PROF("k_col_planes", s, k_col_planes<TY, 2><<<grid, 256, 0, s>>>(src, inv, dst, p.plane, p.ld));
    else
        PROF("k_col_planes", s, k_col_planes<TY, 1><<<grid, 256, 0, s>>>(src, inv, dst, p.plane, p.ld));
}
void col_planes(const PlaneSrc &src, u32 type, const Planes &p, char *ws, hipStream_t s)
{
    type == TY_F32 ? col_planes_of<TY_F32>(src, p, ws, s) : type == TY_BF16 ? col_planes_of<TY_BF16>(src, p, ws, s) : col_planes_of<TY_F16>(src, p, ws, s);
}
void col_stats(const PlaneSrc &src, u32 type, float *d, float *inv, float *sum, hipStream_t s)
{
    const u32 grid = (src.cols + 63u) / 64u;
    switch (type) {
    case TY_F32: PROF("k_col_stats", s, k_col_stats<TY_F32><<<grid, 256, 0, s>>>(src, d, inv, sum)); break;
    case TY_BF16: PROF("k_col_stats", s, k_col_stats<TY_BF16><<<grid, 256, 0, s>>>(src, d, inv, sum)); break;
    default: PROF("k_col_stats", s, k_col_stats<TY_F16><<<grid, 256, 0, s>>>(src, d, inv, sum)); break;
    }
}

// along: the reduction runs along the stored rows
template <int P, bool T>
void weight_planes_of(const WDesc &w, const Planes &p, char *ws, u64 part, hipStream_t s)
{
    const u32 *pm = (const u32 *)(ws + part);
    _Float16 *dst = (_Float16 *)(ws + p.off);
    PROF("k_weight_max", s, k_weight_max<<<WMAX_PARTS, 256, 0, s>>>(w, (u32 *)(ws + part)));
    // (the padding along the reduction belongs to the grid: it is written as zeros)
    const u32 grid = (w.cols + 63u) / 64u * ((w.rows + 63u) / 64u);
    PROF("k_weight_planes", s, k_weight_planes<P, T><<<grid, 256, 0, s>>>(w, pm, dst, p.plane, p.ld));
    if (w.n_outlier) {
        u64 blocks = (w.n_outlier + 255) / 256;
        if (blocks > 2048) blocks = 2048;
        PROF("k_weight_protected", s, k_weight_protected<P, T><<<(u32)blocks, 256, 0, s>>>(w, pm, dst, p.plane, p.ld));
    }
}
void weight_planes(const WDesc &w, bool along, const Planes &p, char *ws, u64 part, hipStream_t s)
{
    if (p.count > 1)
        along ? weight_planes_of<2, false>(w, p, ws, part, s) : weight_planes_of<2, true>(w, p, ws, part, s);
    else
        along ? weight_planes_of<1, false>(w, p, ws, part, s) : weight_planes_of<1, true>(w, p, ws, part, s);
}

// How a product is cut: tiles of 256 x 256 or 128 x 128, and the reduction among several workgroups where there are few tiles.
struct Cut {
    bool large;
    u32 m_tiles, n_tiles, splits, steps;
    u64 partial; // bytes
};
constexpr u32 CUS = 256;
Cut cut_of(u64 M, u64 N, u64 ld)
{
    Cut c;
    const u64 big = up(M, 256) / 256 * (up(N, 256) / 256);
    c.large = big >= CUS;
    const u32 side = c.large ? 256u : 128u;
    c.m_tiles = (u32)((M + side - 1) / side);
    c.n_tiles = (u32)((N + side - 1) / side);
    const u64 tiles = (u64)c.m_tiles * c.n_tiles, steps = ld / KT;
    c.splits = 1;
    while (!c.large && c.splits < 8u && tiles * c.splits < CUS && steps / (2u * c.splits) >= 4u) c.splits *= 2u;
    c.steps = (u32)((steps + c.splits - 1) / c.splits);
    c.splits = (u32)((steps + c.steps - 1) / c.steps); // (none without a step)
    c.partial = c.splits > 1 ? up(N, 8) * M * c.splits * 4u : 0;
    return c;
}

template <u32 TY>
void product_of(const Gemm &g, const Cut &c, hipStream_t s)
{
    const u32 grid = c.m_tiles * c.n_tiles * c.splits;
    if (c.large)
        PROF("k_product", s, k_product<TY, 256, 256, 128, 64><<<grid, 512, 0, s>>>(g));
    else
        PROF("k_product", s, k_product<TY, 128, 128, 64, 64><<<grid, 256, 0, s>>>(g));
    if (c.splits > 1) {
        const u64 all = (u64)g.M * (g.n8 / 8u), blocks = (all + 255) / 256;
        PROF("k_join", s, k_join<TY><<<(u32)(blocks < 4096 ? blocks : 4096), 256, 0, s>>>(g));
    }
}

void product(Gemm g, const Planes &a, const Planes &b, u64 partial, char *ws, hipStream_t s)
{
    g.a = (const _Float16 *)(ws + a.off);
    g.b = (const _Float16 *)(ws + b.off);
    g.plane_a = a.plane;
    g.plane_b = b.plane;
    g.ld = (u32)a.ld;
    // (smallest terms first) l h, h l, h h
    g.pairs = 0;
    g.pa = g.pb = 0;
    if (a.count > 1) g.pa |= 1u << g.pairs++;
    if (b.count > 1) g.pb |= 1u << g.pairs++;
    g.pairs++;
    const Cut c = cut_of(g.M, g.N, a.ld);
    g.m_tiles = c.m_tiles;
    g.n_tiles = c.n_tiles;
    g.splits = c.splits;
    g.steps = c.steps;
    g.n8 = (u32)up(g.N, 8);
    g.partial = c.splits > 1 ? (float *)(ws + partial) : nullptr;
    switch (g.type) {
    case TY_F32: product_of<TY_F32>(g, c, s); break;
    case TY_BF16: product_of<TY_BF16>(g, c, s); break;
    default: product_of<TY_F16>(g, c, s); break;
    }
}

// planes of the sides of a product whose result has this type
u32 planes_x(u32 type) { return type == TY_F32 ? 2u : 1u; }  // activations: bf16 and fp16 are exact in one
u32 planes_w(u32 type) { return type == TY_BF16 ? 1u : 2u; }

struct LinearRoom {
    Planes x, w;
    u64 part, partial, bytes;
    LinearRoom(u64 rows, u32 n_in, u32 n_out, u32 type)
    {
        Room r;
        x = planes_for(r, rows, n_in, planes_x(type));
        w = planes_for(r, n_out, n_in, planes_w(type));
        part = r.take(WMAX_PARTS * 4u);
        partial = r.take(cut_of(rows, n_out, x.ld).partial);
        bytes = r.at;
    }
};
struct GradRoom {
    u64 d = 0, part = 0, partial = 0, bytes = 0;
    Planes dr, w, dc, xc;
    bool own_d;
    GradRoom(u64 rows, u32 n_in, u32 n_out, u32 type, u32 act, bool dx, bool dw)
    {
        Room r;
        own_d = act != ACT_NONE; // the gradient below the activation, in fp32
        if (own_d) d = r.take(rows * n_out * 4u);
        const u32 dt = own_d ? TY_F32 : type;
        if (dx) {
            dr = planes_for(r, rows, n_out, type == TY_BF16 ? 1u : planes_x(dt));
            w = planes_for(r, n_in, n_out, planes_w(type));
            part = r.take(WMAX_PARTS * 4u);
        }
        if (dw) { // (fp32 results)
            dc = planes_for(r, n_out, rows, planes_x(dt));
            xc = planes_for(r, n_in, rows, planes_x(type));
        }
        // (the two products take turns)
        u64 most = dx ? cut_of(rows, n_in, dr.ld).partial : 0;
        if (dw) most = std::max(most, std::max(cut_of(n_out, n_in, dc.ld).partial, cut_of(n_in, n_out, dc.ld).partial));
        partial = r.take(most);
        bytes = r.at;
    }
};

} // namespace

u64 linear_space(u64 rows, u32 n_in, u32 n_out, u32 in_out, u32 type)
{
    return is_few(rows) ? 0 : LinearRoom(rows, n_in, n_out, type).bytes;
}
u64 linear_grad_space(u64 rows, u32 n_in, u32 n_out, u32 in_out, u32 type, u32 act, bool dx, bool dw)
{
    return rows ? GradRoom(rows, n_in, n_out, type, act, dx, dw).bytes : 0;
}

hipError_t launch_linear(const LinearCall &c, hipStream_t s)
{
    if (is_few(c.rows)) return launch_few(c, s);
    const LinearRoom r(c.rows, c.n_in, c.n_out, c.type);
    const PlaneSrc x = {c.x.p, nullptr, c.x.stride, 0, (u32)c.rows, c.n_in, ACT_NONE};
    row_planes(x, c.type, r.x, c.ws, s);
    weight_planes(c.w, !c.in_out, r.w, c.ws, r.part, s);
    Gemm g = {};
    g.M = (u32)c.rows;
    g.N = c.n_out;
    g.inv_a = (const float *)(c.ws + r.x.inv);
    g.wpart = (const u32 *)(c.ws + r.part);
    g.end = {c.bias, c.residual, c.y, c.pre, c.n_out, c.act};
    g.type = c.type;
    product(g, r.x, r.w, r.partial, c.ws, s);
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
    const GradRoom r(c.rows, c.n_in, c.n_out, c.type, c.act, c.dx.p != nullptr, c.dw != nullptr);
    PlaneSrc d = {c.dy.p, c.pre.p, c.dy.stride, c.pre.stride, (u32)c.rows, c.n_out, c.act};
    u32 dt = c.type;
    if (r.own_d || c.dw || c.db)
        col_stats(d, c.type, r.own_d ? (float *)(c.ws + r.d) : nullptr, c.dw ? (float *)(c.ws + r.dc.inv) : nullptr, c.db, s);
    if (r.own_d) {
        d = {c.ws + r.d, nullptr, c.n_out, 0, (u32)c.rows, c.n_out, ACT_NONE};
        dt = TY_F32;
    }
    if (c.dx.p) {
        row_planes(d, dt, r.dr, c.ws, s);
        weight_planes(c.w, c.in_out, r.w, c.ws, r.part, s);
        Gemm g = {};
        g.M = (u32)c.rows;
        g.N = c.n_in;
        g.inv_a = (const float *)(c.ws + r.dr.inv);
        g.wpart = (const u32 *)(c.ws + r.part);
        g.end = {nullptr, {}, c.dx, {}, c.n_in, ACT_NONE};
        g.type = c.type;
        product(g, r.dr, r.w, r.partial, c.ws, s);
    }
    if (c.dw) {
        const PlaneSrc x = {c.x.p, nullptr, c.x.stride, 0, (u32)c.rows, c.n_in, ACT_NONE};
        col_stats(x, c.type, nullptr, (float *)(c.ws + r.xc.inv), nullptr, s);
        col_planes(d, dt, r.dc, c.ws, s);
        col_planes(x, c.type, r.xc, c.ws, s);
        const Planes &a = c.in_out ? r.xc : r.dc, &b = c.in_out ? r.dc : r.xc;
        Gemm g = {};
        g.M = c.in_out ? c.n_in : c.n_out;
        g.N = c.in_out ? c.n_out : c.n_in;
        g.inv_a = (const float *)(c.ws + a.inv);
        g.inv_b = (const float *)(c.ws + b.inv);
        g.end = {nullptr, {}, {c.dw, g.N}, {}, g.N, ACT_NONE};
        g.type = TY_F32;
        product(g, a, b, r.partial, c.ws, s);
    }
    return hipGetLastError();
}

} // namespace inshr
