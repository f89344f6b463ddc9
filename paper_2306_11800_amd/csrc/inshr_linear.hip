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

namespace inshr {

// ------------------------------------------------------------------------------------------
// planes of an operand whose reduction runs along its rows
// ------------------------------------------------------------------------------------------
constexpr u32 KT = 64;  // reduction per step of the product: planes are padded to it with zeros
constexpr u32 RT = 128; // rows and columns of a workgroup's tile
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
    u32 n_tiles;             // along N
    u32 pairs;               // number of passes
    u32 pa, pb;              // plane of pass i: bit i
    const float *inv_a, *inv_b; // per row; inv_b NULL: the weight's
    const u32 *wpart;
    Finish end;
    u32 type;                // of the results
};

template <u32 TY>
__global__ __launch_bounds__(256) void k_product(Gemm g)
{
    constexpr u32 LD = KT + 8;
    __shared__ _Float16 As[RT * LD], Bs[RT * LD];
    const u32 m0 = blockIdx.x / g.n_tiles * RT, n0 = blockIdx.x % g.n_tiles * RT;
    const u32 wave = threadIdx.x >> 6, lane = threadIdx.x & 63u;
    const u32 wm = (wave & 1u) * 64u, wn = (wave >> 1) * 64u;
    f4 acc[4][4] = {};
    for (u32 k0 = 0; k0 < g.ld; k0 += KT)
        for (u32 p = 0; p < g.pairs; p++) {
            const _Float16 *a = g.a + ((g.pa >> p) & 1u) * g.plane_a, *b = g.b + ((g.pb >> p) & 1u) * g.plane_b;
            h8 va[4], vb[4];
#pragma unroll
            for (u32 j = 0; j < 4u; j++) {
                const u32 i = threadIdx.x + 256u * j, r = i >> 3, c = (i & 7u) * 8u;
                // (rows past the last are the last: their results are not stored)
                va[j] = *(const h8 *)(a + (u64)min(m0 + r, g.M - 1u) * g.ld + k0 + c);
                vb[j] = *(const h8 *)(b + (u64)min(n0 + r, g.N - 1u) * g.ld + k0 + c);
            }
            __syncthreads();
#pragma unroll
            for (u32 j = 0; j < 4u; j++) {
                const u32 i = threadIdx.x + 256u * j, r = i >> 3, c = (i & 7u) * 8u;
                *(h8 *)(As + r * LD + c) = va[j];
                *(h8 *)(Bs + r * LD + c) = vb[j];
            }
            __syncthreads();
#pragma unroll
            for (u32 kk = 0; kk < KT; kk += 32u) {
                h8 fa[4], fb[4];
#pragma unroll
                for (u32 t = 0; t < 4u; t++) {
                    fa[t] = *(const h8 *)(As + (wm + t * 16u + (lane & 15u)) * LD + kk + (lane >> 4) * 8u);
                    fb[t] = *(const h8 *)(Bs + (wn + t * 16u + (lane & 15u)) * LD + kk + (lane >> 4) * 8u);
                }
                // (the columns of C are the rows of the instruction's result: a lane gets four consecutive ones)
#pragma unroll
                for (u32 i = 0; i < 4u; i++)
#pragma unroll
                    for (u32 j = 0; j < 4u; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(fb[j], fa[i], acc[i][j], 0, 0, 0);
            }
        }
    float s, inv_w = 1.0f;
    if (!g.inv_b) weight_scale(g.wpart, s, inv_w);
#pragma unroll
    for (u32 i = 0; i < 4u; i++) {
        const u32 m = m0 + wm + i * 16u + (lane & 15u);
        if (m >= g.M) continue;
        const float inv_a = gptr(g.inv_a)[m];
#pragma unroll
        for (u32 j = 0; j < 4u; j++) {
            const u32 n = n0 + wn + j * 16u + (lane >> 4) * 4u;
            if (n >= g.N) continue;
            f4 v = acc[i][j];
#pragma unroll
            for (u32 t = 0; t < 4u; t++) v[t] = v[t] * inv_a * (g.inv_b ? (n + t < g.N ? gptr(g.inv_b)[n + t] : 0.0f) : inv_w);
            epilogue4<TY>(g.end, m, n, v);
        }
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

void product(Gemm g, const Planes &a, const Planes &b, char *ws, hipStream_t s)
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
    g.n_tiles = (g.N + RT - 1) / RT;
    const u32 grid = g.n_tiles * ((g.M + RT - 1) / RT);
    switch (g.type) {
    case TY_F32: PROF("k_product", s, k_product<TY_F32><<<grid, 256, 0, s>>>(g)); break;
    case TY_BF16: PROF("k_product", s, k_product<TY_BF16><<<grid, 256, 0, s>>>(g)); break;
    default: PROF("k_product", s, k_product<TY_F16><<<grid, 256, 0, s>>>(g)); break;
    }
}

// planes of the sides of a product whose result has this type
u32 planes_x(u32 type) { return type == TY_F32 ? 2u : 1u; }  // activations: bf16 and fp16 are exact in one
u32 planes_w(u32 type) { return type == TY_BF16 ? 1u : 2u; }

struct LinearRoom {
    Planes x, w;
    u64 part, bytes;
    LinearRoom(u64 rows, u32 n_in, u32 n_out, u32 type)
    {
        Room r;
        x = planes_for(r, rows, n_in, planes_x(type));
        w = planes_for(r, n_out, n_in, planes_w(type));
        part = r.take(WMAX_PARTS * 4u);
        bytes = r.at;
    }
};
struct GradRoom {
    u64 d = 0, part = 0, bytes = 0;
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
    product(g, r.x, r.w, c.ws, s);
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
        product(g, r.dr, r.w, c.ws, s);
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
        product(g, a, b, c.ws, s);
    }
    return hipGetLastError();
}

} // namespace inshr
