// Products of a few rows with a weight in its compressed form: the symbols go from the stream through a table in LDS
// straight into the operands of the matrix cores.
//
// What bounds it: the stream (w / 8 bytes a weight) and the vector instructions that take the symbols apart (two to place
// a symbol as a table address, one to put its value next to its neighbour's; the table look-up runs beside them).  The
// matrix cores have time to spare, so the factors keep all their bits:
//   bfloat16  the centre as two bfloat16 numbers (16 bits), two instructions
//   fp16      the centre scaled by a power of two as two fp16 numbers (22 bits), two instructions
//   fp32      centre and activation as three bfloat16 numbers each (all 24 bits), the six products that matter
//
// A lane decodes whole runs of consecutive symbols, so that after one funnel shift to the run's first bit all positions
// are constants.  Which k's of the reduction meet in an instruction is free as long as both operands agree:
//   weight [n_out][n_in]  (k_few_rows)  lane (i, g) takes 32 consecutive k of output i, 8 of them per instruction
//   weight [n_in][n_out]  (k_few_cols)  lane (i, g) takes R consecutive outputs of 8 consecutive k; the t-th of them go
//                                        into instruction t, whose outputs are then R apart
// A workgroup's waves share its outputs and split the reduction; their sums are joined in a fixed order.
//
// Protected values are 0 in the table and are added at the end, from the list, in fixed point: whole numbers add up to
// the same sum in any order.
#include "inshr_table.h"

namespace inshr {

typedef __bf16 b8 __attribute__((ext_vector_type(8)));

union Frag { // eight numbers of 16 bits
    u32 u[4];
    u4_16 q;
    h8 h;
    b8 b;
};

// ------------------------------------------------------------------------------------------
// operands
// ------------------------------------------------------------------------------------------
// The parts of eight values, by falling size, from their entries.
template <u32 TY> struct Parts {
    static constexpr int N = TY == TY_F32 ? 3 : 2;
    Frag p[N];
};
template <u32 TY>
__device__ __forceinline__ void put_entries(Parts<TY> &w, int i, const u32 (&a)[2], const u32 (&b)[2]) // values 2i, 2i + 1
{
    w.p[0].u[i] = low_halves(a[0], b[0]);
    w.p[1].u[i] = high_halves(a[0], b[0]);
    if constexpr (TY == TY_F32) w.p[2].u[i] = low_halves(a[1], b[1]);
}

// Eight activations, of which `left` exist, as parts (one for bfloat16 and fp16).
template <u32 TY> struct Xs {
    static constexpr int N = TY == TY_F32 ? 3 : 1;
    Frag p[N];
};
template <u32 TY>
__device__ __forceinline__ void load_xs(const GLOBAL_AS typename Elem<TY>::type *p, u32 left, Xs<TY> &x)
{
    if constexpr (TY == TY_F32) {
        float v[8];
        load8<TY>(p, left, v);
#pragma unroll
        for (int i = 0; i < 4; i++) {
            u32 h[2], m[2], l[2];
#pragma unroll
            for (int j = 0; j < 2; j++) {
                const float a = v[2 * i + j];
                h[j] = __float_as_uint(a);
                const float r1 = a - __uint_as_float(h[j] & 0xffff0000u);
                m[j] = __float_as_uint(r1);
                l[j] = __float_as_uint(r1 - __uint_as_float(m[j] & 0xffff0000u));
            }
            x.p[0].u[i] = high_halves(h[0], h[1]);
            x.p[1].u[i] = high_halves(m[0], m[1]);
            x.p[2].u[i] = high_halves(l[0], l[1]);
        }
    } else {
        x.p[0].q = load_raw8<TY>(p, left).q[0];
    }
}
template <u32 TY>
__device__ __forceinline__ f4 multiply(const Parts<TY> &w, const Xs<TY> &x, f4 c) // smallest products first
{
    if constexpr (TY == TY_F32) {
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.p[2].b, x.p[0].b, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.p[1].b, x.p[1].b, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.p[0].b, x.p[2].b, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.p[1].b, x.p[0].b, c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.p[0].b, x.p[1].b, c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.p[0].b, x.p[0].b, c, 0, 0, 0);
    } else if constexpr (TY == TY_BF16) {
        c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.p[1].b, x.p[0].b, c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w.p[0].b, x.p[0].b, c, 0, 0, 0);
    } else {
        c = __builtin_amdgcn_mfma_f32_16x16x32_f16(w.p[1].h, x.p[0].h, c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(w.p[0].h, x.p[0].h, c, 0, 0, 0);
    }
}

// ------------------------------------------------------------------------------------------
// protected values
// ------------------------------------------------------------------------------------------
// The first entry of the list that is not below `index`, by the lanes of half a wave: 32 places of what is left are
// looked at at once.
__device__ __forceinline__ u64 first_listed(const WDesc &w, u64 index, u32 half_lane, u32 half)
{
    u64 lo = 0, n = w.n_outlier; // the answer lies in lo .. lo + n
    while (__ballot(n > 0)) {    // (the halves of the wave may need different numbers of steps)
        const u64 step = (n + 31) / 32, at = lo + (half_lane + 1u) * step - 1u; // the last entries of 32 parts
        const bool below = n > 0 && at < lo + n && gptr(w.out_idx)[at] < index;
        const u64 past = (u64)__popc((u32)(__ballot(below) >> (32u * half))) * step;
        lo += past;
        n = n == 0 ? 0 : min(step - 1, n - past); // (the next part's last entry is not below, or not there)
    }
    return lo;
}

struct Few {
    WDesc w;
    Finish end;
    Mat x;
    u32 rows, n_in, n_out, in_out;
    u32 cols;        // outputs of a workgroup
    u32 row_blocks;  // blocks of 16 MT rows
    u32 sums_at;     // byte offsets into LDS: the joined sums, ...
    u32 listed_at;   // ... the protected values' part of them
};

// The scale of the centres alone, by every wave.
__device__ __forceinline__ void centre_scale(const WDesc &w, float &s, float &inv)
{
    u32 m = 0u;
    for (u32 i = threadIdx.x & 63u; i < w.K; i += 64u) m = max(m, finite_mag(gptr(w.codebook)[i]));
    scale_of(wave_max_u(m), s, inv);
}

// The joined sums of a workgroup, cols of them per row, lie at `sums`; adds the protected values' part and stores the
// results.  lo .. hi: the entries of the list that may belong to the workgroup.
template <u32 TY, int MT>
__device__ void finish(const Few &f, char *lds, u64 lo, u64 hi, u32 m0, u32 n0, float inv)
{
    typedef typename Elem<TY>::type T;
    const float *sums = (const float *)(lds + f.sums_at);
    unsigned long long *listed = (unsigned long long *)(lds + f.listed_at);
    __shared__ u32 high[16 * MT]; // largest magnitude of a row's products
    const u32 rows = min(f.rows - m0, 16u * MT), cells = rows * f.cols;
    const bool any = hi > lo;
    if (any) {
        // Fixed point: the largest magnitude of a product of the row gets 40 bits, so that nothing is off by more than
        // 2^-41 of it (and 2^22 of them still fit).
        if (threadIdx.x < 16u * MT) high[threadIdx.x] = 0u;
        for (u32 i = threadIdx.x; i < cells; i += blockDim.x) listed[i] = 0ull;
        __syncthreads();
        u32 m_high[16 * MT];
#pragma unroll
        for (int m = 0; m < 16 * MT; m++) m_high[m] = 0u;
        for (int pass = 0; pass < 2; pass++) {
            for (u64 j = lo + threadIdx.x; j < hi; j += blockDim.x) {
                const u32 at = gptr(f.w.out_idx)[j], r = at / f.w.cols, c = at - r * f.w.cols;
                const u32 n = f.in_out ? c : r, k = f.in_out ? r : c;
                if (r >= f.w.rows || n < n0 || n >= n0 + f.cols) continue;
                const float v = protected_value(f.w, j);
                const GLOBAL_AS T *x = (const GLOBAL_AS T *)f.x.p + (u64)m0 * f.x.stride + k;
#pragma unroll
                for (u32 m = 0; m < 16u * MT; m++) {
                    if (m >= rows) continue;
                    const float p = v * Elem<TY>::get(x[(u64)m * f.x.stride]);
                    if (pass == 0)
                        m_high[m] = max(m_high[m], finite_mag(p));
                    else if (mag_bits(p) < 0x7f800000u) // a product below 2^(e - 126) times this is below 2^40
                        atomicAdd(&listed[m * f.cols + n - n0],
                                  (unsigned long long)__double2ll_rn(ldexp((double)p, 166 - (int)(high[m] >> 23))));
                }
            }
            if (pass == 0) {
#pragma unroll
                for (u32 m = 0; m < 16u * MT; m++) {
                    if (m >= rows) continue;
                    const u32 w = wave_max_u(m_high[m]);
                    if ((threadIdx.x & 63u) == 0u) atomicMax(&high[m], w);
                }
            }
            __syncthreads();
        }
    }
    for (u32 i = threadIdx.x; i < cells / 8u; i += blockDim.x) {
        const u32 m = i / (f.cols / 8u), n = (i - m * (f.cols / 8u)) * 8u;
        if (n0 + n >= f.n_out) continue;
        float v[8];
#pragma unroll
        for (u32 t = 0; t < 8u; t++) {
            v[t] = sums[m * f.cols + n + t] * inv;
            if (any) v[t] += (float)ldexp((double)(long long)listed[m * f.cols + n + t], (int)(high[m] >> 23) - 166);
        }
        finish8<TY>(f.end, m0 + m, n0 + n, v);
    }
}

// ------------------------------------------------------------------------------------------
// weight [n_out][n_in]
// ------------------------------------------------------------------------------------------
// 16 outputs, 16 MT rows; the last wave looks the workgroup's part of the protected list up while the others work.
template <u32 TY, int W, int MT>
__global__ __launch_bounds__(1024) void k_few_rows(Few f)
{
    typedef typename Elem<TY>::type T;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ u64 range[2];
    u32 *table = (u32 *)lds;
    f4 *part = (f4 *)(lds + Table<TY, W>::BYTES);
    const u32 wave = threadIdx.x >> 6, lane = threadIdx.x & 63u, waves = (blockDim.x >> 6) - 1u;
    const u32 n0 = blockIdx.x / f.row_blocks * 16u, m0 = blockIdx.x % f.row_blocks * (16u * MT);
    float s = 1.0f, inv = 1.0f;
    if (TY == TY_F16) centre_scale(f.w, s, inv);
    fill_table<TY, W>(f.w, table, s);
    __syncthreads();
    f4 acc[MT] = {};
    if (wave == waves) {
        const u32 half = lane >> 5;
        const u64 first = (u64)min(n0 + half * 16u, f.n_out) * f.n_in;
        const u64 at = f.w.n_outlier ? first_listed(f.w, first, lane & 31u, half) : 0;
        if ((lane & 31u) == 0u) range[half] = at;
    } else {
        const u32 i = lane & 15u, g = lane >> 4, K = f.n_in;
        const u64 row_bit = (u64)min(n0 + i, f.n_out - 1u) * K * W;
        const u32 mine = lane_copy<TY, W>();
        const GLOBAL_AS T *x[MT];
#pragma unroll
        for (int t = 0; t < MT; t++) {
            x[t] = (const GLOBAL_AS T *)f.x.p + (u64)min(m0 + 16u * t + i, f.rows - 1u) * f.x.stride;
        }
        for (u32 k0 = wave * 128u; k0 < K; k0 += waves * 128u) {
            const u32 k = k0 + 32u * g, left = k < K ? K - k : 0u;
            u32 raw[W + 1], d[W];
            const u64 bit = row_bit + (u64)k * W;
            load_words<W + 1>(f.w.packed, bit >> 5, left ? f.w.n_words : 0, raw);
#pragma unroll
            for (int j = 0; j < W; j++) d[j] = __builtin_amdgcn_alignbit(raw[j + 1], raw[j], (u32)bit & 31u);
            if (left < 32u) { // what follows in the stream is another output's
#pragma unroll
                for (int j = 0; j < W; j++) {
                    const int keep = (int)(left * W) - 32 * j;
                    d[j] = keep >= 32 ? d[j] : keep <= 0 ? 0u : d[j] & ((1u << keep) - 1u);
                }
            }
#pragma unroll
            for (int s = 0; s < 4; s++) {
                Parts<TY> w;
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    u32 a[2], b[2];
                    look_up<TY, W>((const char *)table, mine, d, 8 * s + 2 * j, a);
                    look_up<TY, W>((const char *)table, mine, d, 8 * s + 2 * j + 1, b);
                    put_entries<TY>(w, j, a, b);
                }
#pragma unroll
                for (int t = 0; t < MT; t++) {
                    Xs<TY> v;
                    load_xs<TY>(x[t] + k + 8 * s, left > 8u * s ? left - 8u * s : 0u, v);
                    acc[t] = multiply<TY>(w, v, acc[t]);
                }
            }
        }
#pragma unroll
        for (int t = 0; t < MT; t++) part[(wave * MT + t) * 64u + lane] = acc[t];
    }
    __syncthreads();
    // lane (i, g) of a part holds row i, outputs 4 g .. 4 g + 3
    float *sums = (float *)(lds + f.sums_at);
    for (u32 j = threadIdx.x; j < MT * 64u; j += blockDim.x) {
        f4 v = part[j];
        for (u32 q = 1; q < waves; q++) v += part[q * MT * 64u + j];
        *(f4 *)(sums + (j >> 6) * 256u + (j & 15u) * 16u + (j >> 4 & 3u) * 4u) = v;
    }
    __syncthreads();
    finish<TY, MT>(f, lds, range[0], range[1], m0, n0, inv);
}

// ------------------------------------------------------------------------------------------
// weight [n_in][n_out]
// ------------------------------------------------------------------------------------------
// 16 R outputs, 16 MT rows; lane (i, g) decodes outputs i R .. i R + R - 1 of the k's 8 g .. 8 g + 7 of 32.
template <u32 TY, int W, int MT, int R>
__global__ __launch_bounds__(1024) void k_few_cols(Few f)
{
    typedef typename Elem<TY>::type T;
    constexpr int ND = (R * W + 31) / 32; // words of a run
    extern __shared__ __attribute__((aligned(16))) char lds[];
    u32 *table = (u32 *)lds;
    f4 *part = (f4 *)(lds + Table<TY, W>::BYTES);
    const u32 wave = threadIdx.x >> 6, lane = threadIdx.x & 63u, waves = blockDim.x >> 6;
    const u32 n0 = blockIdx.x / f.row_blocks * (16u * R), m0 = blockIdx.x % f.row_blocks * (16u * MT);
    float s = 1.0f, inv = 1.0f;
    if (TY == TY_F16) centre_scale(f.w, s, inv);
    fill_table<TY, W>(f.w, table, s);
    __syncthreads();
    const u32 i = lane & 15u, g = lane >> 4, K = f.n_in;
    const u32 mine = lane_copy<TY, W>();
    const GLOBAL_AS T *x[MT];
#pragma unroll
    for (int t = 0; t < MT; t++) {
        x[t] = (const GLOBAL_AS T *)f.x.p + (u64)min(m0 + 16u * t + i, f.rows - 1u) * f.x.stride;
    }
    f4 acc[MT][R] = {};
    const u64 row_bits = (u64)f.n_out * W, run_bit = (u64)(n0 + i * R) * W;
    for (u32 k0 = wave * 32u; k0 < K; k0 += waves * 32u) {
        const u32 k = k0 + 8u * g, left = k < K ? K - k : 0u;
        u32 e[8][R][2];
#pragma unroll
        for (u32 j = 0; j < 8u; j++) {
            u32 raw[ND + 1], d[ND + 1];
            const u64 bit = (u64)(k + j) * row_bits + run_bit;
            load_words<ND + 1>(f.w.packed, bit >> 5, j < left ? f.w.n_words : 0, raw);
#pragma unroll
            for (int q = 0; q < ND; q++) d[q] = __builtin_amdgcn_alignbit(raw[q + 1], raw[q], (u32)bit & 31u);
            d[ND] = 0u;
#pragma unroll
            for (int t = 0; t < R; t++) look_up<TY, W>((const char *)table, mine, d, t, e[j][t]);
        }
        Xs<TY> v[MT];
#pragma unroll
        for (int t = 0; t < MT; t++) load_xs<TY>(x[t] + k, left, v[t]);
#pragma unroll
        for (int q = 0; q < R; q++) {
            Parts<TY> w;
#pragma unroll
            for (int j = 0; j < 4; j++) put_entries<TY>(w, j, e[2 * j][q], e[2 * j + 1][q]);
#pragma unroll
            for (int t = 0; t < MT; t++) acc[t][q] = multiply<TY>(w, v[t], acc[t][q]);
        }
    }
    // lane (i, g) of instruction q holds row i, outputs (4 g + c) R + q
    float *sums = (float *)(lds + f.sums_at);
#pragma unroll
    for (int q = 0; q < R; q++) {
        __syncthreads();
#pragma unroll
        for (int t = 0; t < MT; t++) part[(wave * MT + t) * 64u + lane] = acc[t][q];
        __syncthreads();
        for (u32 j = threadIdx.x; j < MT * 64u; j += blockDim.x) {
            f4 v = part[j];
            for (u32 o = 1; o < waves; o++) v += part[o * MT * 64u + j];
#pragma unroll
            for (u32 c = 0; c < 4u; c++) sums[((j >> 6) * 16u + (j & 15u)) * (16u * R) + ((j >> 4 & 3u) * 4u + c) * R + q] = v[c];
        }
    }
    __syncthreads();
    finish<TY, MT>(f, lds, 0, f.w.n_outlier, m0, n0, inv);
}

// ------------------------------------------------------------------------------------------
// calls
// ------------------------------------------------------------------------------------------
namespace {

template <u32 TY, int W, int MT>
void start_rows(Few &f, hipStream_t s)
{
    // waves: enough for four to a SIMD over all workgroups, each with two steps of 128 at least where there are as many
    const u32 groups = (f.n_out + 15u) / 16u * f.row_blocks, steps = (f.n_in + 127u) / 128u;
    u32 waves = 4;
    while (waves < 15u && waves * groups < 4096u && waves * 2u < steps) waves = min(waves * 2u, 15u);
    f.cols = 16;
    f.sums_at = Table<TY, W>::BYTES + waves * MT * 1024u;
    f.listed_at = f.sums_at + MT * 1024u;
    const u32 lds = f.listed_at + (f.w.n_outlier ? MT * 2048u : 0u);
    PROF("k_few_rows", s, k_few_rows<TY, W, MT><<<groups, 64u * (waves + 1u), lds, s>>>(f));
}
template <u32 TY, int W, int MT, int R>
void start_cols_of(Few &f, hipStream_t s)
{
    const u32 groups = (f.n_out + 16u * R - 1u) / (16u * R) * f.row_blocks, steps = (f.n_in + 31u) / 32u;
    u32 waves = 4;
    while (waves < 16u / MT && waves * groups < 4096u && waves * 2u < steps) waves *= 2u; // (64 KB of LDS at most)
    f.cols = 16u * R;
    f.sums_at = Table<TY, W>::BYTES + waves * MT * 1024u;
    f.listed_at = f.sums_at + MT * R * 1024u;
    const u32 lds = f.listed_at + (f.w.n_outlier ? MT * R * 2048u : 0u);
    PROF("k_few_cols", s, k_few_cols<TY, W, MT, R><<<groups, 64u * waves, lds, s>>>(f));
}
template <u32 TY, int W, int MT>
void start(Few &f, hipStream_t s)
{
    if (!f.in_out)
        start_rows<TY, W, MT>(f, s);
    else
        start_cols_of<TY, W, MT, TY == TY_F32 ? 2 : 4>(f, s);
}
template <u32 TY>
void start_mt(Few &f, hipStream_t s)
{
    if (f.rows <= 16u) {
        f.row_blocks = 1;
        with_width(f.w.w, [&](auto w) { start<TY, decltype(w)::value, 1>(f, s); });
    } else {
        f.row_blocks = (f.rows + 31u) / 32u;
        with_width(f.w.w, [&](auto w) { start<TY, decltype(w)::value, 2>(f, s); });
    }
}

} // namespace

hipError_t launch_few(const LinearCall &c, hipStream_t s)
{
    Few f = {};
    f.w = c.w;
    f.end = {c.bias, c.residual, c.y, c.pre, c.n_out, c.act};
    f.x = c.x;
    f.rows = (u32)c.rows;
    f.n_in = c.n_in;
    f.n_out = c.n_out;
    f.in_out = c.in_out;
    switch (c.type) {
    case TY_F32: start_mt<TY_F32>(f, s); break;
    case TY_BF16: start_mt<TY_BF16>(f, s); break;
    default: start_mt<TY_F16>(f, s); break;
    }
    return hipGetLastError();
}

} // namespace inshr
