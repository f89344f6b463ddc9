// Products of a few rows with a weight in its compressed form: the symbols go from the stream through a table in LDS
// straight into the operands.
//
// What bounds it: the stream (w / 8 bytes a weight) and the vector instructions that take the symbols apart (two to place
// a symbol as a table address, one to put its value next to its neighbour's or to multiply it; the table look-up runs beside
// them).  A lane decodes whole runs of consecutive symbols, so that after one funnel shift to the run's first bit all
// positions are constants.
//   weight [n_out][n_in]  k_few_rows: the reduction runs along the stream.  Lane (i, g) takes 32 consecutive k of output i, 8 of
//                         them per instruction of the matrix cores (which k's meet in an instruction is free as long as both
//                         operands agree).  The matrix cores have time to spare, so the factors keep all their bits:
//                           bfloat16  the centre as two bfloat16 numbers (16 bits), two instructions
//                           fp16      the centre scaled by a power of two as two fp16 numbers (22 bits), two instructions
//                           fp32      centre and activation as three bfloat16 numbers each (all 24 bits), the six products
//                                     that matter
//   weight [n_in][n_out]  k_few_split: a thread keeps the sums of 16 or 8 consecutive outputs and walks down a part of the rows of
//                         the weight; k_few_join adds the parts.  fp32 throughout, one multiplication per weight and row of
//                         activations, which is why it takes up to FEW_SPLIT rows.
// Measured: one token through 4096 x 11008 bf16 of 6 bits a weight 15.5 us (34 MB of stream: 2.2 TB/s; vector instructions for 45 M
// symbols and the start of the launch share it), 24 rows through 11008 x 4096 fp16 of 7 bits 27.5, one token through 1024 x 4096 stored
// [n_in][n_out] 12.2 (8.7 and 4.0 for the join).
// All sums are taken in a fixed order.  Protected values are 0 in the table and are added from the list.
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

// The scale of the centres alone, by every wave.
__device__ __forceinline__ void centre_scale(const WDesc &w, float &s, float &inv)
{
    u32 m = 0u;
    for (u32 i = threadIdx.x & 63u; i < w.K; i += 64u) m = max(m, finite_mag(gptr(w.codebook)[i]));
    scale_of(wave_max_u(m), s, inv);
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

// Where entries of `index` and above begin among the count ones from lo on, relative to lo (and so at most count).
__device__ __forceinline__ u32 starts_at(const WDesc &w, u64 lo, u32 count, u64 index)
{
    u32 from = 0u;
    while (count) {
        const u32 half = count / 2u;
        const bool below = gptr(w.out_idx)[lo + from + half] < index;
        from += below ? half + 1u : 0u;
        count = below ? count - half - 1u : half;
    }
    return from;
}

// ------------------------------------------------------------------------------------------
// weight [n_out][n_in]
// ------------------------------------------------------------------------------------------
constexpr u32 TURNED = 32; // rows of activations side by side in their turned copy
constexpr u32 FEW_PLAIN = 4; // up to as many rows are read as they are

struct Few {
    WDesc w;
    Finish end;
    Mat x;
    const Frag *packed; // k_few_pack's, or NULL
    const void *turned;
    u32 steps;          // of 128 of the reduction
    float *partial;     // k_few_split: [splits][rows][n8]
    u32 rows, n_in, n_out, n8;
    u32 row_blocks;     // blocks of 16 MT rows
    u32 splits, depth;  // k_few_split: parts of the reduction, rows of a part
};

// What the other kernels read of more than FEW_PLAIN rows of x, so that their loads take whole lines (16 rows of x a load
// were 64 pieces of 16 bytes, and the 512 cycles that a CU takes for a step's addresses were all of its time):
//   packed  the operands of the matrix cores, [tile of 16 rows][step of 128][4 instructions][parts][64 lanes][8]
//   turned  blocks of TURNED rows, the activations that a protected value meets side by side
// The first `tiles * steps` workgroups pack, the others turn.
template <u32 TY>
__global__ __launch_bounds__(256) void k_few_pack(Mat x, u32 rows, u32 cols, u32 tiles, u32 steps, Frag *__restrict__ packed,
                                                  typename Elem<TY>::type *__restrict__ turned)
{
    typedef typename Elem<TY>::type T;
    if (blockIdx.x < tiles * steps) {
        const u32 tile = blockIdx.x / steps, kb = blockIdx.x % steps, s = threadIdx.x >> 6, lane = threadIdx.x & 63u;
        const u32 r = tile * 16u + (lane & 15u), k = kb * 128u + 32u * (lane >> 4) + 8u * s;
        Xs<TY> v;
        load_xs<TY>((const GLOBAL_AS T *)x.p + (u64)min(r, rows - 1u) * x.stride + k, k < cols && r < rows ? cols - k : 0u, v);
#pragma unroll
        for (int q = 0; q < Xs<TY>::N; q++) packed[((u64)(blockIdx.x * 4u + s) * Xs<TY>::N + q) * 64u + lane] = v.p[q];
        return;
    }
    __shared__ T tile[64][TURNED + 2];
    const u32 id = blockIdx.x - tiles * steps, across = (cols + 63u) / 64u, c0 = id % across * 64u, block = id / across, r0 = block * TURNED;
    for (u32 i = threadIdx.x; i < 64u * TURNED; i += 256u) {
        const u32 r = r0 + i / 64u, c = c0 + i % 64u;
        tile[i % 64u][i / 64u] = r < rows && c < cols ? ((const GLOBAL_AS T *)x.p)[(u64)r * x.stride + c] : (T)0;
    }
    __syncthreads();
    for (u32 i = threadIdx.x; i < 64u * TURNED; i += 256u) {
        const u32 c = i / TURNED;
        if (c0 + c < cols) turned[((u64)block * cols + c0 + c) * TURNED + i % TURNED] = tile[c][i % TURNED];
    }
}

constexpr u32 AHEAD = 1; // steps whose part of the stream is asked for before one is worked on (two: fewer waves, 16 -> 20 us for a token)

// This wave's steps of 128 of the reduction, `every` apart.  SAFE: no load of the stream can lead past its end.
template <u32 TY, int W, int MT, bool PACKED, bool SAFE>
__device__ __forceinline__ void few_steps(const Few &f, const char *table, u32 n0, u32 m0, u32 k0, u32 every, u32 (&raw)[AHEAD][W + 1], f4 (&acc)[MT])
{
    typedef typename Elem<TY>::type T;
    const u32 lane = threadIdx.x & 63u, i = lane & 15u, g = lane >> 4, K = f.n_in;
    const u64 row_bit = (u64)min(n0 + i, f.n_out - 1u) * K * W;
    const u32 mine = lane_copy<TY, W>();
    const GLOBAL_AS T *x[MT];
#pragma unroll
    for (int t = 0; t < MT; t++) x[t] = PACKED ? nullptr : (const GLOBAL_AS T *)f.x.p + (u64)min(m0 + 16u * t + i, f.rows - 1u) * f.x.stride;
    for (; k0 < K; k0 += AHEAD * every) {
#pragma unroll
        for (u32 ahead = 0; ahead < AHEAD; ahead++) {
            const u32 kb = k0 + ahead * every, k = kb + 32u * g;
            if (kb >= K) break;
            const u32 left = k < K ? K - k : 0u;
            const bool full = kb + 128u <= K; // (the same for all lanes)
            u32 d[W];
            const u32 shift = (u32)(row_bit + (u64)k * W) & 31u;
#pragma unroll
            for (int j = 0; j < W; j++) d[j] = __builtin_amdgcn_alignbit(raw[ahead][j + 1], raw[ahead][j], shift);
            const u32 next = k + AHEAD * every;
            if (kb + AHEAD * every < K) load_words<W + 1, SAFE>(f.w.packed, (row_bit + (u64)next * W) >> 5, next < K ? f.w.n_words : 0, raw[ahead]);
            if (kb + 128u > K) { // what follows in the stream is another output's
#pragma unroll
                for (int j = 0; j < W; j++) {
                    const int keep = (int)(min(left, 32u) * W) - 32 * j;
                    d[j] = keep >= 32 ? d[j] : keep <= 0 ? 0u : d[j] & ((1u << keep) - 1u);
                }
            }
#pragma unroll
            for (int s = 0; s < 4; s++) {
                Parts<TY> w;
#pragma unroll
                for (int j = 0; j < 4; j++) {
                    u32 a[2], b[2];
                    look_up<TY, W>(table, mine, d, 8 * s + 2 * j, a);
                    look_up<TY, W>(table, mine, d, 8 * s + 2 * j + 1, b);
                    put_entries<TY>(w, j, a, b);
                }
#pragma unroll
                for (int t = 0; t < MT; t++) {
                    Xs<TY> v;
                    if (PACKED) {
                        const Frag *p = f.packed + ((u64)((m0 / 16u + t) * f.steps + kb / 128u) * 4u + s) * (Xs<TY>::N * 64u) + lane;
#pragma unroll
                        for (int q = 0; q < Xs<TY>::N; q++) v.p[q].q = *(const GLOBAL_AS u4_16 *)&gptr(p)[q * 64].q;
                    } else {
                        load_xs<TY>(x[t] + k + 8u * s, full ? 8u : left > 8u * s ? left - 8u * s : 0u, v);
                    }
                    acc[t] = multiply<TY>(w, v, acc[t]);
                }
            }
            __builtin_amdgcn_sched_barrier(0); // (one step's activations in registers at a time)
        }
    }
}
// The stream of the first AHEAD steps: asked for before anything else.
template <int W, bool SAFE>
__device__ __forceinline__ void few_first(const Few &f, u32 n0, u32 k0, u32 every, u32 (&raw)[AHEAD][W + 1])
{
    const u32 lane = threadIdx.x & 63u, K = f.n_in;
    const u64 row_bit = (u64)min(n0 + (lane & 15u), f.n_out - 1u) * K * W;
#pragma unroll
    for (u32 ahead = 0; ahead < AHEAD; ahead++) {
        const u32 kb = k0 + ahead * every, k = kb + 32u * (lane >> 4);
        if (kb < K) load_words<W + 1, SAFE>(f.w.packed, (row_bit + (u64)k * W) >> 5, k < K ? f.w.n_words : 0, raw[ahead]);
    }
}

// Up to FEW_PLAIN rows: the protected values' part of 16 outputs, by one wave while the others work on the stream.  64 entries
// at a time; the entries of an output follow each other and are added up by a scan, and the last one's lane has the sum.
template <u32 TY>
__device__ __forceinline__ void listed_by_wave(const Few &f, u64 lo, u64 hi, u32 n0, float (*listed)[16])
{
    typedef typename Elem<TY>::type T;
    const u32 lane = threadIdx.x & 63u, K = f.n_in;
    if (lane < 16u)
        for (u32 m = 0; m < f.rows; m++) listed[m][lane] = 0.0f;
    for (u64 j0 = lo; j0 < hi; j0 += 64u) {
        const u64 j = j0 + lane;
        const u32 at = j < hi ? gptr(f.w.out_idx)[j] : 0u, row = at / K, k = at - row * K;
        const bool mine = j < hi && row - n0 < 16u;
        const u32 t = mine ? row - n0 : 16u + lane; // (the others: outputs of their own)
        const float v = mine ? protected_value(f.w, j) : 0.0f;
        const u32 after = __shfl_down(t, 1);
        const bool last = mine && (lane == 63u || after != t);
        for (u32 m = 0; m < f.rows; m++) {
            float p = mine ? v * Elem<TY>::get(((const GLOBAL_AS T *)f.x.p)[(u64)m * f.x.stride + k]) : 0.0f;
#pragma unroll
            for (u32 d = 1; d < 64u; d <<= 1) {
                const float up = __shfl_up(p, d);
                const u32 whose = __shfl_up(t, d);
                if (lane >= d && whose == t) p += up;
            }
            if (last) listed[m][t] += p;
        }
    }
}

// 16 outputs, 16 MT rows; the last wave looks the workgroup's part of the protected list up while the others work.
template <u32 TY, int W, int MT, bool PACKED>
__global__ __launch_bounds__(1024) void k_few_rows(Few f)
{
    typedef typename Elem<TY>::type T;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ u64 range[2];
    __shared__ u32 starts[17];
    __shared__ __attribute__((aligned(16))) float sums[16 * MT][16], listed[16 * MT][16];
    u32 *table = (u32 *)lds;
    f4 *part = (f4 *)(lds + Table<TY, W>::BYTES);
    const u32 wave = threadIdx.x >> 6, lane = threadIdx.x & 63u, waves = (blockDim.x >> 6) - 1u;
    const u32 n0 = blockIdx.x / f.row_blocks * 16u, m0 = blockIdx.x % f.row_blocks * (16u * MT), K = f.n_in;
    // the furthest word that a lane may ask for: row n0 + 15, its k rounded up to whole steps
    const bool safe = (((u64)min(n0 + 15u, f.n_out - 1u) * K + K + 128u) * W >> 5) + W + 2u <= f.w.n_words;
    const u32 every = waves * 128u;
    u32 raw[AHEAD][W + 1];
    if (wave < waves) safe ? few_first<W, true>(f, n0, wave * 128u, every, raw) : few_first<W, false>(f, n0, wave * 128u, every, raw);
    float s = 1.0f, inv = 1.0f;
    if (TY == TY_F16) centre_scale(f.w, s, inv);
    fill_table<TY, W>(f.w, table, s);
    __syncthreads();
    if (wave == waves) {
        const u32 half = lane >> 5;
        const u64 first = (u64)min(n0 + half * 16u, f.n_out) * K;
        const u64 at = f.w.n_outlier ? first_listed(f.w, first, lane & 31u, half) : 0;
        if ((lane & 31u) == 0u) range[half] = at;
        const u64 lo = __shfl(at, 0), hi = __shfl(at, 32);
        if (!PACKED) {
            listed_by_wave<TY>(f, lo, hi, n0, listed);
        } else if (lane <= 16u && hi > lo) { // where each output's entries begin, relative to lo
            starts[lane] = starts_at(f.w, lo, (u32)(hi - lo), (u64)min(n0 + lane, f.n_out) * K);
        }
    } else {
        f4 acc[MT] = {};
        if (safe)
            few_steps<TY, W, MT, PACKED, true>(f, (const char *)table, n0, m0, wave * 128u, every, raw, acc);
        else
            few_steps<TY, W, MT, PACKED, false>(f, (const char *)table, n0, m0, wave * 128u, every, raw, acc);
#pragma unroll
        for (int t = 0; t < MT; t++) part[(wave * MT + t) * 64u + lane] = acc[t];
    }
    __syncthreads();
    const u64 lo = range[0], hi = range[1];
    const u32 rows = min(f.rows - m0, 16u * MT);
    // lane (i, g) of a part holds row i, outputs 4 g .. 4 g + 3
    for (u32 j = threadIdx.x; j < MT * 64u; j += blockDim.x) {
        f4 v = part[j];
        for (u32 q = 1; q < waves; q++) v += part[q * MT * 64u + j];
        *(f4 *)&sums[(j >> 6) * 16u + (j & 15u)][(j >> 4 & 3u) * 4u] = v;
    }
    __syncthreads();
    if (PACKED && hi > lo) { // a wave per output; four lanes an entry, eight rows each, four entries a lane at a time
        for (u32 t = wave; t < 16u; t += waves + 1u) {
            const u32 from = starts[t], to = starts[t + 1u], base = (n0 + t) * K; // (at most hi - lo)
            const GLOBAL_AS T *x = (const GLOBAL_AS T *)f.turned + (u64)(m0 / TURNED) * K * TURNED + (lane & 3u) * 8u;
            float sum[8] = {};
            for (u32 j0 = from + (lane >> 2); j0 < to; j0 += 64u) {
                u32 k[4];
                float v[4];
                Raw8<TY> a[4];
#pragma unroll
                for (u32 q = 0; q < 4u; q++) {
                    const u32 j = min(j0 + 16u * q, to - 1u);
                    k[q] = gptr(f.w.out_idx)[lo + j] - base;
                    v[q] = j0 + 16u * q < to && k[q] < K ? protected_value(f.w, lo + j) : 0.0f;
                    k[q] = min(k[q], K - 1u);
                }
#pragma unroll
                for (u32 q = 0; q < 4u; q++) a[q] = load_raw8<TY>(x + (u64)k[q] * TURNED, 8u);
#pragma unroll
                for (u32 q = 0; q < 4u; q++)
#pragma unroll
                    for (int i = 0; i < 8; i++) sum[i] += v[q] != 0.0f ? v[q] * a[q][i] : 0.0f;
            }
#pragma unroll
            for (int d = 4; d < 64; d <<= 1)
#pragma unroll
                for (int q = 0; q < 8; q++) sum[q] += __shfl_xor(sum[q], d);
            if (lane < 2u * MT) {
#pragma unroll
                for (int q = 0; q < 8; q++) listed[lane * 8u + q][t] = sum[q];
            }
        }
        __syncthreads();
    }
    for (u32 j = threadIdx.x; j < rows * 2u; j += blockDim.x) {
        const u32 m = j >> 1, n = (j & 1u) * 8u;
        if (n0 + n >= f.n_out) continue;
        float v[8];
#pragma unroll
        for (u32 t = 0; t < 8u; t++) v[t] = sums[m][n + t] * inv + (hi > lo ? listed[m][n + t] : 0.0f);
        finish8<TY>(f.end, m0 + m, n0 + n, v);
    }
}

// ------------------------------------------------------------------------------------------
// weight [n_in][n_out]
// ------------------------------------------------------------------------------------------
// Consecutive outputs of a thread, 256 of which walk down the rows together.  Runs of 16 take 4 loads where two of 8 take
// 6, but make half the workgroups, and wide symbols take more registers.  One token, runs of 8 / of 16, in us: 2048 x 4096 of 7
// bits 15.9/17.6; 4096 x 4096 of 6 bits 19.1/21.8, of 7 bits 19.0/27.7; 4096 x 8192 of 5 bits 24.0/23.5, of 7 bits 23.4/31.6;
// 4096 x 11008 of 6 bits 33.2/28.4, of 7 bits 32.9/39.2; 1024 x 50257 of 7 bits 52.4/42.8; 8192 x 8192 of 6 bits 35.5/29.8, of 7
// bits 35.0/43.1.  (Four rows' sums of 16 outputs do not fit into the registers.)
inline u32 split_run(u32 rows, u32 n_in, u32 n_out, u32 w)
{
    return rows == 1u && (u64)n_in * n_out >= ((w <= 6u ? 40ull : 48ull) << 20) ? 16u : 8u;
}
constexpr u32 SPLIT_DEPTH = 64;  // most rows of the weight that it walks down

// Rows blockIdx.x % splits * depth .. of the weight.  Table: the values themselves.  Four waves walk down the rows; the
// fifth looks up where the protected entries of each row are meanwhile.
template <u32 TY, int W, int M, u32 R>
__global__ __launch_bounds__(320) void k_few_split(Few f)
{
    typedef typename Elem<TY>::type T;
    typedef Table<TY_BF16, W> Tab; // (one word an entry, as there)
    constexpr u32 COLS = 256u * R, STAGE = 1024, THREADS = 320;
    constexpr int ND = (R * W + 31) / 32;
    constexpr u32 ROWS = 4; // rows asked for before one is worked on
    __shared__ __attribute__((aligned(16))) u32 table[Tab::BYTES / 4];
    __shared__ float xs[SPLIT_DEPTH][M];
    __shared__ float extra[M][COLS];
    __shared__ u32 starts[SPLIT_DEPTH + 1], stage_col[STAGE];
    __shared__ float stage_val[STAGE];
    __shared__ u64 range[2];
    const u32 split = blockIdx.x % f.splits, n0 = blockIdx.x / f.splits * COLS, ka = split * f.depth, kn = min(f.depth, f.n_in - ka);
    const u32 tid = threadIdx.x, run = tid * R, n = n0 + run;
    const bool walks = tid < 256u && n < f.n_out;
    const u64 first_bit = ((u64)ka * f.n_out + n) * W, row_bits = (u64)f.n_out * W;
    u32 raw[ROWS][ND + 1];
    auto ask = [&](u32 j, u32 *d) { // row j of the part
        const u64 bit = first_bit + j * row_bits;
        load_words<ND + 1>(f.w.packed, bit >> 5, walks && j < kn ? f.w.n_words : 0, d);
    };
#pragma unroll
    for (u32 j = 0; j < ROWS; j++) ask(j, raw[j]);
    for (u32 i = tid; i < kn * M; i += THREADS)
        xs[i / M][i % M] = i % M < f.rows ? Elem<TY>::get(((const GLOBAL_AS T *)f.x.p)[(u64)(i % M) * f.x.stride + ka + i / M]) : 0.0f;
    for (u32 i = tid; i < (1u << W) * Tab::COPIES; i += THREADS) table[i] = __float_as_uint(symbol_value(f.w, i / Tab::COPIES));
    const bool any = f.w.n_outlier != 0;
    if (any)
        for (u32 i = tid; i < M * COLS; i += THREADS) extra[i / COLS][i % COLS] = 0.0f;
    __syncthreads();
    float acc[M][R] = {};
    if (tid >= 256u) {
        const u32 lane = tid & 63u, half = lane >> 5;
        const u64 at = any ? first_listed(f.w, (u64)(ka + half * kn) * f.n_out, lane & 31u, half) : 0;
        if ((lane & 31u) == 0u) range[half] = at;
        const u64 lo = __shfl(at, 0), hi = __shfl(at, 32);
        if (hi > lo)
            for (u32 t = lane; t <= kn; t += 64u) starts[t] = starts_at(f.w, lo, (u32)(hi - lo), (u64)(ka + t) * f.n_out);
    } else {
        const u32 mine = lane_copy<TY_BF16, W>();
        for (u32 j0 = 0; j0 < kn; j0 += ROWS) {
#pragma unroll
            for (u32 q = 0; q < ROWS; q++) {
                const u32 j = j0 + q;
                if (j >= kn) break;
                const u32 shift = (u32)(first_bit + j * row_bits) & 31u;
                u32 d[ND + 1];
#pragma unroll
                for (int t = 0; t < ND; t++) d[t] = __builtin_amdgcn_alignbit(raw[q][t + 1], raw[q][t], shift);
                d[ND] = 0u;
                ask(j + ROWS, raw[q]);
                float x[M];
#pragma unroll
                for (int m = 0; m < M; m++) x[m] = xs[j][m];
#pragma unroll
                for (int t = 0; t < (int)R; t++) {
                    u32 e[2];
                    look_up<TY_BF16, W>((const char *)table, mine, d, t, e);
#pragma unroll
                    for (int m = 0; m < M; m++) acc[m][t] = fmaf(x[m], __uint_as_float(e[0]), acc[m][t]);
                }
            }
        }
    }
    __syncthreads();
    // the protected values row by row, as a row has an output once; a part of the list at a time in LDS
    const u64 lo = range[0], hi = range[1];
    if (hi > lo) {
        const u32 count = (u32)(hi - lo);
        u32 j = 0; // the first row that is not done
        for (u32 s0 = 0; s0 < count; s0 += STAGE) {
            const u32 s1 = min(count, s0 + STAGE);
            for (u32 i = s0 + tid; i < s1; i += THREADS) {
                stage_col[i - s0] = gptr(f.w.out_idx)[lo + i];
                stage_val[i - s0] = protected_value(f.w, lo + i);
            }
            __syncthreads();
            for (; j < kn; j++) {
                const u32 from = max(starts[j], s0), to = min(starts[j + 1u], s1);
                for (u32 i = from + tid; i < to; i += THREADS) {
                    const u32 c = stage_col[i - s0] - (ka + j) * f.n_out - n0;
                    if (c >= COLS || c + n0 >= f.n_out) continue;
#pragma unroll
                    for (int m = 0; m < M; m++) extra[m][c] = fmaf(xs[j][m], stage_val[i - s0], extra[m][c]);
                }
                __syncthreads();
                if (starts[j + 1u] > s1) break; // (the rest of the row is in the next part)
            }
        }
    }
    if (!walks) return;
#pragma unroll
    for (int m = 0; m < M; m++) {
        if ((u32)m >= f.rows) break;
        float *to = f.partial + ((u64)split * f.rows + m) * f.n8 + n;
#pragma unroll
        for (u32 q = 0; q < R; q += 4u) {
            if (n + q >= f.n8) break;
            f4 a;
#pragma unroll
            for (u32 t = 0; t < 4u; t++) a[t] = acc[m][q + t] + (any ? extra[m][run + q + t] : 0.0f);
            *(f4 *)(to + q) = a;
        }
    }
}

// 64 outputs of a row: thread (part, i) adds the splits part, part + 32, ... of outputs 8 i .. 8 i + 7.
template <u32 TY>
__global__ __launch_bounds__(256) void k_few_join(Few f)
{
    __shared__ __attribute__((aligned(16))) float sums[32][64];
    const u32 blocks = (f.n_out + 63u) / 64u, m = blockIdx.x / blocks, n0 = blockIdx.x % blocks * 64u;
    const u32 i = (threadIdx.x & 7u) * 8u, part = threadIdx.x >> 3;
    f4 a = {}, b = {};
    if (n0 + i < f.n_out) {
#pragma unroll 8
        for (u32 q = part; q < f.splits; q += 32u) {
            const GLOBAL_AS f4 *p = (const GLOBAL_AS f4 *)(gptr(f.partial) + ((u64)q * f.rows + m) * f.n8 + n0 + i);
            a += p[0];
            b += p[1];
        }
    }
    *(f4 *)&sums[part][i] = a;
    *(f4 *)&sums[part][i + 4] = b;
    for (u32 d = 16; d; d >>= 1) {
        __syncthreads();
        if (part < d) {
            *(f4 *)&sums[part][i] += *(const f4 *)&sums[part + d][i];
            *(f4 *)&sums[part][i + 4] += *(const f4 *)&sums[part + d][i + 4];
        }
    }
    if (part == 0u && n0 + i < f.n_out) {
        float v[8];
#pragma unroll
        for (u32 t = 0; t < 8u; t++) v[t] = sums[0][i + t];
        finish8<TY>(f.end, m, n0 + i, v);
    }
}

// ------------------------------------------------------------------------------------------
// calls
// ------------------------------------------------------------------------------------------
namespace {

struct FewRoom {
    u64 packed = 0, turned = 0, partial = 0; // bytes (the last, or the others)
    u32 tiles = 0, steps = 0;                // of `packed`
    u32 splits = 1, depth = 1;
    FewRoom(u64 rows, u32 n_in, u32 n_out, bool in_out, u32 type, u32 w, bool listed)
    {
        if (!in_out) {
            steps = (n_in + 127u) / 128u;
            if (rows <= FEW_PLAIN) return;
            tiles = rows <= 16u ? 1u : ((u32)rows + 31u) / 32u * 2u;
            packed = (u64)tiles * steps * 4096u * (type == TY_F32 ? Xs<TY_F32>::N : 1);
            if (listed) turned = (rows + TURNED - 1) / TURNED * TURNED * n_in * elem_size(type);
            return;
        }
        // about 768 workgroups (three a CU) where the weight has 4 rows for each at least, SPLIT_DEPTH at most
        const u32 cols = 256u * split_run((u32)rows, n_in, n_out, w), blocks = (n_out + cols - 1u) / cols;
        depth = (u32)(((u64)n_in * blocks + 767u) / 768u);
        depth = depth < 4u ? 4u : depth > SPLIT_DEPTH ? SPLIT_DEPTH : depth;
        splits = (n_in + depth - 1u) / depth;
        partial = (u64)splits * rows * ((n_out + 7u) / 8u * 8u) * 4u;
    }
};

template <u32 TY, int W, int MT, bool PACKED>
void start_rows(Few &f, hipStream_t s)
{
    // As many waves as let all workgroups run at once, at 24 waves a CU (16 with two tiles of rows, which take more
    // registers), but not more than there are steps for.  A token through 4096 x 11008, 688 workgroups: 5 waves each 18.4 us,
    // 6 16.9, 8 15.6, 10 19.7; 9 waves in two rounds 25.
    const u32 groups = (f.n_out + 15u) / 16u * f.row_blocks, per_cu = (groups + 255u) / 256u, slots = MT == 1 ? 24u : 16u;
    u32 waves = per_cu >= slots / 3u ? 2u : slots / per_cu - 1u;
    waves = waves < 15u ? waves : 15u;
    waves = waves < f.steps ? waves : f.steps;
    PROF("k_few_rows", s, k_few_rows<TY, W, MT, PACKED><<<groups, 64u * (waves + 1u), Table<TY, W>::BYTES + waves * MT * 1024u, s>>>(f));
}
template <u32 TY>
void start_few(Few &f, const LinearCall &c, hipStream_t s)
{
    const FewRoom r(c.rows, c.n_in, c.n_out, c.in_out != 0, c.type, c.w.w, c.w.n_outlier != 0);
    if (!c.in_out) {
        f.steps = r.steps;
        f.row_blocks = f.rows <= 16u ? 1u : (f.rows + 31u) / 32u;
        if (r.packed) {
            f.packed = (const Frag *)c.ws;
            f.turned = c.ws + r.packed;
            const u32 grid = r.tiles * r.steps + (r.turned ? (c.n_in + 63u) / 64u * ((f.rows + TURNED - 1u) / TURNED) : 0u);
            PROF("k_few_pack", s, k_few_pack<TY><<<grid, 256, 0, s>>>(c.x, f.rows, c.n_in, r.tiles, r.steps, (Frag *)c.ws,
                                                                      (typename Elem<TY>::type *)(c.ws + r.packed)));
        }
        with_width(f.w.w, [&](auto w) {
            constexpr int W = decltype(w)::value;
            if (f.rows <= FEW_PLAIN)
                start_rows<TY, W, 1, false>(f, s);
            else if (f.rows <= 16u)
                start_rows<TY, W, 1, true>(f, s);
            else
                start_rows<TY, W, 2, true>(f, s);
        });
        return;
    }
    f.partial = (float *)c.ws;
    f.splits = r.splits;
    f.depth = r.depth;
    f.n8 = (f.n_out + 7u) / 8u * 8u;
    const u32 run = split_run(f.rows, f.n_in, f.n_out, f.w.w), grid = r.splits * ((f.n_out + 256u * run - 1u) / (256u * run));
    with_width(f.w.w, [&](auto w) {
        constexpr int W = decltype(w)::value;
        if (f.rows > 1u)
            PROF("k_few_split", s, k_few_split<TY, W, (int)FEW_SPLIT, 8><<<grid, 320, 0, s>>>(f));
        else if (run == 16u)
            PROF("k_few_split", s, k_few_split<TY, W, 1, 16><<<grid, 320, 0, s>>>(f));
        else
            PROF("k_few_split", s, k_few_split<TY, W, 1, 8><<<grid, 320, 0, s>>>(f));
    });
    PROF("k_few_join", s, k_few_join<TY><<<f.rows * ((f.n_out + 63u) / 64u), 256, 0, s>>>(f));
}

} // namespace

u64 few_space(u64 rows, u32 n_in, u32 n_out, bool in_out, u32 type, u32 w, bool listed)
{
    const FewRoom r(rows, n_in, n_out, in_out, type, w, listed);
    return rows ? r.packed + r.turned + r.partial : 0;
}

hipError_t launch_few(const LinearCall &c, hipStream_t s)
{
    Few f = {};
    f.w = c.w;
    f.end = {c.bias, c.residual, c.y, c.pre, c.n_out, c.act};
    f.x = c.x;
    f.rows = (u32)c.rows;
    f.n_in = c.n_in;
    f.n_out = c.n_out;
    switch (c.type) {
    case TY_F32: start_few<TY_F32>(f, c, s); break;
    case TY_BF16: start_few<TY_BF16>(f, c, s); break;
    default: start_few<TY_F16>(f, c, s); break;
    }
    return hipGetLastError();
}

} // namespace inshr
