// A teacher's largest logits with the mass of the others, and the distillation loss on them with its gradient.
//
// One workgroup takes a row.  Sums of exponentials run over the row once, every thread with the largest value it has
// seen so far (what it holds is scaled down when a larger one comes), and are joined in fp64.
#include "inshr_answer.h"

namespace inshr {

constexpr double LOG2E = 1.4426950408889634, LN2 = 0.69314718055994531;

// log sum e^(x / T) as it grows: `m` the largest value seen, `s` the sum of e^((x - m) / T)
struct RowSum {
    float m, s;
};
__device__ __forceinline__ RowSum row_sum() { return {-INFINITY, 0.0f}; }
__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }
// eight more values; the ones that do not count are -inf.  c: log2 e / T
__device__ __forceinline__ void add8(RowSum &a, const float (&v)[8], float c)
{
    float m = fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
    m = fmaxf(m, a.m);
    if (m == -INFINITY) { // (nothing yet, or a NaN, which the sum then keeps)
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (v[i] != v[i]) a.s = v[i];
        return;
    }
    float s = a.s * pow2((a.m - m) * c);
#pragma unroll
    for (int i = 0; i < 8; i++) s += pow2((v[i] - m) * c);
    a.m = m;
    a.s = s;
}

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ double wave_max(double v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v = fmax(v, __shfl_xor(v, d));
    return v;
}
// Over all threads of the workgroup, the same for everybody; `room`: a double per wave.
template <int WAVES>
__device__ double block_sum(double v, double *room)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63u) == 0u) room[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0.0;
    for (int i = 0; i < WAVES; i++) v += room[i];
    return v;
}
template <int WAVES>
__device__ double block_max(double v, double *room)
{
    v = wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63u) == 0u) room[threadIdx.x >> 6] = v;
    __syncthreads();
    v = room[0];
    for (int i = 1; i < WAVES; i++) v = fmax(v, room[i]);
    return v;
}
// log of the sum that the threads hold together, -inf where nothing counts
template <int WAVES>
__device__ double block_log(const RowSum &a, double inv_T, double *room)
{
    const double m = block_max<WAVES>((double)a.m, room);
    const double part = a.s > 0.0f ? (double)a.s * exp(((double)a.m - m) * inv_T) : (a.s != a.s ? (double)a.s : 0.0);
    const double s = block_sum<WAVES>(part, room);
    return s > 0.0 ? m * inv_T + log(s) : s != s ? s : -INFINITY;
}

template <u32 TY>
__device__ __forceinline__ const GLOBAL_AS typename Elem<TY>::type *row_of(const Mat &m, u64 r)
{
    return (const GLOBAL_AS typename Elem<TY>::type *)m.p + r * m.stride;
}

// ------------------------------------------------------------------------------------------
// the largest logits
// ------------------------------------------------------------------------------------------
constexpr u32 TOP_BLOCK = 1024, TOP_ROOM = 2048;

__device__ __forceinline__ u32 logit_key(float x) { return x != x ? 0xFFFFFFFFu : key_of_float(x); }
__device__ __forceinline__ float logit_of(u32 key) { return __uint_as_float(bits_of_key(key)); }

template <class T>
__device__ void sort_descending(T *v, u32 n) // n: a power of two
{
    for (u32 size = 2; size <= n; size <<= 1)
        for (u32 step = size >> 1; step; step >>= 1) {
            __syncthreads();
            for (u32 i = threadIdx.x; i < n / 2u; i += blockDim.x) {
                const u32 a = 2u * i - (i & (step - 1u)), b = a + step;
                const T x = v[a], y = v[b];
                if ((x < y) == ((a & size) == 0u)) {
                    v[a] = y;
                    v[b] = x;
                }
            }
        }
    __syncthreads();
}

template <u32 TY>
__global__ __launch_bounds__(TOP_BLOCK) void k_top_logits(LogitsCall c, int *__restrict__ index, float *__restrict__ value, float *__restrict__ tail)
{
    constexpr int WAVES = TOP_BLOCK / 64;
    __shared__ u64 cand[TOP_ROOM];
    __shared__ u32 maxima[TOP_BLOCK];
    __shared__ double room[WAVES];
    __shared__ u32 n_cand, count;
    const u64 r = blockIdx.x;
    const auto *p = row_of<TY>(c.logits, r);
    const bool wide = ((u64)p & 15u) == 0u;
    const u32 V = c.n_vocab, k = c.k, tid = threadIdx.x;
    const double inv_T = 1.0 / (double)c.temperature;
    const float c2 = (float)(LOG2E * inv_T);

    // The k-th of the threads' largest keys: at least k elements are not below it.
    u32 top = 0u;
    for (u32 i = tid * 8u; i < V; i += TOP_BLOCK * 8u) {
        float v[8];
        load8<TY>(p + i, wide, V - i, v);
#pragma unroll
        for (u32 j = 0; j < 8u; j++)
            if (i + j < V) top = max(top, logit_key(v[j]));
    }
    maxima[tid] = top;
    if (tid == 0) n_cand = 0u;
    sort_descending(maxima, TOP_BLOCK);
    const u32 thr = maxima[k - 1u], highest = maxima[0];

    // Everything from it on is a candidate; the others are added up.
    RowSum rest = row_sum();
    for (u32 i = tid * 8u; i < V; i += TOP_BLOCK * 8u) {
        float v[8];
        load8<TY>(p + i, wide, V - i, v);
#pragma unroll
        for (u32 j = 0; j < 8u; j++) {
            const u32 key = logit_key(v[j]);
            if (i + j >= V) {
                v[j] = -INFINITY;
            } else if (key >= thr) {
                const u32 at = atomicAdd(&n_cand, 1u);
                if (at < TOP_ROOM) cand[at] = (u64)key << 32 | (u32)~(i + j);
                v[j] = -INFINITY;
            }
        }
        add8(rest, v, c2);
    }
    __syncthreads();
    u32 n = n_cand;
    if (n > TOP_ROOM) {
        // Too many equal ones: the key of rank k by halving, then the larger ones and the first of the equal ones.
        u32 lo = thr, hi = 0xFFFFFFFFu; // count(>= lo) >= k
        while (lo < hi) {
            const u32 mid = lo + (hi - lo) / 2u + 1u;
            __syncthreads();
            if (tid == 0) count = 0u;
            __syncthreads();
            u32 have = 0u;
            for (u32 i = tid; i < V; i += TOP_BLOCK) have += logit_key(Elem<TY>::get(p[i])) >= mid ? 1u : 0u;
            if (have) atomicAdd(&count, have);
            __syncthreads();
            if (count >= k)
                lo = mid;
            else
                hi = mid - 1u;
        }
        __syncthreads();
        if (tid == 0) n_cand = 0u;
        __syncthreads();
        rest = row_sum();
        for (u32 i = tid; i < V; i += TOP_BLOCK) {
            const float x = Elem<TY>::get(p[i]);
            const u32 key = logit_key(x);
            if (key > lo) cand[atomicAdd(&n_cand, 1u)] = (u64)key << 32 | (u32)~i; // (fewer than k)
            if (key < lo) {
                const float one[8] = {x, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY};
                add8(rest, one, c2);
            }
        }
        __syncthreads();
        n = n_cand;
        u32 equal = 0u; // equal ones before this step of the row, the same in all threads
        for (u32 i0 = 0; i0 < V; i0 += TOP_BLOCK) {
            const u32 i = i0 + tid;
            const bool is = i < V && logit_key(Elem<TY>::get(p[i])) == lo;
            const u64 mask = __ballot(is);
            __syncthreads();
            if ((tid & 63u) == 0u) maxima[tid >> 6] = (u32)__popcll(mask);
            __syncthreads();
            u32 before = equal, all = 0u;
            for (int w = 0; w < WAVES; w++) {
                if (w < (int)(tid >> 6)) before += maxima[w];
                all += maxima[w];
            }
            if (is) {
                const u32 at = n + before + (u32)__popcll(mask & ((1ull << (tid & 63u)) - 1ull));
                if (at < k)
                    cand[at] = (u64)lo << 32 | (u32)~i;
                else if (lo != key_of_float(-INFINITY)) {
                    const float one[8] = {logit_of(lo), -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY};
                    add8(rest, one, c2);
                }
            }
            equal += all;
        }
        __syncthreads();
        n = k;
    }
    u32 size = 2u;
    while (size < n) size <<= 1;
    for (u32 i = n + tid; i < size; i += TOP_BLOCK) cand[i] = 0ull;
    sort_descending(cand, size);
    for (u32 i = tid; i < n; i += TOP_BLOCK) {
        const u32 key = (u32)(cand[i] >> 32);
        if (i < k) {
            gptr(index)[r * k + i] = (int)~(u32)cand[i];
            gptr(value)[r * k + i] = Elem<TY>::get(p[~(u32)cand[i]]);
        } else {
            const float one[8] = {logit_of(key), -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY, -INFINITY};
            add8(rest, one, c2);
        }
    }
    if (tail) {
        const double l = block_log<WAVES>(rest, inv_T, room);
        if (tid == 0) gptr(tail)[r] = highest >= key_of_float(INFINITY) ? __uint_as_float(0x7fc00000u) : (float)l;
    }
}

// ------------------------------------------------------------------------------------------
// the loss
// ------------------------------------------------------------------------------------------
constexpr u32 DIST_BLOCK = 256; // threads; at least MAX_LISTED
static_assert(DIST_BLOCK >= MAX_LISTED, "a thread per listed entry");
// Saved per row: log of the student's sum, log of its part that is not listed, log of the teacher's sum, and what the
// unlisted ones' gradient is of their share of that part: q - P_tail e^(u - log_out) = e^(u - log_out) (q_rest - P_tail).
constexpr int SAVED = 4;

// This thread's entry of the list, or -1: no thread, no index of the vocabulary, or one that stands earlier in the list.
__device__ __forceinline__ int listed_entry(const LogitsCall &c, u64 r, int *idx)
{
    int i = -1;
    if (threadIdx.x < c.k) {
        i = gptr(c.index)[r * c.k + threadIdx.x];
        if (i < 0 || (u32)i >= c.n_vocab) i = -1;
        idx[threadIdx.x] = i;
    }
    __syncthreads();
    for (u32 j = 0; j < threadIdx.x && j < c.k; j++)
        if (idx[j] == i) i = -1;
    return i;
}

template <u32 TY>
__global__ __launch_bounds__(DIST_BLOCK) void k_distill(LogitsCall c, float *__restrict__ loss, double *__restrict__ saved)
{
    constexpr int WAVES = DIST_BLOCK / 64;
    extern __shared__ u32 bits[]; // which logits are listed
    __shared__ int idx[MAX_LISTED];
    __shared__ double room[WAVES];
    const u64 r = blockIdx.x;
    const auto *p = row_of<TY>(c.logits, r);
    const bool wide = ((u64)p & 15u) == 0u;
    const u32 V = c.n_vocab, tid = threadIdx.x;
    const double inv_T = 1.0 / (double)c.temperature;
    const float c2 = (float)(LOG2E * inv_T);
    for (u32 i = tid; i < (V + 31u) / 32u; i += DIST_BLOCK) bits[i] = 0u;
    const int mine = listed_entry(c, r, idx); // (a barrier inside)
    if (mine >= 0) atomicOr(&bits[mine >> 5], 1u << (mine & 31));
    __syncthreads();
    RowSum rest = row_sum();
    for (u32 i = tid * 8u; i < V; i += DIST_BLOCK * 8u) {
        float v[8];
        load8<TY>(p + i, wide, V - i, v);
        const u32 b = ((const unsigned char *)bits)[i >> 3];
#pragma unroll
        for (u32 j = 0; j < 8u; j++)
            if (i + j >= V || (b >> j & 1u)) v[j] = -INFINITY;
        add8(rest, v, c2);
    }
    const double log_out = block_log<WAVES>(rest, inv_T, room);
    // the listed ones, and the teacher's, in fp64: the loss is a small difference of logarithms
    const double t = mine >= 0 ? (double)gptr(c.value)[r * c.k + tid] * inv_T : -INFINITY;
    const double u = mine >= 0 ? (double)Elem<TY>::get(p[mine]) * inv_T : -INFINITY;
    const double tail = c.tail ? (double)gptr(c.tail)[r] : -INFINITY;
    const double mt = fmax(block_max<WAVES>(t, room), tail), ms = fmax(block_max<WAVES>(u, room), log_out);
    const double any = block_sum<WAVES>(mine >= 0 ? 1.0 : 0.0, room);
    const double st = block_sum<WAVES>(t == -INFINITY ? 0.0 : exp(t - mt), room);
    const double ss = block_sum<WAVES>(u == -INFINITY ? 0.0 : exp(u - ms), room);
    const double log_t = mt + log(st + (tail == -INFINITY ? 0.0 : exp(tail - mt)));
    const double log_s = ms + log(ss + (log_out == -INFINITY ? 0.0 : exp(log_out - ms)));
    const bool empty = any == 0.0 || mt == -INFINITY || ms == -INFINITY;
    // sum P (e^d - 1 - d), d = log q - log P: as the listed ones and the rest add up to 1 on both sides, errors of the two
    // logarithms of sums cancel to first order
    double one = 0.0;
    if (mine >= 0 && !empty) {
        const double lp = t - log_t, d = (u - log_s) - lp;
        one = t == -INFINITY ? exp(u - log_s) : exp(lp) * (expm1(d) - d);
    }
    double all = block_sum<WAVES>(one, room);
    if (tid == 0) {
        double over = 0.0;
        if (!empty) {
            const double lp = tail - log_t, lq = log_out - log_s;
            all += tail == -INFINITY ? exp(lq) : exp(lp) * (expm1(lq - lp) - (lq - lp));
            if (log_out != -INFINITY) over = tail == -INFINITY ? exp(lq) : lp > lq ? exp(lp) * expm1(lq - lp) : -exp(lq) * expm1(lp - lq);
        }
        gptr(loss)[r] = empty ? 0.0f : (float)all;
        if (saved) {
            gptr(saved)[r * SAVED + 0] = empty ? INFINITY : log_s;
            gptr(saved)[r * SAVED + 1] = log_out == -INFINITY ? 0.0 : log_out;
            gptr(saved)[r * SAVED + 2] = log_t;
            gptr(saved)[r * SAVED + 3] = over;
        }
    }
}

template <u32 TY>
__global__ __launch_bounds__(DIST_BLOCK) void k_distill_grad(LogitsCall c, const double *__restrict__ saved, const float *__restrict__ g, Mat grad)
{
    typedef typename Elem<TY>::type T;
    __shared__ int idx[MAX_LISTED];
    const u64 r = blockIdx.x;
    const auto *p = row_of<TY>(c.logits, r);
    GLOBAL_AS T *out = (GLOBAL_AS T *)grad.p + r * grad.stride;
    const bool wide = (((u64)p | (u64)out) & 15u) == 0u;
    const u32 V = c.n_vocab, tid = threadIdx.x;
    const double inv_T = 1.0 / (double)c.temperature;
    const double log_s = gptr(saved)[r * SAVED + 0];
    const bool empty = log_s == INFINITY;
    const double up = (g ? (double)gptr(g)[r] : 1.0) * inv_T;
    const int mine = listed_entry(c, r, idx);
    float at_mine = 0.0f;
    if (mine >= 0 && !empty) {
        const double t = (double)gptr(c.value)[r * c.k + tid] * inv_T;
        const double u = (double)Elem<TY>::get(p[mine]) * inv_T;
        at_mine = (float)(up * (exp(u - log_s) - exp(t - gptr(saved)[r * SAVED + 2])));
    }
    __syncthreads(); // (the gradient may take the logits' place)
    const float f = empty ? 0.0f : (float)(up * gptr(saved)[r * SAVED + 3]);
    // e^(z / T - log_out) = 2^(z c - l), c and l in two parts each
    const double c64 = LOG2E * inv_T, l64 = empty ? 0.0 : gptr(saved)[r * SAVED + 1] * LOG2E;
    const float ch = (float)c64, cl = (float)(c64 - (double)ch), lh = (float)l64, ll = (float)(l64 - (double)lh);
    for (u32 i = tid * 8u; i < V; i += DIST_BLOCK * 8u) {
        float v[8];
        load8<TY>(p + i, wide, V - i, v);
#pragma unroll
        for (int j = 0; j < 8; j++) v[j] = empty || v[j] == -INFINITY ? 0.0f : f * pow2(fmaf(v[j], ch, -lh) + fmaf(v[j], cl, -ll));
        if (wide && V - i >= 8u) {
            union {
                u4_16 q[sizeof(T) / 2];
                T e[8];
            } x;
#pragma unroll
            for (int j = 0; j < 8; j++) x.e[j] = Elem<TY>::put(v[j]);
#pragma unroll
            for (u32 j = 0; j < sizeof(T) / 2; j++) ((GLOBAL_AS u4_16 *)(out + i))[j] = x.q[j];
        } else {
#pragma unroll
            for (u32 j = 0; j < 8u; j++)
                if (i + j < V) out[i + j] = Elem<TY>::put(v[j]);
        }
    }
    __syncthreads();
    if (mine >= 0) out[mine] = Elem<TY>::put(at_mine);
}

// ------------------------------------------------------------------------------------------
// calls
// ------------------------------------------------------------------------------------------
hipError_t launch_top_logits(const LogitsCall &c, int *index, float *value, float *tail, hipStream_t s)
{
    const u32 grid = (u32)c.rows;
    switch (c.type) {
    case TY_F32: PROF("k_top_logits", s, k_top_logits<TY_F32><<<grid, TOP_BLOCK, 0, s>>>(c, index, value, tail)); break;
    case TY_BF16: PROF("k_top_logits", s, k_top_logits<TY_BF16><<<grid, TOP_BLOCK, 0, s>>>(c, index, value, tail)); break;
    default: PROF("k_top_logits", s, k_top_logits<TY_F16><<<grid, TOP_BLOCK, 0, s>>>(c, index, value, tail)); break;
    }
    return hipGetLastError();
}
hipError_t launch_distill(const LogitsCall &c, float *loss, double *saved, hipStream_t s)
{
    const u32 grid = (u32)c.rows, lds = (c.n_vocab + 31u) / 32u * 4u;
    switch (c.type) {
    case TY_F32: PROF("k_distill", s, k_distill<TY_F32><<<grid, DIST_BLOCK, lds, s>>>(c, loss, saved)); break;
    case TY_BF16: PROF("k_distill", s, k_distill<TY_BF16><<<grid, DIST_BLOCK, lds, s>>>(c, loss, saved)); break;
    default: PROF("k_distill", s, k_distill<TY_F16><<<grid, DIST_BLOCK, lds, s>>>(c, loss, saved)); break;
    }
    return hipGetLastError();
}
hipError_t launch_distill_grad(const LogitsCall &c, const double *saved, const float *g, const Mat &grad, hipStream_t s)
{
    const u32 grid = (u32)c.rows;
    switch (c.type) {
    case TY_F32: PROF("k_distill_grad", s, k_distill_grad<TY_F32><<<grid, DIST_BLOCK, 0, s>>>(c, saved, g, grad)); break;
    case TY_BF16: PROF("k_distill_grad", s, k_distill_grad<TY_BF16><<<grid, DIST_BLOCK, 0, s>>>(c, saved, g, grad)); break;
    default: PROF("k_distill_grad", s, k_distill_grad<TY_F16><<<grid, DIST_BLOCK, 0, s>>>(c, saved, g, grad)); break;
    }
    return hipGetLastError();
}

} // namespace inshr
