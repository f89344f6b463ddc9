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
// the largest of eight, NaN if one is
__device__ __forceinline__ float largest(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float largest8(const float (&v)[8])
{
    return largest(largest(largest(largest(v[0], v[1]), v[2]), largest(largest(v[3], v[4]), v[5])), largest(v[6], v[7]));
}
// eight more values, m8 the largest; the ones that do not count are -inf.  c: log2 e / T
__device__ __forceinline__ void add8(RowSum &a, const float (&v)[8], float m8, float c)
{
    if (m8 > a.m) {
        a.s *= pow2((a.m - m8) * c);
        a.m = m8;
    } else if (a.m == -INFINITY) { // (nothing yet, or a NaN, which the sum then keeps)
        if (m8 != m8) a.s = m8;
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; i++) a.s += pow2((v[i] - a.m) * c);
}
// `n` more of one value
__device__ __forceinline__ void add_equal(RowSum &a, float x, float n, float c)
{
    if (x > a.m) {
        a.s = a.s * pow2((a.m - x) * c) + n;
        a.m = x;
    } else if (a.m != -INFINITY) {
        a.s += n * pow2((x - a.m) * c);
    }
}
__device__ __forceinline__ void add1(RowSum &a, float x, float c) { add_equal(a, x, 1.0f, c); }

// A row in steps of eight elements a thread: work(first element, the eight, number of them there) for all of them, four
// steps asked for at a time.  Steps that are there for every thread are worked on without a look at the row's end.
template <u32 TY, u32 BLOCK, class F>
__device__ __forceinline__ void each_step(const GLOBAL_AS typename Elem<TY>::type *p, u32 n, F work)
{
    constexpr u32 STEP = BLOCK * 8u;
    const u32 mine = threadIdx.x * 8u;
    u32 i0 = 0u;
    for (; i0 + 4u * STEP <= n; i0 += 4u * STEP) {
        Raw8<TY> x[4];
#pragma unroll
        for (u32 j = 0; j < 4u; j++) x[j] = load_raw8<TY>(p + i0 + j * STEP + mine, 8u);
#pragma unroll
        for (u32 j = 0; j < 4u; j++) work(i0 + j * STEP + mine, x[j], 8u, j);
    }
    if (i0 < n) {
        Raw8<TY> x[4];
#pragma unroll
        for (u32 j = 0; j < 4u; j++) {
            const u32 i = i0 + j * STEP + mine;
            x[j] = load_raw8<TY>(p + i, i < n ? n - i : 0u);
        }
#pragma unroll
        for (u32 j = 0; j < 4u; j++) {
            const u32 i = i0 + j * STEP + mine;
            if (i < n) work(i, x[j], min(n - i, 8u), j);
        }
    }
}

__device__ __forceinline__ double wave_sum(double v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ u32 wave_sum_u(u32 v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    return v;
}
__device__ __forceinline__ u32 wave_min_u(u32 v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v = min(v, __shfl_xor(v, d));
    return v;
}
__device__ __forceinline__ double wave_max(double v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v = fmax(v, __shfl_xor(v, d));
    return v;
}
// What the threads' sums are together, for every wave to join from `room` (a place per wave) after a barrier.
__device__ __forceinline__ void put_sum(const RowSum &a, double c, double2 *room)
{
    float m = a.m;
#pragma unroll
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    double s = a.m == m && a.s == a.s ? (double)a.s : a.s > 0.0f ? (double)a.s * exp2(((double)a.m - (double)m) * c) : a.s != a.s ? (double)a.s : 0.0;
    s = wave_sum(s);
    if ((threadIdx.x & 63u) == 0u) room[threadIdx.x >> 6] = make_double2((double)m, s);
}
// The whole sum: the largest logit (x) and the sum of e^((logit - x) / T) (y), 0 where nothing counts, NaN where one is NaN
// or +inf; by all lanes of a wave.
template <int WAVES>
__device__ __forceinline__ double2 joined_sum(const double2 *room, double inv_T)
{
    const u32 lane = threadIdx.x & 63u;
    double2 v = make_double2(-INFINITY, 0.0);
    if (lane < (u32)WAVES) v = room[lane];
    double m = v.x;
#pragma unroll
    for (int d = 8; d; d >>= 1) m = fmax(m, __shfl_xor(m, d)); // (up to 16 waves)
    double s = v.y > 0.0 ? v.y * exp((v.x - m) * inv_T) : v.y;
#pragma unroll
    for (int d = 8; d; d >>= 1) s += __shfl_xor(s, d);
    return make_double2(__shfl(m, 0), __shfl(s, 0));
}

template <u32 TY>
__device__ __forceinline__ const GLOBAL_AS typename Elem<TY>::type *row_of(const Mat &m, u64 r)
{
    return (const GLOBAL_AS typename Elem<TY>::type *)m.p + r * m.stride;
}

// ------------------------------------------------------------------------------------------
// the largest logits
// ------------------------------------------------------------------------------------------
constexpr u32 TOP_ROOM = 2048; // candidates
// a thread keeps the largest of as many parts of its elements: every fourth step, or in a row of one step two elements each
constexpr int TOP_MAXIMA = 4;

__device__ __forceinline__ u32 logit_key(float x) { return x != x ? 0xFFFFFFFFu : key_of_float(x); }
__device__ __forceinline__ float logit_of(u32 key) { return __uint_as_float(bits_of_key(key)); }
constexpr u32 KEY_OF_NONE = 0x007FFFFFu; // of -inf: the least of all

// A number that at least k of the wave's keys are not below: the k-th largest, cut to its upper 20 bits.
__device__ __forceinline__ u32 wave_kth(const u32 (&m)[TOP_MAXIMA], u32 k)
{
    u32 t = 0u;
    for (int b = 31; b >= 12; b--) {
        const u32 c = t | 1u << b;
        u32 n = 0u;
#pragma unroll
        for (int i = 0; i < TOP_MAXIMA; i++) n += (u32)__popcll(__ballot(m[i] >= c));
        if (n >= k) t = c;
    }
    return t;
}

// The same of the workgroup's keys, for rows whose elements lie in a few waves (the others are masked, or the row is short).
template <int WAVES>
__device__ __forceinline__ u32 group_kth(const u32 (&m)[TOP_MAXIMA], u32 k, u32 (&counts)[2][WAVES])
{
    u32 t = 0u;
    for (int b = 31; b >= 12; b--) {
        const u32 c = t | 1u << b;
        u32 n = 0u;
#pragma unroll
        for (int i = 0; i < TOP_MAXIMA; i++) n += (u32)__popcll(__ballot(m[i] >= c));
        if ((threadIdx.x & 63u) == 0u) counts[b & 1][threadIdx.x >> 6] = n;
        __syncthreads(); // (the step after the next writes here again, and waits for this one's readers in between)
        n = 0u;
#pragma unroll
        for (int w = 0; w < WAVES; w++) n += counts[b & 1][w];
        if (n >= k) t = c;
    }
    return t;
}

template <class T>
__device__ __forceinline__ void sort_descending(T *v, u32 n) // n: a power of two
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

// The k largest in three steps.  Every wave finds a number that ceil(k / waves) of the largest keys its threads have
// seen are not below; at least k elements of the row are not below the smallest of these (about 1.2 k for logits in no
// particular order).  Where a wave has seen too few that are allowed, or its share is half of its threads in a short row, the
// waves look for a number together, with 20 barriers (without it all of a row was candidates: 1000 rows of 1000 bf16, k = 64,
// 33 -> 14 us, 100 rows of 8192 with the last eighth masked 82 -> 15; where it is not needed it costs 1 to 2 us).  A second reading of the row picks them out and adds the others up.  Each candidate's place is the
// number of larger ones.
// Bound by vector instructions: 4096 rows of 32000 bf16, k = 64, 93 us (two readings of 262 MB each, 5.6 TB/s); one row of 50257 fp32
// 14.3 us, read by one workgroup.  Keeping the row in registers for the second reading took longer (95 -> 102 us), and
// so did a bound from a part of the row (92 -> 102).
template <u32 TY, u32 BLOCK>
__global__ __launch_bounds__(BLOCK) void k_top_logits(LogitsCall c, int *__restrict__ index, float *__restrict__ value, float *__restrict__ tail)
{
    constexpr int WAVES = BLOCK / 64;
    __shared__ u64 cand[TOP_ROOM];
    __shared__ u32 low[WAVES], counts[2][WAVES];
    __shared__ double2 room[WAVES];
    __shared__ u32 n_cand, count;
    const u64 r = blockIdx.x;
    const auto *p = row_of<TY>(c.logits, r);
    const u32 V = c.n_vocab, k = c.k, tid = threadIdx.x;
    const double inv_T = 1.0 / (double)c.temperature;
    const float c2 = (float)(LOG2E * inv_T);

    float high[TOP_MAXIMA] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    if (V <= BLOCK * 8u) {
        const u32 left = V - min(tid * 8u, V);
        const Raw8<TY> x = load_raw8<TY>(p + tid * 8u, left);
#pragma unroll
        for (u32 q = 0; q < 8u; q++)
            if (q < left) high[q / 2u] = largest(high[q / 2u], x[q]);
    } else {
        each_step<TY, BLOCK>(p, V, [&](u32, const Raw8<TY> &x, u32 there, u32 j) {
            float v[8];
#pragma unroll
            for (u32 q = 0; q < 8u; q++) v[q] = q < there ? x[q] : -INFINITY;
            high[j] = largest(high[j], largest8(v));
        });
    }
    u32 top[TOP_MAXIMA];
#pragma unroll
    for (int j = 0; j < TOP_MAXIMA; j++) top[j] = logit_key(high[j]);
    const u32 share = (k + WAVES - 1u) / WAVES, mine = wave_kth(top, share);
    if ((tid & 63u) == 0u) low[tid >> 6] = mine;
    if (tid == 0) n_cand = 0u;
    __syncthreads();
    u32 thr = low[0];
#pragma unroll
    for (int w = 1; w < WAVES; w++) thr = min(thr, low[w]);

    if (thr <= KEY_OF_NONE || (share >= 32u && V <= BLOCK * 16u)) thr = group_kth<WAVES>(top, k, counts);
    if (thr <= KEY_OF_NONE) thr = KEY_OF_NONE + 1u; // (all that is allowed, which may be fewer than k)
    const float bound = logit_of(thr); // (NaN where the keys that were cut off it are those of NaN)
    RowSum rest = row_sum();
    u32 least = ~0u;  // of the candidates' keys
    bool odd = false; // NaN or +inf
    each_step<TY, BLOCK>(p, V, [&](u32 i, const Raw8<TY> &x, u32 there, u32) {
        float v[8];
#pragma unroll
        for (u32 q = 0; q < 8u; q++) v[q] = q < there ? x[q] : -INFINITY;
        float m8 = largest8(v);
        if (!(m8 < bound)) {
#pragma unroll
            for (u32 q = 0; q < 8u; q++)
                if (!(v[q] < bound) && q < there) {
                    odd = odd || !(v[q] < INFINITY);
                    const u32 at = atomicAdd(&n_cand, 1u), key = logit_key(v[q]);
                    if (at < TOP_ROOM) cand[at] = (u64)key << 32 | (u32)~(i + q);
                    least = min(least, key);
                    v[q] = -INFINITY;
                }
            m8 = largest8(v);
        }
        add8(rest, v, m8, c2);
    });
    odd = __syncthreads_or(odd ? 1 : 0) != 0;
    u32 n = n_cand;
    if (n > TOP_ROOM || n < k) {
        // Too few: the first of those that are not allowed.  Too many, mostly equal ones (masked by a finite value): the key of
        // rank k, the larger ones, and the first of the equal ones.  The first try is whether fewer than k lie above the least
        // candidate, as in such a row; then by halving.
        u32 lo = KEY_OF_NONE;
        if (n > TOP_ROOM) {
            if (tid == 0) count = ~0u;
            __syncthreads();
            least = wave_min_u(least);
            if ((tid & 63u) == 0u) atomicMin(&count, least);
            __syncthreads();
            lo = count;
            u32 hi = 0xFFFFFFFFu, there_are = n; // not below lo, at least k
            for (bool first = true; lo < hi; first = false) {
                const u32 mid = first ? lo + 1u : lo + (hi - lo) / 2u + 1u;
                __syncthreads();
                if (tid == 0) count = 0u;
                __syncthreads();
                u32 have = 0u;
                each_step<TY, BLOCK>(p, V, [&](u32, const Raw8<TY> &x, u32 there, u32) {
#pragma unroll
                    for (u32 q = 0; q < 8u; q++) have += q < there && logit_key(x[q]) >= mid ? 1u : 0u;
                });
                have = wave_sum_u(have);
                if ((tid & 63u) == 0u) atomicAdd(&count, have);
                __syncthreads();
                if (count >= k) {
                    lo = mid;
                    there_are = count;
                } else {
                    hi = mid - 1u;
                }
            }
            __syncthreads();
            if (tid == 0) n_cand = 0u;
            __syncthreads();
            rest = row_sum();
            const float equal_to = logit_of(lo);
            each_step<TY, BLOCK>(p, V, [&](u32 i, const Raw8<TY> &x, u32 there, u32) {
                float v[8];
#pragma unroll
                for (u32 q = 0; q < 8u; q++) v[q] = q < there ? x[q] : -INFINITY;
                float m8 = largest8(v);
                if (!(m8 < equal_to)) {
#pragma unroll
                    for (u32 q = 0; q < 8u; q++) {
                        const u32 key = logit_key(v[q]);
                        if (key < lo || q >= there) continue;
                        if (key > lo) cand[atomicAdd(&n_cand, 1u)] = (u64)key << 32 | (u32)~(i + q); // (fewer than k)
                        v[q] = -INFINITY;
                    }
                    m8 = largest8(v);
                }
                add8(rest, v, m8, c2);
            });
            if (tid == 0 && there_are > k) add_equal(rest, equal_to, (float)(there_are - k), c2);
            __syncthreads();
            n = n_cand;
        }
        u32 equal = 0u; // equal ones before this step of the row, the same in all threads
        for (u32 i0 = 0; i0 < V && n + equal < k; i0 += BLOCK) {
            const u32 i = i0 + tid;
            const bool is = i < V && logit_key(Elem<TY>::get(p[i])) == lo;
            const u64 mask = __ballot(is);
            __syncthreads();
            if ((tid & 63u) == 0u) counts[0][tid >> 6] = (u32)__popcll(mask);
            __syncthreads();
            u32 before = equal;
            for (int w = 0; w < WAVES; w++) {
                if (w < (int)(tid >> 6)) before += counts[0][w];
                equal += counts[0][w];
            }
            const u32 at = n + before + (u32)__popcll(mask & ((1ull << (tid & 63u)) - 1ull));
            if (is && at < k) cand[at] = (u64)lo << 32 | (u32)~i;
        }
        __syncthreads();
        n = k;
    }
    if (n > BLOCK) { // (a place for every thread's candidate: the largest ones first)
        u32 size = 2u;
        while (size < n) size <<= 1;
        for (u32 i = n + tid; i < size; i += BLOCK) cand[i] = 0ull;
        sort_descending(cand, size);
        for (u32 i = k + tid; i < n; i += BLOCK) add1(rest, logit_of((u32)(cand[i] >> 32)), c2);
        n = k;
    }
    // (candidates stand in the order in which they were found, which is another one every time: those that are not listed
    // are added up in the order of their places)
    __shared__ float late[BLOCK];
    if (tid < n) {
        const u64 own = cand[tid];
        u32 place = 0u;
#pragma unroll 8
        for (u32 i = 0; i < n; i++) place += cand[i] > own ? 1u : 0u;
        const u32 at = (u32)~(u32)own;
        if (place < k) {
            gptr(index)[r * k + place] = (int)at;
            gptr(value)[r * k + place] = Elem<TY>::get(p[at]); // (of the two zeros the one that is there)
        } else {
            late[place] = logit_of((u32)(own >> 32));
        }
    }
    if (tail) {
        __syncthreads();
        if (tid >= k && tid < n) add1(rest, late[tid], c2);
        put_sum(rest, LOG2E * inv_T, room);
        __syncthreads();
        if (tid >= 64u) return;
        const double2 l = joined_sum<WAVES>(room, inv_T);
        if (tid == 0) gptr(tail)[r] = odd || l.y != l.y ? __uint_as_float(0x7fc00000u) : l.y > 0.0 ? (float)(l.x * inv_T + log(l.y)) : -INFINITY;
    }
}

// ------------------------------------------------------------------------------------------
// the loss
// ------------------------------------------------------------------------------------------
static_assert(MAX_LISTED <= 256, "a thread per listed entry");
// Logarithms of sums are held as the largest member and the logarithm of what the sum is relative to it: added up, a
// logit / T of 2^53 takes all digits of the second (a row masked by the type's lowest value throughout).  Saved per row:
//   0  the student's second part; +inf for a row whose loss is 0 by definition, NaN for a row with NaN or +inf
//   1  two floats: the student's largest logit, the largest of those that are not listed (0 where there are none)
//   2  the teacher's second part, -0.0 or less where its largest member is the tail (as they are not below 0)
//   3  two floats: the teacher's largest member, a listed logit or the tail; and what the gradient of an unlisted logit is
//      of e^((logit - largest) / T): q_rest - P_tail, divided by the sum of these (by 1 where q_rest is so small that fp64 has
//      no digits of the sum in its logarithm: unlisted logits 2^53 T below the listed ones)
constexpr int SAVED = 4;
__device__ __forceinline__ double two_floats(float a, float b) { return __longlong_as_double((long long)((u64)__float_as_uint(a) << 32 | __float_as_uint(b))); }
__device__ __forceinline__ float first_float(double v) { return __uint_as_float((u32)((u64)__double_as_longlong(v) >> 32)); }
__device__ __forceinline__ float second_float(double v) { return __uint_as_float((u32)(u64)__double_as_longlong(v)); }

// Entry j of the row's list into idx[j], -1 for an index outside the vocabulary; idx has room for MAX_LISTED and is -1
// past the list.  A barrier has to follow.
__device__ __forceinline__ void read_list(const LogitsCall &c, u64 r, int *idx)
{
    for (u32 j = threadIdx.x; j < MAX_LISTED; j += blockDim.x) {
        const int i = j < c.k ? gptr(c.index)[r * c.k + j] : -1;
        idx[j] = (u32)i < c.n_vocab ? i : -1;
    }
}
// Entry j, or -1 where its index stands earlier in the list.
__device__ __forceinline__ int first_of(const int *idx, u32 j)
{
    const int i = idx[j];
    const int4 *four = (const int4 *)idx;
    bool again = false;
    for (u32 q = 0; 4u * q < j; q++) {
        const int4 v = four[q];
        again = again || v.x == i || (v.y == i && 4u * q + 1u < j) || (v.z == i && 4u * q + 2u < j) || (v.w == i && 4u * q + 3u < j);
    }
    return again ? -1 : i;
}

// P (e^d - 1 - d), d = log q - log P, of the logarithms.  Past d = 1 nothing cancels, and e^d may leave fp64 where P e^d = q
// does not; a P that is 0 in fp64 counts as 0.
__device__ __forceinline__ double divergence(double lp, double lq)
{
    const double p = exp(lp), d = lq - lp;
    if (d > 1.0) return exp(lq) - (p == 0.0 ? 0.0 : p * (1.0 + d));
    return p == 0.0 ? 0.0 : p * (expm1(d) - d);
}

// A listed logit of the teacher's / T and its tail, relative to the largest member of its sum.  (Of equal logits the difference
// is 0: taken before it is divided, as the compiler may leave a product unrounded before a subtraction.)
struct Teacher {
    double high, tail, inv_T; // the largest listed logit, the tail
    bool by_tail;             // the tail is the largest
    __device__ __forceinline__ double listed(double value) const { return by_tail ? value * inv_T - tail : (value - high) * inv_T; }
    __device__ __forceinline__ double rest() const { return by_tail ? 0.0 : tail - high * inv_T; }
};

// One reading of the row, the first wave ends it: 64 lanes with up to four listed entries each, in fp64.  4096 rows of 50257
// bf16, 64 listed: 135 us behind a gradient that has written 412 MB (3.1 TB/s; an exponential and five other vector instructions
// a logit beside the reading), 86 when the same rows have just been read (the last-level cache has part of them).
template <u32 TY, u32 BLOCK>
__global__ __launch_bounds__(BLOCK) void k_distill(LogitsCall c, float *__restrict__ loss, double *__restrict__ saved)
{
    constexpr int WAVES = BLOCK / 64;
    extern __shared__ u32 bits[]; // which logits are listed
    __shared__ __attribute__((aligned(16))) int idx[MAX_LISTED];
    __shared__ double2 room[WAVES];
    const u64 r = blockIdx.x;
    const auto *p = row_of<TY>(c.logits, r);
    const u32 V = c.n_vocab, tid = threadIdx.x;
    const double inv_T = 1.0 / (double)c.temperature;
    const float c2 = (float)(LOG2E * inv_T);
    for (u32 i = tid; i < (V + 31u) / 32u; i += BLOCK) bits[i] = 0u;
    read_list(c, r, idx);
    __syncthreads();
    if (tid < c.k && idx[tid] >= 0) atomicOr(&bits[idx[tid] >> 5], 1u << (idx[tid] & 31));
    __syncthreads();
    RowSum rest = row_sum();
    each_step<TY, BLOCK>(p, V, [&](u32 i, const Raw8<TY> &x, u32 there, u32) {
        const u32 b = ((const unsigned char *)bits)[i >> 3];
        float v[8];
#pragma unroll
        for (u32 q = 0; q < 8u; q++) v[q] = q < there ? x[q] : -INFINITY;
        if (b) {
#pragma unroll
            for (u32 q = 0; q < 8u; q++)
                if (b >> q & 1u) v[q] = -INFINITY;
        }
        add8(rest, v, largest8(v), c2);
    });
    put_sum(rest, LOG2E * inv_T, room);
    __syncthreads();
    if (tid >= 64u) return;
    // the listed ones, and the teacher's, in fp64: the loss is a small difference of logarithms
    double t[4], u[4], high = -INFINITY, ms = -INFINITY;
    const double tail = c.tail ? (double)gptr(c.tail)[r] : -INFINITY;
    // what there is (NaN is there too: the maxima below pass it over)
    bool any = false, taught = tail != -INFINITY, student = false, odd = !(tail < INFINITY);
#pragma unroll
    for (u32 q = 0; q < 4u; q++) {
        t[q] = u[q] = -INFINITY;
        if (64u * q >= c.k) continue; // (the same for all lanes)
        const int i = first_of(idx, tid + 64u * q);
        if (i < 0) continue;
        any = true;
        t[q] = (double)gptr(c.value)[r * c.k + tid + 64u * q];
        u[q] = (double)Elem<TY>::get(p[i]);
        high = fmax(high, t[q]);
        ms = fmax(ms, u[q]);
        taught = taught || t[q] != -INFINITY;
        student = student || u[q] != -INFINITY;
        odd = odd || !(t[q] < INFINITY) || !(u[q] < INFINITY);
    }
    const double2 out = joined_sum<WAVES>(room, inv_T);
    const bool untaught = __ballot(any) == 0 || __ballot(taught) == 0;
    odd = !untaught && __ballot(odd || out.y != out.y) != 0;
    const bool empty = untaught || (!odd && __ballot(student || out.y > 0.0) == 0);
    high = wave_max(high);
    const Teacher teacher = {high, tail, inv_T, !(tail <= high * inv_T)};
    ms = fmax(wave_max(ms), out.x);
    double st = 0.0, ss = 0.0;
#pragma unroll
    for (u32 q = 0; q < 4u; q++) {
        if (64u * q >= c.k) continue;
        if (t[q] != -INFINITY) st += exp(teacher.listed(t[q]));
        if (u[q] != -INFINITY) ss += exp((u[q] - ms) * inv_T);
    }
    st = wave_sum(st);
    ss = wave_sum(ss);
    const double lt = log(st + (tail == -INFINITY ? 0.0 : exp(teacher.rest())));
    const double ls = log(ss + (out.y > 0.0 ? out.y * exp((out.x - ms) * inv_T) : 0.0));
    // the sum of the divergences: as the listed ones and the rest add up to 1 on both sides, errors of the two
    // logarithms of sums cancel to first order
    double all = 0.0;
#pragma unroll
    for (u32 q = 0; q < 4u; q++) {
        if (64u * q >= c.k || empty) continue;
        if (t[q] != -INFINITY)
            all += divergence(teacher.listed(t[q]) - lt, (u[q] - ms) * inv_T - ls);
        else if (u[q] != -INFINITY)
            all += exp((u[q] - ms) * inv_T - ls);
    }
    all = wave_sum(all);
    if (tid == 0) {
        double over = 0.0;
        if (!empty) {
            const double lp = teacher.rest() - lt, one = (out.x - ms) * inv_T - ls, lq = out.y > 0.0 ? one + log(out.y) : -INFINITY;
            all += tail == -INFINITY ? exp(lq) : divergence(lp, lq);
            if (out.y > 0.0) {
                over = tail == -INFINITY ? exp(lq) : lp > lq ? exp(lp) * expm1(lq - lp) : -exp(lq) * expm1(lp - lq);
                over *= exp(one - lq); // (1 / out.y, or 1 where lq has no digits for it)
            }
        }
        gptr(loss)[r] = empty ? 0.0f : odd ? __uint_as_float(0x7fc00000u) : (float)all;
        if (saved) {
            GLOBAL_AS double *to = gptr(saved) + r * SAVED;
            to[0] = empty ? INFINITY : odd ? NAN : ls;
            to[1] = two_floats((float)ms, out.y > 0.0 ? (float)out.x : 0.0f);
            to[2] = copysign(lt, teacher.by_tail ? -1.0 : 1.0);
            to[3] = two_floats((float)(teacher.by_tail ? tail : high), (float)over);
        }
    }
}

// A reading and a writing of the row: 4096 rows of 50257 bf16 in 167 us (4.9 TB/s, more than a plain copy of the library reaches).
template <u32 TY, u32 BLOCK>
__global__ __launch_bounds__(BLOCK) void k_distill_grad(LogitsCall c, const double *__restrict__ saved, const float *__restrict__ g, Mat grad)
{
    typedef typename Elem<TY>::type T;
    __shared__ __attribute__((aligned(16))) int idx[MAX_LISTED];
    const u64 r = blockIdx.x;
    const auto *p = row_of<TY>(c.logits, r);
    GLOBAL_AS T *out = (GLOBAL_AS T *)grad.p + r * grad.stride;
    const u32 V = c.n_vocab, tid = threadIdx.x;
    const double inv_T = 1.0 / (double)c.temperature;
    const GLOBAL_AS double *kept = gptr(saved) + r * SAVED;
    const double ls = kept[0], lt = kept[2];
    const bool empty = ls == INFINITY, odd = ls != ls;
    const double up = (g ? (double)gptr(g)[r] : 1.0) * inv_T;
    read_list(c, r, idx);
    __syncthreads();
    const int mine = tid < c.k ? first_of(idx, tid) : -1;
    float at_mine = 0.0f;
    if (mine >= 0 && !empty) {
        const double most = (double)first_float(kept[3]);
        const Teacher teacher = {most, most, inv_T, (bool)signbit(lt)};
        const double t = teacher.listed((double)gptr(c.value)[r * c.k + tid]);
        const double u = ((double)Elem<TY>::get(p[mine]) - (double)first_float(kept[1])) * inv_T;
        at_mine = (float)(up * (exp(u - ls) - exp(t - fabs(lt))));
    }
    __syncthreads(); // (the gradient may take the logits' place)
    const float none = odd ? __uint_as_float(0x7fc00000u) : 0.0f; // of a logit that is -inf
    const float f = empty || odd ? none : (float)(up * (double)second_float(kept[3]));
    const double c64 = LOG2E * inv_T, m = empty ? 0.0 : (double)second_float(kept[1]), l64 = m * c64;
    const float ch = (float)c64, cl = (float)(c64 - (double)ch);
    // The steps begin where the results' lines of 128 bytes begin; an element of a step is read before it is written.
    auto row = [&](auto share) {
        auto slope = [&](float x) {
            const float s = f * share(x);
            return empty || x == -INFINITY ? none : s;
        };
        const u32 head = min((u32)((0ull - (u64)out) & 127ull) / (u32)sizeof(T), V);
        if (tid < head) out[tid] = Elem<TY>::put(slope(Elem<TY>::get(p[tid])));
        each_step<TY, BLOCK>(p + head, V - head, [&](u32 i, const Raw8<TY> &x, u32 there, u32) {
            float v[8];
#pragma unroll
            for (int q = 0; q < 8; q++) v[q] = slope(x[q]);
            store8<TY>(out + head + i, there, v);
        });
    };
    // e^((z - m) / T) = 2^(z c - l), l = m c, c and l in two parts each; where l has too many digits before the point, or z c may leave
    // fp32, 2^((z - m) c), with z - m rounded, and what is less than 2^-300 taken for that, so that no term is infinite
    if (fabs(l64) < 1048576.0 && c64 < 1048576.0) {
        const float lh = (float)l64, ll = (float)(l64 - (double)lh);
        row([&](float x) { return pow2(fmaf(x, ch, -lh) + fmaf(x, cl, -ll)); });
    } else {
        const float mf = (float)m, least = -(float)fmin(300.0 / c64, 3.4e38);
        row([&](float x) {
            const float d = fmaxf(x - mf, least);
            return pow2(fmaf(d, ch, d * cl));
        });
    }
    __syncthreads();
    if (mine >= 0) out[mine] = Elem<TY>::put(at_mine);
}

// ------------------------------------------------------------------------------------------
// calls
// ------------------------------------------------------------------------------------------
namespace {

// A workgroup per row: 256 threads where the rows fill the chip (eight workgroups a CU), 1024 where there are few, each of
// which is then read in fewer steps.  256 threads / 1024, in us:
//   k_top_logits, one workgroup of 1024 a CU, two of which would take turns   256 rows of 50257 bf16 22.5/19.8, fp32 26.8/25.9, of
//       131072 bf16 38/30; 384 rows of 20000 fp32 16.6/24.8, of 50257 bf16 26.8/33.0
//   loss and gradient, two a CU   384 rows of 50257 bf16 37.1/34.5, fp32 48.5/50.4, of 131072 bf16 68/62; 768 rows of 50257 bf16
//       50.6/54.2, of 20000 fp32 41.8/52.3
constexpr u64 FEW_TOP_ROWS = 257, FEW_LOGIT_ROWS = 512;

template <u32 TY, u32 BLOCK>
void start_top(const LogitsCall &c, int *index, float *value, float *tail, hipStream_t s)
{
    PROF("k_top_logits", s, k_top_logits<TY, BLOCK><<<(u32)c.rows, BLOCK, 0, s>>>(c, index, value, tail));
}
template <u32 TY, u32 BLOCK>
void start_distill(const LogitsCall &c, float *loss, double *saved, hipStream_t s)
{
    PROF("k_distill", s, k_distill<TY, BLOCK><<<(u32)c.rows, BLOCK, (c.n_vocab + 31u) / 32u * 4u, s>>>(c, loss, saved));
}
template <u32 TY, u32 BLOCK>
void start_grad(const LogitsCall &c, const double *saved, const float *g, const Mat &grad, hipStream_t s)
{
    PROF("k_distill_grad", s, k_distill_grad<TY, BLOCK><<<(u32)c.rows, BLOCK, 0, s>>>(c, saved, g, grad));
}

} // namespace

hipError_t launch_top_logits(const LogitsCall &c, int *index, float *value, float *tail, hipStream_t s)
{
    // (k of 1024 threads' maxima: every wave has to have seen k / 16 elements' worth of them)
    const bool few = c.rows < FEW_TOP_ROWS && c.n_vocab >= 8192u;
    switch (c.type) {
    case TY_F32: few ? start_top<TY_F32, 1024>(c, index, value, tail, s) : start_top<TY_F32, 256>(c, index, value, tail, s); break;
    case TY_BF16: few ? start_top<TY_BF16, 1024>(c, index, value, tail, s) : start_top<TY_BF16, 256>(c, index, value, tail, s); break;
    default: few ? start_top<TY_F16, 1024>(c, index, value, tail, s) : start_top<TY_F16, 256>(c, index, value, tail, s); break;
    }
    return hipGetLastError();
}
hipError_t launch_distill(const LogitsCall &c, float *loss, double *saved, hipStream_t s)
{
    const bool few = c.rows < FEW_LOGIT_ROWS;
    switch (c.type) {
    case TY_F32: few ? start_distill<TY_F32, 1024>(c, loss, saved, s) : start_distill<TY_F32, 256>(c, loss, saved, s); break;
    case TY_BF16: few ? start_distill<TY_BF16, 1024>(c, loss, saved, s) : start_distill<TY_BF16, 256>(c, loss, saved, s); break;
    default: few ? start_distill<TY_F16, 1024>(c, loss, saved, s) : start_distill<TY_F16, 256>(c, loss, saved, s); break;
    }
    return hipGetLastError();
}
hipError_t launch_distill_grad(const LogitsCall &c, const double *saved, const float *g, const Mat &grad, hipStream_t s)
{
    const bool few = c.rows < FEW_LOGIT_ROWS;
    switch (c.type) {
    case TY_F32: few ? start_grad<TY_F32, 1024>(c, saved, g, grad, s) : start_grad<TY_F32, 256>(c, saved, g, grad, s); break;
    case TY_BF16: few ? start_grad<TY_BF16, 1024>(c, saved, g, grad, s) : start_grad<TY_BF16, 256>(c, saved, g, grad, s); break;
    default: few ? start_grad<TY_F16, 1024>(c, saved, g, grad, s) : start_grad<TY_F16, 256>(c, saved, g, grad, s); break;
    }
    return hipGetLastError();
}

} // namespace inshr
