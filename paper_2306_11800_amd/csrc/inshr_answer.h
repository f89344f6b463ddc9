// Descriptors of the operators that run layers from their compressed form and compare answers
// (inshr_linear.hip, inshr_logits.hip), and what their kernels share.
#pragma once
#include "inshr_launch.h"

namespace inshr {

// element types of activations and logits; the numbers are those of the C ABI
constexpr u32 TY_F32 = 0u, TY_BF16 = 1u, TY_F16 = 2u;
// activations; the numbers are those of the C ABI
constexpr u32 ACT_NONE = 0u, ACT_RELU = 1u, ACT_GELU = 2u, ACT_GELU_TANH = 3u, ACT_SILU = 4u;

__host__ __device__ inline u64 elem_size(u32 type) { return type == TY_F32 ? 4u : 2u; }

struct WDesc { // a weight as the quantizer left it, row-major [rows][cols]
    const u32 *packed;      // the symbol stream as 32-bit words, n_words of them
    const float *codebook;
    const u32 *out_idx;
    const void *out_val;    // fp32, or bfloat16 where val_bf16 is set
    u64 n_words, n_outlier;
    u32 rows, cols, w, K, val_bf16, pad;
};

struct Mat { // rows of a matrix in the caller's memory
    void *p;
    u64 stride; // elements between rows
};

struct LinearCall {
    WDesc w;
    const float *bias;
    Mat x, residual, y, pre; // p == NULL: not given, not wanted
    u64 rows;
    u32 n_in, n_out, in_out, type, act;
    char *ws;                // workspace, linear_space() bytes
};
struct LinearGradCall {
    WDesc w;
    Mat x, dy, pre, dx;
    float *dw, *db;
    u64 rows;
    u32 n_in, n_out, in_out, type, act;
    char *ws;                // workspace, linear_grad_space() bytes
};
u64 linear_space(u64 rows, u32 n_in, u32 n_out, u32 in_out, u32 type, u32 w, bool listed); // (w: bits of a symbol)
u64 linear_grad_space(u64 rows, u32 n_in, u32 n_out, u32 in_out, u32 type, u32 act, bool dx, bool dw);
hipError_t launch_linear(const LinearCall &c, hipStream_t s);
// Few rows: straight from the stream.  Every block of 32 rows decodes the weight once more, which takes longer for wide symbols
// and for fp32 (three parts, six products) and, of two weights of one size, for the one with more outputs; planes are decoded
// once, and multiplied in two passes for fp16 and three for fp32.  Straight / by planes in us:
//   96 rows  2048 x 2048 fp32 23/31, 4096 x 4096 bf16 of 5 bits 33/35, of 8 bits 50/38, fp32 72/48, 11008 x 4096 fp16 56/87,
//            8192 x 8192 fp16 85/148, 1024 x 11008 bf16 40/32
//   64 rows  8192 x 8192 fp32 98/157, 4096 x 11008 bf16 of 5 bits 53/59, of 8 bits 71/65, fp16 54/84, fp32 109/94,
//            1024 x 50257 bf16 86/61
//   32 rows  1024 x 50257 bf16 52/60, fp32 71/100, 256 x 30000 bf16 26/24
// Weights stored [in][out] have no such way for more than 4 rows (4096 x 11008 bf16: 4 rows 60, 5 by planes 67).
constexpr u32 FEW_ROWS = 96, FEW_SPLIT = 4;
inline bool is_few(u64 rows, u32 n_out, bool in_out, u32 type, u32 w)
{
    const u32 most = type == TY_F32 || w > 7u ? 2048u : type == TY_BF16 ? 4096u : 8192u; // outputs for three blocks
    return rows <= (in_out ? FEW_SPLIT : n_out <= most ? FEW_ROWS : n_out <= 4u * most ? 64u : 32u);
}
u64 few_space(u64 rows, u32 n_in, u32 n_out, bool in_out, u32 type, u32 w, bool listed);
hipError_t launch_few(const LinearCall &c, hipStream_t s);
hipError_t launch_linear_grad(const LinearGradCall &c, hipStream_t s);

constexpr u32 MAX_VOCAB = 1u << 18; // a bit per logit of a row fits into 32 KB of LDS
constexpr u32 MAX_LISTED = 256u;
struct LogitsCall {
    Mat logits;
    u64 rows;
    u32 type, n_vocab, k;
    float temperature;
    const int *index;   // [rows][k]
    const float *value; // [rows][k]
    const float *tail;  // [rows] or NULL
};
hipError_t launch_top_logits(const LogitsCall &c, int *index, float *value, float *tail, hipStream_t s);
hipError_t launch_distill(const LogitsCall &c, float *loss, double *saved, hipStream_t s);
hipError_t launch_distill_grad(const LogitsCall &c, const double *saved, const float *g, const Mat &grad, hipStream_t s);

// ------------------------------------------------------------------------------------------
// elements
// ------------------------------------------------------------------------------------------
template <u32 TY> struct Elem;
template <> struct Elem<TY_F32> {
    typedef float type;
    static __device__ __forceinline__ float get(float v) { return v; }
    static __device__ __forceinline__ float put(float v) { return v; }
};
template <> struct Elem<TY_BF16> {
    typedef u16 type;
    static __device__ __forceinline__ float get(u16 v) { return __uint_as_float((u32)v << 16); }
    static __device__ __forceinline__ u16 put(float v) { return __builtin_bit_cast(u16, (__bf16)v); } // (to nearest even)
};
template <> struct Elem<TY_F16> {
    typedef _Float16 type;
    static __device__ __forceinline__ float get(_Float16 v) { return (float)v; }
    static __device__ __forceinline__ _Float16 put(float v) { return (_Float16)v; }
};

typedef u32 u4_16 __attribute__((ext_vector_type(4)));
// 16 bytes at an address aligned to an element of E bytes: one instruction all the same
template <u32 E> struct Any16;
template <> struct Any16<2> { typedef u32 type __attribute__((ext_vector_type(4), aligned(2))); };
template <> struct Any16<4> { typedef u32 type __attribute__((ext_vector_type(4), aligned(4))); };

// Eight consecutive elements as they lie in memory.
template <u32 TY> union Raw8 {
    typedef typename Elem<TY>::type T;
    u4_16 q[sizeof(T) / 2];
    T e[8];
    __device__ __forceinline__ Raw8() {}
    __device__ __forceinline__ float operator[](int i) const { return Elem<TY>::get(e[i]); }
};
// `left` of them exist, the others read as 0.
template <u32 TY>
__device__ __forceinline__ Raw8<TY> load_raw8(const GLOBAL_AS typename Elem<TY>::type *p, u32 left)
{
    typedef typename Elem<TY>::type T;
    typedef typename Any16<sizeof(T)>::type V;
    Raw8<TY> x;
    if (left >= 8u) {
#pragma unroll
        for (u32 i = 0; i < sizeof(T) / 2; i++) x.q[i] = ((const GLOBAL_AS V *)p)[i];
    } else {
#pragma unroll
        for (u32 i = 0; i < 8u; i++) x.e[i] = i < left ? p[i] : (T)0;
    }
    return x;
}
template <u32 TY>
__device__ __forceinline__ void load8(const GLOBAL_AS typename Elem<TY>::type *p, u32 left, float (&v)[8])
{
    const Raw8<TY> x = load_raw8<TY>(p, left);
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = x[i];
}
template <u32 TY>
__device__ __forceinline__ void store8(GLOBAL_AS typename Elem<TY>::type *p, u32 left, const float (&v)[8])
{
    typedef typename Elem<TY>::type T;
    typedef typename Any16<sizeof(T)>::type V;
    Raw8<TY> x;
#pragma unroll
    for (int i = 0; i < 8; i++) x.e[i] = Elem<TY>::put(v[i]);
    if (left >= 8u) {
#pragma unroll
        for (u32 i = 0; i < sizeof(T) / 2; i++) ((GLOBAL_AS V *)p)[i] = x.q[i];
    } else {
#pragma unroll
        for (u32 i = 0; i < 8u; i++)
            if (i < left) p[i] = x.e[i];
    }
}

} // namespace inshr
