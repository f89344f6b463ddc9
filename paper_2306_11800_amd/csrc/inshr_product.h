// What the kernels of the products share: vector types, scales, activations, what follows a sum.
#pragma once
#include "inshr_answer.h"

namespace inshr {

typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef float f4 __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------------------------------
// scales
// ------------------------------------------------------------------------------------------
// The power of two that brings a largest magnitude (bits of |x|) into [2^14, 2^15), and its inverse; both normal.  An
// infinity counts as the largest finite exponent: it stays infinite under any scale.
__device__ __forceinline__ void scale_of(u32 mag, float &s, float &inv)
{
    u32 e = mag >> 23;
    e = e > 254u ? 254u : e;
    const u32 sb = e < 15u ? 253u : 268u - e;
    s = __uint_as_float(sb << 23);
    inv = __uint_as_float((254u - sb) << 23);
}
__device__ __forceinline__ int exponent_of(float scale) { return (int)(__float_as_uint(scale) >> 23) - 127; } // of a power of two
__device__ __forceinline__ u32 mag_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }
__device__ __forceinline__ u32 wave_max_u(u32 v)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        const u32 o = __shfl_xor(v, d);
        v = v > o ? v : o;
    }
    return v;
}
// (magnitudes of infinities and NaN say nothing of the finite values' scale)
__device__ __forceinline__ u32 finite_mag(float x)
{
    const u32 m = mag_bits(x);
    return m < 0x7f800000u ? m : 0u;
}

// ------------------------------------------------------------------------------------------
// activations
// ------------------------------------------------------------------------------------------
// 1 / (1 + e^-x), by the instructions for powers of two and reciprocals: each is off by one unit of 2^-24 or so, and the
// argument's rounding by 2^-24 of it, which tells in e^-x alone where the result is near e^x (a fifth of the instructions
// of the library's expf and division; 256 x 256 results with silu 20 -> 5 us).
__device__ __forceinline__ float logistic(float x)
{
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(x * -1.44269504f));
}
// ... and `rest` = 1 - logistic(x) = e^-x logistic(x), which keeps its digits where the logistic is near 1
__device__ __forceinline__ float logistic(float x, float &rest)
{
    const float e = __builtin_amdgcn_exp2f(fminf(x * -1.44269504f, 126.0f)), s = __builtin_amdgcn_rcpf(1.0f + e);
    rest = e * s;
    return s;
}
__device__ __forceinline__ float bend(float a) { return 1.59576912160573071f * (a + 0.044715f * a * a * a); } // 2 u

template <int N>
__device__ __forceinline__ void act_of(float (&v)[N], u32 act)
{
    switch (act) {
    case ACT_RELU:
#pragma unroll
        for (int i = 0; i < N; i++) v[i] = v[i] < 0.0f ? 0.0f : v[i];
        break;
    case ACT_GELU:
#pragma unroll
        for (int i = 0; i < N; i++) v[i] = 0.5f * v[i] * (1.0f + erff(v[i] * 0.70710678118654752f));
        break;
    case ACT_GELU_TANH: // 0.5 a (1 + tanh u) = a / (1 + e^-2u)
#pragma unroll
        for (int i = 0; i < N; i++) v[i] *= logistic(bend(v[i]));
        break;
    case ACT_SILU:
#pragma unroll
        for (int i = 0; i < N; i++) v[i] *= logistic(v[i]);
        break;
    }
}
// a for the slopes' polynomials: past `end` the slope is 0 or 1 (to 2^-100), and powers of a would outrun the exponential,
// which ends at 2^126; NaN stays
__device__ __forceinline__ float within(float a, float end)
{
    return __builtin_elementwise_minimum(__builtin_elementwise_maximum(a, -end), end);
}
// v times the slope at a
template <int N>
__device__ __forceinline__ void act_grad(float (&v)[N], const float (&a)[N], u32 act)
{
    switch (act) {
    case ACT_RELU:
#pragma unroll
        for (int i = 0; i < N; i++) v[i] = a[i] > 0.0f ? v[i] : a[i] != a[i] ? a[i] : 0.0f * v[i];
        break;
    case ACT_GELU:
#pragma unroll
        for (int i = 0; i < N; i++)
            v[i] *= 0.5f * (1.0f + erff(a[i] * 0.70710678118654752f)) +
                    a[i] * 0.39894228040143268f * __builtin_amdgcn_exp2f(a[i] * a[i] * -0.72134752f);
        break;
    case ACT_GELU_TANH: // with s = 1 / (1 + e^-2u): s + 2 a s (1 - s) u'
#pragma unroll
        for (int i = 0; i < N; i++) {
            float rest;
            const float x = within(a[i], 16.0f), s = logistic(bend(x), rest);
            v[i] *= s + x * s * rest * 1.59576912160573071f * (1.0f + 0.134145f * x * x);
        }
        break;
    case ACT_SILU:
#pragma unroll
        for (int i = 0; i < N; i++) {
            float rest;
            const float x = within(a[i], 120.0f), s = logistic(x, rest);
            v[i] *= s * (1.0f + x * rest);
        }
        break;
    }
}

// ------------------------------------------------------------------------------------------
// a weight's values
// ------------------------------------------------------------------------------------------
__device__ __forceinline__ float protected_value(const WDesc &w, u64 j)
{
    return w.val_bf16 ? __uint_as_float((u32)((const GLOBAL_AS u16 *)w.out_val)[j] << 16) : ((const GLOBAL_AS float *)w.out_val)[j];
}

// Values of the symbols: 0 for pruned, 0 for protected (their values follow from the list), the centres, and NaN for
// what is no symbol of the codebook.
__device__ __forceinline__ float symbol_value(const WDesc &w, u32 s)
{
    return s < 2u ? 0.0f : s < w.K + 2u ? gptr(w.codebook)[s - 2u] : __uint_as_float(0x7fc00000u);
}

// ------------------------------------------------------------------------------------------
// what follows a sum
// ------------------------------------------------------------------------------------------
struct Finish {
    const float *bias;
    Mat residual, out, pre;
    u32 N, act;
};

// Results (m, n) .. (m, n + 7), n < N, the columns past N left out: bias, activation, residual, one rounding.
template <u32 TY>
__device__ __forceinline__ void finish8(const Finish &g, u32 m, u32 n, float (&v)[8])
{
    typedef typename Elem<TY>::type T;
    const u32 there = min(g.N - n, 8u);
    if (g.bias) {
        float b[8];
        load8<TY_F32>(gptr(g.bias) + n, there, b);
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] += b[i];
    }
    if (g.pre.p) store8<TY>((GLOBAL_AS T *)g.pre.p + (u64)m * g.pre.stride + n, there, v);
    act_of(v, g.act);
    if (g.residual.p) {
        float r[8];
        load8<TY>((const GLOBAL_AS T *)g.residual.p + (u64)m * g.residual.stride + n, there, r);
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] += r[i];
    }
    store8<TY>((GLOBAL_AS T *)g.out.p + (u64)m * g.out.stride + n, there, v);
}

} // namespace inshr
