// Symbols from the stream to values: a table in LDS with a copy of every entry for each of the lanes that read together.
#pragma once
#include "inshr_product.h"

#include <type_traits>

namespace inshr {

// ------------------------------------------------------------------------------------------
// the table
// ------------------------------------------------------------------------------------------
// Copies of an entry, one per bank (or two) that the lanes of a read meet in; at most 16 KB in all.
template <u32 TY, int W> struct Table {
    static constexpr u32 WORDS = TY == TY_F32 ? 2u : 1u; // 32-bit words of an entry
    static constexpr u32 COPIES = (W <= 7 ? 32u : W == 8 ? 16u : 8u) / WORDS;
    static constexpr u32 BYTES = (1u << W) * COPIES * WORDS * 4u;
};
__device__ __forceinline__ u32 bf16_cut(float x) { return __float_as_uint(x) & 0xffff0000u; } // towards zero: what is left over is exact
template <u32 TY>
__device__ __forceinline__ void entry_of(float v, float s, u32 (&e)[2])
{
    if (TY == TY_BF16) {
        // (to nearest, but not to infinity: past the largest bfloat16 number the second part takes what is cut off)
        const u32 m = __float_as_uint(v) & 0x7fffffffu, hi = m >= 0x7f7f8000u && m < 0x7f800000u ? bf16_cut(v) >> 16 : Elem<TY_BF16>::put(v);
        const float rest = v - __uint_as_float(hi << 16);
        e[0] = hi | (u32)Elem<TY_BF16>::put(rest) << 16;
    } else if (TY == TY_F16) {
        union { _Float16 h; u16 u; } a, b;
        a.h = (_Float16)(v * s);
        b.h = (_Float16)(v * s - (float)a.h);
        e[0] = a.u | (u32)b.u << 16;
    } else {
        const u32 h = bf16_cut(v);
        const float r1 = v - __uint_as_float(h);
        const u32 m = bf16_cut(r1);
        e[0] = h >> 16 | m;
        e[1] = __float_as_uint(r1 - __uint_as_float(m)) >> 16;
    }
}
// Fills the table with the values times s (fp16 only).  A barrier has to follow.
template <u32 TY, int W>
__device__ __forceinline__ void fill_table(const WDesc &w, u32 *table, float s)
{
    typedef Table<TY, W> T;
    constexpr u32 C = T::COPIES;
    for (u32 i = threadIdx.x; i < (1u << W) * C; i += blockDim.x) {
        u32 e[2];
        entry_of<TY>(symbol_value(w, i / C), s, e);
        table[i * T::WORDS] = e[0];
        if (T::WORDS > 1) table[i * T::WORDS + 1] = e[1];
    }
}
// where this lane's copy of entry 0 is (bytes)
template <u32 TY, int W>
__device__ __forceinline__ u32 lane_copy()
{
    return (threadIdx.x & (Table<TY, W>::COPIES - 1u)) * Table<TY, W>::WORDS * 4u;
}
// The entry of symbol j of a run whose first bit is bit 0 of d[0].
template <u32 TY, int W>
__device__ __forceinline__ void look_up(const char *table, u32 mine, const u32 *d, int j, u32 (&e)[2])
{
    typedef Table<TY, W> T;
    constexpr int SH = __builtin_ctz(T::COPIES * T::WORDS * 4u); // an entry's copies: 2^SH bytes
    constexpr u32 MASK = ((1u << W) - 1u) << SH;
    const int bit = j * W, at = bit >> 5, off = bit & 31;
    u32 a;
    if (off + W > 32) // in two words
        a = __builtin_amdgcn_alignbit(d[at + 1], d[at], (u32)off) << SH;
    else if (off >= SH)
        a = d[at] >> (off - SH);
    else
        a = d[at] << (SH - off);
    const char *p = table + ((a & MASK) | mine);
    if (T::WORDS > 1) {
        const uint2 v = *(const uint2 *)p;
        e[0] = v.x;
        e[1] = v.y;
    } else {
        e[0] = *(const u32 *)p;
    }
}
__device__ __forceinline__ u32 low_halves(u32 a, u32 b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ u32 high_halves(u32 a, u32 b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// ------------------------------------------------------------------------------------------
// the stream
// ------------------------------------------------------------------------------------------
typedef u32 u4_any __attribute__((ext_vector_type(4), aligned(4)));
// N consecutive words, those from word `end` on as 0.  SAFE: they are there whatever `end` says.
template <int N, bool SAFE = false>
__device__ __forceinline__ void load_words(const u32 *packed, u64 at, u64 end, u32 *d)
{
    const GLOBAL_AS u32 *p = gptr(packed) + at;
    if (SAFE || at + N <= end) {
#pragma unroll
        for (int i = 0; i + 4 <= N; i += 4) {
            const u4_any v = *(const GLOBAL_AS u4_any *)(p + i);
            d[i] = v.x;
            d[i + 1] = v.y;
            d[i + 2] = v.z;
            d[i + 3] = v.w;
        }
#pragma unroll
        for (int i = N & ~3; i < N; i++) d[i] = p[i];
    } else {
#pragma unroll
        for (int i = 0; i < N; i++) d[i] = at + i < end ? p[i] : 0u;
    }
}

// A kernel for the width of a symbol: run(std::integral_constant<int, w>).
template <class F>
inline void with_width(u32 w, F run)
{
    switch (w) {
    case 2: run(std::integral_constant<int, 2>()); break;
    case 3: run(std::integral_constant<int, 3>()); break;
    case 4: run(std::integral_constant<int, 4>()); break;
    case 5: run(std::integral_constant<int, 5>()); break;
    case 6: run(std::integral_constant<int, 6>()); break;
    case 7: run(std::integral_constant<int, 7>()); break;
    case 8: run(std::integral_constant<int, 8>()); break;
    default: run(std::integral_constant<int, 9>()); break;
    }
}

} // namespace inshr
