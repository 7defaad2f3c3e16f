// Device-side helpers of attention: operands of the matrix cores in the types of a cache.
#pragma once

#include "cache_device.h"

namespace dcnn {

typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef f16 f16x8v __attribute__((ext_vector_type(8)));
typedef bf16 bf16x8v __attribute__((ext_vector_type(8)));

// What a type's queries, weights, keys and values are on the matrix cores: TERMS operands whose sum is the number.  Codes times a power of two are
// exact in bf16 (and, from 2^-24 to 2^16, in fp16), fp32 numbers are three bf16 ones.
// Weights of 16-bit types are one operand, rounded by half a step of each at most.  Another one for what that leaves over (weights as good as fp32's) was
// measured: one row of 262143 tokens 54 us in place of 50, 64 rows of up to 8192 70 in place of 64, prompts in tiles 820 in place of 655, flagged pixels 657
// in place of 442.  A call that wants them kept takes the cache's memory, which is the same in all types, as fp32's.
template <typename T> struct Operand {
    typedef f16x8v type;
    static constexpr int TERMS = 1;
    static constexpr float RAISE = 15.0f;      // weights are 2^15 at most: below 2^-14 fp16 has fewer digits, below 2^-25 none
    static __device__ __forceinline__ void split(const float (&v)[8], type (&o)[TERMS]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) o[0][e] = (f16)v[e];
    }
    template <int SEL> static __device__ __forceinline__ uint32_t pair(uint32_t w, float s) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(w, s, SEL)); }
    static __device__ __forceinline__ f32x4 mfma16(type a, type b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x16 mfma32(type a, type b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
template <> struct Operand<bf16> {
    typedef bf16x8v type;
    static constexpr int TERMS = 1;
    static constexpr float RAISE = 0.0f;
    static __device__ __forceinline__ void split(const float (&v)[8], type (&o)[TERMS]) {
#pragma unroll
        for (int e = 0; e < 8; ++e) o[0][e] = (bf16)v[e];
    }
    template <int SEL> static __device__ __forceinline__ uint32_t pair(uint32_t w, float s) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, SEL)); }
    static __device__ __forceinline__ f32x4 mfma16(type a, type b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
    static __device__ __forceinline__ f32x16 mfma32(type a, type b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
// (cut, not rounded: eight bits of the 24 to a term are exact too, and the largest numbers do not become infinity)
template <> struct Operand<float> : Operand<bf16> {
    static constexpr int TERMS = 3;
    static __device__ __forceinline__ void split(const float (&v)[8], type (&o)[TERMS]) {
        u32x4 w[TERMS];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
            float a = v[e], b = v[e + 1];
#pragma unroll
            for (int t = 0; t < TERMS; ++t) {
                const uint32_t x = __builtin_bit_cast(uint32_t, a), y = __builtin_bit_cast(uint32_t, b);
                w[t][e / 2] = __builtin_amdgcn_perm(y, x, 0x07060302u);
                a -= __builtin_bit_cast(float, x & 0xffff0000u), b -= __builtin_bit_cast(float, y & 0xffff0000u);
            }
        }
#pragma unroll
        for (int t = 0; t < TERMS; ++t) o[t] = __builtin_bit_cast(type, w[t]);
    }
};
// Eight codes of a word, one scale.
template <typename T> __device__ __forceinline__ typename Operand<T>::type decode8(uint32_t w, float s) {
    typedef Operand<T> O;
    const u32x4 v = {O::template pair<0>(w, s), O::template pair<1>(w, s), O::template pair<2>(w, s), O::template pair<3>(w, s)};
    return __builtin_bit_cast(typename O::type, v);
}
// Eight codes of a word, a scale for each: a pair is converted with both, and halves of the two are put together.
template <typename T> __device__ __forceinline__ typename Operand<T>::type decode8(uint32_t w, const float (&s)[8]) {
    typedef Operand<T> O;
    const u32x4 v = {__builtin_amdgcn_perm(O::template pair<0>(w, s[1]), O::template pair<0>(w, s[0]), 0x07060100u),
                     __builtin_amdgcn_perm(O::template pair<1>(w, s[3]), O::template pair<1>(w, s[2]), 0x07060100u),
                     __builtin_amdgcn_perm(O::template pair<2>(w, s[5]), O::template pair<2>(w, s[4]), 0x07060100u),
                     __builtin_amdgcn_perm(O::template pair<3>(w, s[7]), O::template pair<3>(w, s[6]), 0x07060100u)};
    return __builtin_bit_cast(typename O::type, v);
}
// Eight values of queries as operands, or their opposites.
template <typename T> __device__ __forceinline__ void load_operand(const T* p, int negate, typename Operand<T>::type (&o)[Operand<T>::TERMS]) {
    if constexpr (sizeof(T) == 2) {
        u32x4 v = __builtin_bit_cast(u32x4, *reinterpret_cast<const typename RowVec<T>::type*>(p));
        v ^= negate ? 0x80008000u : 0u;
        o[0] = __builtin_bit_cast(typename Operand<T>::type, v);
    } else {
        float v[8];
        const typename RowVec<T>::type a = *reinterpret_cast<const typename RowVec<T>::type*>(p), b = *reinterpret_cast<const typename RowVec<T>::type*>(p + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = negate ? -a[e] : a[e], v[4 + e] = negate ? -b[e] : b[e];
        Operand<T>::split(v, o);
    }
}

// The larger of a lane's value and that of the lane 32 on, or before.
__device__ __forceinline__ float max_of_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
    return fmaxf(__builtin_bit_cast(float, (uint32_t)r[0]), __builtin_bit_cast(float, (uint32_t)r[1]));
}

// Waves to a SIMD of the kernel for tiles of rows: as many as leave a lane's queries, sums, products and weights (heads of 32 NB values, numbers of
// `terms` operands) room for addresses and codes.  Heads of 64 with three in place of two: 655 us and 548 (26240 rows of 8 heads, 4096 tokens each).
constexpr int tile_waves(int nb, int terms) {
    const int registers = nb * 8 * terms + nb * 16 + 32 + 16 * terms;
    return registers <= 112 ? 3 : registers <= 176 ? 2 : 1;
}

// Tiles that each of the `shares` workgroups of a head takes: a tile for each wave at least.
__device__ __forceinline__ int share_of(int tiles, int shares) {
    const int n = (tiles + shares - 1) / shares;
    return n < 4 ? 4 : n;
}
// Where the first of a part's 16 columns lies: a workgroup has one of the row that it begins in (0) and one of the row that it ends in (1) at most.
__device__ __forceinline__ int64_t part_at(int hb, int share, int shares, int which) { return (((int64_t)hb * shares + share) * 2 + which) * 16; }

// Tokens that a row sees: lo .. hi-1.
struct Span { int lo, hi; };
__device__ __forceinline__ Span span_of(const AttendArgs& a, const Token& t) {
    if (!t.here || (uint32_t)t.stream >= (uint32_t)a.cache.streams) return {0, 0};
    int lo = 0, hi = a.cache.length;
    if (a.lens != nullptr) {
        const int n = a.lens[t.stream];
        hi = n < 0 ? 0 : (n < hi ? n : hi);
    }
    // (in 64 bits: positions may be any number)
    if (a.causal != 0 && (int64_t)t.pos + 1 < hi) hi = t.pos + 1;
    if (a.window > 0) {
        const int64_t first = (int64_t)t.pos - a.window + 1, end = (int64_t)t.pos + a.window;
        if (end < hi) hi = (int)end;
        if (first > lo) lo = first < hi ? (int)first : hi;
    }
    if (hi <= lo) return {0, 0};
    return {lo, hi};
}

}  // namespace dcnn
