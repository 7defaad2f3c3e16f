// Device-side helpers of the row operators: element types, 16-byte vectors at any element address, reductions over a row's lanes.
#pragma once

#include "device_utils.h"
#include "rows.h"

namespace dcnn {

typedef __bf16 bf16;
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// 16 bytes of a row: E elements, and a vector of them where rows lie.  Rows start at any multiple of the element's size (odd widths,
// views), and the memory path takes vectors at such addresses: the alignment is the element's.
template <typename T> struct RowVec {
    static constexpr int E = 16 / (int)sizeof(T);
    typedef T type __attribute__((ext_vector_type(16 / sizeof(T)), aligned(sizeof(T))));
};
// Four consecutive outputs.
template <typename T> struct RowQuad { typedef T type __attribute__((ext_vector_type(4), aligned(sizeof(T)))); };

// The same in LDS, where they are aligned.
template <typename T> using AlignedVec = T __attribute__((ext_vector_type(16 / sizeof(T))));
template <typename T> using AlignedQuad = T __attribute__((ext_vector_type(4)));

// Rows of this call, read on the GPU where a list's length is.
__device__ __forceinline__ int row_count(const int32_t* count, int rows) {
    if (count == nullptr) return rows;
    const int n = *count;
    return n < 0 ? 0 : (n < rows ? n : rows);
}

struct SumOp {
    typedef float type;
    static __device__ __forceinline__ float op(float a, float b) { return a + b; }
};
struct MaxOp {                   // bit patterns of magnitudes: NaN above infinity above every number
    typedef uint32_t type;
    static __device__ __forceinline__ uint32_t op(uint32_t a, uint32_t b) { return a > b ? a : b; }
};
template <typename Op, int CTRL> __device__ __forceinline__ typename Op::type dpp_step(typename Op::type u) {
    const int v = __builtin_bit_cast(int, u);
    return Op::op(u, __builtin_bit_cast(typename Op::type, __builtin_amdgcn_update_dpp(v, v, CTRL, 0xf, 0xf, true)));
}
// Over aligned groups of L lanes of a wave, delivered to all of them; every step adds the same two numbers on both sides, so
// the lanes of a group hold the same bits.  (Within 16 lanes by lane permutations, see group_max.)
template <typename Op, int L> __device__ __forceinline__ typename Op::type wave_reduce(typename Op::type u) {
    if constexpr (L >= 2) u = dpp_step<Op, 0xB1>(u);
    if constexpr (L >= 4) u = dpp_step<Op, 0x4E>(u);
    if constexpr (L >= 8) u = dpp_step<Op, 0x141>(u);
    if constexpr (L >= 16) u = dpp_step<Op, 0x140>(u);
    if constexpr (L >= 32) u = Op::op(u, __shfl_xor(u, 16, kWave));
    if constexpr (L >= 64) u = Op::op(u, __shfl_xor(u, 32, kWave));
    return u;
}
// Over the L lanes of a row: a part of a wave, or the whole workgroup.  `red` is 2 * waves words of LDS, `turn` alternates: a
// reduction's words are overwritten two reductions later, behind the barrier of the one between.
template <typename Op, int L> __device__ __forceinline__ typename Op::type row_reduce(typename Op::type u, uint32_t* red, int& turn) {
    u = wave_reduce<Op, (L < kWave ? L : kWave)>(u);
    if constexpr (L > kWave) {
        constexpr int W = L / kWave;
        uint32_t* s = red + turn * W;
        turn ^= 1;
        if (threadIdx.x % kWave == 0) s[threadIdx.x / kWave] = __builtin_bit_cast(uint32_t, u);
        __syncthreads();
        u = __builtin_bit_cast(typename Op::type, s[0]);
#pragma unroll
        for (int i = 1; i < W; ++i) u = Op::op(u, __builtin_bit_cast(typename Op::type, s[i]));
    }
    return u;
}

// A product's output before its activation: the sum, the factor and the output are rounded to fp32, one after the other, whatever comes
// behind.  (Left alone, the compiler folds the last of these into the rounding to fp16 where nothing stands between, and a row's outputs
// would depend on the kernel that makes them, once in 20000.)
__device__ __forceinline__ float scaled_sum(int32_t sum, float row_scale, float w_scale, float bias) {
    float v = __builtin_fmaf((float)sum, row_scale * w_scale, bias);
    asm("" : "+v"(v));
    return v;
}
// ReLU up to hi of a product's outputs.  A NaN (of a row that held one) stays one: maximum and minimum hand it on.  (Two instructions; with
// comparisons four and their waits, 26214 x 256 -> 1024 took 21.8 us in place of 19.2.)
__device__ __forceinline__ void act_keep_nan(float (&v)[4], float hi) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __builtin_elementwise_minimum(__builtin_elementwise_maximum(v[e], 0.0f), hi);
}

// Four channels of a bias, zero where there is none.
template <typename T> __device__ __forceinline__ f32x4 load_bias(const void* bias, int ch, int n) {
    f32x4 v = {0.0f, 0.0f, 0.0f, 0.0f};
    const T* b = static_cast<const T*>(bias);
    if (b == nullptr || ch >= n) return v;
    if (ch + 4 <= n) {
        const typename RowQuad<T>::type q = *reinterpret_cast<const typename RowQuad<T>::type*>(b + ch);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = (float)q[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (ch + e < n) v[e] = (float)b[ch + e];
    }
    return v;
}

// v -> round_half_even(v * inv) as the low byte of the result.  |v * inv| <= 127.5: adding 1.5 * 2^23 leaves the integer in the
// low bits, rounded half to even.  The product is rounded by itself first (no fused multiply-add): that is the definition.
__device__ __forceinline__ uint32_t quantize_bits(float v, float inv) {
#pragma clang fp contract(off)
    const float p = v * inv;
    return __builtin_bit_cast(uint32_t, p + 12582912.0f);
}
// low bytes of four words
__device__ __forceinline__ uint32_t pack_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x0c0c0400u), hi = __builtin_amdgcn_perm(d, c, 0x0c0c0400u);
    return lo | hi << 16;
}
constexpr float kQuantMin = 1e-36f;            // below it 127 / max|v| overflows: such a row is zeros
// The scale of a row and what its values are multiplied with; bits: max|v| as bits
__device__ __forceinline__ float quantize_scale(uint32_t bits, float* inv) {
    const float amax = __builtin_bit_cast(float, bits);
    *inv = 0.0f;
    if (bits >= 0x7f800000u) return __builtin_nanf("");
    if (amax < kQuantMin) return 0.0f;
    *inv = 127.0f / amax;
    return amax / 127.0f;
}

// ---- rows in registers ----------------------------------------------------------------------------------------------
// A row is cut into vectors of 16 bytes; where its length is no multiple of that the last one ends where the row does, and its first
// elements are the vector's before it once more: they count in no sum and are stored twice, with the same values.  (So no load is masked
// and no store is in pieces, wherever rows start.)
// Vector `base` of a row of c elements: where it lies (below c), and the elements that do not count (E: all, it is behind the row).
struct RowPart { int at, skip; };
template <typename T> __device__ __forceinline__ RowPart row_part(int base, int c) {
    constexpr int E = RowVec<T>::E;
    if (base + E <= c || c < E) return {base, base < c ? 0 : E};           // (rows shorter than a vector: the first one)
    return base < c ? RowPart{c - E, base + E - c} : RowPart{base, E};
}
template <typename T> __device__ __forceinline__ u32x4 row_load(const T* row, int base, int c) {
    constexpr int E = RowVec<T>::E;
    const RowPart p = row_part<T>(base, c);
    u32x4 v = {0u, 0u, 0u, 0u};
    if (p.skip >= E) return v;
    if (c >= E) return __builtin_bit_cast(u32x4, *reinterpret_cast<const typename RowVec<T>::type*>(row + p.at));
    typedef std::conditional_t<sizeof(T) == 4, uint32_t, uint16_t> Bits;
#pragma unroll
    for (int e = 0; e < E; ++e)
        if (e < c) v[e * (int)sizeof(T) / 4] |= (uint32_t) reinterpret_cast<const Bits*>(row)[e] << (e * (int)sizeof(T) % 4 * 8);
    return v;
}
template <typename T> __device__ __forceinline__ float row_get(u32x4 v, int e) {
    typedef T Vec __attribute__((ext_vector_type(16 / sizeof(T))));
    return (float)__builtin_bit_cast(Vec, v)[e];
}
// Stored past the L2: none of a row's elements is wanted there again before the kernel's end, and its lines would take the inputs' places
// (16384 x 4096 bf16, y and z: 111 us -> 90; 26214 rows of 256 by a list 14.3 -> 12.4.)
template <typename T> __device__ __forceinline__ void row_store(T* row, int base, int c, const float* o) {
    constexpr int E = RowVec<T>::E;
    const RowPart p = row_part<T>(base, c);
    if (p.skip >= E) return;
    typename RowVec<T>::type v;
#pragma unroll
    for (int e = 0; e < E; ++e) v[e] = (T)o[e];
    if (c >= E) {
        __builtin_nontemporal_store(v, reinterpret_cast<typename RowVec<T>::type*>(row + p.at));
    } else {
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (e < c) row[e] = v[e];
    }
}

// The same value, of which the compiler knows nothing: what is made of it in a loop is not made once before it and kept.  (Parameters held
// as 16-bit values would be held as fp32 values, in twice the registers.)
__device__ __forceinline__ u32x4 unknown(u32x4 v) {
    asm volatile("" : "+v"(v));
    return v;
}

// A norm's parameters for the channels of a lane: read once for many rows (HOLD), or where they are used.
template <typename T, int L, int NV, bool HOLD> struct NormParams {
    const T *w, *b;
    u32x4 wv[HOLD ? NV : 1], bv[HOLD ? NV : 1];
    __device__ __forceinline__ void read(const void* w_, const void* b_, int lane, int c) {
        w = static_cast<const T*>(w_), b = static_cast<const T*>(b_);
        if constexpr (HOLD) {
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (w != nullptr) wv[j] = row_load<T>(w, (j * L + lane) * RowVec<T>::E, c);
                if (b != nullptr) bv[j] = row_load<T>(b, (j * L + lane) * RowVec<T>::E, c);
            }
        }
    }
    __device__ __forceinline__ u32x4 weight(int j, int lane, int c) const { return HOLD ? unknown(wv[HOLD ? j : 0]) : row_load<T>(w, (j * L + lane) * RowVec<T>::E, c); }
    __device__ __forceinline__ u32x4 bias(int j, int lane, int c) const { return HOLD ? unknown(bv[HOLD ? j : 0]) : row_load<T>(b, (j * L + lane) * RowVec<T>::E, c); }
};

// s = f(s, v[j][e]) over the elements that count in the row's sums, over the row's lanes.  Where a part of a wave has more than one vector to a
// lane the vectors are added up as twice, four or eight times as many lanes would: a row's sums have the same bits either way.
template <typename T, int L, int NV, typename F>
__device__ __forceinline__ float row_sum(const float (&v)[NV][RowVec<T>::E], int lane, int c, uint32_t* red, int& turn, F&& f) {
    constexpr int E = RowVec<T>::E, S = L < kWave ? NV : 1;
    static_assert(S == 1 || ((S & (S - 1)) == 0 && S * L <= kWave), "pairs of vectors");
    float s[S] = {};
    if (c % E == 0) {                                          // (what lies behind the row is zero)
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e) s[j % S] = f(s[j % S], v[j][e]);
    } else {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int skip = c < E ? 0 : row_part<T>((j * L + lane) * E, c).skip;
#pragma unroll
            for (int e = 0; e < E; ++e) s[j % S] = e >= skip ? f(s[j % S], v[j][e]) : s[j % S];
        }
    }
#pragma unroll
    for (int j = 0; j < S; ++j) s[j] = row_reduce<SumOp, L>(s[j], red, turn);
#pragma unroll
    for (int d = 1; d < S; d *= 2)
#pragma unroll
        for (int j = 0; j < S; j += 2 * d) s[j] += s[j + d];
    return s[0];
}

// v <- norm(v); vectors behind the row's end are zero before and after.  (What is fused into one rounding is written so: rows that
// fit a wave have the same bits in every kernel that norms them.)
template <typename T, int L, int NV, bool HOLD>
__device__ __forceinline__ void norm_row(float (&v)[NV][RowVec<T>::E], int kind, float eps, const NormParams<T, L, NV, HOLD>& params, int lane, int c, float inv_c,
                                         uint32_t* red, int& turn) {
#pragma clang fp contract(off)
    constexpr int E = RowVec<T>::E;
    if (kind == DCNN_NORM_LAYER) {
        const float mean = row_sum<T, L, NV>(v, lane, c, red, turn, [](float s, float a) { return s + a; }) * inv_c;
#pragma unroll
        for (int j = 0; j < NV; ++j) {
            const int base = (j * L + lane) * E;
            if (c < E) {
#pragma unroll
                for (int e = 0; e < E; ++e) v[j][e] = base + e < c ? v[j][e] - mean : 0.0f;
            } else {
                const float m = base < c ? mean : 0.0f;
#pragma unroll
                for (int e = 0; e < E; ++e) v[j][e] -= m;
            }
        }
    }
    const float squares = row_sum<T, L, NV>(v, lane, c, red, turn, [](float s, float a) { return __builtin_fmaf(a, a, s); });
    const float r = 1.0f / sqrtf(__builtin_fmaf(squares, inv_c, eps));
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        // (the four cases apart: a vector of factors held between them is registers that large rows have not left)
        if (params.w != nullptr) {
            const u32x4 w = params.weight(j, lane, c);
            if (params.b != nullptr) {
                const u32x4 b = params.bias(j, lane, c);
#pragma unroll
                for (int e = 0; e < E; ++e) v[j][e] = __builtin_fmaf(v[j][e], r * row_get<T>(w, e), row_get<T>(b, e));
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) v[j][e] *= r * row_get<T>(w, e);
            }
        } else if (params.b != nullptr) {
            const u32x4 b = params.bias(j, lane, c);
#pragma unroll
            for (int e = 0; e < E; ++e) v[j][e] = __builtin_fmaf(v[j][e], r, row_get<T>(b, e));
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) v[j][e] *= r;
        }
    }
}

// A row's largest magnitude, as bits, over its lanes.
template <int L, int NV, int E> __device__ __forceinline__ uint32_t row_amax(const float (&v)[NV][E], uint32_t* red, int& turn) {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) m = MaxOp::op(m, __builtin_bit_cast(uint32_t, v[j][e]) & 0x7fffffffu);
    return row_reduce<MaxOp, L>(m, red, turn);
}
// E values in 8 bits.
template <typename T> struct QuantWords {
    typedef uint32_t type __attribute__((ext_vector_type(16 / sizeof(T) / 4), aligned(1)));
};
template <typename T> __device__ __forceinline__ typename QuantWords<T>::type quantized(const float (&v)[RowVec<T>::E], float inv) {
    typename QuantWords<T>::type w;
#pragma unroll
    for (int e = 0; e < RowVec<T>::E; e += 4)
        w[e / 4] = inv == 0.0f ? 0u : pack_bytes(quantize_bits(v[e], inv), quantize_bits(v[e + 1], inv), quantize_bits(v[e + 2], inv), quantize_bits(v[e + 3], inv));
    return w;
}
// Vector `base` of a row of c in 8 bits.  (A row shorter than a vector has room for one.)
template <typename T> __device__ __forceinline__ void row_store_quantized(int8_t* row, int base, int c, const float (&v)[RowVec<T>::E], float inv) {
    const RowPart p = row_part<T>(base, c);
    if (p.skip < RowVec<T>::E) *reinterpret_cast<typename QuantWords<T>::type*>(row + p.at) = quantized<T>(v, inv);
}

}  // namespace dcnn
