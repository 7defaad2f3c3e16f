// Heads normed and rotated, appended to the cache in 4 bits, and read from it.
//
//   u = norm(x[r, h]),  rotated: (a, b) -> (a cos - b sin, b cos + a sin)
//   appended: 32 values share the smallest power of two s with max|u| <= 6 s, each becomes the code next to u / s
//
// A head's D values lie in the registers of D / 8 lanes (eight to a lane), its statistics and a block's largest magnitude are lane
// permutations, and a value's partner in a rotation by halves is read again (from the L1) rather than passed between lanes.  A workgroup
// takes 256 / L rows and goes through some of their heads, so a row's position, page, angles and a norm's parameters are read once.
// Rows beside each other are tokens beside each other, as a rule: the few bytes of a head and token fill whole lines of the cache.
// Keys are fp64 from the norm to the code (their cost hides behind the memory): a code is the same whatever the order of a sum.
#include "cache_device.h"

namespace dcnn {

template <typename T> __device__ __forceinline__ void load8(const T* p, float (&v)[8]) {
    constexpr int E = RowVec<T>::E;
#pragma unroll
    for (int i = 0; i < 8; i += E) {
        const typename RowVec<T>::type x = *reinterpret_cast<const typename RowVec<T>::type*>(p + i);
#pragma unroll
        for (int e = 0; e < E; ++e) v[i + e] = (float)x[e];
    }
}
template <typename T> __device__ __forceinline__ void store8(T* p, const float (&v)[8]) {
    constexpr int E = RowVec<T>::E;
#pragma unroll
    for (int i = 0; i < 8; i += E) {
        typename RowVec<T>::type x;
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = (T)v[i + e];
        __builtin_nontemporal_store(x, reinterpret_cast<typename RowVec<T>::type*>(p + i));
    }
}

// Sum over aligned groups of L lanes, delivered to all of them (see wave_reduce).
template <int L> __device__ __forceinline__ float sum_lanes(float v) { return wave_reduce<SumOp, L>(v); }
template <int CTRL> __device__ __forceinline__ double dpp64(double v) {
    const uint64_t u = __builtin_bit_cast(uint64_t, v);
    const int lo = (int)(uint32_t)u, hi = (int)(uint32_t)(u >> 32);
    const uint32_t l = (uint32_t)__builtin_amdgcn_update_dpp(lo, lo, CTRL, 0xf, 0xf, true), h = (uint32_t)__builtin_amdgcn_update_dpp(hi, hi, CTRL, 0xf, 0xf, true);
    return __builtin_bit_cast(double, (uint64_t)h << 32 | l);
}
template <int L> __device__ __forceinline__ double sum_lanes(double v) {
    v += dpp64<0xB1>(v);
    v += dpp64<0x4E>(v);
    if constexpr (L >= 8) v += dpp64<0x141>(v);
    if constexpr (L >= 16) v += dpp64<0x140>(v);
    if constexpr (L >= 32) v += __shfl_xor(v, 16, kWave);
    return v;
}
// Largest magnitude of a block of 32, over its four lanes; an infinity where there is one or a NaN.
__device__ __forceinline__ double block_amax(const double (&v)[8]) {
    double m = 0.0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const double a = __builtin_fabs(v[e]);
        m = a <= 1.7976931348623157e308 ? (a > m ? a : m) : __builtin_inf();
    }
    const double n = dpp64<0xB1>(m);
    m = n > m ? n : m;
    const double o = dpp64<0x4E>(m);
    return o > m ? o : m;
}

// A head's eight values of a lane, normed: what stays the same for all heads of a job.
template <typename T> struct HeadNorm {
    int kind;
    float eps;
    const T *w, *b;
};
// v (and p, the partners' values, where `both`) <- norm.  Lanes behind the head (`!in`) hold zeros.
template <typename T, typename A, int D, int L>
__device__ __forceinline__ void norm_head(A (&v)[8], A (&p)[8], bool both, const HeadNorm<T>& n, int at, int partner, bool in) {
    if (n.kind == DCNN_NORM_NONE) return;
    A mean = 0;
    if (n.kind == DCNN_NORM_LAYER) {
        A s = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) s += v[e];
        mean = sum_lanes<L>(s) / (A)D;
    }
    A s = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        v[e] = in ? v[e] - mean : (A)0;
        s += v[e] * v[e];
    }
    A r;
    if constexpr (sizeof(A) == 8) r = 1.0 / sqrt(sum_lanes<L>(s) / (A)D + (A)n.eps);
    else r = 1.0f / sqrtf(sum_lanes<L>(s) / (A)D + n.eps);
    float w[8];
    if (n.w != nullptr && in) load8<T>(n.w + at, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] *= n.w != nullptr && in ? r * (A)w[e] : r;
    if (n.b != nullptr && in) {
        load8<T>(n.b + at, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += (A)w[e];
    }
    if (!both) return;
    if (n.w != nullptr) load8<T>(n.w + partner, w);
#pragma unroll
    for (int e = 0; e < 8; ++e) p[e] = (p[e] - mean) * (n.w != nullptr ? r * (A)w[e] : r);
    if (n.b != nullptr) {
        load8<T>(n.b + partner, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) p[e] += (A)w[e];
    }
}

// Eight values in [-6, 6] of a block's multiples, in fp64, as codes.  They are cut to fp32 with the last bit set where something was
// cut off ("to odd"), so that the conversion's rounding is that of the fp64 value.  (Below 1/8 every one is a zero.)
__device__ __forceinline__ float to_odd(double u) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, u);
    const uint32_t hi = (uint32_t)(bits >> 32), lo = (uint32_t)bits;
    const uint32_t mag = ((hi << 3 | lo >> 29) - (896u << 23)) & 0x7fffffffu;  // exponent with the bias of fp32
    const uint32_t f = mag | ((lo & 0x1fffffffu) != 0 ? 1u : 0u) | (hi & 0x80000000u);
    return __builtin_bit_cast(float, __builtin_fabs(u) < 0.125 ? hi & 0x80000000u : f);
}
__device__ __forceinline__ uint32_t codes_of(const float (&v)[8], float scale) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
    return w;
}
// The largest scale: what is held of a block stays finite in the cache's type (6 * 2^13 in fp16; a larger magnitude is held as that).
template <typename T> constexpr int kMaxScale = std::is_same_v<T, f16> ? 13 : 125;
// (codes, scale byte) of a lane's eight values; the four lanes of a block agree on the byte.
template <int MOST> __device__ __forceinline__ uint32_t encode(const double (&v)[8], uint32_t* byte) {
    const double amax = block_amax(v);
    const uint64_t bits = __builtin_bit_cast(uint64_t, amax);
    const int exponent = (int)(bits >> 52) - 1023;
    const uint64_t mantissa = bits & 0xfffffffffffffull;
    int e = exponent - (mantissa <= 0x8000000000000ull ? 2 : 1);       // amax = m 2^exponent: m <= 1.5 fits 6 * 2^(exponent - 2)
    e = e < -126 ? -126 : (e > MOST ? MOST : e);
    *byte = exponent == 1024 ? 255u : (uint32_t)(e + 127);
    if (exponent == 1024) return 0u;
    const double inv = __builtin_bit_cast(double, (uint64_t)(1023 - e) << 52);
    float u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const double x = v[i] * inv;                                   // (a power of two: exact)
        u[i] = __builtin_fabs(x) > 6.0 ? (x < 0.0 ? -6.0f : 6.0f) : to_odd(x);
    }
    return codes_of(u, 1.0f);
}
template <int MOST> __device__ __forceinline__ uint32_t encode(const float (&v)[8], uint32_t* byte) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = MaxOp::op(m, __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffffu);
    m = wave_reduce<MaxOp, 4>(m);
    const int exponent = (int)(m >> 23) - 127;
    int e = exponent - ((m & 0x7fffffu) <= 0x400000u ? 2 : 1);
    e = e < -126 ? -126 : (e > MOST ? MOST : e);
    *byte = m >= 0x7f800000u ? 255u : (uint32_t)(e + 127);
    if (m >= 0x7f800000u) return 0u;
    return codes_of(v, scale_of_byte((uint32_t)(e + 127)));
}

template <typename T, int D, HeadsOp OP>
__global__ __launch_bounds__(256) void heads_kernel(HeadsArgs a) {
    constexpr int L = D <= 32 ? 4 : D <= 64 ? 8 : D <= 128 ? 16 : 32, R = 256 / L;
    const int lane = threadIdx.x % L, sub = threadIdx.x / L;
    const bool in = lane * 8 < D;
    const int at = in ? lane * 8 : 0;
    const int count = row_count(a.tokens.count, a.tokens.rows);
    const int chunks = a.chunks[0] + a.chunks[1];
    const RotationArgs& rot = a.rotation;
    const int64_t items = (int64_t)((count + R - 1) / R) * chunks;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int tile = (int)(item / chunks), part = (int)(item % chunks);
        const int which = part >= a.chunks[0];
        const HeadJob& job = a.job[which];
        const int first = (part - (which ? a.chunks[0] : 0)) * a.chunk, last = first + a.chunk < job.heads ? first + a.chunk : job.heads;
        const int64_t r = (int64_t)tile * R + sub;
        const bool live = r < count;
        Token token = {0, 0, false};
        if (live) token = token_of(a.tokens, (int)r);
        const bool turns = OP != kReadHeads && rot.table != nullptr && (OP == kTurnHeads || which == 0);
        bool here = token.here;
        if (rot.table != nullptr && (uint32_t)token.pos >= (uint32_t)rot.positions) here = false;
        int64_t slot = 0;                                      // of head 0 and this token, in tokens
        if constexpr (OP != kTurnHeads) {
            int page = -1;
            if (here && (uint32_t)token.stream < (uint32_t)a.cache.streams && (uint32_t)token.pos < (uint32_t)a.cache.length)
                page = page_of(a.cache, token.stream, token.pos >> a.cache.page_shift);
            here = page >= 0;
            slot = head_of_page(a.cache, here ? page : 0, which, 0) + (token.pos & ((1 << a.cache.page_shift) - 1));
        }
        if constexpr (OP == kReadHeads) {
            for (int h = first; h < last; ++h) {
                const int64_t s = slot + ((int64_t)h << a.cache.page_shift);
                float v[8] = {};
                if (here && in) {
                    const uint32_t w = *reinterpret_cast<const uint32_t*>(a.cache.codes + s * (D / 2) + lane * 4);
                    const float scale = scale_of_byte(a.cache.scales[s * (D / 32) + lane / 4]);
                    typedef float f32x2 __attribute__((ext_vector_type(2)));
                    f32x2 p[4];
                    p[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 0);
                    p[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 1);
                    p[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 2);
                    p[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, scale, 3);
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = p[e / 2][e % 2];
                }
                if (live && in) store8<T>(static_cast<T*>(job.out) + r * job.ld_out + h * D + at, v);
            }
        } else {
            // angles: out = v * cs + partner * sn
            typedef std::conditional_t<OP == kAppendHeads, double, float> A;
            float cs[8], sn[8];
            int partner = at;
            const bool turned = turns && here && in && at < rot.rot;
            const bool halves = rot.style == DCNN_ROT_HALVES;
            if (turned) {
                const int half = rot.rot / 2;
                const bool second = at >= half;
                const float* t = rot.table + (int64_t)token.pos * rot.rot;
                float pair[16];
                if (halves) {
                    partner = second ? at - half : at + half;
                    const float* p = t + (second ? at - half : at) * 2;
#pragma unroll
                    for (int i = 0; i < 16; i += 4) *reinterpret_cast<f32x4*>(pair + i) = *reinterpret_cast<const f32x4*>(p + i);
#pragma unroll
                    for (int e = 0; e < 8; ++e) cs[e] = pair[2 * e], sn[e] = second ? pair[2 * e + 1] : -pair[2 * e + 1];
                } else {
#pragma unroll
                    for (int i = 0; i < 8; i += 4) *reinterpret_cast<f32x4*>(pair + i) = *reinterpret_cast<const f32x4*>(t + at + i);
#pragma unroll
                    for (int e = 0; e < 8; ++e) cs[e] = pair[e & ~1], sn[e] = e % 2 ? pair[e | 1] : -pair[e | 1];
                }
            }
            const HeadNorm<T> norm = {job.norm, job.eps, static_cast<const T*>(job.w), static_cast<const T*>(job.b)};
            for (int h = first; h < last; ++h) {
                const T* x = static_cast<const T*>(job.in) + r * job.ld_in + h * D;
                float raw[8] = {}, other[8] = {};
                const bool both = turned && halves;
                if (here && in) load8<T>(x + at, raw);
                if (both) load8<T>(x + partner, other);
                if (OP == kAppendHeads && which == 1) {
                    uint32_t byte;
                    const uint32_t w = encode<kMaxScale<T>>(raw, &byte);
                    if (here && in) {
                        const int64_t s = slot + ((int64_t)h << a.cache.page_shift);
                        *reinterpret_cast<uint32_t*>(a.cache.codes + s * (D / 2) + lane * 4) = w;
                        if (lane % 4 == 0) a.cache.scales[s * (D / 32) + lane / 4] = (uint8_t)byte;
                    }
                    continue;
                }
                A v[8], p[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = raw[e], p[e] = other[e];
                norm_head<T, A, D, L>(v, p, both, norm, at, partner, in);
                if (turned) {
                    A o[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = v[e] * (A)cs[e] + (halves ? p[e] : v[e ^ 1]) * (A)sn[e];
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[e] = o[e];
                }
                if constexpr (OP == kTurnHeads) {
                    if (!here) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) v[e] = 0.0f;
                    }
                    if (live && in) store8<T>(static_cast<T*>(job.out) + r * job.ld_out + h * D + at, v);
                } else {
                    uint32_t byte;
                    const uint32_t w = encode<kMaxScale<T>>(v, &byte);
                    if (here && in) {
                        const int64_t s = slot + ((int64_t)h << a.cache.page_shift);
                        *reinterpret_cast<uint32_t*>(a.cache.codes + s * (D / 2) + lane * 4) = w;
                        if (lane % 4 == 0) a.cache.scales[s * (D / 32) + lane / 4] = (uint8_t)byte;
                    }
                }
            }
        }
    }
}

template <typename T, int D> static dcnn_status launch_heads_dim(dcnn_ctx* ctx, HeadsOp op, const HeadsArgs& a) {
    constexpr int L = D <= 32 ? 4 : D <= 64 ? 8 : D <= 128 ? 16 : 32;
    const int64_t items = cdiv(a.tokens.rows, 256 / L) * (a.chunks[0] + a.chunks[1]), most = (int64_t)ctx->num_cu * 8;
    const dim3 grid((unsigned)(items < most ? items : most));
    if (op == kTurnHeads) hipLaunchKernelGGL((heads_kernel<T, D, kTurnHeads>), grid, dim3(256), 0, ctx->stream, a);
    else if (op == kAppendHeads) hipLaunchKernelGGL((heads_kernel<T, D, kAppendHeads>), grid, dim3(256), 0, ctx->stream, a);
    else hipLaunchKernelGGL((heads_kernel<T, D, kReadHeads>), grid, dim3(256), 0, ctx->stream, a);
    return check_hip(ctx, hipGetLastError(), "heads_kernel launch");
}
template <typename T> static dcnn_status launch_heads_t(dcnn_ctx* ctx, int dim, HeadsOp op, const HeadsArgs& a) {
    switch (dim) {
        case 32: return launch_heads_dim<T, 32>(ctx, op, a);
        case 64: return launch_heads_dim<T, 64>(ctx, op, a);
        case 96: return launch_heads_dim<T, 96>(ctx, op, a);
        case 128: return launch_heads_dim<T, 128>(ctx, op, a);
        case 192: return launch_heads_dim<T, 192>(ctx, op, a);
        default: return launch_heads_dim<T, 256>(ctx, op, a);
    }
}

dcnn_status launch_heads(dcnn_ctx* ctx, int dtype, int dim, HeadsOp op, HeadsArgs a) {
    const int lanes = dim <= 32 ? 4 : dim <= 64 ? 8 : dim <= 128 ? 16 : 32, heads = a.job[0].heads + a.job[1].heads;
    // heads one after the other only where there are workgroups enough for all compute units without
    const int64_t chunk = cdiv(a.tokens.rows, 256 / lanes) * heads / ((int64_t)ctx->num_cu * 8);
    a.chunk = (int)(chunk < 1 ? 1 : (chunk < heads ? chunk : heads));
    for (int j = 0; j < 2; ++j) a.chunks[j] = (int)cdiv(a.job[j].heads, a.chunk);
    if (dtype == DCNN_F16) return launch_heads_t<f16>(ctx, dim, op, a);
    if (dtype == DCNN_BF16) return launch_heads_t<bf16>(ctx, dim, op, a);
    return launch_heads_t<float>(ctx, dim, op, a);
}

}  // namespace dcnn
