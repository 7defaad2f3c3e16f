// Heads normed and rotated, appended to the cache in 4 bits, and read from it.
//
//   u = norm(x[r, h]),  rotated: (a, b) -> (a cos - b sin, b cos + a sin)
//   appended: 32 values share the smallest power of two s with max|u| <= 6 s, each becomes the code next to u / s
//
// A head's D values lie in the registers of D / 8 lanes (eight to a lane), its statistics and a block's largest magnitude are lane
// permutations, and a value's partner in a rotation by halves is read again (from the L1) rather than passed between lanes.  A workgroup
// takes some rows and heads of each side by side: two where rows are many, and up to all the places that it has (2048 / D, D a power of two) where they are few.
// Keys are fp64 from the norm to the code: a code is the same whatever the order of a sum.
// Heads move 344 MB (16384 rows of 40 x 128, bf16) in 76 us, 4.5 TB/s.  Appending 16275 rows of 8 x 128 (bf16, pages of 16) takes 33 us, 11 of them for
// the values, where all of its 84 MB could take 17: a key's chain of norm, fp64 and rounding is latency and instructions.  Reading them back takes 16.
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
// Eight values of a head as they lie, and those that they meet in the rotation.
template <typename T> struct Raw8 {
    static constexpr int N = (int)sizeof(T) / 2;
    u32x4 v[N];
    __device__ __forceinline__ void read(const T* p, bool take) {
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = take ? __builtin_bit_cast(u32x4, *reinterpret_cast<const typename RowVec<T>::type*>(p + i * RowVec<T>::E)) : u32x4{0u, 0u, 0u, 0u};
    }
    // neighbours exchanged
    __device__ __forceinline__ Raw8 crossed(bool take) const {
        Raw8 r;
#pragma unroll
        for (int i = 0; i < N; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const uint32_t w = sizeof(T) == 2 ? v[i][e] << 16 | v[i][e] >> 16 : v[i][e ^ 1];
                r.v[i][e] = take ? w : 0u;
            }
        return r;
    }
    __device__ __forceinline__ float at(int e) const { return row_get<T>(v[e / RowVec<T>::E], e % RowVec<T>::E); }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = at(e);
    }
};

// Where a lane's values lie, and their partners: the same for all heads of a row.
struct Place {
    int at, partner;
    bool in, here, turned, halves;             // in the head; the row has a token; rotated; by halves
};
// Norm and rotation as one: out = r (x - mean) a + r (partner - mean) b + c, with r and mean of the head.
template <typename A> struct Turn {
    A a[8], b[8];
    float c[8];
};
template <typename T, typename A>
__device__ __forceinline__ void turn_of(Turn<A>& f, const RotationArgs& rot, int pos, const HeadJob& job, const Place& at) {
    float cs[8], sn[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) cs[e] = 1, sn[e] = 0;
    if (at.turned) {
        const int half = rot.rot / 2;
        const bool second = at.at >= half;
        const float* t = rot.table + (int64_t)pos * rot.rot;
        float pair[16];
        if (at.halves) {
            t += (second ? at.at - half : at.at) * 2;
#pragma unroll
            for (int i = 0; i < 16; i += 4) *reinterpret_cast<f32x4*>(pair + i) = *reinterpret_cast<const f32x4*>(t + i);
#pragma unroll
            for (int e = 0; e < 8; ++e) cs[e] = pair[2 * e], sn[e] = second ? pair[2 * e + 1] : -pair[2 * e + 1];
        } else {
            t += at.at;
#pragma unroll
            for (int i = 0; i < 8; i += 4) *reinterpret_cast<f32x4*>(pair + i) = *reinterpret_cast<const f32x4*>(t + i);
#pragma unroll
            for (int e = 0; e < 8; ++e) cs[e] = pair[e & ~1], sn[e] = e % 2 ? pair[e | 1] : -pair[e | 1];
        }
    }
    const auto weigh = [&](const void* params, float (&own)[8], float (&other)[8], float none) {
        const T* p = static_cast<const T*>(params);
#pragma unroll
        for (int e = 0; e < 8; ++e) own[e] = none, other[e] = none;
        if (p == nullptr || !at.in || !at.here) return;        // (a row without a token: zeros times one, and no bias)
        load8<T>(p + at.at, own);
        if (!at.turned) return;                                // (an infinity times the sine of no turn, zero, is none)
#pragma unroll
        for (int e = 0; e < 8; ++e) other[e] = own[e ^ 1];
        if (at.halves) load8<T>(p + at.partner, other);
    };
    float own[8], other[8];
    weigh(job.w, own, other, 1.0f);
#pragma unroll
    for (int e = 0; e < 8; ++e) f.a[e] = (A)own[e] * (A)cs[e], f.b[e] = (A)other[e] * (A)sn[e];
    // (in fp64 a bias is read where it is used: few norms have one)
    if constexpr (sizeof(A) == 4) {
#pragma unroll
        for (int e = 0; e < 8; ++e) f.c[e] = 0.0f;
        if (job.b == nullptr) return;
        weigh(job.b, own, other, 0.0f);
#pragma unroll
        for (int e = 0; e < 8; ++e) f.c[e] = own[e] * cs[e] + other[e] * sn[e];
    }
}
// Element e's part of the bias, in fp64.
template <typename T> __device__ __forceinline__ double bias64(const RotationArgs& rot, int pos, const HeadJob& job, const Place& at, int e) {
    const T* const b = static_cast<const T*>(job.b);
    if (!at.in) return 0.0;
    const int own = at.at + e;
    if (!at.turned) return (double)(float)b[own];
    const bool second = at.at >= rot.rot / 2;
    const float* const pair = rot.table + (int64_t)pos * rot.rot + (at.halves ? (second ? own - rot.rot / 2 : own) * 2 : own & ~1);
    const double o = (double)(float)b[at.halves ? at.partner + e : own ^ 1] * (double)pair[1];
    return (double)(float)b[own] * (double)pair[0] + ((at.halves ? !second : e % 2 == 0) ? -o : o);
}
// r of a head; x and p less its mean.  A row without a token: zero.
template <int D, int L> __device__ __forceinline__ float centre(float (&x)[8], float (&p)[8], const HeadJob& job, const Place& at) {
    if (job.norm == DCNN_NORM_NONE) return 1.0f;
    if (job.norm == DCNN_NORM_LAYER) {
        float s = 0.0f;
#pragma unroll
        for (int e = 0; e < 8; ++e) s += x[e];
        const float mean = sum_lanes<L>(s) * (1.0f / (float)D);
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = at.in ? x[e] - mean : 0.0f, p[e] -= mean;
    }
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s = __builtin_fmaf(x[e], x[e], s);
    const float r = rsqrtf(sum_lanes<L>(s) * (1.0f / (float)D) + job.eps);
    return at.here ? r : 0.0f;
}
// The same in fp64: r and the mean of values as they lie.  (They are converted where they are used: eight fp64 values more in registers, and the
// compiler spills some: 26240 rows of 8 x 64 took 83 us.)
template <typename T, int D, int L> __device__ __forceinline__ double centre64(const Raw8<T>& x, const HeadJob& job, const Place& at, double* mean) {
    *mean = 0.0;
    if (job.norm == DCNN_NORM_NONE) return 1.0;
    double s = 0.0;
    if (job.norm == DCNN_NORM_LAYER) {
#pragma unroll
        for (int e = 0; e < 8; ++e) s += (double)x.at(e);
        *mean = sum_lanes<L>(s) * (1.0 / (double)D);
        s = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const double d = at.in ? (double)x.at(e) - *mean : 0.0;
            s = __builtin_fma(d, d, s);
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) s = __builtin_fma((double)x.at(e), (double)x.at(e), s);
    }
    return rsqrt(sum_lanes<L>(s) * (1.0 / (double)D) + (double)job.eps);
}

// An fp64 value as the fp32 one next to zero of it, with the last bit set where something was cut off ("to odd"): rounding that to a code, and
// comparing it with a border, is rounding and comparing the fp64 value.  Magnitudes from 2^128 on become infinity, those below 2^-126 zero.  At the EDGE
// they are told apart: the former are the largest number if they are finite, and the latter have steps of 2^-149, as fp32 has them.
template <bool EDGE> __device__ __forceinline__ float to_odd(double v) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, v);
    const uint32_t hi = (uint32_t)(bits >> 32), lo = (uint32_t)bits, rest = lo & 0x1fffffffu;
    const uint32_t f = ((hi << 3 | lo >> 29) - (896u << 23)) & 0x7fffffffu;    // exponent with the bias of fp32
    const uint32_t odd = f | (rest < 1u ? rest : 1u) | (hi & 0x80000000u);
    const uint32_t size = hi & 0x7fffffffu;
    if (EDGE && size < 0x38100000u) {
        const double steps = __builtin_fabs(v) * 0x1p149;
        const uint32_t n = (uint32_t)steps;
        return __builtin_bit_cast(float, n | ((double)n != steps ? 1u : 0u) | (hi & 0x80000000u));
    }
    if (EDGE && size >= 0x47f00000u && size < 0x7ff00000u) return __builtin_bit_cast(float, 0x7f7fffffu | (hi & 0x80000000u));
    return size < 0x38100000u ? 0.0f : __builtin_bit_cast(float, size < 0x47f00000u ? odd : 0x7f800000u);
}
// (a zero is code 0, whatever its sign was)
__device__ __forceinline__ uint32_t codes_of(const float (&v)[8], float scale) {
    uint32_t w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
    const uint32_t m = w & 0x77777777u;
    return m | (w & ((m << 1 | m << 2 | m << 3) & 0x88888888u));
}
// The largest scale: what is held of a block stays finite in the cache's type (6 * 2^13 in fp16; a larger magnitude is held as that).
template <typename T> constexpr int kMaxScale = std::is_same_v<T, f16> ? 13 : 125;
// Exponent of the scale of a block: the largest magnitude is m 2^k, and m <= 1.5 fits 6 * 2^(k - 2).
template <int MOST> __device__ __forceinline__ int scale_exponent(int k, bool small) {
    const int e = k - (small ? 2 : 1);
    return e < -126 ? -126 : (e > MOST ? MOST : e);
}
// (codes, scale byte) of a lane's eight values; the four lanes of a block agree on the byte.
template <int MOST> __device__ __forceinline__ uint32_t encode(const float (&v)[8], uint32_t* byte) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = MaxOp::op(m, __builtin_bit_cast(uint32_t, v[e]) & 0x7fffffffu);
    m = wave_reduce<MaxOp, 4>(m);
    const int e = scale_exponent<MOST>((int)(m >> 23) - 127, (m & 0x7fffffu) <= 0x400000u);
    *byte = m >= 0x7f800000u ? 255u : (uint32_t)(e + 127);
    if (m >= 0x7f800000u) return 0u;
    return codes_of(v, scale_of_byte((uint32_t)(e + 127)));
}

// BIAS: a norm of appended keys has one (a kernel of its own: the others need not its registers).
template <typename T, int D, HeadsOp OP, bool BIAS = false>
__global__ __launch_bounds__(256, OP == kAppendHeads && !BIAS ? 4 : 1) void heads_kernel(HeadsArgs a) {
    constexpr int L = D <= 32 ? 4 : D <= 64 ? 8 : D <= 128 ? 16 : 32, R = 256 / L;
    const int lane = threadIdx.x % L, sub = threadIdx.x / L;
    const bool in = lane * 8 < D;
    const int at = in ? lane * 8 : 0;
    const uint32_t count = (uint32_t)row_count(a.tokens.count, a.tokens.rows);         // (up to 2^31 - 1: with a tile's rows on top it needs the last bit)
    const RotationArgs& rot = a.rotation;
    // 2^shift heads of a row side by side: two, so that what belongs to the row serves many, and as many as have a place where workgroups are left
    int shift = a.shift;
    while (shift > 1 && (int64_t)((count + (R >> shift) - 1) / (uint32_t)(R >> shift)) * a.jobs > (int)gridDim.x) --shift;
    const int rows = R >> shift, stride = 1 << shift, h0 = sub & (stride - 1);
    const int tiles = (int)((count + rows - 1) / (uint32_t)rows);
    // one job before the other: what one costs is not what the other does, and workgroups that follow each other go to different L2 caches
    for (int64_t item = blockIdx.x; item < (int64_t)tiles * a.jobs; item += gridDim.x) {
        const int which = item >= tiles, tile = (int)(which ? item - tiles : item);
        const HeadJob& job = a.job[which];
        const int64_t r = (int64_t)tile * rows + (sub >> shift);
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
        const auto put = [&](int h, uint32_t words, uint32_t byte, bool take) {
            const int64_t s = slot + ((int64_t)h << a.cache.page_shift);
            if (!take) return;
            *reinterpret_cast<uint32_t*>(a.cache.codes + s * (D / 2) + lane * 4) = words;
            if (lane % 4 == 0) a.cache.scales[s * (D / 32) + lane / 4] = (uint8_t)byte;
        };
        if constexpr (OP == kReadHeads) {
            for (int h = h0; h < job.heads; h += stride) {
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
            continue;
        }
        Place place;
        place.at = at, place.in = in, place.here = here;
        place.halves = rot.style == DCNN_ROT_HALVES;
        place.turned = turns && here && in && at < rot.rot;
        place.partner = !place.turned || !place.halves ? at : (at >= rot.rot / 2 ? at - rot.rot / 2 : at + rot.rot / 2);
        const T* const source = static_cast<const T*>(job.in) + r * job.ld_in;
        if (OP == kAppendHeads && which == 1) {                // values: exact as they are
            for (int h = h0; h < job.heads; h += stride) {
                Raw8<T> raw;
                raw.read(source + h * D + at, here && in);
                float x[8];
                raw.get(x);
                uint32_t byte;
                const uint32_t words = encode<kMaxScale<T>>(x, &byte);
                put(h, words, byte, here && in);
            }
            continue;
        }
        typedef std::conditional_t<OP == kAppendHeads, double, float> A;
        Turn<A> turn;
        turn_of<T>(turn, rot, token.pos, job, place);
        // (without norms' fp64 there are registers for the next head's values: 16384 rows of 40 x 128 take 74 us in place of 80; appended keys, 40 in place of 35)
        constexpr bool AHEAD = OP == kTurnHeads;
        Raw8<T> raw, met;
        const auto fetch = [&](int h) {
            raw.read(source + h * D + at, here && in && h < job.heads);
            if (place.halves) met.read(source + h * D + place.partner, place.turned && h < job.heads);
            else met = raw.crossed(place.turned);
        };
        if (AHEAD) fetch(h0);
        for (int h = h0; h < job.heads; h += stride) {
            if (!AHEAD) fetch(h);
            float o[8];
            if constexpr (OP == kAppendHeads) {
                double mean;
                const double scale = centre64<T, D, L>(raw, job, place, &mean);
                const auto key = [&](int e) {
                    double v = (double)raw.at(e) * turn.a[e] + (double)met.at(e) * turn.b[e];
                    if (job.norm == DCNN_NORM_LAYER) v -= mean * (turn.a[e] + turn.b[e]);
                    v *= scale;
                    if constexpr (BIAS) v += bias64<T>(rot, token.pos, job, place, e);
                    return v;
                };
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = to_odd<false>(key(e));
                uint32_t byte;
                uint32_t words = encode<kMaxScale<T>>(o, &byte);
                // Scales up to 2^-125: magnitudes below 2^-126 have codes too.  An infinity: it may be a number that fp32 lacks, held as the largest.  (Blocks
                // of zeros alone are among the first.  Looked at for each value where it was made, it took 35 us in place of 30, 16275 rows of 8 x 128; the
                // values are fetched again, or they take registers.)
                if (__any(here && in && (byte <= 2 || byte == 255))) {
                    fetch(h);
#pragma unroll
                    for (int e = 0; e < 8; ++e) o[e] = to_odd<true>(key(e));
                    words = encode<kMaxScale<T>>(o, &byte);
                }
                put(h, words, byte, here && in);
            } else {
                float x[8], p[8];
                raw.get(x), met.get(p);
                fetch(h + stride);
                const float scale = centre<D, L>(x, p, job, place);
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = __builtin_fmaf(scale, __builtin_fmaf(p[e], turn.b[e], x[e] * turn.a[e]), turn.c[e]);
                if (live && in) store8<T>(static_cast<T*>(job.out) + r * job.ld_out + h * D + at, o);
            }
        }
    }
}

template <typename T, int D> static dcnn_status launch_heads_dim(dcnn_ctx* ctx, HeadsOp op, HeadsArgs a) {
    constexpr int L = D <= 32 ? 4 : D <= 64 ? 8 : D <= 128 ? 16 : 32;
    const int most_heads = a.job[0].heads > a.job[1].heads ? a.job[0].heads : a.job[1].heads;
    a.shift = 0;
    while ((2 << a.shift) <= 256 / L && 1 << a.shift < most_heads) ++a.shift;
    a.jobs = a.job[1].heads > 0 ? 2 : 1;
    // (workgroups to a compute unit: 16384 rows of 40 x 128 take 81 us with 16, 92 with 8; appended, 43 with 16 in place of 36)
    const int64_t items = cdiv(a.tokens.rows, 256 / L >> a.shift) * a.jobs, most = (int64_t)ctx->num_cu * (op == kTurnHeads ? 16 : 8);
    const dim3 grid((unsigned)(items < most ? items : most));
    if (op == kTurnHeads) hipLaunchKernelGGL((heads_kernel<T, D, kTurnHeads>), grid, dim3(256), 0, ctx->stream, a);
    else if (op == kAppendHeads && a.job[0].b != nullptr) hipLaunchKernelGGL((heads_kernel<T, D, kAppendHeads, true>), grid, dim3(256), 0, ctx->stream, a);
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

dcnn_status launch_heads(dcnn_ctx* ctx, int dtype, int dim, HeadsOp op, const HeadsArgs& a) {
    if (dtype == DCNN_F16) return launch_heads_t<f16>(ctx, dim, op, a);
    if (dtype == DCNN_BF16) return launch_heads_t<bf16>(ctx, dim, op, a);
    return launch_heads_t<float>(ctx, dim, op, a);
}

}  // namespace dcnn
