// Attention over the cache for rows by themselves: one of each stream, or some (attend_plan).
//
//   S = K q,  p = exp2(S * scale log2(e) - max),  y = V^T p / sum p, the maximum and the sums kept up to date from tile to tile
//
// The cache is read once and nothing else is large: HBM bounds it, so every step serves to keep loads in flight.  A workgroup has one row, one
// head of keys and up to 16 query heads of it (the columns of an operand) at a time; its four waves go through tiles of 64 tokens in turn, each
// with its own sums, which are joined at the end.  A tile:
//   * lane (g, i), g = lane / 16, i = lane % 16.  Operand rows are tokens in the order that puts the products of tokens 16 g .. 16 g + 15
//     into lane group g: row i of the kt-th sixteen is token 16 (i / 4) + 4 kt + i % 4.  Group g multiplies the words [g NB, (g + 1) NB) of a
//     token's codes: one wide load, mostly one scale.
//   * values lie in LDS as they came (rows of D / 2 bytes, columns of 16 bytes permuted against bank conflicts) and are read transposed: 16
//     tokens of a channel to a lane, the ones whose weights the lane has.  Their 16 scales come straight from the cache.
//   * codes become operands by conversions that take the scale: one instruction for two values.
// The next tile's codes and scales are in flight meanwhile.  Where rows are long, the tokens of all of them are dealt out evenly to as many workgroups
// as are resident (two to a compute unit), whatever the rows' lengths, and attend_join_kernel makes their parts one.
// Measured (32 heads on 8 of 128, bf16 and fp16): 64 rows of up to 8192 tokens, 309 MB, 67 us, 4.6 TB/s; one row of 262143, 285 MB, 57 us, 5.0 TB/s.
#include "attend_device.h"

namespace dcnn {

typedef __attribute__((address_space(3))) i32x2 lds_i32x2;

// A tile's part of a lane.
template <int NB> struct KvTile {
    uint32_t k[4][NB];
    uint32_t ks[4][2];                         // scale bytes of a word's block: the first and the last word's
    u32x4 v[NB];
    u32x4 vs[NB];                              // 16 tokens, NB bytes each
    bool page;                                 // the lane's sixteen tokens have a page
};

template <int NB> __device__ __forceinline__ int value_column(int row, int col) {
    if constexpr (NB == 2 || NB == 6) return col ^ (row >> 3 & 1);
    if constexpr (NB == 4) return col ^ (row >> 2 & 3);
    if constexpr (NB == 8) return col ^ (row >> 1 & 7);
    return col;
}

// The page of a tile (WHOLE: pages hold whole tiles), or of its sixteen tokens `lane % 4`.
template <bool WHOLE> __device__ __forceinline__ int tile_page(const CacheArgs& c, int stream, int first, int lane) {
    if constexpr (WHOLE) return page_of_all(c, stream, first >> c.page_shift);
    else return page_of(c, stream, (first + 16 * (lane & 3)) >> c.page_shift);
}

template <int NB, bool WHOLE> __device__ __forceinline__ void load_tile(KvTile<NB>& t, const CacheArgs& c, int page, int head, int first, int lane) {
    constexpr int ROW = NB * 16;
    const int g = lane / 16, i = lane % 16, mask = (1 << c.page_shift) - 1;
    const int64_t page_tokens = (int64_t)c.heads << c.page_shift;      // tokens of a page's keys, or values
    // where sixteen tokens of the page `p` begin; with whole tiles that is the same for all lanes, and what differs between them are 32-bit offsets
    const auto token_at = [&](int p, int group, int which) {
        return ((int64_t)(p < 0 ? 0 : p) * 2 + which) * page_tokens + ((int64_t)head << c.page_shift) + ((first + 16 * group) & mask);
    };
    const int64_t keys = WHOLE ? token_at(page, 0, 0) : token_at(__shfl(page, i / 4, kWave), i / 4, 0);
    const uint32_t row = (WHOLE ? 16 * (i / 4) : 0) + i % 4;
    const uint8_t *const kp = c.codes + keys * ROW, *const sp = c.scales + keys * NB;
#pragma unroll
    for (int kt = 0; kt < 4; ++kt) {
#pragma unroll
        for (int j = 0; j < NB; ++j) t.k[kt][j] = *reinterpret_cast<const uint32_t*>(kp + (row * ROW + g * NB * 4 + kt * 4 * ROW + j * 4));
        t.ks[kt][0] = sp[row * NB + kt * 4 * NB + g * NB / 4];
        if constexpr (NB % 4 != 0 && NB > 2) t.ks[kt][1] = sp[row * NB + kt * 4 * NB + (g * NB + NB - 1) / 4];
        if constexpr (NB == 8) t.ks[kt][1] = sp[row * NB + kt * 4 * NB + g * 2 + 1];
    }
    if constexpr (WHOLE) {
        const int64_t values = token_at(page, 0, 1);
        const uint8_t *const vp = c.codes + values * ROW, *const wp = c.scales + values * NB;
#pragma unroll
        for (int n = 0; n < NB; ++n) t.v[n] = *reinterpret_cast<const u32x4*>(vp + (uint32_t)(lane * 16 + n * 1024));
#pragma unroll
        for (int n = 0; n < NB; ++n) t.vs[n] = *reinterpret_cast<const u32x4*>(wp + (uint32_t)(g * 16 * NB + n * 16));
        t.page = page >= 0;
    } else {
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            const int chunk = lane + 64 * n, group = chunk / (16 * NB), within = chunk % (16 * NB);
            const int64_t at = token_at(__shfl(page, group, kWave), group, 1);
            t.v[n] = *reinterpret_cast<const u32x4*>(c.codes + at * ROW + within * 16);
        }
        const int v_page = __shfl(page, g, kWave);
        t.page = v_page >= 0;
        const u32x4* wp = reinterpret_cast<const u32x4*>(c.scales + token_at(v_page, g, 1) * NB);
#pragma unroll
        for (int n = 0; n < NB; ++n) t.vs[n] = wp[n];
    }
}

// Scale of token e and block b among a lane's value scales, as a conversion takes it.
template <int NB> __device__ __forceinline__ float value_scale(const u32x4 (&vs)[NB], int e, int b) {
    const int byte = e * NB + b, word = byte / 4, at = byte % 4;
    const uint32_t w = vs[word / 4][word % 4];
    return __builtin_bit_cast(float, at == 3 ? w >> 1 : w << (23 - 8 * at));
}

__device__ __forceinline__ int tiles_of(const Span& s) { return (s.hi - (s.lo & ~63) + 63) / 64; }

template <typename T, int NB, bool WHOLE>
__global__ __launch_bounds__(256, NB * Operand<T>::TERMS <= 6 ? 2 : 1) void attend_few_kernel(AttendArgs a) {
    typedef Operand<T> O;
    typedef typename O::type Op;
    constexpr int D = NB * 32, ROW = NB * 16, TERMS = O::TERMS;
    __shared__ __attribute__((aligned(16))) uint8_t lds[4 * 64 * ROW];         // values of the waves' tiles, then sums
    __shared__ float stat[4][16][2];
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave), g = lane / 16, i = lane % 16;
    uint8_t* const mine = lds + wave * 64 * ROW;
    // the rows' tiles of tokens, one row's behind the other's: each of the workgroups of a head takes as many of them
    __shared__ int before[kShareRows + 1], row_stream[kShareRows], row_lo[kShareRows], row_hi[kShareRows], wave_sum[4];
    const int count = row_count(a.tokens.count, a.tokens.rows);
    const int shares = a.splits, column_blocks = a.cache.heads * a.blocks;
    int first_row, last_row, begin = 0, end = 0, total_tiles = 0, hb, share_index = 0, share_tiles = 0;
    if (shares > 0) {
        constexpr int PER = kShareRows / 256;
        hb = blockIdx.x % column_blocks, share_index = blockIdx.x / column_blocks;
        int mine_tiles[PER], sum_tiles = 0;
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int r = threadIdx.x * PER + k;
            Span span = {0, 0};
            Token token = {0, 0, false};
            if (r < count) {
                token = token_of(a.tokens, r);
                span = span_of(a, token);
            }
            row_stream[r] = token.stream, row_lo[r] = span.lo, row_hi[r] = span.hi;
            mine_tiles[k] = tiles_of(span);
            sum_tiles += mine_tiles[k];
        }
        int scan = sum_tiles;
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) {
            const int other = __shfl_up(scan, d, kWave);
            if (lane >= d) scan += other;
        }
        if (lane == kWave - 1) wave_sum[wave] = scan;
        __syncthreads();
        int at = scan - sum_tiles;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            if (w < wave) at += wave_sum[w];
            total_tiles += wave_sum[w];
        }
#pragma unroll
        for (int k = 0; k < PER; ++k) before[threadIdx.x * PER + k] = at, at += mine_tiles[k];
        if (threadIdx.x == 255) before[kShareRows] = at;
        __syncthreads();
        share_tiles = share_of(total_tiles, shares);
        if (blockIdx.x == 0) {                                 // (what the joining kernel goes by)
            for (int r = threadIdx.x; r <= count; r += 256) a.plan[1 + r] = before[r];
            if (threadIdx.x == 0) a.plan[0] = share_tiles;
        }
        begin = share_index * share_tiles, end = begin + share_tiles < total_tiles ? begin + share_tiles : total_tiles;
        if (begin >= total_tiles && share_index > 0) return;
        // the first row that begins here or later, or the one before it, if that reaches into this part
        int low = 0, high = count;
        while (low < high) {
            const int middle = (low + high) / 2;
            if (before[middle] < begin) low = middle + 1;
            else high = middle;
        }
        first_row = low > 0 && (low == count || before[low] > begin) ? low - 1 : low;
        last_row = count;
    } else {
        first_row = 0, last_row = 0, hb = 0;
    }
    // one row after the other of this part, or, where rows are many, of all that this workgroup strides through
    const int64_t units = (int64_t)count * column_blocks;
    int row = first_row;
    for (int64_t item = blockIdx.x;; item += gridDim.x, ++row) {
        int r, from, to, start;
        Span span;
        int stream;
        if (shares > 0) {
            if (row >= last_row || !(before[row] < end || (before[row] == total_tiles && end == total_tiles))) break;
            r = row;
            span.lo = row_lo[r], span.hi = row_hi[r], stream = row_stream[r];
            from = begin > before[r] ? begin - before[r] : 0, to = (end < before[r + 1] ? end : before[r + 1]) - before[r];
        } else {
            if (item >= units) break;
            r = (int)(item / column_blocks), hb = (int)(item % column_blocks);
            const Token token = token_of(a.tokens, r);
            span = span_of(a, token), stream = token.stream;
            from = 0, to = tiles_of(span);
        }
        // (the same for all lanes, and the compiler is told: what is made of it takes no vector registers)
        r = __builtin_amdgcn_readfirstlane(r), stream = __builtin_amdgcn_readfirstlane(stream);
        from = __builtin_amdgcn_readfirstlane(from), to = __builtin_amdgcn_readfirstlane(to);
        span.lo = __builtin_amdgcn_readfirstlane(span.lo), span.hi = __builtin_amdgcn_readfirstlane(span.hi);
        start = span.lo & ~63;
        const bool whole = from == 0 && to == tiles_of(span);
        const int block = hb % a.blocks, head = hb / a.blocks;
        // this lane's query head, and its values that meet the lane's part of a key
        const int column = block * 16 + i;
        const bool asks = column < a.group;
        const T* q = static_cast<const T*>(a.q) + (int64_t)r * a.ldq + ((int64_t)head * a.group + (asks ? column : 0)) * D + g * NB * 8;
        Op qo[NB][TERMS];
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            load_operand<T>(q + j * 8, a.negate, qo[j]);
            if (!asks) {
#pragma unroll
                for (int t = 0; t < TERMS; ++t) qo[j][t] = Op{};
            }
        }
        f32x4 o[2 * NB];
#pragma unroll
        for (int d = 0; d < 2 * NB; ++d) o[d] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
        float top = -INFINITY, sum = 0.0f;

        int tile = from + wave;
        KvTile<NB> tiles_ahead[2];
        int page = -1;
        const auto page_at = [&](int t) { return tile_page<WHOLE>(a.cache, stream, start + t * 64, lane); };
        if (tile < to) {
            page = page_at(tile);
            load_tile<NB, WHOLE>(tiles_ahead[0], a.cache, page, head, start + tile * 64, lane);
            if (tile + 4 < to) page = page_at(tile + 4);
        }
        // a tile in work while the next one's codes are on the way, into the other of two places
        const auto work = [&](KvTile<NB>& now, KvTile<NB>& next) {
            const int first = start + tile * 64;
            // (a wave's accesses to LDS follow each other: what it reads of the tile before has been read)
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                const int chunk = lane + 64 * n, row = chunk / NB, col = chunk % NB;
                *reinterpret_cast<u32x4*>(mine + row * ROW + value_column<NB>(row, col) * 16) = now.v[n];
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            if (tile + 4 < to) {
                load_tile<NB, WHOLE>(next, a.cache, page, head, first + 256, lane);
                if (tile + 8 < to) page = page_at(tile + 8);
            }
            float p[16];
#pragma unroll
            for (int kt = 0; kt < 4; ++kt) {
                f32x4 s = {0.0f, 0.0f, 0.0f, 0.0f};
                const float s0 = scale_of_byte(now.ks[kt][0]), s1 = NB % 4 != 0 && NB <= 2 ? s0 : NB == 4 ? s0 : scale_of_byte(now.ks[kt][1]);
#pragma unroll
                for (int j = 0; j < NB; ++j) {
                    const float sj = (NB == 8 ? j < 4 : (g * NB + j) / 4 == g * NB / 4) ? s0 : s1;
                    const Op k = decode8<T>(now.k[kt][j], sj);
#pragma unroll
                    for (int t = 0; t < TERMS; ++t) s = O::mfma16(k, qo[j][t], s);
                }
#pragma unroll
                for (int e = 0; e < 4; ++e) p[kt * 4 + e] = s[e];
            }
            // the lane's column, tokens first + 16 g + 0 .. 15
            if (__builtin_amdgcn_readfirstlane(first < span.lo || first + 64 > span.hi || !__all(now.page))) {
                const int t = first + 16 * g;
                uint32_t seen = 0;
#pragma unroll
                for (int e = 0; e < 16; ++e) seen |= now.page && t + e >= span.lo && t + e < span.hi ? 1u << e : 0u;
#pragma unroll
                for (int e = 0; e < 16; ++e) p[e] = seen >> e & 1 ? p[e] : -INFINITY;
                // (what lies in masked places may be anything, and a zero times NaN is one: their values' scales become the smallest)
#pragma unroll
                for (int w = 0; w < 4 * NB; ++w) {
                    uint32_t keep = 0;
#pragma unroll
                    for (int byte = 0; byte < 4; ++byte) keep |= seen >> ((4 * w + byte) / NB) & 1 ? 0xffu << 8 * byte : 0u;
                    now.vs[w / 4][w % 4] &= keep;
                }
            }
            float m = p[0];
#pragma unroll
            for (int e = 1; e < 16; ++e) m = fmaxf(m, p[e]);
            m = fmaxf(m, __shfl_xor(m, 16, kWave));
            m = fmaxf(m, __shfl_xor(m, 32, kWave));
            m = fmaxf(m * a.factor, top);                              // (the factor is above zero)
            if (__any(m > top)) {
                const float factor = m > top ? __builtin_amdgcn_exp2f(top - m) : 1.0f;        // (top may be -inf: 0)
                top = m;
                sum *= factor;
#pragma unroll
                for (int d = 0; d < 2 * NB; ++d) o[d] *= factor;
            }
            const float base = top == -INFINITY ? 0.0f : top - O::RAISE;       // (sums of weights and of values are raised alike)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                p[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[e], a.factor, -base));
                sum += p[e];
            }
            Op w[2][TERMS];
#pragma unroll
            for (int s = 0; s < 2; ++s) O::split(*reinterpret_cast<const float(*)[8]>(p + 8 * s), w[s]);
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                float vs[2][8];
#pragma unroll
                for (int e = 0; e < 16; ++e) vs[e / 8][e % 8] = value_scale<NB>(now.vs, e, b);
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    const int d = 2 * b + half;
                    const i32x2 v = __builtin_amdgcn_ds_read_tr4_b64_v2i32((lds_i32x2*)(mine + lane * ROW + value_column<NB>(lane, b) * 16 + half * 8));
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const Op k = decode8<T>((uint32_t)v[s], vs[s]);
#pragma unroll
                        for (int t = 0; t < TERMS; ++t) o[d] = O::mfma16(k, w[s][t], o[d]);
                    }
                }
            }
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        };
        while (tile < to) {
            work(tiles_ahead[0], tiles_ahead[1]);
            tile += 4;
            if (tile >= to) break;
            work(tiles_ahead[1], tiles_ahead[0]);
            tile += 4;
        }

        // the waves' sums as one: those of waves 2 and 3 to waves 0 and 1, then wave 1's to wave 0
        sum += __shfl_xor(sum, 16, kWave);
        sum += __shfl_xor(sum, 32, kWave);
        if (g == 0) stat[wave][i][0] = top, stat[wave][i][1] = sum;
        __syncthreads();
        float all = stat[0][i][0], total = 0.0f;
#pragma unroll
        for (int w = 1; w < 4; ++w) all = fmaxf(all, stat[w][i][0]);
        const float base = all == -INFINITY ? 0.0f : all;
#pragma unroll
        for (int w = 0; w < 4; ++w) total += stat[w][i][1] * (all == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(stat[w][i][0] - base));
        const float factor = all == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top - base);
#pragma unroll
        for (int d = 0; d < 2 * NB; ++d) o[d] *= factor;
        f32x4* const sums = reinterpret_cast<f32x4*>(lds);
        if (wave >= 2) {
#pragma unroll
            for (int d = 0; d < 2 * NB; ++d) sums[((wave - 2) * 2 * NB + d) * kWave + lane] = o[d];
        }
        __syncthreads();
        if (wave < 2) {
#pragma unroll
            for (int d = 0; d < 2 * NB; ++d) o[d] += sums[(wave * 2 * NB + d) * kWave + lane];
        }
        __syncthreads();
        if (wave == 1) {
#pragma unroll
            for (int d = 0; d < 2 * NB; ++d) sums[d * kWave + lane] = o[d];
        }
        __syncthreads();
        if (wave == 0 && asks) {
#pragma unroll
            for (int d = 0; d < 2 * NB; ++d) o[d] += sums[d * kWave + lane];
            if (whole) {
                T* y = static_cast<T*>(a.y) + (int64_t)r * a.ldy + ((int64_t)head * a.group + column) * D + 4 * g;
                const float inv = total == 0.0f ? 0.0f : 1.0f / total;
#pragma unroll
                for (int d = 0; d < 2 * NB; ++d) {
                    typename RowQuad<T>::type v;
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = (T)(total == 0.0f ? 0.0f : o[d][e] * inv);
                    *reinterpret_cast<typename RowQuad<T>::type*>(y + d * 16) = v;
                }
            } else {
                const int64_t at = part_at(hb, share_index, shares, before[r] > begin) + i;
#pragma unroll
                for (int d = 0; d < 2 * NB; ++d) *reinterpret_cast<f32x4*>(a.part + at * D + d * 16 + 4 * g) = o[d];
                if (g == 0) a.stat[at * 2] = all, a.stat[at * 2 + 1] = total;
            }
        }
        __syncthreads();                                               // (the sums have been read: the next row's values may come)
    }
}

template <typename T, int NB> static dcnn_status launch_few(dcnn_ctx* ctx, const AttendArgs& a) {
    const int64_t columns = (int64_t)a.cache.heads * a.blocks, units = a.splits > 0 ? columns * a.splits : a.tokens.rows * columns, most = (int64_t)ctx->num_cu * 16;
    const dim3 grid((unsigned)(a.splits > 0 || units < most ? units : most));
    if (a.cache.page_shift >= 6) hipLaunchKernelGGL((attend_few_kernel<T, NB, true>), grid, dim3(256), 0, ctx->stream, a);
    else hipLaunchKernelGGL((attend_few_kernel<T, NB, false>), grid, dim3(256), 0, ctx->stream, a);
    return check_hip(ctx, hipGetLastError(), "attend_few_kernel launch");
}
template <typename T> static dcnn_status launch_few_t(dcnn_ctx* ctx, int dim, const AttendArgs& a) {
    switch (dim) {
        case 32: return launch_few<T, 1>(ctx, a);
        case 64: return launch_few<T, 2>(ctx, a);
        case 96: return launch_few<T, 3>(ctx, a);
        case 128: return launch_few<T, 4>(ctx, a);
        case 192: return launch_few<T, 6>(ctx, a);
        default: return launch_few<T, 8>(ctx, a);
    }
}
dcnn_status launch_attend_few(dcnn_ctx* ctx, int dtype, int dim, const AttendArgs& a) {
    if (dtype == DCNN_F16) return launch_few_t<f16>(ctx, dim, a);
    if (dtype == DCNN_BF16) return launch_few_t<bf16>(ctx, dim, a);
    return launch_few_t<float>(ctx, dim, a);
}

}  // namespace dcnn
