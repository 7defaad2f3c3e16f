// Attention over the cache for many rows of a stream.
//
//   S^T = K Q^T,  P = exp2(S * scale log2(e) - max),  Y^T = V^T P^T / sum P, the maximum and the sums kept up to date from tile to tile
//
// A workgroup has 128 vectors of queries (rows and the query heads of one head of keys, rows first), 32 to a wave: the columns of its operands.
// It goes through the tokens that any of them sees, 64 at a time.  A tile's codes come in registers two tiles ahead, become operands in LDS
// (two buffers) by conversions that take the scale, one tile ahead, and every wave multiplies all of them:
//   * S^T: rows are tokens, so a lane has one column's products with 32 tokens, in registers; a column's maximum takes one exchange
//     between lanes, and the weights are the second product's operand as they are, in the order of tokens that the first leaves;
//   * V^T: values lie in LDS as rows of tokens and are read transposed, four tokens of a channel at a time, in that same order.
// Rows of several streams in a tile of rows are taken one stream after the other ("segments": columns outside of it see nothing).
// Instruction issue bounds it: eight vector instructions for each product of a query and a key that a lane has, an exponential among them, stand
// between the matrix products, and the two or three workgroups of a compute unit overlap them in part.  Measured: 14348 rows of 32 heads on 8 of
// 128 (bf16, causal, three prompts of up to 6000 tokens) 654 us, 0.90 PFLOP/s, matrix cores 37 % busy; 26240 flagged pixels of 8 heads of 64 (fp16,
// 4096 tokens each) 453 us with the join of halves (34).  A wave with 32 columns and a workgroup with 128 leave room for two waves to a SIMD at
// heads of 128.  With 256 vectors to a workgroup the prompts took 770 us and more with the products of one tile between the exponentials of the one
// before, 818 with two groups of four waves, one at the matrix cores while the other weighs and stages.
#include "attend_device.h"

namespace dcnn {

typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

constexpr int kVectors = 128, kTokens = 64;
constexpr float kSlack = 8.0f;                  // how far a column's maximum may lie above the one that its sums are relative to, as a power of two

// 16-byte columns of a row of LDS (4 NB of them), permuted so that sixteen lanes meet sixteen different ones of the 256 bytes that the banks span: the same
// column of sixteen rows in a row (keys), four columns of four rows (values, read transposed).
template <int NB> __device__ __forceinline__ int tile_column(int row, int col) {
    if constexpr (NB % 4 == 0) return col ^ ((row & 3) << 2 | (row >> 2 & 3));
    if constexpr (NB % 2 == 0) return col ^ ((row >> 1 & 1) << 2 | (row >> 2 & 3));
    return col ^ (row >> 2 & 3);
}
// The token of the x-th group of lanes that writes a tile: those that write together differ in the bits that permute columns.
template <int NB> __device__ __forceinline__ int staged_token(int x) {
    if constexpr (NB == 1) return x;
    if constexpr (NB % 4 == 0 || NB == 3) return (x & ~15) | (x & 3) << 2 | (x >> 2 & 3);
    return (x & ~14) | (x & 6) << 1 | (x >> 2 & 2);
}

__device__ __forceinline__ int wave_min(int v) {
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const int o = __shfl_xor(v, d, kWave);
        v = o < v ? o : v;
    }
    return __builtin_amdgcn_readfirstlane(v);
}

template <typename T, int NB> struct TileShape {
    static constexpr int waves = tile_waves(NB, Operand<T>::TERMS);
    static constexpr int bytes = 2 * 2 * kTokens * NB * 64;            // two buffers of keys and values
};

// WHOLE: pages hold whole tiles of tokens.
template <typename T, int NB, bool WHOLE>
__global__ __launch_bounds__(256, (TileShape<T, NB>::waves)) void attend_tile_kernel(AttendArgs a) {
    typedef Operand<T> O;
    typedef typename O::type Op;
    constexpr int D = NB * 32, ROW = D * 2, TERMS = O::TERMS, CHUNKS = (NB + 1) / 2, PLANE = kTokens * ROW;
    extern __shared__ __attribute__((aligned(16))) uint8_t lds[];
    __shared__ int streams[kVectors], lows[kVectors], highs[kVectors];
    // blocks of values that are NaN, in the order in which they are written, and whether there were any.  (Looked at word by word, and written, only
    // where there are.)
    __shared__ uint64_t broken[2][NB];
    __shared__ int any_broken;
    const int tid = threadIdx.x, lane = tid % kWave, wave = __builtin_amdgcn_readfirstlane(tid / kWave), half = lane / 32, col = lane % 32;
    const int count = row_count(a.tokens.count, a.tokens.rows);
    const int vectors = count * a.group, tiles = (vectors + kVectors - 1) / kVectors, heads = a.cache.heads;
    if (tiles == 0) return;
    // a few tiles of rows: their segments to workgroups of their own
    int turns = 512 / ((int64_t)tiles * heads * a.splits < 512 ? tiles * heads * a.splits : 512);
    turns = turns < kVectors ? turns : kVectors;
    const int page_mask = (1 << a.cache.page_shift) - 1;
    const uint32_t page_tokens = (uint32_t)heads << a.cache.page_shift;
    for (int64_t item = blockIdx.x; item < (int64_t)tiles * heads * a.splits * turns; item += gridDim.x) {
        int rest = (int)(item / heads);
        const int head = (int)(item % heads), part = rest % a.splits;
        rest /= a.splits;
        const int turn = rest % turns, place = rest / turns, tile = a.causal ? tiles - 1 - place : place;      // (later rows see more: they go first)
        const int v = tile * kVectors + wave * 32 + col;
        const bool active = v < vectors;
        const int r = active ? (int)fast_div((uint32_t)v, a.by_group) : 0, in_group = active ? v - r * a.group : 0;
        Token token = {-1, 0, false};
        Span span = {0, 0};
        if (active) {
            token = token_of(a.tokens, r);
            span = span_of(a, token);
        }
        const int stream = token.here && (uint32_t)token.stream < (uint32_t)a.cache.streams ? token.stream : -1;
        if (half == 0) streams[wave * 32 + col] = stream, lows[wave * 32 + col] = span.lo, highs[wave * 32 + col] = span.hi;
        // queries, as operands
        Op q[2 * NB][TERMS];
        const T* qp = static_cast<const T*>(a.q) + (int64_t)r * a.ldq + ((int64_t)head * a.group + in_group) * D + half * 8;
#pragma unroll
        for (int j = 0; j < 2 * NB; ++j) load_operand<T>(qp + j * 16, a.negate, q[j]);
        f32x16 o[NB];
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int e = 0; e < 16; ++e) o[b][e] = 0.0f;
        float top = -INFINITY, sum = 0.0f;
        bool mine = false;
        if (tid < 2 * NB) broken[tid / NB][tid % NB] = 0;
        if (tid == 2 * NB) any_broken = 0;
        uint32_t dirty = 0;                                            // words of this wave that are not zero
        __syncthreads();
        const uint64_t starts0 = __ballot(lane == 0 || streams[lane] != streams[lane == 0 ? 0 : lane - 1]), starts1 = __ballot(streams[lane + 64] != streams[lane + 63]);
        int index = 0;
        for (int begin = 0, end; begin < kVectors; begin = end, ++index) {
            const uint64_t later0 = begin < 63 ? starts0 >> (begin + 1) : 0, later1 = begin < 63 ? starts1 : (begin < 127 ? starts1 >> (begin - 63) : 0);
            end = later0 ? begin + 1 + __builtin_ctzll(later0) : (later1 ? (begin < 63 ? 64 : begin + 1) + __builtin_ctzll(later1) : kVectors);
            if (index % turns != turn) continue;
            const int at = wave * 32 + col;
            const bool in_segment = at >= begin && at < end;
            mine = mine || in_segment;
            const int lo = in_segment ? span.lo : 0, hi = in_segment ? span.hi : 0;
            int first = 0x7fffffff, last = 0;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int w = lane + 64 * i;
                if (w >= begin && w < end && lows[w] < highs[w]) {
                    first = lows[w] < first ? lows[w] : first;
                    last = highs[w] > last ? highs[w] : last;
                }
            }
            first = wave_min(first), last = -wave_min(-last);
            if (last <= first) continue;
            const int of = __builtin_amdgcn_readfirstlane(streams[begin]);
            // what all of the wave's columns see, and what any of them does
            const int see_from = -wave_min(-(lo < hi ? lo : 0x7fffffff)), see_to = wave_min(hi);
            const int any_from = wave_min(lo < hi ? lo : 0x7fffffff), any_to = -wave_min(-hi);
            const int start = first & ~(kTokens - 1), all = (last - start + kTokens - 1) / kTokens, share = (all + a.splits - 1) / a.splits;
            const int from = part * share, to = from + share < all ? from + share : all;
            if (from >= to) continue;

            // ---- codes of a tile: from memory, to operands in LDS
            u32x4 raw[CHUNKS];
            uint8_t byte[CHUNKS];                                      // (as words, they would be waited for where they were asked for: to cut them to bytes)
            bool drop[CHUNKS];
            // (keys 0, values 1, nothing 2: one for all of a wave's lanes)
            const auto which_of = [&](int n) { return NB % 4 == 0 ? 4 * n / NB : (wave + 4 * n) / NB; };
            // The page of a tile, or of its sixteen tokens `lane % 4`: 64 pages are asked for at once, a lane each.  (One by one, through either cache, every
            // tile waits for them, and for what was asked for before.)
            constexpr int PER = WHOLE ? 1 : 4, SPAN = kTokens / PER;
            int pages = -1;
            const auto page_at = [&](int t) {
                const int at = (t - from) * PER % 64;
                if (at == 0) pages = page_of(a.cache, of, (start + t * kTokens + lane * SPAN) >> a.cache.page_shift);
                if constexpr (WHOLE) return __builtin_amdgcn_readlane(pages, at);
                else return __shfl(pages, at + lane % 4, kWave);
            };
            const auto load = [&](int t, int page) {
                const uint64_t tile_slot = (uint64_t)(uint32_t)(page < 0 ? 0 : page) * (2 * page_tokens) + ((start + t * kTokens) & page_mask);
#pragma unroll
                for (int n = 0; n < CHUNKS; ++n) {
                    const int within = (tid + 256 * n) % (kTokens * NB), token_in = staged_token<NB>(within / NB), b = within % NB;
                    const int which = which_of(n), t_at = start + t * kTokens + token_in;
                    if (NB % 2 != 0 && which > 1) break;
                    bool counts = (uint32_t)(t_at - first) < (uint32_t)(last - first);
                    if constexpr (WHOLE) {
                        // the tile's first token, one for all lanes, and 32-bit offsets from it
                        const uint64_t slot = tile_slot + ((uint32_t)(which * heads + head) << a.cache.page_shift);
                        const uint8_t *const codes = a.cache.codes + slot * (D / 2), *const scales = a.cache.scales + slot * NB;
                        raw[n] = *reinterpret_cast<const u32x4*>(codes + (uint32_t)(token_in * (D / 2) + b * 16));
                        byte[n] = scales[(uint32_t)(token_in * NB + b)];
                        counts = counts && page >= 0;
                    } else {
                        const int p = __shfl(page, token_in / 16, kWave);
                        const int64_t slot = ((int64_t)(p < 0 ? 0 : p) * 2 + which) * page_tokens + ((int64_t)head << a.cache.page_shift) + (t_at & page_mask);
                        raw[n] = *reinterpret_cast<const u32x4*>(a.cache.codes + slot * (D / 2) + b * 16);
                        byte[n] = a.cache.scales[slot * NB + b];
                        counts = counts && p >= 0;
                    }
                    drop[n] = !counts;                                 // (what lies there may be anything)
                }
            };
            const auto stage = [&](int buffer) {
#pragma unroll
                for (int n = 0; n < CHUNKS; ++n) {
                    const int within = (tid + 256 * n) % (kTokens * NB), token_in = staged_token<NB>(within / NB), b = within % NB, which = which_of(n);
                    if (NB % 2 != 0 && which > 1) break;
                    float scale = scale_of_byte(byte[n]);
                    // keys of tokens that do not count may be anything: their products are not looked at.  Values are multiplied by weights of zero there,
                    // and so is a value that is NaN for rows that do not see it: they become zeros, and the second kind is noted
                    if (which == 1) {
                        const uint64_t noted = __ballot(byte[n] == 255 && !drop[n]);
                        const uint32_t bit = 1u << (buffer * CHUNKS + n);
                        if (noted != 0 || (dirty & bit) != 0) {
                            if (lane == 0) broken[buffer][within / 64] = noted;
                            if (noted != 0) any_broken = 1;
                            dirty = noted != 0 ? dirty | bit : dirty & ~bit;
                        }
                        scale = drop[n] || byte[n] == 255 ? 0.0f : scale;
                    }
                    uint8_t* const row = lds + (buffer * 2 + which) * PLANE + token_in * ROW;
#pragma unroll
                    for (int i = 0; i < 4; ++i) *reinterpret_cast<Op*>(row + tile_column<NB>(token_in, 4 * b + i) * 16) = decode8<T>(raw[n][i], scale);
                }
            };
            // which sixteens of a tile's tokens have a page
            const auto sixteens = [&](int p) { return WHOLE ? (p >= 0 ? 15u : 0u) : (uint32_t)__ballot(p >= 0) & 15u; };
            int page = page_at(from);
            uint32_t paged = sixteens(page), paged_next = 0;
            load(from, page);
            page = page_at(from + 1);
            __syncthreads();                                           // (a segment before this one is done with the buffers)
            stage(from & 1);
            if (from + 1 < to) {
                paged_next = sixteens(page);
                load(from + 1, page);
                page = page_at(from + 2);
            }
            for (int t = from; t < to; ++t) {
                __syncthreads();                                       // this tile is there, and all are done with the one before it
                if (t + 1 < to) stage((t + 1) & 1);
                const uint32_t has_page = paged;
                paged = paged_next;
                if (t + 2 < to) {                                      // (nothing of these loads is looked at before the next tile's turn)
                    paged_next = sixteens(page);
                    load(t + 2, page);
                    page = page_at(t + 3);
                }
                const int t0 = start + t * kTokens;
                if (t0 + kTokens <= any_from || t0 >= any_to) continue;
                // (lane's parts of addresses: made anew for each tile, or the compiler keeps one in a register for each read)
                int key_x = half ^ tile_column<NB>(col, 0), value_x = (lane % 32 / 16 * 2 + lane % 4 / 2) ^ tile_column<NB>(4 * half + lane % 16 / 4, 0);
                asm volatile("" : "+v"(key_x), "+v"(value_x));
                const uint8_t* const keys = lds + (t & 1) * 2 * PLANE + col * ROW;
                const uint8_t* const vals = lds + (t & 1) * 2 * PLANE + PLANE + (4 * half + lane % 16 / 4) * ROW + lane % 2 * 8;
                // operands are read four products ahead: one at a time, each product waits for its own (the prompts above took 850 us)
                f32x16 s[2];
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int e = 0; e < 16; ++e) s[kb][e] = 0.0f;
                Op k[2][4];
                const auto read_keys = [&](int group) {
#pragma unroll
                    for (int n = 0; n < 4; ++n) k[group % 2][n] = *reinterpret_cast<const Op*>(keys + n % 2 * 32 * ROW + (key_x ^ 2 * (group * 2 + n / 2)) * 16);
                };
                read_keys(0);
#pragma unroll
                for (int group = 0; group < NB; ++group) {
                    if (group + 1 < NB) read_keys(group + 1);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int n = 0; n < 4; ++n)
#pragma unroll
                        for (int m = 0; m < TERMS; ++m) s[n % 2] = O::mfma32(k[group % 2][n], q[group * 2 + n / 2][m], s[n % 2]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                // values: two blocks of channels side by side; step n is tokens 16 * (n / 2 % 4) on and block 2 * (n / 8) + n % 2
                constexpr auto block_of = [](int n) { return n < NB / 2 * 8 ? n / 8 * 2 + n % 2 : NB - 1; };
                constexpr auto tokens_of = [](int n) { return n < NB / 2 * 8 ? n / 2 % 4 : n % 4; };
                Op x[2][4];
                const auto read_values = [&](int group) {
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        i16x4 part[2];
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            part[i] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(vals + (16 * tokens_of(group * 4 + n) + 8 * i) * ROW +
                                                                                            (value_x ^ (4 * block_of(group * 4 + n) + 2 * i)) * 16));
                        x[group % 2][n] = __builtin_bit_cast(Op, __builtin_shufflevector(part[0], part[1], 0, 1, 2, 3, 4, 5, 6, 7));
                    }
                };
                read_values(0);
                // the column's product with token t0 + 32 kb + 8 (e / 4) + 4 half + e % 4
                if (t0 < see_from || t0 + kTokens > see_to || has_page != 15u) {
#pragma unroll
                    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const int in_tile = 32 * kb + 8 * (e / 4) + 4 * half + e % 4;
                            const bool seen = (uint32_t)(t0 + in_tile - lo) < (uint32_t)(hi - lo) && (has_page >> (2 * kb + e / 8) & 1);
                            s[kb][e] = seen ? s[kb][e] : -INFINITY;
                        }
                }
                float m = s[0][0];
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int e = 0; e < 16; ++e) m = fmaxf(m, s[kb][e]);
                m = max_of_halves(m);
                m *= a.factor;                                         // (the factor is above zero)
                // (weights up to 2^kSlack do as well as those up to one: sums are scaled anew where a column's maximum has grown by more than that)
                if (__any(m > top + kSlack)) {
                    m = fmaxf(m, top);
                    const float factor = m > top ? __builtin_amdgcn_exp2f(top - m) : 1.0f;
                    top = m;
                    sum *= factor;
#pragma unroll
                    for (int b = 0; b < NB; ++b) o[b] *= factor;
                }
                constexpr float RAISE = O::RAISE > 0.0f ? O::RAISE - kSlack : 0.0f;
                const float base = top == -INFINITY ? 0.0f : top - RAISE;      // (sums of weights and of values are raised alike)
                Op p[2][2][TERMS];
#pragma unroll
                for (int kb = 0; kb < 2; ++kb)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        float w[8];
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][8 * u + e], a.factor, -base));
                            sum += w[e];
                        }
                        O::split(w, p[kb][u]);
                    }
#pragma unroll
                for (int group = 0; group < NB; ++group) {
                    if (group + 1 < NB) read_values(group + 1);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int n = 0; n < 4; ++n) {
                        const int b = block_of(group * 4 + n), tokens = tokens_of(group * 4 + n);
#pragma unroll
                        for (int m = 0; m < TERMS; ++m) o[b] = O::mfma32(x[group % 2][n], p[tokens / 2][tokens % 2][m], o[b]);
                    }
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (__builtin_amdgcn_readfirstlane(any_broken) != 0) {
                    for (int w = 0; w < NB; ++w)
                        for (uint64_t bits = broken[t & 1][w]; bits != 0; bits &= bits - 1) {
                            const int bit = w * 64 + __builtin_ctzll(bits), in_tile = staged_token<NB>(bit / NB);
                            if ((uint32_t)(t0 + in_tile - lo) < (uint32_t)(hi - lo)) {
#pragma unroll
                                for (int b = 0; b < NB; ++b)
                                    if (bit % NB == b) {
#pragma unroll
                                        for (int e = 0; e < 16; ++e) o[b][e] = __builtin_nanf("");
                                    }
                            }
                        }
                }
            }
        }
        // sums of both halves' tokens; the column's channels 32 b + 8 (e / 4) + 4 half + e % 4
        sum += __shfl_xor(sum, 32, kWave);
        if (mine && active) {
            if (a.splits == 1) {
                T* y = static_cast<T*>(a.y) + (int64_t)r * a.ldy + ((int64_t)head * a.group + in_group) * D + 4 * half;
                const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        typename RowQuad<T>::type w;
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[e] = (T)(o[b][4 * i + e] * inv);
                        *reinterpret_cast<typename RowQuad<T>::type*>(y + b * 32 + 8 * i) = w;
                    }
            } else {
                const int64_t at = ((int64_t)r * heads * a.group + head * a.group + in_group) * a.splits + part;
#pragma unroll
                for (int b = 0; b < NB; ++b)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        *reinterpret_cast<f32x4*>(a.part + at * D + b * 32 + 8 * i + 4 * half) = f32x4{o[b][4 * i], o[b][4 * i + 1], o[b][4 * i + 2], o[b][4 * i + 3]};
                if (half == 0) a.stat[at * 2] = top, a.stat[at * 2 + 1] = sum;
            }
        }
        __syncthreads();                                               // (streams and spans have been read)
    }
}

template <typename T, int NB> static dcnn_status launch_tile(dcnn_ctx* ctx, const AttendArgs& a) {
    constexpr int bytes = TileShape<T, NB>::bytes;
    auto* const kern = a.cache.page_shift >= 6 ? &attend_tile_kernel<T, NB, true> : &attend_tile_kernel<T, NB, false>;
    if (bytes > 64 * 1024) {
        const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (err != hipSuccess) return check_hip(ctx, err, "hipFuncSetAttribute(attend_tile_kernel)");
    }
    const int64_t items = cdiv((int64_t)a.tokens.rows * a.group, kVectors) * a.cache.heads * a.splits;
    // a list's length is not known here: workgroups stride through what there is
    int64_t grid = items < 512 ? 512 : items;
    if (a.tokens.count != nullptr && grid > 2048) grid = 2048;
    hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(256), bytes, ctx->stream, a);
    return check_hip(ctx, hipGetLastError(), "attend_tile_kernel launch");
}
template <typename T> static dcnn_status launch_tile_t(dcnn_ctx* ctx, int dim, const AttendArgs& a) {
    switch (dim) {
        case 32: return launch_tile<T, 1>(ctx, a);
        case 64: return launch_tile<T, 2>(ctx, a);
        case 96: return launch_tile<T, 3>(ctx, a);
        case 128: return launch_tile<T, 4>(ctx, a);
        case 192: return launch_tile<T, 6>(ctx, a);
        default: return launch_tile<T, 8>(ctx, a);
    }
}
dcnn_status launch_attend_tile(dcnn_ctx* ctx, int dtype, int dim, const AttendArgs& a) {
    if (dtype == DCNN_F16) return launch_tile_t<f16>(ctx, dim, a);
    if (dtype == DCNN_BF16) return launch_tile_t<bf16>(ctx, dim, a);
    return launch_tile_t<float>(ctx, dim, a);
}

}  // namespace dcnn
