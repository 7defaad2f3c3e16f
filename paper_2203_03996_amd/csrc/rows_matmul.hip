// Products of rows in 8-bit integers with weights in 8-bit integers: a scale for each row and for each output channel.
//
//   y[r][j] = act( (sum_k q[r][k] w[k][j]) * (q_scale[r] * w_scale[j]) + bias[j] )
//
// The sums are exact in 32-bit integers, so how a sum is cut up never changes a result.
#include "rows_device.h"
#include "tile_schedule.h"

namespace dcnn {

// ---- weights ------------------------------------------------------------------------------------------------------
// One workgroup per block of 32 channels: the largest magnitude of each channel over k (or the scale that came with the weights), then
// the 8-bit values in the order that the products read them.  Runs once per weight tensor.
constexpr int kPackThreads = 256;
template <typename T> __global__ __launch_bounds__(kPackThreads) void rows_pack_kernel(const T* w, int64_t ldw, int k, int n, int kp, const float* scale,
                                                                                       int8_t* packed, float* packed_scale) {
    constexpr int P = kPackThreads / kPackC;
    __shared__ uint32_t part[P][kPackC];
    const int ch = threadIdx.x % kPackC, part_k = threadIdx.x / kPackC;
    const int64_t j = (int64_t)blockIdx.x * kPackC + ch;
    const bool in = j < n;
    float inv = 1.0f;
    if constexpr (!std::is_same_v<T, int8_t>) {
        uint32_t m = 0;
        if (in)
            for (int kk = part_k; kk < k; kk += P) m = MaxOp::op(m, __builtin_bit_cast(uint32_t, (float)w[kk * ldw + j]) & 0x7fffffffu);
        part[part_k][ch] = m;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < P; ++i) m = MaxOp::op(m, part[i][ch]);
        const float s = quantize_scale(m, &inv);
        if (part_k == 0) packed_scale[j] = in ? s : 0.0f;
    } else {
        if (part_k == 0) packed_scale[j] = in ? scale[j] : 0.0f;
    }
    for (int k16 = part_k; k16 < kp / 16; k16 += P) {
        uint32_t word[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t b[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const int kk = k16 * 16 + i * 4 + e;
                b[e] = 0;
                if (in && kk < k) {
                    if constexpr (std::is_same_v<T, int8_t>) b[e] = (uint8_t)w[kk * ldw + j];
                    else b[e] = inv == 0.0f ? 0u : quantize_bits((float)w[kk * ldw + j], inv);
                }
            }
            word[i] = pack_bytes(b[0], b[1], b[2], b[3]);
        }
        *reinterpret_cast<uint4*>(packed + (((int64_t)blockIdx.x * (kp / 16) + k16) * kPackC + ch) * 16) = make_uint4(word[0], word[1], word[2], word[3]);
    }
}

dcnn_status launch_rows_pack(dcnn_ctx* ctx, int dtype, int64_t k, int64_t n, const void* w, int64_t ldw, const float* scale, int8_t* packed,
                             float* packed_scale) {
    const dim3 grid((unsigned)(packed_n(n) / kPackC)), block(kPackThreads);
    const int kp = (int)packed_k(k);
#define DCNN_PACK(T) hipLaunchKernelGGL((rows_pack_kernel<T>), grid, block, 0, ctx->stream, static_cast<const T*>(w), ldw, (int)k, (int)n, kp, scale, packed, packed_scale)
    if (dtype == DCNN_I8) DCNN_PACK(int8_t);
    else if (dtype == DCNN_F16) DCNN_PACK(f16);
    else if (dtype == DCNN_BF16) DCNN_PACK(bf16);
    else DCNN_PACK(float);
#undef DCNN_PACK
    return check_hip(ctx, hipGetLastError(), "rows_pack_kernel launch");
}

// ---- products -----------------------------------------------------------------------------------------------------
// A workgroup of TW x CW waves computes TW*FT*32 rows by CW*FC*32 channels over K-tiles of 128.  The channels are the matrix cores' rows
// and the tokens their columns: a lane ends with four consecutive channels of one token.
//
// K-tiles go from memory straight into one of NB LDS buffers, NB - 1 K-tiles ahead of their use, the first ones of the workgroup's next
// tile behind the last ones of this (which and when: tile_schedule.h); the operands of a step of 32 k are read from LDS one step ahead, the
// first ones of the next K-tile behind the one barrier, which stands a step before the tile's end.  So the matrix cores wait for memory and
// LDS only where a K-tile takes longer to come than to multiply: with two buffers a K-tile has the time of one on its way.  Three buffers
// give it the time of two, but at every third K-tile, where the first buffer is read, the compiler waits for all copies.
// Weights lie in LDS as they are packed (an operand load of a wave is 1 KB in a row).  A row's eight chunks of 16 k are exchanged by bits
// of its number: the 16 lanes of a quarter of an operand load, 16 rows at one k, then cover all 64 banks.
//
// The sums leave through LDS, a wave's 32 tokens by 128 bytes at a time: pieces of rows, 16 bytes a lane, where the matrix cores' order
// would store 16 bytes from 32 rows; past the L2, which has the operands to keep (26214 x 256 -> 1024: 20.3 us -> 18.7, 8000 x 256 -> 256:
// 8.4 -> 6.9; 4096 -> 4096 the same, or 4 % at 60000 rows).  An output costs three and a half instructions and an activation two more: that,
// and not the matrix cores, is what a short k waits for.
//
// 16384 x 4096 -> 4096 in bf16: 237-247 us in a row (the same matrices again, or others from memory), 2.2-2.3 POP/s; 8192 x 8192 -> 4096:
// 225-245, 2.2-2.4 (a library's 8-bit product that leaves its 32-bit sums: 248 and 226).  Power bounds these: the same product of zeros takes
// 183 us in place of 230; the clock is at 1.8 GHz, and the matrix cores are busy 60 % of its cycles.  Per tile of 256 x 256 about 5 us of 60
// are the outputs'.  What it took, us for the first of them: one K-tile staged through registers behind a barrier 328; loads two K-tiles and
// operands a step ahead 295; copies straight into LDS 272; scales and bias by one load each, dealt out in LDS, and no wait for stores 250.
// 26214 x 256 -> 1024 in fp16 is bound by its outputs: 17-18 us in a row where the rows are in the caches, 25 where all comes from memory.
constexpr int kChunks = kPackK / 16, kSteps = kPackK / 32;
constexpr int kPlanCus = 256;                  // compute units of an MI355X: what a plan counts on
constexpr int kPanelTiles = 2;                 // K-tiles of rows that a workgroup makes for itself and keeps
enum TileMode { kWhole, kParts, kPanel };      // rows_matmul_kernel: see there
template <typename T, int TW, int CW, int FT, int FC, int NB, TileMode MODE> struct TileShape {
    static constexpr int waves = TW * CW, threads = waves * kWave, tokens = TW * FT * 32, channels = CW * FC * 32;
    static constexpr int row = FC * 32 * (int)sizeof(T) < 128 ? FC * 32 * (int)sizeof(T) : 128;      // bytes of a token on their way out
    static constexpr int copied = MODE == kPanel ? 0 : tokens;                                       // tokens of a buffer
    static constexpr int stage = (copied + channels) * kPackK, unit = 32 * row, lds = NB * stage + waves * unit;
};
__device__ __forceinline__ int chunk_swizzle(int row) { return (row >> 1) & 7; }

// Tiles in the order that workgroups take them: four rows of tiles side by side, so that the tiles in work on an XCD share what its L2 holds.
struct TileAt { int t, c; };
__device__ __forceinline__ TileAt tile_at(int tile, int tiles_t, int tiles_c) {
    const int group = tile / (4 * tiles_c), first = group * 4, size = tiles_t - first < 4 ? tiles_t - first : 4;
    const int r = tile - group * 4 * tiles_c;
    return {first + r % size, r / size};
}

// 16 bytes a lane from memory to 1 KB of LDS, in the order of the lanes.
__device__ __forceinline__ void copy_to_lds(__amdgpu_buffer_rsrc_t from, int offset, int uniform, int8_t* to) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(from, (__attribute__((address_space(3))) void*)to, 16, offset, uniform, 0, 0);
}
// at most N loads of this wave still on their way
template <int N> __device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0f70); }

// All waves are here, and what they have read from LDS is in their registers.  (A fence would wait for the copies into LDS as well.)
__device__ __forceinline__ void meet() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xc07f);                        // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Workgroups that share a tile: each leaves its sums, in the order of its registers, and counts itself; the last one to do so adds up the
// others' (32-bit integers: in any order the same) and goes on.  Nobody waits for anybody.
// Sums and count go past the XCDs' caches, one access at a time (atomic accesses of the GPU's scope); a thread's stores are done before its
// workgroup counts itself.  A fence in their place writes a whole L2 back for every workgroup: 256 of them took 35 us.
template <int N, int THREADS>
__device__ __forceinline__ bool last_part(i32x16* acc, int32_t* partial, uint32_t* arrived, int tile, int part, int parts, int8_t* lds) {
    uint64_t* const sums = reinterpret_cast<uint64_t*>(partial) + (int64_t)tile * parts * (N * 8 * THREADS);
    uint64_t* mine = sums + part * (N * 8 * THREADS) + threadIdx.x;
#pragma unroll
    for (int i = 0; i < N; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j)
            __hip_atomic_store(mine + (i * 8 + j) * THREADS, (uint64_t)(uint32_t)acc[i][j * 2] | (uint64_t)(uint32_t)acc[i][j * 2 + 1] << 32,
                               __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("" ::: "memory");
    wait_loads<0>();                                           // (stores count as loads do)
    __syncthreads();
    uint32_t* const before = reinterpret_cast<uint32_t*>(lds);
    if (threadIdx.x == 0) *before = __hip_atomic_fetch_add(arrived + tile, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    if (*before != (uint32_t)parts - 1) return false;
    constexpr int K = 4;                                       // parts whose sums are on their way together
    for (int p = 1; p < parts; p += K) {
        uint64_t v[K][N * 8];
#pragma unroll
        for (int k = 0; k < K; ++k) {                          // (behind the last one: the last one again)
            const int at = part + (p + k < parts ? p + k : parts - 1);
            const uint64_t* from = sums + (at < parts ? at : at - parts) * (N * 8 * THREADS) + threadIdx.x;
#pragma unroll
            for (int i = 0; i < N * 8; ++i) v[k][i] = __hip_atomic_load(from + i * THREADS, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        }
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (p + k >= parts) break;
#pragma unroll
            for (int i = 0; i < N; ++i)
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    acc[i][j * 2] += (int32_t)(uint32_t)v[k][i * 8 + j];
                    acc[i][j * 2 + 1] += (int32_t)(uint32_t)(v[k][i * 8 + j] >> 32);
                }
        }
    }
    if (threadIdx.x == 0) __hip_atomic_store(arrived + tile, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();                                           // (the LDS word is about to be overwritten)
    return true;
}

template <int I> using Int = std::integral_constant<int, I>;
template <int N, int I = 0, typename F> __device__ __forceinline__ void unrolled(F&& f) {
    if constexpr (I < N) {
        f(Int<I>{});
        unrolled<N, I + 1>(f);
    }
}

struct FewRows {                 // the rows that a kernel norms and quantises for itself
    const void *x, *w, *b;
    const int32_t* idx;
    int ldx, map_rows, c, kind;
    float eps;
};

// kPanel: the rows of a token tile, normed (or not), in 8 bits, in LDS: K-tiles one behind the other, laid out as the others' buffers are.
// Eight lanes to a row, so that a wave has its eight rows in hand at once: a wave to a row, eight rows one behind the other, took 5 to 10 us
// longer (reductions that wait for each other, code that is run once).
constexpr int kPanelLanes = 8;
template <typename T, int NV, int TOKENS, int WAVES>
__device__ __forceinline__ void make_panel(const FewRows& n, int t0, int count, int8_t* panel, float* scales) {
    constexpr int E = RowVec<T>::E, L = kPanelLanes;
    static_assert(TOKENS == WAVES * (kWave / L), "a row for each eight lanes");
    const int lane = threadIdx.x % L, r = threadIdx.x / L, c = n.c;
    const float inv_c = 1.0f / (float)c;
    const bool in = in_rows(t0, r, count);
    int turn = 0, i = in ? t0 + r : -1;
    if (n.idx != nullptr && in) i = n.idx[i];
    const bool token = i >= 0 && i < n.map_rows;
    const T* x = static_cast<const T*>(n.x) + (int64_t)(token ? i : 0) * n.ldx;
    u32x4 raw[NV];
#pragma unroll
    for (int j = 0; j < NV; ++j) raw[j] = row_load<T>(x, (j * L + lane) * E, token ? c : 0);
    NormParams<T, L, NV, true> params;
    params.read(n.w, n.b, lane, c);
    float v[NV][E];
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int e = 0; e < E; ++e) v[j][e] = row_get<T>(raw[j], e);
    if (n.kind != DCNN_NORM_NONE) norm_row<T, L, NV, true>(v, n.kind, n.eps, params, lane, c, inv_c, nullptr, turn);
    if (!token) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
            for (int e = 0; e < E; ++e) v[j][e] = 0.0f;
    }
    float inv;
    const float scale = quantize_scale(row_amax<L, NV, E>(v, nullptr, turn), &inv);
    if (lane == 0) scales[r] = scale;
    auto place = [&](int k) { return panel + (k / kPackK * TOKENS + r) * kPackK + ((k % kPackK / 16 ^ chunk_swizzle(r)) * 16 + k % 16); };
#pragma unroll
    for (int j = 0; j < NV; ++j) {
        const RowPart part = row_part<T>((j * L + lane) * E, c);
        if (part.skip >= E) continue;
        const typename QuantWords<T>::type w = quantized<T>(v[j], inv);
        if (part.at % E == 0) {
            typedef uint32_t Words __attribute__((ext_vector_type(E / 4)));
            *reinterpret_cast<Words*>(place(part.at)) = w;
        } else {                                               // (a row's last vector where its length is odd: across two chunks)
#pragma unroll
            for (int e = 0; e < E; ++e) *place(part.at + e) = (int8_t)(w[e / 4] >> (e % 4 * 8));
        }
    }
}

// kWhole: workgroups stride through the tiles.  kParts: `splits` workgroups share a tile, each `share` of its K-tiles.  kPanel: a workgroup
// has one tile and makes the 8-bit rows of its tokens itself.
template <typename T, int TW, int CW, int FT, int FC, int NB, TileMode MODE>
__global__ __launch_bounds__(TW * CW * kWave, 2) void rows_matmul_kernel(MatmulArgs a, int splits, int share, std::conditional_t<MODE == kPanel, FewRows, int> n) {
    using S = TileShape<T, TW, CW, FT, FC, NB, MODE>;
    constexpr int QL = S::copied / 8 / S::waves, WL = S::channels / 8 / S::waves;        // copies of 1 KB per K-tile and wave
    static_assert(S::threads >= S::channels && S::threads >= S::tokens && (2 * S::channels + S::tokens) * 4 <= S::waves * S::unit, "a thread for each factor");
    static_assert(QL * 8 * S::waves == S::copied && WL * 8 * S::waves == S::channels, "whole rounds of copies");
    // (an array each: what is read from the second and third does not wait for copies into the others; of the first the compiler is not so
    // sure, and waits for every copy before it is read)
    __shared__ __align__(1024) int8_t buf0[S::stage], buf1[S::stage], buf2[NB > 2 ? S::stage : 16], out_lds[S::waves * S::unit];
    static_assert(NB == 2 || NB == 3, "an array for each buffer");
    auto buffer = [&](auto i) -> int8_t* {
        constexpr int I = decltype(i)::value % NB;
        if constexpr (I == 0) return buf0;
        else if constexpr (I == 1) return buf1;
        else return buf2;
    };
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int tw = wave / CW, cw = wave % CW;
    const int count = row_count(a.count, a.rows);
    const int tiles_t = tiles_of(count, S::tokens), tiles_c = tiles_of(a.n, S::channels);
    const int blocks_c = (a.n + kPackC - 1) / kPackC;
    const int w_block_bytes = a.kt * kPackK * kPackC;          // 2 MB at most
    // (workgroups that share a tile, or the rows of one, are neighbours, so on one XCD; the grid has one for each)
    const WgTileRange range = wg_tile_range((int64_t)tiles_t * tiles_c * (MODE == kParts ? splits : 1));
    if (range.begin >= range.end) return;
    const int part = MODE == kParts ? (int)(range.begin % splits) : 0, k0 = MODE == kParts ? part * share : 0;
    const int kts = MODE == kParts ? (a.kt - k0 < share ? a.kt - k0 : share) : a.kt;
    const TileAt only = MODE == kPanel ? TileAt{(int)((uint32_t)range.begin / (uint32_t)tiles_c), (int)((uint32_t)range.begin % (uint32_t)tiles_c)} : TileAt{};
    auto place_of = [&](int64_t tile) -> TileAt {
        if constexpr (MODE == kPanel) return only;
        else return tile_at((int)(MODE == kParts ? tile / splits : tile), tiles_t, tiles_c);
    };
    extern __shared__ __align__(16) int8_t panel[];

    // of the tile that is being copied: rows behind the last one read the last one, blocks behind the last one the last one
    __amdgpu_buffer_rsrc_t q_tile, w_tile;
    int q_at[QL > 0 ? QL : 1], w_at[WL];
    auto aim = [&](int64_t tile) {
        const TileAt at = place_of(tile);
        const int t0 = at.t * S::tokens, b0 = at.c * (S::channels / kPackC);
        if constexpr (QL > 0) q_tile = ws_rsrc(a.q + (int64_t)t0 * a.ldq, kWsMaxBytes);
        w_tile = ws_rsrc(a.w + (int64_t)b0 * w_block_bytes, kWsMaxBytes);
#pragma unroll
        for (int i = 0; i < QL; ++i) {
            const int row = (i * S::waves + wave) * 8 + lane / 8;
            q_at[i] = (row < count - t0 ? row : count - t0 - 1) * a.ldq;
        }
#pragma unroll
        for (int i = 0; i < WL; ++i) {
            const int j = i * S::waves + wave, block = j / 4;
            w_at[i] = (block < blocks_c - b0 ? block : blocks_c - b0 - 1) * w_block_bytes + j % 4 * 1024 + lane * 16;
        }
    };
    // (rows 8 on: their low bits are the same but for one)
    const int q_chunk[2] = {lane % 8 ^ chunk_swizzle(lane / 8), lane % 8 ^ chunk_swizzle(lane / 8 + 8)};
    auto copy = [&](int8_t* buf, int tile_kt) {
        const int kt = k0 + tile_kt;
        int at[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {                          // chunks behind a row's last one: any, their weights are zero
            const int chunk = kt * kChunks + q_chunk[i];
            at[i] = (chunk < a.kc ? chunk : 0) * 16;
        }
#pragma unroll
        for (int i = 0; i < QL; ++i) {
            const int rows = (i * S::waves + wave) * 8;
            copy_to_lds(q_tile, q_at[i] + (S::waves % 2 == 0 ? (wave % 2 ? at[1] : at[0]) : (rows / 8 % 2 ? at[1] : at[0])), 0, buf + rows * kPackK);
        }
#pragma unroll
        for (int i = 0; i < WL; ++i) copy_to_lds(w_tile, w_at[i], kt * (kPackK * kPackC), buf + S::copied * kPackK + (i * S::waves + wave) * 1024);
    };
    i32x4 qf[2][FT], wf[2][FC];
    // (32 rows on, the low bits that exchange chunks are the same)
    const int q_lane = (tw * FT * 32 + lane % 32) * kPackK + (lane / 32 ^ chunk_swizzle(lane % 32)) * 16;
    const int w_lane = S::copied * kPackK + cw * FC * (kPackK * kPackC) + lane * 16;
    auto operands = [&](int8_t* buf, int kt, int ks) {
        const int8_t* rows = MODE == kPanel ? panel + kt * (S::tokens * kPackK) : buf;
#pragma unroll
        for (int t = 0; t < FT; ++t) qf[ks % 2][t] = *reinterpret_cast<const i32x4*>(rows + (q_lane ^ ks * 32) + t * (32 * kPackK));
#pragma unroll
        for (int f = 0; f < FC; ++f) wf[ks % 2][f] = *reinterpret_cast<const i32x4*>(buf + w_lane + f * (kPackK * kPackC) + ks * 1024);
    };
    i32x16 acc[FT][FC];
    auto multiply = [&](int ks) {
#pragma unroll
        for (int t = 0; t < FT; ++t)
#pragma unroll
            for (int f = 0; f < FC; ++f) acc[t][f] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[ks % 2][f], qf[ks % 2][t], acc[t][f], 0, 0, 0);
    };
    int64_t ahead = range.begin;                               // the tile whose K-tiles are copied
    auto wait_but = [&](int tiles) {                           // until all but the last so many copied K-tiles have arrived
        unrolled<NB>([&](auto i) {
            constexpr int J = NB - 1 - decltype(i)::value;
            if (tiles == J) wait_loads<J * (QL + WL)>();
        });
    };
    int arrived;                                               // of this workgroup's tile, before it began
    // K-tile kt of this workgroup's tile lies in `buf`, kt + 1 in `next`.
    auto k_tile = [&](int kt, int8_t* buf, int8_t* next) {
#pragma unroll
        for (int ks = 0; ks < kSteps - 1; ++ks) {
            operands(buf, kt, ks + 1);
            if constexpr (FT * FC < 8) __builtin_amdgcn_sched_barrier(0);
            multiply(ks);
            if constexpr (FT * FC >= 8) {                      // an operand read between two products (2 % of large tiles)
#pragma unroll
                for (int i = 0; i < FT + FC; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if (kt + 1 >= arrived) {                               // K-tile kt + 1: those behind it may be on their way
            static_assert(NB == 2 || NB == 3, "none or one");
            if (may_be_in_flight(kt, kts, NB, ahead < range.end) == NB - 2) wait_loads<(NB - 2) * (QL + WL)>();
            else wait_loads<0>();
        }
        meet();
        operands(next, kt + 1 < kts ? kt + 1 : kt, 0);         // (behind a tile's last K-tile: anything, nobody uses it)
        int from = kt + NB;
        if (from >= kts) {                                     // the next tile's K-tile of this buffer
            if (turns_to_next(kt, kts, NB)) {
                ahead += range.step;
                if (ahead < range.end) aim(ahead);
            }
            from = copied_behind(kt, kts, NB);
        }
        if (ahead < range.end) copy(buf, from);
        __builtin_amdgcn_sched_barrier(0);
        multiply(kSteps - 1);
    };
    aim(ahead);
    unrolled<NB>([&](auto i) {
        if (decltype(i)::value < kts) copy(buffer(i), decltype(i)::value);
    });
    if constexpr (MODE == kPanel) {
        float* const scales = reinterpret_cast<float*>(panel + kts * (S::tokens * kPackK));
        constexpr int X = 8 / RowVec<T>::E;                    // (vectors of a lane: twice as many in fp32)
        const int t0 = only.t * S::tokens;
        if (n.c <= 64) make_panel<T, X, S::tokens, S::waves>(n, t0, count, panel, scales);
        else if (n.c <= 128) make_panel<T, 2 * X, S::tokens, S::waves>(n, t0, count, panel, scales);
        else make_panel<T, 4 * X, S::tokens, S::waves>(n, t0, count, panel, scales);
        static_assert(kPanelTiles * kPackK == 256, "... of rows that long");
    }
    wait_but((kts < NB ? kts : NB) - 1);
    arrived = 1;
    meet();
    operands(buf0, 0, 0);
    const float hi = act_hi(a.act);
    for (int64_t tile = range.begin; tile < range.end; tile += range.step) {
        const TileAt at = place_of(tile);
        const int t0 = at.t * S::tokens, c0 = at.c * S::channels;
#pragma unroll
        for (int t = 0; t < FT; ++t)
#pragma unroll
            for (int f = 0; f < FC; ++f) acc[t][f] = i32x16{};
        // what the sums are scaled with: a channel's and a row's by each thread, dealt out when the sums are there
        const int my_ch = c0 + (int)threadIdx.x;
        float my_ws = 0.0f, my_bias = 0.0f, my_rs = 0.0f;
        if ((int)threadIdx.x < S::channels && my_ch < a.n) {
            my_ws = a.w_scale[my_ch];
            if (a.bias != nullptr) my_bias = (float)static_cast<const T*>(a.bias)[my_ch];
        }
        if constexpr (MODE != kPanel)
            if ((int)threadIdx.x < S::tokens && in_rows(t0, (int)threadIdx.x, count)) my_rs = a.q_scale[t0 + (int)threadIdx.x];
        int kt = 0;
#pragma clang loop unroll(disable)
        for (; kt + NB <= kts; kt += NB)
            unrolled<NB>([&](auto i) { k_tile(kt + decltype(i)::value, buffer(i), buffer(Int<decltype(i)::value + 1>{})); });
        unrolled<NB - 1>([&](auto i) {
            if (kt + decltype(i)::value < kts) k_tile(kt + decltype(i)::value, buffer(i), buffer(Int<decltype(i)::value + 1>{}));
        });
        arrived = NB;
        if constexpr (MODE == kParts) {
            if (!last_part<FT * FC, S::threads>(reinterpret_cast<i32x16*>(acc), a.partial, a.arrived, (int)(tile / splits), part, splits, out_lds)) return;
        }
        wait_loads<0>();                                       // the next tile's first K-tiles have arrived, ...
        float* const factors = reinterpret_cast<float*>(out_lds);
        if ((int)threadIdx.x < S::channels) {
            factors[threadIdx.x] = my_ws;
            factors[S::channels + threadIdx.x] = my_bias;
        }
        if constexpr (MODE != kPanel)
            if ((int)threadIdx.x < S::tokens) factors[2 * S::channels + threadIdx.x] = my_rs;
        const float* row_factors = MODE == kPanel ? reinterpret_cast<const float*>(panel + kts * (S::tokens * kPackK)) : factors + 2 * S::channels;
        meet();                                                // ... everybody's
        f32x4 ws[FC][4], bias[FC][4];
        float rs[FT];
#pragma unroll
        for (int t = 0; t < FT; ++t) rs[t] = row_factors[(tw * FT + t) * 32 + lane % 32];
#pragma unroll
        for (int f = 0; f < FC; ++f)
#pragma unroll
            for (int g = 0; g < 4; ++g) {
                const int ch = (cw * FC + f) * 32 + g * 8 + lane / 32 * 4;
                ws[f][g] = *reinterpret_cast<const f32x4*>(factors + ch);
                bias[f][g] = *reinterpret_cast<const f32x4*>(factors + S::channels + ch);
            }
        meet();
        int8_t* mine = out_lds + wave * S::unit;
        constexpr int E = RowVec<T>::E, PW = S::row / 16, UF = PW * E / 32;
        // this lane's first 16 bytes on their way out: row r0 of the tile, channel ch0
        const int r0 = tw * FT * 32 + lane / PW, ch0 = c0 + cw * FC * 32 + lane % PW * E;
        T* const y0 = static_cast<T*>(a.y) + ((int64_t)t0 + r0) * a.ldy + ch0;
        const bool cut = c0 + S::channels > a.n && a.n % E != 0;
        constexpr int kAsk = 2;
        auto leave = [&](auto acts) {                          // 0: no activation, 1: one, kAsk: see there
#pragma unroll
            for (int t = 0; t < FT; ++t)
#pragma unroll
                for (int u = 0; u < FC / UF; ++u) {
                    // PW places of 16 bytes to a token, exchanged by the token's low bits
#pragma unroll
                    for (int fu = 0; fu < UF; ++fu)
#pragma unroll
                        for (int g = 0; g < 4; ++g) {
                            const int f = u * UF + fu, c = fu * 32 + g * 8 + lane / 32 * 4;
                            float v[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) v[e] = scaled_sum(acc[t][f][g * 4 + e], rs[t], ws[f][g][e], bias[f][g][e]);
                            if (decltype(acts)::value == kAsk ? a.act != DCNN_ACT_NONE : decltype(acts)::value != 0) act_keep_nan(v, hi);
                            AlignedQuad<T> out;
#pragma unroll
                            for (int e = 0; e < 4; ++e) out[e] = (T)v[e];
                            *reinterpret_cast<AlignedQuad<T>*>(mine + ((lane % 32) * PW + (c / E ^ lane % PW)) * 16 + c % E * sizeof(T)) = out;
                        }
                    lds_wave_sync();
                    const int8_t* from = mine + (lane / PW * PW + (lane % PW ^ lane / PW % PW)) * 16;      // (rows further on: the same low bits)
                    static_assert(kWave / PW % PW == 0, "whole exchanges of places");
                    T* y = y0 + (int64_t)(t * 32) * a.ldy + u * UF * 32;
                    const auto piece = [&](int i) { return *reinterpret_cast<const AlignedVec<T>*>(from + i * kWave * 16); };
                    const int ch = ch0 + u * UF * 32, left = count - t0 - r0 - t * 32;   // rows from this lane's first one on
                    const int whole = ch + E <= a.n ? left : 0;
#pragma unroll
                    for (int i = 0; i < 32 * PW / kWave; ++i) {
                        const AlignedVec<T> v = piece(i);
                        if (i * (kWave / PW) < whole)
                            __builtin_nontemporal_store((typename RowVec<T>::type)v, reinterpret_cast<typename RowVec<T>::type*>(y + (int64_t)(i * (kWave / PW)) * a.ldy));
                    }
                    if (__builtin_expect(cut, 0) && ch < a.n && ch + E > a.n) {          // a lane's last 16 bytes are not all there
#pragma clang loop unroll(disable)
                        for (int i = 0; i < 32 * PW / kWave && i * (kWave / PW) < left; ++i, y += (int64_t)(kWave / PW) * a.ldy)
#pragma clang loop unroll(disable)
                            for (int e = 0; e < a.n - ch; ++e) y[e] = reinterpret_cast<const T*>(from + i * kWave * 16)[e];
                    }
                    lds_wave_sync();
                }
        };
        // (a copy for each, where tiles follow one another: 26214 x 256 -> 1024 17.5 us, asked at every four outputs 18.3.  The largest tile's
        // wants more registers than there are, 8000 x 4096 -> 4096 144 us in place of 127; the smallest is a workgroup's only one: 4.2 / 3.8
        // for 512 x 256 -> 1024, the code is read once)
        if constexpr (FT * FC >= 8 || FT * FC == 1) leave(Int<kAsk>{});
        else if (a.act == DCNN_ACT_NONE) leave(Int<0>{});
        else leave(Int<1>{});
        operands(buf0, 0, 0);                                  // (read here and not at the tile's begin: nothing is left to be waited for)
    }
}

template <typename T, int TW, int CW, int FT, int FC, int NB, TileMode MODE = kWhole>
static dcnn_status launch_tile(dcnn_ctx* ctx, const MatmulArgs& a, int splits = 1, int share = 0, const FewRows* rows = nullptr) {
    using S = TileShape<T, TW, CW, FT, FC, NB, MODE>;
    const int64_t tiles = cdiv(a.rows, S::tokens) * cdiv(a.n, S::channels) * splits;
    const int64_t most = MODE != kWhole ? tiles : (int64_t)ctx->num_cu * (int64_t)(ctx->max_lds / S::lds);
    const int64_t grid = cdiv(tiles < most ? tiles : most, kXcd) * kXcd;   // (tile_range deals out to whole rounds of XCDs)
    if constexpr (MODE == kPanel) {
        auto kern = rows_matmul_kernel<T, TW, CW, FT, FC, NB, MODE>;
        const size_t panel = (size_t)a.kt * S::tokens * kPackK + S::tokens * sizeof(float);
        static bool attr_set = false;
        if (!attr_set) {
            const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize,
                                                       kPanelTiles * S::tokens * kPackK + S::tokens * (int)sizeof(float));
            if (err != hipSuccess) return check_hip(ctx, err, "hipFuncSetAttribute(rows_matmul_kernel)");
            attr_set = true;
        }
        hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(S::threads), panel, ctx->stream, a, splits, share, *rows);
    } else {
        hipLaunchKernelGGL((rows_matmul_kernel<T, TW, CW, FT, FC, NB, MODE>), dim3((unsigned)grid), dim3(S::threads), 0, ctx->stream, a, splits, share, 0);
    }
    return check_hip(ctx, hipGetLastError(), "rows_matmul_kernel launch");
}

// ---- few rows -----------------------------------------------------------------------------------------------------
// Up to G*16 tokens: the weights are all there is to read, once, and every workgroup reads its own: F*16 channels, whose k the workgroup's
// waves deal out among themselves in steps of 64, with kAhead steps of a wave on their way at a time.  A step is one instruction of the
// matrix cores (16 channels by 16 tokens) per F and G.  The waves' sums meet in LDS.
//
// NORM > 0: up to NORM tokens are normed and quantised on the spot, by every workgroup for itself (a row is 8 KB that the caches hold, a
// launch of its own takes longer), while the first weights are on their way.
//
// Bound by the weights' bytes and the launch (3.2 us): 1 x 4096 -> 4096 6.2 us in a row with weights from memory (3.7 where the caches hold
// them), 16 rows 7.4, 32 rows 9.1 to 10.9 (their 8-bit rows from L2 or memory, as many bytes as the weights); 1 x 8192 -> 1024 5.5 to 7.0.
constexpr int kFewWaves = 8, kAhead = 8;
template <int G, int F> struct FewShape {
    static constexpr int sums = kFewWaves * G * F * kWave * 16;
};

template <typename T, int G, int F, int NORM, int NV>
__global__ __launch_bounds__(kFewWaves * kWave) void rows_few_kernel(MatmulArgs a, FewRows n) {
    constexpr int L = kFewWaves * kWave;
    extern __shared__ __align__(16) int8_t lds[];              // sums, then (NORM) the 8-bit rows
    __shared__ uint32_t red[2 * kFewWaves];
    __shared__ float scales[NORM > 0 ? NORM : 1];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int count = row_count(a.count, a.rows);
    const int steps = (a.kc + 3) / 4;                          // of 64 k
    const int c0 = blockIdx.x * (F * 16);
    if (count == 0) return;
    // 16 channels of a block of 32, four chunks of 16 k to a step
    const int w_block_bytes = a.kt * kPackK * kPackC;
    const __amdgpu_buffer_rsrc_t w = ws_rsrc(a.w + (int64_t)(c0 / kPackC) * w_block_bytes, kWsMaxBytes);
    const int w_lane = c0 % kPackC * 16 + lane / 16 * (kPackC * 16) + lane % 16 * 16;
    auto weights = [&](int step, int f) {                      // (F = 2: both halves of a block)
        const uint32_t at = step < steps ? (uint32_t)(w_lane + step * (64 * kPackC) + f * 256) : kOob;
        return ws_load16<i32x4>(w, at);
    };
    i32x4 wv[kAhead][F];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
#pragma unroll
        for (int f = 0; f < F; ++f) wv[i][f] = weights(wave + i * kFewWaves, f);

    // what this thread's four sums are scaled with at the end (G * F waves have some): lane: channels lane / 16 * 4 .. + 3 of token lane % 16
    static_assert(G * F <= kFewWaves, "a wave for each 16 x 16 sums");
    const int out_row = wave / F * 16 + lane % 16, out_ch = c0 + wave % F * 16 + lane / 16 * 4;
    const bool out = wave < G * F && out_row < count && out_ch < a.n;
    f32x4 ws{}, bias{};
    float rs = 0.0f;
    if (out) {
        ws = *reinterpret_cast<const f32x4*>(a.w_scale + out_ch);
        bias = load_bias<T>(a.bias, out_ch, a.n);
        if constexpr (NORM == 0) rs = a.q_scale[out_row];
    }

    const int row_bytes = steps * 64 + 16;                     // (16: rows start on different banks)
    int8_t* rows = lds + FewShape<G, F>::sums;
    if constexpr (NORM > 0) {
        constexpr int E = RowVec<T>::E;
        int turn = 0;
        const float inv_c = 1.0f / (float)n.c;
        NormParams<T, L, NV, true> params;
        params.read(n.w, n.b, threadIdx.x, n.c);
#pragma unroll
        for (int r = 0; r < NORM; ++r) {
            int i = r;
            if (n.idx != nullptr) i = r < count ? n.idx[r] : -1;
            const bool token = r < count && i >= 0 && i < n.map_rows;
            const T* x = static_cast<const T*>(n.x) + (int64_t)(token ? i : 0) * n.ldx;
            float v[NV][E];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const u32x4 xv = row_load<T>(x, token ? (j * L + (int)threadIdx.x) * E : n.c, n.c);
#pragma unroll
                for (int e = 0; e < E; ++e) v[j][e] = row_get<T>(xv, e);
            }
            if (n.kind != DCNN_NORM_NONE)
                norm_row<T, L, NV, true>(v, n.kind, n.eps, params, threadIdx.x, n.c, inv_c, red, turn);
            if (!token) {
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int e = 0; e < E; ++e) v[j][e] = 0.0f;
            }
            float inv;
            const float scale = quantize_scale(row_amax<L, NV, E>(v, red, turn), &inv);
#pragma unroll
            for (int j = 0; j < NV; ++j) row_store_quantized<T>(rows + r * row_bytes, (j * L + (int)threadIdx.x) * E, n.c, v[j], inv);
            if (threadIdx.x == 0) scales[r] = scale;
        }
        __syncthreads();
    }
    const __amdgpu_buffer_rsrc_t q = ws_rsrc(a.q, NORM > 0 ? 0 : kWsMaxBytes);
    const int token = lane % 16 < count ? lane % 16 : count - 1;
    uint32_t q_lane[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {                              // tokens behind the last one read the last one
        const int row = g * 16 + lane % 16;
        q_lane[g] = (uint32_t)(row < count ? row : count - 1) * (uint32_t)a.ldq;
    }
    auto tokens = [&](int step, int g) {
        const int chunk = step * 4 + lane / 16;
        if constexpr (NORM > 0) {                              // (steps behind the last one have no weights: any tokens do)
            return *reinterpret_cast<const i32x4*>(rows + (token < NORM ? token : 0) * row_bytes + (step < steps ? chunk : 0) * 16);
        } else {
            return ws_load16<i32x4>(q, chunk < a.kc ? q_lane[g] + (uint32_t)chunk * 16 : kOob);
        }
    };
    i32x4 acc[G][F] = {};
    for (int s0 = wave; s0 < steps; s0 += kAhead * kFewWaves) {
        i32x4 qv[kAhead][G];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int g = 0; g < G; ++g) qv[i][g] = tokens(s0 + i * kFewWaves, g);
        i32x4 next[kAhead][F];
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int f = 0; f < F; ++f) next[i][f] = weights(s0 + (kAhead + i) * kFewWaves, f);
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int g = 0; g < G; ++g)
#pragma unroll
                for (int f = 0; f < F; ++f) acc[g][f] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[i][f], qv[i][g], acc[g][f], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int f = 0; f < F; ++f) wv[i][f] = next[i][f];
    }
    i32x4* sums = reinterpret_cast<i32x4*>(lds);
#pragma unroll
    for (int g = 0; g < G; ++g)
#pragma unroll
        for (int f = 0; f < F; ++f) sums[((wave * G + g) * F + f) * kWave + lane] = acc[g][f];
    __syncthreads();
    if (!out) return;
    i32x4 s = sums[wave * kWave + lane];
#pragma unroll
    for (int i = 1; i < kFewWaves; ++i) s += sums[(i * G * F + wave) * kWave + lane];
    if constexpr (NORM > 0) rs = scales[out_row < NORM ? out_row : 0];
    float v[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = scaled_sum(s[e], rs, ws[e], bias[e]);
    if (a.act != DCNN_ACT_NONE) act_keep_nan(v, act_hi(a.act));
    T* y = static_cast<T*>(a.y) + (int64_t)out_row * a.ldy + out_ch;
    if (out_ch + 4 <= a.n) {
        typename RowQuad<T>::type quad;
#pragma unroll
        for (int e = 0; e < 4; ++e) quad[e] = (T)v[e];
        *reinterpret_cast<typename RowQuad<T>::type*>(y) = quad;
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (out_ch + e < a.n) y[e] = (T)v[e];
    }
}

template <typename T, int G, int F, int NORM, int NV> static dcnn_status launch_few(dcnn_ctx* ctx, const MatmulArgs& a, const FewRows& n) {
    const size_t lds = FewShape<G, F>::sums + (NORM > 0 ? (size_t)NORM * (cdiv(a.kc, 4) * 64 + 16) : 0);
    hipLaunchKernelGGL((rows_few_kernel<T, G, F, NORM, NV>), dim3((unsigned)cdiv(a.n, F * 16)), dim3(kFewWaves * kWave), lds, ctx->stream, a, n);
    return check_hip(ctx, hipGetLastError(), "rows_few_kernel launch");
}

// ---- norm, 8-bit rows and product in one kernel ---------------------------------------------------------------------------
// Rows that every workgroup norms for itself: 512 lanes hold a row in one or two vectors each.
constexpr int kFewNorm = 4;
static bool fuses_few(int dtype, int64_t rows, int64_t k) { return rows <= kFewNorm && align_up((size_t)k, 64) <= (dtype == DCNN_F32 ? 4096 : 8192); }
// Short rows of which all tiles are in work at a time, in workgroups that norm 64 of them each.
static int64_t panel_tiles(int64_t rows, int64_t n, bool counted) { return cdiv(counted ? cdiv(rows, 4) : rows, 64) * cdiv(n, 128); }
bool rows_linear_fuses(int dtype, int64_t rows, int64_t k, int64_t n, bool counted) {
    return fuses_few(dtype, rows, k) || (packed_k(k) <= kPanelTiles * kPackK && panel_tiles(rows, n, counted) <= 2 * kPlanCus);
}

template <typename T> static dcnn_status launch_linear_t(dcnn_ctx* ctx, const FewRows& n, const MatmulArgs& a) {
    if (!fuses_few(sizeof(T) == 4 ? DCNN_F32 : DCNN_F16, a.rows, n.c)) return launch_tile<T, 2, 4, 1, 1, 2, kPanel>(ctx, a, 1, 0, &n);
    const bool one = (int64_t)cdiv(n.c, 64) * 64 <= kFewWaves * kWave * RowVec<T>::E;
    if (a.rows == 1) return one ? launch_few<T, 1, 1, 1, 1>(ctx, a, n) : launch_few<T, 1, 1, 1, 2>(ctx, a, n);
    return one ? launch_few<T, 1, 1, kFewNorm, 1>(ctx, a, n) : launch_few<T, 1, 1, kFewNorm, 2>(ctx, a, n);
}

dcnn_status launch_rows_linear_fused(dcnn_ctx* ctx, int dtype, const NormArgs& norm, const MatmulArgs& a) {
    const FewRows n{norm.x, norm.pre_w, norm.pre_b, norm.idx, norm.ldx, norm.map_rows, norm.c, norm.pre, norm.pre_eps};
    if (dtype == DCNN_F16) return launch_linear_t<f16>(ctx, n, a);
    if (dtype == DCNN_BF16) return launch_linear_t<bf16>(ctx, n, a);
    return launch_linear_t<float>(ctx, n, a);
}

// ---- which kernel ------------------------------------------------------------------------------------------------------
// us, in a row on the GPU, weights from memory, rows that the caches hold (rows, k -> n); a launch alone is 3.2:
//   17 to 32 rows: few / tiles of 64   24, 4096 -> 4096: 8.9 / 11.1   24, 1024 -> 256: 4.6 / 5.1   32, 8192 -> 1024: 11.3 / 10.9   32, 16384 -> 512: 19.5 / 12.5
//   tiles of 64 / 128 deep / 128 / 256   500, 4096 -> 4096 (128 tiles of 128): 20 / 23 / 32 / 50   1000, 4096 -> 4096 (256): 35 / 25 / 33 / 50
//                                        2000, 4096 -> 4096 (512): 67 / 46 / 40 / 50   4000, 4096 -> 4096 (1024; 256 of 256): 128 / 94 / 78 / 63
//                                        8000, 8192 -> 1024 (504; 128): 123 / 90 / 69 / 93   16384, 1000 -> 1531 (1536; 384): 61 / 45 / 43 / 53
//   128 in eight waves, three buffers / four   500, 2048 -> 8192: 13.8 / 14.4   2000, 2048 -> 2048: 13.6 / 14.2   1000, 4096 -> 4096: 25.0 / 24.5
//   pairs of 128, in four waves each / in eight   26214, 256 -> 1024: 18.0 / 18.6   6000, 512 -> 1024: 9.1 / 8.6   26214, 1000 -> 1531: 65 / 73
//   pairs of 128 / 256                   26214, 256 -> 1024: 17.9 / 19.4   16384, 512 -> 2048: 29.5 / 27.5   16384, 1000 -> 1531: 43 / 53   8000, 4096 -> 4096: 150 / 132
//   k of a tile of 64 in one / in parts  64, 8192 -> 1024: 22 / 10.9 (8)   64, 4096 -> 4096: 17 / 11.0 (4)   200, 8192 -> 1024: 22 / 12.5 (4), 14.4 (8)
//                                        500, 8192 -> 1024: 24 / 18.2 (2), 16.4 (4)   64, 1024 -> 256: 5.1 / 6.7 (2)
// A list's length is on the GPU: its plan is that of a quarter of its room, a guess that was measured only afterwards.  Product behind a count
// of 3, 10, 30 and 100 % of the room / of as many rows without one, the same matrices again:
//   262144, 256 -> 1024: 7.0 / 7.0, 19.8 / 17.7, 49 / 47, 156 / 152      65536, 512 -> 512: 6.0 / 4.4, 6.6 / 6.4, 11.5 / 11.5, 32 / 29
//   16384, 1024 -> 4096: 15.6 / 6.6, 16.4 / 11.8, 34 / 28, 80 / 78       16384, 256 -> 1024: 4.8 / 3.6, 5.1 / 4.3, 7.7 / 6.1, 14.1 / 10.9
MatmulPlan matmul_plan(int64_t rows, int64_t k, int64_t n, bool counted) {
    MatmulPlan p{kFewRows, 1, 0};
    const int64_t kt = packed_k(k) / kPackK;
    if (rows <= 16 || (rows <= 32 && kt < 64)) return p;
    const int64_t likely = counted ? cdiv(rows, 4) : rows;
    const int64_t tiles64 = cdiv(rows, 64) * cdiv(n, 64), tiles128 = cdiv(likely, 128) * cdiv(n, 128), tiles256 = cdiv(likely, 256) * cdiv(n, 256);
    if (tiles128 <= kPlanCus / 2) {
        p.kernel = kTile64;
        // few tiles: workgroups for all compute units, which take eight K-tiles at least; of a long k, four parts where there are twice as many
        const auto least = [](int64_t a, int64_t b) { return a < b ? a : b; };
        int64_t splits = least(least(kPlanCus / tiles64, kt / 8), 8);
        const int64_t more = least(2 * kPlanCus / tiles64, 4);
        if (kt >= 64 && splits < more) splits = more;
        if (splits > 1) {
            p.share = (int)cdiv(kt, splits);
            p.splits = (int)cdiv(kt, p.share);
        }
    } else if (tiles128 <= kPlanCus) {
        p.kernel = kTile128Deep;
    } else {
        // a round of tiles of 256 takes 1.7 times as long as one of tiles of 128 (two to a compute unit), of a short k or where it is not full 2.1
        const int64_t rounds256 = cdiv(tiles256, kPlanCus), rounds128 = cdiv(tiles128, 2 * kPlanCus);
        const bool full = 10 * tiles256 >= 8 * rounds256 * kPlanCus;
        p.kernel = (kt >= 8 && full ? 17 : 21) * rounds256 <= 10 * rounds128 ? kTile256 : kTile128;
    }
    return p;
}

// Room for the partial sums of calls with up to so many rows, whichever plan they get: workgroups that share tiles are at most eight to a tile
// and no more than the plan above allows in all.
size_t partial_bytes(int64_t rows, int64_t k, int64_t n) {
    const int64_t kt = packed_k(k) / kPackK, tiles_c = cdiv(n, 64), most = kt >= 64 ? 2 * kPlanCus : kPlanCus;
    if (rows <= 16 || kt < 16 || 2 * tiles_c > most) return 0;
    const int64_t parts = 8 * cdiv(rows, 64) * tiles_c;
    return (size_t)(parts < most ? parts : most) * 64 * 64 * sizeof(int32_t);
}

template <typename T> static dcnn_status launch_matmul_t(dcnn_ctx* ctx, const MatmulPlan& p, const MatmulArgs& a) {
    switch (p.kernel) {
        case kFewRows:
            // 32 channels to a workgroup where that makes one for every compute unit: 32, 2048 -> 8192: 9.3 against 10.2; 4096 -> 4096: 10.7, 9.3
            if (a.n >= 32 * kPlanCus) return a.rows <= 16 ? launch_few<T, 1, 2, 0, 1>(ctx, a, FewRows{}) : launch_few<T, 2, 2, 0, 1>(ctx, a, FewRows{});
            return a.rows <= 16 ? launch_few<T, 1, 1, 0, 1>(ctx, a, FewRows{}) : launch_few<T, 2, 1, 0, 1>(ctx, a, FewRows{});
        case kTile64: return p.splits > 1 ? launch_tile<T, 2, 2, 1, 1, 3, kParts>(ctx, a, p.splits, p.share) : launch_tile<T, 2, 2, 1, 1, 3>(ctx, a);
        case kTile128Deep: return launch_tile<T, 2, 4, 2, 1, 3>(ctx, a);
        case kTile128: return launch_tile<T, 2, 2, 2, 2, 2>(ctx, a);
        case kTile256: return launch_tile<T, 2, 4, 4, 2, 2>(ctx, a);
    }
    return DCNN_EINVAL;
}

dcnn_status launch_rows_matmul(dcnn_ctx* ctx, int dtype, const MatmulPlan& plan, const MatmulArgs& a) {
    if (a.rows == 0) return DCNN_OK;
    if (dtype == DCNN_F16) return launch_matmul_t<f16>(ctx, plan, a);
    if (dtype == DCNN_BF16) return launch_matmul_t<bf16>(ctx, plan, a);
    return launch_matmul_t<float>(ctx, plan, a);
}

}  // namespace dcnn
