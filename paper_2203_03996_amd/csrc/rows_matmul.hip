// Products of rows in 8-bit integers with weights in 8-bit integers: a scale for each row and for each output channel.
//
//   y[r][j] = act( (sum_k q[r][k] w[k][j]) * (q_scale[r] * w_scale[j]) + bias[j] )
//
// The sums are exact in 32-bit integers, so how a sum is cut up never changes a result.
#include "rows_device.h"

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
// A workgroup of TW x CW waves computes TW*FT*32 rows by CW*FC*32 channels, K-tiles of 128 at a time.  A K-tile of both operands is
// staged through registers into one of two LDS buffers while the other is multiplied.  Weights lie in LDS as they are packed
// (an operand load of a wave is 1 KB in a row); a row's eight chunks of 16 k are exchanged by the low bits of its number, so
// that the lanes of an operand load, 32 rows at one k, start on different banks.  The channels are the matrix cores' rows and
// the tokens their columns: a lane ends with four consecutive channels of one token.
template <typename T, int TW, int CW, int FT, int FC> struct TileShape {
    static constexpr int threads = TW * CW * kWave, tokens = TW * FT * 32, channels = CW * FC * 32;
    static constexpr int stage = (tokens + channels) * kPackK;
};

template <typename T, int TW, int CW, int FT, int FC>
__global__ __launch_bounds__(TW * CW * kWave) void rows_matmul_kernel(MatmulArgs a) {
    using S = TileShape<T, TW, CW, FT, FC>;
    constexpr int CH = kPackK / 16;                            // chunks of a row of a K-tile
    constexpr int QL = S::tokens * CH / S::threads, WL = S::channels * CH / S::threads;
    extern __shared__ __align__(16) int8_t lds[];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const int tw = wave / CW, cw = wave % CW;
    const int count = row_count(a.count, a.rows);
    const int tiles_t = (count + S::tokens - 1) / S::tokens, tiles_c = (a.n + S::channels - 1) / S::channels;
    const int blocks_c = (a.n + kPackC - 1) / kPackC;
    const int q_row = tid / CH, q_chunk = (tid % CH) ^ (q_row % CH);       // rows tid/8 + i*threads/8: the same low bits
    const int w_ch = tid % kPackC, w_k = tid / kPackC % CH, w_block = tid / (kPackC * CH);
    constexpr int w_step = S::threads / (kPackC * CH);
    static_assert(S::threads % (kPackC * CH) == 0, "a round of loads is whole blocks of packed weights");
    const int64_t w_block_bytes = (int64_t)a.kt * kPackK * kPackC;
    const WgTileRange range = wg_tile_range((int64_t)tiles_t * tiles_c);
    for (int64_t tile = range.begin; tile < range.end; tile += range.step) {
        const int t0 = (int)(tile / tiles_c) * S::tokens, c0 = (int)(tile % tiles_c) * S::channels;
        const int8_t* q_at[QL];
        const int8_t* w_at[WL];
#pragma unroll
        for (int i = 0; i < QL; ++i) {                         // rows behind the last one read the last one
            const int row = t0 + q_row + i * (S::threads / CH);
            q_at[i] = a.q + (int64_t)(row < count ? row : count - 1) * a.ldq;
        }
#pragma unroll
        for (int i = 0; i < WL; ++i) {
            const int block = c0 / kPackC + w_block + i * w_step;
            w_at[i] = a.w + (block < blocks_c ? block : blocks_c - 1) * w_block_bytes + (w_k * kPackC + w_ch) * 16;
        }
        u32x4 qv[QL], wv[WL];
        auto load = [&](int kt) {
            const int chunk = kt * CH + q_chunk;               // chunks behind a row's last one: any, their weights are zero
            const int at = (chunk < a.kc ? chunk : 0) * 16;
#pragma unroll
            for (int i = 0; i < QL; ++i) qv[i] = *reinterpret_cast<const u32x4*>(q_at[i] + at);
#pragma unroll
            for (int i = 0; i < WL; ++i) wv[i] = *reinterpret_cast<const u32x4*>(w_at[i] + (int64_t)kt * (kPackK * kPackC));
        };
        auto stage = [&](int buf) {
            int8_t* s = lds + buf * S::stage;
#pragma unroll
            for (int i = 0; i < QL; ++i) *reinterpret_cast<u32x4*>(s + (tid + i * S::threads) * 16) = qv[i];
            s += S::tokens * kPackK;
#pragma unroll
            for (int i = 0; i < WL; ++i) *reinterpret_cast<u32x4*>(s + (tid + i * S::threads) * 16) = wv[i];
        };
        i32x16 acc[FT][FC] = {};
        load(0);
        stage(0);
        __syncthreads();
        for (int kt = 0; kt < a.kt; ++kt) {
            if (kt + 1 < a.kt) load(kt + 1);
            const int8_t* s = lds + (kt & 1) * S::stage;
#pragma unroll
            for (int ks = 0; ks < kPackK / 32; ++ks) {
                i32x4 qf[FT], wf[FC];
                const int chunk = 2 * ks + lane / 32;
#pragma unroll
                for (int t = 0; t < FT; ++t) {
                    const int row = (tw * FT + t) * 32 + lane % 32;
                    qf[t] = *reinterpret_cast<const i32x4*>(s + row * kPackK + (chunk ^ (row % CH)) * 16);
                }
#pragma unroll
                for (int f = 0; f < FC; ++f)
                    wf[f] = *reinterpret_cast<const i32x4*>(s + S::tokens * kPackK + ((cw * FC + f) * CH + chunk) * (kPackC * 16) + lane % 32 * 16);
#pragma unroll
                for (int t = 0; t < FT; ++t)
#pragma unroll
                    for (int f = 0; f < FC; ++f) acc[t][f] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wf[f], qf[t], acc[t][f], 0, 0, 0);
            }
            if (kt + 1 < a.kt) stage((kt + 1) & 1);
            __syncthreads();
        }
        const float hi = act_hi(a.act);
#pragma unroll
        for (int t = 0; t < FT; ++t) {
            const int row = t0 + (tw * FT + t) * 32 + lane % 32;
            if (row >= count) continue;
            const float rs = a.q_scale[row];
            T* y = static_cast<T*>(a.y) + (int64_t)row * a.ldy;
#pragma unroll
            for (int f = 0; f < FC; ++f)
#pragma unroll
                for (int g = 0; g < 4; ++g) {
                    const int ch = c0 + (cw * FC + f) * 32 + g * 8 + lane / 32 * 4;
                    if (ch >= a.n) continue;
                    // (the channel scales are padded to whole blocks)
                    const f32x4 ws = *reinterpret_cast<const f32x4*>(a.w_scale + ch);
                    typename RowQuad<T>::type out;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float v = (float)acc[t][f][g * 4 + e] * (rs * ws[e]);
                        if (a.bias != nullptr && ch + e < a.n) v += (float)static_cast<const T*>(a.bias)[ch + e];
                        out[e] = (T)(a.act == DCNN_ACT_NONE ? v : act_keep_nan(v, hi));
                    }
                    if (ch + 4 <= a.n) {
                        *reinterpret_cast<typename RowQuad<T>::type*>(y + ch) = out;
                    } else {
#pragma unroll
                        for (int e = 0; e < 4; ++e)
                            if (ch + e < a.n) y[ch + e] = out[e];
                    }
                }
        }
    }
}

template <typename T, int TW, int CW, int FT, int FC> static dcnn_status launch_tile(dcnn_ctx* ctx, const MatmulArgs& a) {
    using S = TileShape<T, TW, CW, FT, FC>;
    auto kern = rows_matmul_kernel<T, TW, CW, FT, FC>;
    static bool attr_set = false;
    if (!attr_set) {
        const hipError_t err = hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, 2 * S::stage);
        if (err != hipSuccess) return check_hip(ctx, err, "hipFuncSetAttribute(rows_matmul_kernel)");
        attr_set = true;
    }
    const int64_t tiles = cdiv(a.rows, S::tokens) * cdiv(a.n, S::channels);
    const int64_t most = (int64_t)ctx->num_cu * (int64_t)(ctx->max_lds / (2 * S::stage));
    const int64_t grid = cdiv(tiles < most ? tiles : most, kXcd) * kXcd;   // (tile_range deals out to whole rounds of XCDs)
    hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(S::threads), 2 * S::stage, ctx->stream, a);
    return check_hip(ctx, hipGetLastError(), "rows_matmul_kernel launch");
}

template <typename T> static dcnn_status launch_matmul_t(dcnn_ctx* ctx, const MatmulArgs& a) {
    return launch_tile<T, 2, 2, 2, 2>(ctx, a);
}

dcnn_status launch_rows_matmul(dcnn_ctx* ctx, int dtype, const MatmulArgs& a) {
    if (a.rows == 0) return DCNN_OK;
    if (dtype == DCNN_F16) return launch_matmul_t<f16>(ctx, a);
    if (dtype == DCNN_BF16) return launch_matmul_t<bf16>(ctx, a);
    return launch_matmul_t<float>(ctx, a);
}

}  // namespace dcnn
