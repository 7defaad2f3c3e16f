// Norms before and after a block, fused with its gate and residual scale, and rows in 8 bits.
//
//   y = x + scale * gate * post(h),  z = pre(y),  q = z in 8 bits with a scale of its own
//
// One pass: a row of c channels lives in the registers of its L lanes (8 to 64 lanes of a wave, or a workgroup of 256 to 1024), NV vectors
// of 16 bytes to a lane, so its mean, its variance (from the centred values, not from a difference of squares) and its largest magnitude
// are reductions over registers and nothing is read twice.  Few vectors and many lanes: with four vectors to a lane (what y needs, what
// the parameters hold) registers left one wave to a SIMD, 8192 rows of 8192 in 8 bits took 116 us in place of 40.
// fp32 all through; y, z and q are rounded once each, z and q from the unrounded y.
// y and z are stored past the L2 (non-temporal; see row_store): 5 to 20 % of the time.  x and h are not read so: 5 to 15 % more.
//
// Bound by HBM, 2 * c elements read and up to 2 * c written a row, and by the launch (3 us) below some 10 MB:
// (us in a row on the GPU: all matrices from memory / the same ones again, which the caches hold in part; a copy of 2 GB: 4.94 TB/s)
//   16384 x 4096 bf16, both norms, gate, y and z     104 (5.2 TB/s) / 90
//   16384 x 1024 bf16                                31  (4.4) / 25
//   26214 of 262144 x 256 fp16 by a list             13  (4.1)
//   4099 x 1037 fp32                                 22  (3.0) / 18     20000 x 500 fp16 19, x 512 19 (rows at odd addresses cost little)
//   8192 x 8192 fp16 to 8 bits                       40  (5.0) / 33     26214 x 256 by a list 9.6
//   1 x 2048 fp16                                    3.7
#include "rows_device.h"

namespace dcnn {

template <typename T, int L> struct NormShape {
    static constexpr int threads = L > 256 ? L : 256, rows = threads / L;
};

// BLOCK: there is an h.  (Without one six waves fit a SIMD; with five of them 8192 rows of 8192 in 8 bits took 30 % longer.)  HOLD: a lane's part of the parameters stays in registers from row to row.
template <typename T, int L, int NV, bool BLOCK>
__global__ __launch_bounds__((NormShape<T, L>::threads), !BLOCK && NV <= 2 ? 6 : 4) void rows_norm_kernel(NormArgs a) {
    constexpr int E = RowVec<T>::E, R = NormShape<T, L>::rows;
    constexpr bool HOLD = NV <= 2;
    __shared__ uint32_t red[2 * (L > kWave ? L / kWave : 1)];
    int turn = 0;
    const int lane = threadIdx.x % L, sub = threadIdx.x / L, c = a.c;
    const int count = row_count(a.count, a.rows);
    const float inv_c = 1.0f / (float)c;
    const T* const gate = static_cast<const T*>(a.gate);
    const bool gates = a.gate_div.d != 0;                      // a row of gate for each so many tokens
    NormParams<T, L, NV, HOLD> post, pre;
    u32x4 gv[BLOCK ? NV : 1];
    if constexpr (BLOCK) {
        post.read(a.post_w, a.post_b, lane, c);
        if (gate != nullptr && !gates) {
#pragma unroll
            for (int j = 0; j < NV; ++j) gv[j] = row_load<T>(gate, (j * L + lane) * E, c);
        }
    }
    pre.read(a.pre_w, a.pre_b, lane, c);
    for (int64_t base = (int64_t)blockIdx.x * R; base < count; base += (int64_t)gridDim.x * R) {
        const int64_t r = base + sub;
        const bool live = r < count;                           // (lanes without a row take part in the reductions)
        int64_t i = r;
        if (a.idx != nullptr) i = live ? a.idx[r] : -1;
        const bool token = live && i >= 0 && i < a.map_rows;
        const int width = token ? c : 0;
        float v[NV][E];
        u32x4 xv[NV];
        const bool have_x = a.x != nullptr;
        if (have_x) {
            const T* x = static_cast<const T*>(a.x) + i * a.ldx;
#pragma unroll
            for (int j = 0; j < NV; ++j) xv[j] = row_load<T>(x, (j * L + lane) * E, width);
        }
        if constexpr (BLOCK) {
            const T* h = static_cast<const T*>(a.h) + r * a.ldh;
            u32x4 hv[NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) hv[j] = row_load<T>(h, (j * L + lane) * E, width);
            if (gates) {
                const T* g = gate + (token ? (int64_t)fast_div((uint32_t)i, a.gate_div) * a.ldg : 0);
#pragma unroll
                for (int j = 0; j < NV; ++j) gv[j] = row_load<T>(g, (j * L + lane) * E, c);
            }
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < E; ++e) v[j][e] = row_get<T>(hv[j], e);
            if (a.post != DCNN_NORM_NONE) norm_row<T, L, NV, HOLD>(v, a.post, a.post_eps, post, lane, c, inv_c, red, turn);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                if (gate != nullptr) {
                    const u32x4 g = unknown(gv[j]);
#pragma unroll
                    for (int e = 0; e < E; ++e) v[j][e] *= row_get<T>(g, e);
                }
#pragma unroll
                for (int e = 0; e < E; ++e) v[j][e] = have_x ? row_get<T>(xv[j], e) + a.scale * v[j][e] : a.scale * v[j][e];
            }
            // in place, where a row's last vector holds elements of the one before it and another wave may have that one: all of the row has
            // been read before any of it is written
            if (L > kWave && a.y == a.x && c % E != 0) {
                __builtin_amdgcn_s_waitcnt(0x0f70);            // vmcnt(0)
                __syncthreads();
            }
            if (a.y != nullptr && token) {
                T* y = static_cast<T*>(a.y) + i * a.ldy;
#pragma unroll
                for (int j = 0; j < NV; ++j) row_store<T>(y, (j * L + lane) * E, c, v[j]);
            }
        } else {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < E; ++e) v[j][e] = row_get<T>(xv[j], e);
        }
        if (a.z == nullptr && a.q == nullptr) continue;
        if (a.pre != DCNN_NORM_NONE) norm_row<T, L, NV, HOLD>(v, a.pre, a.pre_eps, pre, lane, c, inv_c, red, turn);
        if (a.idx != nullptr && !token) {
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < E; ++e) v[j][e] = 0.0f;
        }
        if (a.z != nullptr && live) {
            T* z = static_cast<T*>(a.z) + r * a.ldz;
#pragma unroll
            for (int j = 0; j < NV; ++j) row_store<T>(z, (j * L + lane) * E, c, v[j]);
        }
        if (a.q != nullptr) {
            float inv;
            const float scale = quantize_scale(row_amax<L, NV, E>(v, red, turn), &inv);
            if (live) {
                int8_t* q = a.q + r * a.ldq;
#pragma unroll
                for (int j = 0; j < NV; ++j) row_store_quantized<T>(q, (j * L + lane) * E, c, v[j], inv);
                if (lane == 0) a.q_scale[r] = scale;
            }
        }
    }
}

template <typename T, int L, int NV, bool BLOCK> static dcnn_status launch_norm_shape(dcnn_ctx* ctx, const NormArgs& a) {
    constexpr int R = NormShape<T, L>::rows, threads = NormShape<T, L>::threads;
    // about as many workgroups as are resident at a time, 24 waves to a compute unit; they stride through the rows
    const int64_t most = (int64_t)ctx->num_cu * (24 * kWave / threads);
    const int64_t grid = cdiv(a.rows, R) < most ? cdiv(a.rows, R) : most;
    hipLaunchKernelGGL((rows_norm_kernel<T, L, NV, BLOCK>), dim3((unsigned)grid), dim3(threads), 0, ctx->stream, a);
    return check_hip(ctx, hipGetLastError(), "rows_norm_kernel launch");
}

template <typename T, bool BLOCK> static dcnn_status launch_norm_t(dcnn_ctx* ctx, const NormArgs& a) {
    const int64_t v = cdiv(a.c, RowVec<T>::E);                 // 16-byte vectors of a row
    if (v <= 8) return launch_norm_shape<T, 8, 1, BLOCK>(ctx, a);
    if (v <= 16) return launch_norm_shape<T, 16, 1, BLOCK>(ctx, a);
    if (v <= 32) return launch_norm_shape<T, 32, 1, BLOCK>(ctx, a);
    if (v <= 64) return launch_norm_shape<T, 64, 1, BLOCK>(ctx, a);
    if (v <= 128) return launch_norm_shape<T, 64, 2, BLOCK>(ctx, a);
    if (v <= 256) return launch_norm_shape<T, 256, 1, BLOCK>(ctx, a);
    if (v <= 512) return launch_norm_shape<T, 256, 2, BLOCK>(ctx, a);
    if (v <= 1024) return launch_norm_shape<T, 512, 2, BLOCK>(ctx, a);
    if (v <= 2048) return launch_norm_shape<T, 1024, 2, BLOCK>(ctx, a);
    if constexpr (kRowsMaxC / RowVec<T>::E > 4096)             // (fp32 alone)
        if (v > 4096) return launch_norm_shape<T, 1024, 8, BLOCK>(ctx, a);
    return launch_norm_shape<T, 1024, 4, BLOCK>(ctx, a);
}
template <typename T> static dcnn_status launch_norm_any(dcnn_ctx* ctx, const NormArgs& a) {
    return a.h != nullptr ? launch_norm_t<T, true>(ctx, a) : launch_norm_t<T, false>(ctx, a);
}

dcnn_status launch_rows_norm(dcnn_ctx* ctx, int dtype, const NormArgs& a) {
    if (a.rows == 0) return DCNN_OK;
    if (dtype == DCNN_F16) return launch_norm_any<f16>(ctx, a);
    if (dtype == DCNN_BF16) return launch_norm_any<bf16>(ctx, a);
    return launch_norm_any<float>(ctx, a);
}

}  // namespace dcnn
