// Norms before and after a block, fused with its gate and residual scale, and rows in 8 bits.
//
//   y = x + scale * gate * post(h),  z = pre(y),  q = z in 8 bits with a scale of its own
//
// One pass: a row of c channels lives in the registers of its L lanes (8 .. 64 lanes of a wave, or a workgroup of 256 or 1024), so
// its mean, its variance (from the centred values, not from a difference of squares) and its largest magnitude are reductions
// over registers and nothing is read twice.  Bound by HBM: 2 * c elements read and up to 2 * c written per row.
#include "rows_device.h"

namespace dcnn {

template <typename T, int L> struct NormShape {
    static constexpr int threads = L > 256 ? L : 256, rows = threads / L;
};

template <typename T, int L, int NV> __global__ __launch_bounds__((NormShape<T, L>::threads)) void rows_norm_kernel(NormArgs a) {
    constexpr int E = RowVec<T>::E, R = NormShape<T, L>::rows;
    typedef typename RowVec<T>::type Vec;
    __shared__ uint32_t red[2 * (L > kWave ? L / kWave : 1)];
    int turn = 0;
    const int lane = threadIdx.x % L, sub = threadIdx.x / L, c = a.c;
    const int count = row_count(a.count, a.rows);
    const float inv_c = 1.0f / (float)c;
    for (int64_t base = (int64_t)blockIdx.x * R; base < count; base += (int64_t)gridDim.x * R) {
        const int64_t r = base + sub;
        const bool live = r < count;                           // (lanes without a row take part in the reductions)
        int64_t i = r;
        if (a.idx != nullptr) i = live ? a.idx[r] : -1;
        const bool token = live && i >= 0 && i < a.map_rows;
        float v[NV][E];
        Vec xv[NV];
        const T* x = static_cast<const T*>(a.x) + i * a.ldx;
        const bool have_x = a.x != nullptr && token;
        if (have_x) {
#pragma unroll
            for (int j = 0; j < NV; ++j) xv[j] = row_load<T>(x, (j * L + lane) * E, c);
        }
        if (a.h != nullptr) {
            const T* h = static_cast<const T*>(a.h) + r * a.ldh;
            const T* gate = static_cast<const T*>(a.gate);
            if (gate != nullptr && a.gate_div.d != 0 && token) gate += (int64_t)fast_div((uint32_t)i, a.gate_div) * a.ldg;
            Vec gv[NV];
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                const int at = token ? (j * L + lane) * E : c;
                const Vec hv = row_load<T>(h, at, c);
                if (gate != nullptr) gv[j] = row_load<T>(gate, at, c);
#pragma unroll
                for (int e = 0; e < E; ++e) v[j][e] = (float)hv[e];
            }
            if (a.post != DCNN_NORM_NONE)
                norm_row<T, L, NV>(v, a.post, a.post_eps, static_cast<const T*>(a.post_w), static_cast<const T*>(a.post_b), lane, c, inv_c, red, turn);
#pragma unroll
            for (int j = 0; j < NV; ++j)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    v[j][e] *= a.scale;
                    if (gate != nullptr) v[j][e] *= (float)gv[j][e];
                    if (have_x) v[j][e] += (float)xv[j][e];
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
                for (int e = 0; e < E; ++e) v[j][e] = have_x ? (float)xv[j][e] : 0.0f;
        }
        if (a.z == nullptr && a.q == nullptr) continue;
        if (a.pre != DCNN_NORM_NONE)
            norm_row<T, L, NV>(v, a.pre, a.pre_eps, static_cast<const T*>(a.pre_w), static_cast<const T*>(a.pre_b), lane, c, inv_c, red, turn);
        if (!token) {
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
                for (int j = 0; j < NV; ++j) {
                    // (a row's last vector ends within the multiple of 16 that a row of 8-bit integers takes)
                    const int at = (j * L + lane) * E;
                    if (at < c) store_quantized<E>(q + at, v[j], inv);
                }
                if (lane == 0) a.q_scale[r] = scale;
            }
        }
    }
}

template <typename T, int L, int NV> static dcnn_status launch_norm_shape(dcnn_ctx* ctx, const NormArgs& a) {
    constexpr int R = NormShape<T, L>::rows, threads = NormShape<T, L>::threads;
    // as many workgroups as are resident at a time (eight of 256 threads to a compute unit); they stride through the rows
    const int64_t most = (int64_t)ctx->num_cu * (2048 / threads);
    const int64_t grid = cdiv(a.rows, R) < most ? cdiv(a.rows, R) : most;
    hipLaunchKernelGGL((rows_norm_kernel<T, L, NV>), dim3((unsigned)grid), dim3(threads), 0, ctx->stream, a);
    return check_hip(ctx, hipGetLastError(), "rows_norm_kernel launch");
}

template <typename T> static dcnn_status launch_norm_t(dcnn_ctx* ctx, const NormArgs& a) {
    const int64_t v = cdiv(a.c, RowVec<T>::E);                 // 16-byte vectors of a row
    if (v <= 8) return launch_norm_shape<T, 8, 1>(ctx, a);
    if (v <= 16) return launch_norm_shape<T, 16, 1>(ctx, a);
    if (v <= 32) return launch_norm_shape<T, 32, 1>(ctx, a);
    if (v <= 64) return launch_norm_shape<T, 64, 1>(ctx, a);
    if (v <= 128) return launch_norm_shape<T, 64, 2>(ctx, a);
    if (v <= 256) return launch_norm_shape<T, 64, 4>(ctx, a);
    if (v <= 512) return launch_norm_shape<T, 256, 2>(ctx, a);
    if (v <= 1024) return launch_norm_shape<T, 256, 4>(ctx, a);
    if (v <= 2048) return launch_norm_shape<T, 1024, 2>(ctx, a);
    if (v <= 4096) return launch_norm_shape<T, 1024, 4>(ctx, a);
    return launch_norm_shape<T, 1024, 8>(ctx, a);
}

dcnn_status launch_rows_norm(dcnn_ctx* ctx, int dtype, const NormArgs& a) {
    if (a.rows == 0) return DCNN_OK;
    if (dtype == DCNN_F16) return launch_norm_t<f16>(ctx, a);
    if (dtype == DCNN_BF16) return launch_norm_t<bf16>(ctx, a);
    return launch_norm_t<float>(ctx, a);
}

}  // namespace dcnn
