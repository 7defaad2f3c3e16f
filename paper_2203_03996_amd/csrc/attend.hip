// Attention over the cache: which kernel, and what joins the parts of rows whose tokens are shared among workgroups.
#include "attend_device.h"

namespace dcnn {

// The parts of a row and head as one.
template <typename T, int D> __global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a) {
    constexpr int E = (D + 63) / 64;
    __shared__ float sums[4][D];
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    const int count = row_count(a.tokens.count, a.tokens.rows);
    const int q_heads = a.cache.heads * a.group;
    for (int unit = blockIdx.x; unit < count * q_heads; unit += gridDim.x) {
        const int r = unit / q_heads, q_head = unit % q_heads;
        const int64_t first = (int64_t)unit * a.splits;
        float top = -INFINITY;
        for (int s = lane; s < a.splits; s += kWave) top = fmaxf(top, a.stat[(first + s) * 2]);
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) top = fmaxf(top, __shfl_xor(top, d, kWave));
        const float base = top == -INFINITY ? 0.0f : top;
        float total = 0.0f, o[E] = {};
#pragma unroll 4
        for (int s = wave; s < a.splits; s += 4) {
            const int64_t at = first + s;
            const float m = a.stat[at * 2], w = top == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(m - base);
            total += a.stat[at * 2 + 1] * w;
#pragma unroll
            for (int e = 0; e < E; ++e)
                if (lane + 64 * e < D) o[e] += a.part[at * D + lane + 64 * e] * w;
        }
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (lane + 64 * e < D) sums[wave][lane + 64 * e] = o[e];
        __shared__ float totals[4];
        if (lane == 0) totals[wave] = total;
        __syncthreads();
        total = totals[0] + totals[1] + totals[2] + totals[3];
        if ((int)threadIdx.x < D) {
            const int d = threadIdx.x;
            const float v = sums[0][d] + sums[1][d] + sums[2][d] + sums[3][d];
            static_cast<T*>(a.y)[(int64_t)r * a.ldy + (int64_t)q_head * D + d] = (T)(total == 0.0f ? 0.0f : v / total);
        }
        __syncthreads();
    }
}

AttendPlan attend_plan(int64_t rows, int q_heads, int heads, int64_t streams, int64_t length) {
    const int64_t group = q_heads / heads;
    AttendPlan p;
    p.tiles = rows > 2 * streams;
    const int64_t units = p.tiles ? cdiv(rows * group, 128) * heads : rows * heads * cdiv(group, 16);
    const int64_t wanted = cdiv(p.tiles ? 512 : 2048, units < 1 ? 1 : units), most = cdiv(length, p.tiles ? 512 : 256);
    p.splits = (int)(wanted < most ? wanted : most);
    return p;
}

template <typename T> static dcnn_status launch_join(dcnn_ctx* ctx, int dim, const AttendArgs& a) {
    const int64_t outs = (int64_t)a.tokens.rows * a.cache.heads * a.group, most = (int64_t)ctx->num_cu * 16;
    const dim3 grid((unsigned)(outs < most ? outs : most));
    switch (dim) {
        case 32: hipLaunchKernelGGL((attend_join_kernel<T, 32>), grid, dim3(256), 0, ctx->stream, a); break;
        case 64: hipLaunchKernelGGL((attend_join_kernel<T, 64>), grid, dim3(256), 0, ctx->stream, a); break;
        case 96: hipLaunchKernelGGL((attend_join_kernel<T, 96>), grid, dim3(256), 0, ctx->stream, a); break;
        case 128: hipLaunchKernelGGL((attend_join_kernel<T, 128>), grid, dim3(256), 0, ctx->stream, a); break;
        case 192: hipLaunchKernelGGL((attend_join_kernel<T, 192>), grid, dim3(256), 0, ctx->stream, a); break;
        default: hipLaunchKernelGGL((attend_join_kernel<T, 256>), grid, dim3(256), 0, ctx->stream, a); break;
    }
    return check_hip(ctx, hipGetLastError(), "attend_join_kernel launch");
}

dcnn_status launch_attend(dcnn_ctx* ctx, int dtype, int dim, const AttendPlan& plan, const AttendArgs& a) {
    const dcnn_status st = plan.tiles ? launch_attend_tile(ctx, dtype, dim, a) : launch_attend_few(ctx, dtype, dim, a);
    if (st != DCNN_OK || a.splits == 1) return st;
    if (dtype == DCNN_F16) return launch_join<f16>(ctx, dim, a);
    if (dtype == DCNN_BF16) return launch_join<bf16>(ctx, dim, a);
    return launch_join<float>(ctx, dim, a);
}

}  // namespace dcnn
