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
        // the row's parts: those of its tile, or those of the workgroups that its tokens were shared among
        int parts = a.splits, from = 0, tiles_before = 0, share = 0;
        if (a.plan != nullptr) {
            share = a.plan[0], tiles_before = a.plan[1 + r];
            const int tiles = a.plan[2 + r] - tiles_before;
            from = tiles_before / share;
            parts = tiles > 0 ? (tiles_before + tiles - 1) / share - from + 1 : 1;
            if (parts == 1) continue;                          // (written already)
        }
        const int column = q_head % a.group, hb = q_head / a.group * a.blocks + column / 16;
        const auto part = [&](int s) {
            if (a.plan == nullptr) return (int64_t)unit * a.splits + s;
            return part_at(hb, from + s, a.splits, s == 0 && tiles_before % share != 0) + column % 16;
        };
        float top = -INFINITY;
        for (int s = lane; s < parts; s += kWave) top = fmaxf(top, a.stat[part(s) * 2]);
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) top = fmaxf(top, __shfl_xor(top, d, kWave));
        const float base = top == -INFINITY ? 0.0f : top;
        float total = 0.0f, o[E] = {};
#pragma unroll 4
        for (int s = wave; s < parts; s += 4) {
            const int64_t at = part(s);
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

AttendPlan attend_plan(int dtype_size, int64_t rows, int q_heads, int heads, int dim, int64_t streams, int64_t length) {
    const int64_t group = q_heads / heads;
    AttendPlan p;
    p.tiles = rows > 2 * streams;
    if (p.tiles) {
        const int64_t units = cdiv(rows * group, 128) * heads, wanted = cdiv(512, units < 1 ? 1 : units), most = cdiv(length, 512);
        p.splits = (int)(wanted < most ? wanted : most);
        p.parts = p.splits > 1 ? rows * q_heads * p.splits : 0;
    } else {
        // as many workgroups as are resident at a time; where every row is a few tiles, or rows are many, one takes whole rows
        const int64_t columns = heads * cdiv(group, 16), resident = dim * (dtype_size == 4 ? 3 : 1) <= 192 ? 512 : 256;
        const int64_t shares = resident / columns;
        p.splits = shares > 1 && rows <= kShareRows && length > 256 && rows * cdiv(length, 64) < 1 << 30 ? (int)shares : 0;
        p.parts = columns * p.splits * 32;
    }
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
    if (st != DCNN_OK || plan.parts == 0) return st;
    if (dtype == DCNN_F16) return launch_join<f16>(ctx, dim, a);
    if (dtype == DCNN_BF16) return launch_join<bf16>(ctx, dim, a);
    return launch_join<float>(ctx, dim, a);
}

}  // namespace dcnn
