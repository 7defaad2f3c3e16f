// Attention over the cache: which kernel, and what joins the parts of rows whose tokens are shared among workgroups.
#include "attend_device.h"

namespace dcnn {

// The parts of a row and head as one: out = sum_s 2^(top_s - top) part_s / sum_s 2^(top_s - top) sum_s.  What it takes is the way to memory and back:
// few parts are asked for all at once, by a wave for itself (512 rows of 32 heads of 128 in two parts took 22 us with four waves and a barrier); of rows
// alone, one may have most of the parts, and four waves share them.
constexpr int kFewParts = 8;

template <typename T, int D> __global__ __launch_bounds__(256) void attend_join_few_kernel(AttendArgs a) {
    constexpr int E = (D + 63) / 64;
    const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
    const int q_heads = a.cache.heads * a.group, units = row_count(a.tokens.count, a.tokens.rows) * q_heads, parts = a.splits;
    for (int unit = (int)blockIdx.x * 4 + wave; unit < units; unit += gridDim.x * 4) {
        const int64_t at = (int64_t)unit * parts;
        float v[kFewParts][E], top = -INFINITY, sum = 0.0f;
        if (lane < parts) top = a.stat[(at + lane) * 2], sum = a.stat[(at + lane) * 2 + 1];
#pragma unroll
        for (int s = 0; s < kFewParts; ++s)
#pragma unroll
            for (int e = 0; e < E; ++e) v[s][e] = s < parts && lane + 64 * e < D ? a.part[(at + s) * D + lane + 64 * e] : 0.0f;
        float most = top;
#pragma unroll
        for (int d = 1; d < kFewParts; d *= 2) most = fmaxf(most, __shfl_xor(most, d, kWave));
        // (a part that sees nothing has sums of zero)
        const float w = most == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(top - most);
        float total = sum * w;
#pragma unroll
        for (int d = 1; d < kFewParts; d *= 2) total += __shfl_xor(total, d, kWave);
        total = __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, total)));
        float o[E] = {};
#pragma unroll
        for (int s = 0; s < kFewParts; ++s) {
            const float ws = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, w), s));
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = s < parts ? __builtin_fmaf(v[s][e], ws, o[e]) : o[e];
        }
        const int r = unit / q_heads, q_head = unit - r * q_heads;
        T* const y = static_cast<T*>(a.y) + (int64_t)r * a.ldy + (int64_t)q_head * D;
#pragma unroll
        for (int e = 0; e < E; ++e)
            if (lane + 64 * e < D) y[lane + 64 * e] = (T)(total == 0.0f ? 0.0f : o[e] / total);
    }
}
template <typename T, int D> __global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a) {
    constexpr int E = (D + 63) / 64;
    __shared__ float sums[4][D], totals[4];
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
#pragma unroll 8
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
    // A tile of 128 query vectors reads its tokens once, a row alone reads them for itself: some rows of a stream find them in the caches.
    // (16 streams of 4096 tokens, 32 heads on 8 of 128: four rows each take 48 us alone and 57 in tiles, six 72 and 79, eight 87 and 56.)
    // `rows` are those that the call has room for, taken as spread over all streams: fewer, or those of a few streams, are known on the GPU alone.
    p.tiles = rows > 6 * streams;
    if (p.tiles) {
        // two workgroups to a compute unit, with 256 tokens each at least (512 rows of a stream of 8192 tokens, the same heads: 278 us unsplit, 96 us;
        // 64 rows of 2048: 78, 31 with 512 tokens at least, 24)
        const int64_t units = cdiv(rows * group, 128) * heads, wanted = cdiv(512, units < 1 ? 1 : units), most = cdiv(length, 256);
        p.splits = (int)(wanted < most ? wanted : most);
        // A few more tiles than are resident at a time leave most of the card to the last ones: halves or thirds fill it better, up to where the join
        // costs as much (2080 rows of 32 heads on 8 of 128, 8192 tokens: 376, 349 and 342 us whole, in halves, in thirds; 3000 rows 380, 388, 400, but
        // of 2048 tokens 165, 150, 155; 4000 rows 439, 475, 493; of heads of 64 the sums of parts are small: 20000 rows of 8, 4096 tokens, 242, 224, 226)
        const int waves = tile_waves(dim / 32, dtype_size == 4 ? 3 : 1);
        const int64_t slots = 256 * waves;
        if (units > slots && length >= 2048) p.splits = units * 10 <= slots * 13 ? 3 : units * 2 <= slots * (waves > 2 ? 5 : 3) ? 2 : p.splits;
        p.parts = p.splits > 1 ? rows * q_heads * p.splits : 0;
    } else {
        // As many workgroups as are resident at a time, each an equal part of the tokens of all rows: their lengths may be any.  Where every row is a
        // few tiles, or rows are many, workgroups take whole rows and need neither the plan nor the join (a row of the same heads: 512 tokens take
        // 8.3 us whole and 10.5 shared, 1024 11.3 and 10.7, 2048 17.0 and 11.1; 512 rows of 1024, 113 and 126).
        const int64_t columns = heads * cdiv(group, 16), resident = dim * (dtype_size == 4 ? 3 : 1) <= 192 ? 512 : 256;
        const int64_t shares = resident / columns;
        p.splits = shares > 1 && rows <= kShareRows && length > 1024 && rows * cdiv(length, 64) < 1 << 30 ? (int)shares : 0;
        p.parts = columns * p.splits * 32;
    }
    return p;
}

template <typename T, int D> static dcnn_status launch_join_dim(dcnn_ctx* ctx, const AttendArgs& a) {
    const int64_t outs = (int64_t)a.tokens.rows * a.cache.heads * a.group, most = (int64_t)ctx->num_cu * 16;
    if (a.plan == nullptr && a.splits <= kFewParts) {
        const int64_t groups = cdiv(outs, 4);
        hipLaunchKernelGGL((attend_join_few_kernel<T, D>), dim3((unsigned)(groups < most ? groups : most)), dim3(256), 0, ctx->stream, a);
    } else hipLaunchKernelGGL((attend_join_kernel<T, D>), dim3((unsigned)(outs < most ? outs : most)), dim3(256), 0, ctx->stream, a);
    return check_hip(ctx, hipGetLastError(), "attend_join_kernel launch");
}
template <typename T> static dcnn_status launch_join(dcnn_ctx* ctx, int dim, const AttendArgs& a) {
    switch (dim) {
        case 32: return launch_join_dim<T, 32>(ctx, a);
        case 64: return launch_join_dim<T, 64>(ctx, a);
        case 96: return launch_join_dim<T, 96>(ctx, a);
        case 128: return launch_join_dim<T, 128>(ctx, a);
        case 192: return launch_join_dim<T, 192>(ctx, a);
        default: return launch_join_dim<T, 256>(ctx, a);
    }
}

dcnn_status launch_attend(dcnn_ctx* ctx, int dtype, int dim, const AttendPlan& plan, const AttendArgs& a) {
    const dcnn_status st = plan.tiles ? launch_attend_tile(ctx, dtype, dim, a) : launch_attend_few(ctx, dtype, dim, a);
    if (st != DCNN_OK || plan.parts == 0) return st;
    if (dtype == DCNN_F16) return launch_join<f16>(ctx, dim, a);
    if (dtype == DCNN_BF16) return launch_join<bf16>(ctx, dim, a);
    return launch_join<float>(ctx, dim, a);
}

}  // namespace dcnn
