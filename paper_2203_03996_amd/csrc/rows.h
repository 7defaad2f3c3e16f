// Row operators: what their translation units share (internal).
#pragma once

#include "common.h"

namespace dcnn {

constexpr int kRowsMaxC = 32768;               // channels of a row that is normed or quantised: it stays in registers
constexpr int64_t kRowsMaxK = 65536;           // 65536 products of 8-bit integers: at most 2^30 in magnitude, exact in 32 bits
constexpr int64_t kRowsMaxN = 1 << 24;
constexpr int64_t kRowsMax = 0x7fffffff;       // rows of a map or of a compact matrix
constexpr int64_t kLdMax = 0x7fffffff;         // leading dimensions travel in 32 bits, offsets are formed in 64
constexpr int kPackC = 32;                     // channels of a block of packed weights
constexpr int kPackK = 128;                    // the packed weights' k is padded with zeros to a multiple of this

inline size_t rows_dtype_size(int dt) { return dt == DCNN_F32 ? 4 : (dt == DCNN_I8 ? 1 : 2); }
inline bool rows_float(int dt) { return dt == DCNN_F32 || dt == DCNN_F16 || dt == DCNN_BF16; }

// Packed weights: [n / 32][k / 16][32 channels][16 bytes of k], then the channel scales [n rounded up to 32].  Sixteen consecutive
// k of a channel are one operand register quad of a lane, and the 32 channels of a block are the 32 lanes that want them.
inline int64_t packed_k(int64_t k) { return cdiv(k, kPackK) * kPackK; }
inline int64_t packed_n(int64_t n) { return cdiv(n, kPackC) * kPackC; }
inline size_t packed_scale_offset(int64_t k, int64_t n) { return (size_t)(packed_k(k) * packed_n(n)); }

// Kernel arguments (leading dimensions and row counts fit 31 bits: the launchers' callers check it).
struct NormArgs {
    const void *x, *h, *gate, *post_w, *post_b, *pre_w, *pre_b;
    void *y, *z;
    int8_t* q;
    float* q_scale;
    const int32_t *idx, *count;
    int rows, map_rows;
    int ldx, ldh, ldg, ldy, ldz, ldq;
    int c, post, pre;
    float post_eps, pre_eps, scale;
    FastDiv gate_div;            // d = 0: one row of gate for all
};
dcnn_status launch_rows_norm(dcnn_ctx* ctx, int dtype, const NormArgs& a);

struct MatmulArgs {
    const int8_t* q;
    const float* q_scale;
    const int8_t* w;             // packed
    const float* w_scale;
    const void* bias;            // may be null
    void* y;
    const int32_t* count;        // may be null
    int rows, n;
    int ldq, ldy;
    int kc, kt;                  // chunks of 16 k that a row holds, K-tiles of kPackK
    int act;
    int32_t* partial;            // sums of workgroups that share a tile, and a count of those that are done for each tile:
    uint32_t* arrived;           //    zero before the launch and after it
};
// Which kernel: a function of the sizes alone.
enum MatmulKernel { kFewRows, kTile64, kTile128Deep, kTile128, kTile256 };
struct MatmulPlan {
    MatmulKernel kernel;
    int splits;                  // workgroups that share a tile's k (kTile64), each `share` K-tiles of it
    int share;
};
MatmulPlan matmul_plan(int64_t rows, int64_t k, int64_t n, bool counted);
size_t partial_bytes(int64_t rows, int64_t k, int64_t n);
constexpr size_t kArrivedBytes = 2048;         // counts of the workgroups of 512 tiles
dcnn_status launch_rows_matmul(dcnn_ctx* ctx, int dtype, const MatmulPlan& plan, const MatmulArgs& a);
// Norm, 8-bit rows and product in one kernel, for a token or a few: x, idx, map_rows, ldx, c and pre of NormArgs, all of MatmulArgs but q.
bool rows_linear_fuses(int dtype, int64_t rows, int64_t k, int64_t n, bool counted);
dcnn_status launch_rows_linear_fused(dcnn_ctx* ctx, int dtype, const NormArgs& norm, const MatmulArgs& a);
dcnn_status launch_rows_pack(dcnn_ctx* ctx, int dtype, int64_t k, int64_t n, const void* w, int64_t ldw, const float* scale,
                             int8_t* packed, float* packed_scale);

}  // namespace dcnn
