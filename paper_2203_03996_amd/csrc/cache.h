// Heads, the cache in 4 bits and attention over it: what their translation units share (internal).
#pragma once

#include "rows.h"

namespace dcnn {

constexpr int64_t kCacheMaxLength = 1 << 30;   // positions, with a tile of tokens behind them, fit 31 bits
constexpr int64_t kMaxHeadRows = 1 << 30;      // rows * heads of a call
constexpr int64_t kMaxPageBytes = 0xffffffff;  // of a page's codes: the factor of a page's number fits 32 bits
constexpr int kMxBlock = 32;                   // values that share a scale

inline bool cache_dim(int d) { return d == 32 || d == 64 || d == 96 || d == 128 || d == 192 || d == 256; }

// Which token a row is (see dcnn_row_tokens).
struct TokenArgs {
    const int32_t *idx, *count, *stream, *pos;
    int rows, map_rows;
    FastDiv period;
};
struct CacheArgs {
    uint8_t *codes, *scales;
    const int32_t* pages;
    int heads, dim, page_shift, num_pages;
    int streams, length, per_stream;           // per_stream: pages of a stream
};
struct RotationArgs {
    const float* table;                        // null: none
    int positions, rot, style;
};
// One matrix of heads of a call.
struct HeadJob {
    const void *in, *w, *b;
    void* out;
    int64_t ld_in, ld_out;
    int heads, norm;
    float eps;
};
enum HeadsOp { kTurnHeads, kAppendHeads, kReadHeads };
struct HeadsArgs {
    TokenArgs tokens;
    CacheArgs cache;                           // append, read
    RotationArgs rotation;                     // of both jobs' heads (kTurnHeads), of the keys (kAppendHeads)
    HeadJob job[2];                            // queries and keys, or keys and values
    int jobs, shift;                           // 2^shift heads of a row are side by side in a workgroup at most (filled in at the launch)
};
dcnn_status launch_heads(dcnn_ctx* ctx, int dtype, int dim, HeadsOp op, const HeadsArgs& a);

struct AttendArgs {
    TokenArgs tokens;
    CacheArgs cache;
    const void* q;
    void* y;
    int64_t ldq, ldy;
    int group;                                 // query heads of a head of keys
    int blocks;                                // sixteens of them
    float factor;                              // |scale| * log2(e), above zero
    int negate;                                // scale is below zero: the queries' opposites
    int causal;
    int64_t window;                            // 0: none
    const int32_t* lens;
    FastDiv by_group;
    int splits;                                // tiles: workgroups that share the tokens of a tile of rows; else: that share all rows' of a head (0: none do)
    int* plan;                                 // (shared rows) tiles of a share, then the tiles before each row and behind the last
    float *part, *stat;                        // sums of parts [part][dim], their maxima and sums of weights [part][2]
};
constexpr int kShareRows = 512;                // rows at most whose tokens are shared evenly
// Which kernel: a function of the sizes alone.
struct AttendPlan {
    bool tiles;                                // rows of one stream share its tiles of tokens
    int splits;
    int64_t parts;                             // of the sums of workgroups that share a row
};
AttendPlan attend_plan(int dtype_size, int64_t rows, int q_heads, int heads, int dim, int64_t streams, int64_t length);
dcnn_status launch_attend(dcnn_ctx* ctx, int dtype, int dim, const AttendPlan& plan, const AttendArgs& a);
dcnn_status launch_attend_few(dcnn_ctx* ctx, int dtype, int dim, const AttendArgs& a);
dcnn_status launch_attend_tile(dcnn_ctx* ctx, int dtype, int dim, const AttendArgs& a);

}  // namespace dcnn
