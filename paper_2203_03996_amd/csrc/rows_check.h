// Checks of arguments that the entry points of row operators and of the cache share (host code).
#pragma once

#include "overlap.h"
#include "rows.h"

namespace dcnn {

inline bool aligned(const void* p, size_t a) { return reinterpret_cast<uintptr_t>(p) % a == 0; }

inline dcnn_status check_list(dcnn_ctx* ctx, const char* what, const dcnn_row_list& l) {
    if (l.rows < 0 || l.rows > kRowsMax) return fail(ctx, DCNN_EINVAL, "%s: %lld rows", what, (long long)l.rows);
    if (!aligned(l.idx_dev, 4) || !aligned(l.count_dev, 4)) return fail(ctx, DCNN_EINVAL, "%s: idx or count not 4-byte aligned", what);
    return DCNN_OK;
}
// the part of the list that maps need
inline dcnn_status check_map(dcnn_ctx* ctx, const char* what, const dcnn_row_list& l) {
    if (l.map_rows < 0 || l.map_rows > kRowsMax) return fail(ctx, DCNN_EINVAL, "%s: maps of %lld rows", what, (long long)l.map_rows);
    if (l.idx_dev == nullptr && l.map_rows < l.rows)
        return fail(ctx, DCNN_ESHAPE, "%s: %lld rows of maps that have %lld", what, (long long)l.rows, (long long)l.map_rows);
    return DCNN_OK;
}
inline dcnn_status check_ld(dcnn_ctx* ctx, const char* what, const char* name, const void* p, int64_t ld, int64_t c, size_t es) {
    if (p == nullptr) return DCNN_OK;
    if (ld < c) return fail(ctx, DCNN_ESHAPE, "%s: leading dimension %lld of %s is less than its %lld columns", what, (long long)ld, name, (long long)c);
    if (ld > kLdMax) return fail(ctx, DCNN_EUNSUPPORTED, "%s: leading dimension %lld of %s", what, (long long)ld, name);
    if (!aligned(p, es)) return fail(ctx, DCNN_EINVAL, "%s: %s is not aligned to its elements", what, name);
    return DCNN_OK;
}
inline dcnn_status check_norm(dcnn_ctx* ctx, const char* what, const dcnn_row_norm& n, size_t es) {
    if (n.kind < DCNN_NORM_NONE || n.kind > DCNN_NORM_LAYER) return fail(ctx, DCNN_EINVAL, "%s: norm %d", what, n.kind);
    if (n.kind == DCNN_NORM_NONE) return DCNN_OK;
    if (!(n.eps >= 0.0f) || n.eps > 3.0e38f) return fail(ctx, DCNN_EINVAL, "%s: a norm's eps must be finite and not negative", what);
    if (!aligned(n.w_dev, es) || !aligned(n.b_dev, es)) return fail(ctx, DCNN_EINVAL, "%s: a norm's parameters are not aligned to their elements", what);
    return DCNN_OK;
}
inline void set_norm(const dcnn_row_norm& n, int* kind, float* eps, const void** w, const void** b) {
    *kind = n.kind;
    *eps = n.eps;
    *w = n.kind == DCNN_NORM_NONE ? nullptr : n.w_dev;
    *b = n.kind == DCNN_NORM_NONE ? nullptr : n.b_dev;
}
// An output shares no byte with an input or another output: workgroups run in any order, and what one of them reads another may have
// written over.  (`x` may be `y`, and `x2` `y2`, the caller says where: a row is read before it is written.)
template <int OUTS, int INS>
inline dcnn_status check_apart(dcnn_ctx* ctx, const char* what, const Bytes (&outs)[OUTS], const Bytes (&ins)[INS], const Bytes* y = nullptr, const Bytes* x = nullptr,
                               const Bytes* y2 = nullptr, const Bytes* x2 = nullptr) {
    for (int i = 0; i < OUTS; ++i) {
        for (int j = i + 1; j < OUTS; ++j)
            if (overlap(outs[i], outs[j])) return fail(ctx, DCNN_EINVAL, "%s: %s overlaps %s", what, outs[i].name, outs[j].name);
        for (int j = 0; j < INS; ++j)
            if (!(&outs[i] == y && &ins[j] == x) && !(&outs[i] == y2 && &ins[j] == x2) && overlap(outs[i], ins[j])) return fail(ctx, DCNN_EINVAL, "%s: %s overlaps %s", what, outs[i].name, ins[j].name);
    }
    return DCNN_OK;
}
inline Bytes vector_bytes(const char* name, const void* p, int64_t bytes) { return {name, p, 1, bytes, bytes}; }
inline Bytes matrix_bytes(const char* name, const void* p, int64_t rows, int64_t ld, int64_t c, size_t es) { return {name, p, rows, ld * (int64_t)es, c * (int64_t)es}; }

}  // namespace dcnn
