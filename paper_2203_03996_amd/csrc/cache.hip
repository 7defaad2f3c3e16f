// C entry points of heads, the cache in 4 bits and attention: checks of arguments, no kernels.
#include "cache.h"
#include "rows_check.h"

using namespace dcnn;

namespace {

constexpr size_t kPlanBytes = 4096;            // of the scratch: the tiles of a share, and those before each of up to kShareRows rows
static_assert((kShareRows + 2) * sizeof(int) <= kPlanBytes, "room for the rows");

dcnn_status check_tokens(dcnn_ctx* ctx, const char* what, const dcnn_row_tokens& t, bool streams, bool positions, TokenArgs* a) {
    dcnn_status st = check_list(ctx, what, t.list);
    if (st == DCNN_OK) st = check_map(ctx, what, t.list);
    if (st != DCNN_OK) return st;
    if (!aligned(t.stream_dev, 4) || !aligned(t.pos_dev, 4)) return fail(ctx, DCNN_EINVAL, "%s: streams or positions not 4-byte aligned", what);
    const bool divides = (streams && t.stream_dev == nullptr) || (positions && t.pos_dev == nullptr);
    if (divides && (t.period < 1 || t.period > kRowsMax)) return fail(ctx, DCNN_EINVAL, "%s: a period of %lld tokens", what, (long long)t.period);
    a->idx = t.list.idx_dev, a->count = t.list.count_dev;
    a->stream = streams ? t.stream_dev : nullptr, a->pos = positions ? t.pos_dev : nullptr;
    a->rows = (int)t.list.rows, a->map_rows = (int)t.list.map_rows;
    a->period = make_fastdiv(divides ? (uint32_t)t.period : 1u);
    return DCNN_OK;
}
dcnn_status check_rotation(dcnn_ctx* ctx, const char* what, const dcnn_rotation& r, int dim, RotationArgs* a) {
    *a = RotationArgs{nullptr, 0, 0, 0};
    if (r.table_dev == nullptr) return DCNN_OK;
    if (r.rot < 16 || r.rot > dim || r.rot % 16 != 0) return fail(ctx, DCNN_EINVAL, "%s: %d of %d values rotated (a multiple of 16)", what, r.rot, dim);
    if (r.style != DCNN_ROT_HALVES && r.style != DCNN_ROT_PAIRS) return fail(ctx, DCNN_EINVAL, "%s: rotation of style %d", what, r.style);
    if (r.positions < 1 || r.positions > kRowsMax) return fail(ctx, DCNN_EINVAL, "%s: a rotation of %lld positions", what, (long long)r.positions);
    if (!aligned(r.table_dev, 16)) return fail(ctx, DCNN_EINVAL, "%s: the rotation's table is not 16-byte aligned", what);
    *a = RotationArgs{r.table_dev, (int)r.positions, r.rot, r.style};
    return DCNN_OK;
}
dcnn_status check_cache(dcnn_ctx* ctx, const char* what, const dcnn_cache& c, CacheArgs* a) {
    if (!rows_float(c.dtype)) return fail(ctx, DCNN_EDTYPE, "%s: dtype %d", what, c.dtype);
    if (!cache_dim(c.dim)) return fail(ctx, DCNN_EUNSUPPORTED, "%s: heads of %d values", what, c.dim);
    if (c.heads < 1 || c.heads > 65536) return fail(ctx, DCNN_EINVAL, "%s: %d heads", what, c.heads);
    if (c.page < 16 || c.page > 4096 || (c.page & (c.page - 1)) != 0) return fail(ctx, DCNN_EINVAL, "%s: pages of %d tokens", what, c.page);
    if (c.streams < 1 || c.streams > kRowsMax) return fail(ctx, DCNN_EINVAL, "%s: %lld streams", what, (long long)c.streams);
    if (c.length < 1 || c.length > kCacheMaxLength) return fail(ctx, DCNN_EINVAL, "%s: streams of %lld tokens", what, (long long)c.length);
    if (c.num_pages < 1 || c.num_pages > kRowsMax) return fail(ctx, DCNN_EINVAL, "%s: %lld pages", what, (long long)c.num_pages);
    if ((int64_t)c.heads * c.page * c.dim > kMaxPageBytes) return fail(ctx, DCNN_EUNSUPPORTED, "%s: pages of %d heads, %d tokens", what, c.heads, c.page);
    const int64_t per_stream = cdiv(c.length, c.page);
    if (c.pages_dev == nullptr && c.num_pages < c.streams * per_stream)
        return fail(ctx, DCNN_ESHAPE, "%s: %lld pages for %lld streams of %lld", what, (long long)c.num_pages, (long long)c.streams, (long long)per_stream);
    if (c.codes_dev == nullptr || c.scales_dev == nullptr) return fail(ctx, DCNN_EINVAL, "%s: the cache's codes or scales are null", what);
    if (!aligned(c.codes_dev, 16) || !aligned(c.scales_dev, 16) || !aligned(c.pages_dev, 4)) return fail(ctx, DCNN_EINVAL, "%s: the cache is not aligned", what);
    *a = CacheArgs{c.codes_dev, c.scales_dev, c.pages_dev, c.heads, c.dim, __builtin_ctz(c.page), (int)c.num_pages, (int)c.streams, (int)c.length, (int)per_stream};
    return DCNN_OK;
}
Bytes codes_bytes(const dcnn_cache& c) { return vector_bytes("the cache's codes", c.codes_dev, c.num_pages * c.heads * c.page * c.dim); }
Bytes scales_bytes(const dcnn_cache& c) { return vector_bytes("the cache's scales", c.scales_dev, c.num_pages * c.heads * c.page * (c.dim / 16)); }
Bytes pages_bytes(const dcnn_cache& c) { return vector_bytes("the page table", c.pages_dev, c.streams * cdiv(c.length, c.page) * 4); }
Bytes idx_bytes(const dcnn_row_tokens& t) { return vector_bytes("idx", t.list.idx_dev, t.list.rows * 4); }
Bytes count_bytes(const dcnn_row_tokens& t) { return vector_bytes("count", t.list.count_dev, 4); }
Bytes stream_bytes(const dcnn_row_tokens& t) { return vector_bytes("streams", t.stream_dev, t.list.map_rows * 4); }
Bytes pos_bytes(const dcnn_row_tokens& t) { return vector_bytes("positions", t.pos_dev, t.list.map_rows * 4); }
Bytes table_bytes(const dcnn_rotation& r) { return vector_bytes("the rotation's table", r.table_dev, r.positions * r.rot * 4); }

dcnn_status check_heads_matrix(dcnn_ctx* ctx, const char* what, const char* name, const void* p, int64_t ld, int64_t c, size_t es) {
    if (p == nullptr) return fail(ctx, DCNN_EINVAL, "%s: %s is null", what, name);
    return check_ld(ctx, what, name, p, ld, c, es);
}

}  // namespace

extern "C" {

dcnn_status dcnn_rows_heads(dcnn_ctx* ctx, const dcnn_rows_heads_args* p) {
    const char* what = "rows_heads";
    if (!ctx || !p) return DCNN_EINVAL;
    if (!rows_float(p->dtype)) return fail(ctx, DCNN_EDTYPE, "%s: dtype %d", what, p->dtype);
    if (!cache_dim(p->dim)) return fail(ctx, DCNN_EUNSUPPORTED, "%s: heads of %d values", what, p->dim);
    if (p->q_heads < 1 || p->q_heads > 65536 || p->k_heads < 0 || p->k_heads > 65536)
        return fail(ctx, DCNN_EINVAL, "%s: %d heads of queries, %d of keys", what, p->q_heads, p->k_heads);
    HeadsArgs a{};
    dcnn_status st = check_rotation(ctx, what, p->rotation, p->dim, &a.rotation);
    if (st == DCNN_OK) st = check_tokens(ctx, what, p->tokens, false, a.rotation.table != nullptr, &a.tokens);
    if (st != DCNN_OK || p->tokens.list.rows == 0) return st;  // (buffers of no rows may be null)
    const int64_t rows = p->tokens.list.rows, qc = (int64_t)p->q_heads * p->dim, kc = (int64_t)p->k_heads * p->dim;
    if (rows * (p->q_heads + p->k_heads) > kRowsMax) return fail(ctx, DCNN_EUNSUPPORTED, "%s: %lld rows of %d heads", what, (long long)rows, p->q_heads + p->k_heads);
    const size_t es = rows_dtype_size(p->dtype);
    st = check_heads_matrix(ctx, what, "q", p->q_dev, p->ldq, qc, es);
    if (st == DCNN_OK) st = check_heads_matrix(ctx, what, "q_out", p->q_out_dev, p->ldq_out, qc, es);
    if (st == DCNN_OK && kc > 0) st = check_heads_matrix(ctx, what, "k", p->k_dev, p->ldk, kc, es);
    if (st == DCNN_OK && kc > 0) st = check_heads_matrix(ctx, what, "k_out", p->k_out_dev, p->ldk_out, kc, es);
    if (st == DCNN_OK) st = check_norm(ctx, what, p->q_norm, es);
    if (st == DCNN_OK && kc > 0) st = check_norm(ctx, what, p->k_norm, es);
    if (st != DCNN_OK) return st;
    const void *k = kc > 0 ? p->k_dev : nullptr, *k_out = kc > 0 ? p->k_out_dev : nullptr;
    const bool q_here = p->q_dev == p->q_out_dev, k_here = k != nullptr && k == k_out;
    if ((q_here && rows > 1 && p->ldq != p->ldq_out) || (k_here && rows > 1 && p->ldk != p->ldk_out))
        return fail(ctx, DCNN_ESHAPE, "%s: in place with two leading dimensions", what);
    a.job[0].in = p->q_dev, a.job[0].out = p->q_out_dev, a.job[0].ld_in = p->ldq, a.job[0].ld_out = p->ldq_out, a.job[0].heads = p->q_heads;
    set_norm(p->q_norm, &a.job[0].norm, &a.job[0].eps, &a.job[0].w, &a.job[0].b);
    if (kc > 0) {
        a.job[1].in = k, a.job[1].out = p->k_out_dev, a.job[1].ld_in = p->ldk, a.job[1].ld_out = p->ldk_out, a.job[1].heads = p->k_heads;
        set_norm(p->k_norm, &a.job[1].norm, &a.job[1].eps, &a.job[1].w, &a.job[1].b);
    }
    const Bytes outs[] = {matrix_bytes("q_out", p->q_out_dev, rows, p->ldq_out, qc, es), matrix_bytes("k_out", k_out, rows, p->ldk_out, kc, es)};
    const int64_t d = p->dim * (int64_t)es;
    const Bytes ins[] = {matrix_bytes("q", p->q_dev, rows, p->ldq, qc, es), matrix_bytes("k", k, rows, p->ldk, kc, es),
                         vector_bytes("a norm's weight", a.job[0].w, d), vector_bytes("a norm's bias", a.job[0].b, d),
                         vector_bytes("a norm's weight", a.job[1].w, d), vector_bytes("a norm's bias", a.job[1].b, d),
                         idx_bytes(p->tokens), count_bytes(p->tokens), vector_bytes("positions", a.tokens.pos, p->tokens.list.map_rows * 4), table_bytes(p->rotation)};
    st = check_apart(ctx, what, outs, ins, q_here ? &outs[0] : nullptr, &ins[0], k_here ? &outs[1] : nullptr, &ins[1]);
    if (st != DCNN_OK) return st;
    return launch_heads(ctx, p->dtype, p->dim, kTurnHeads, a);
}

dcnn_status dcnn_cache_append(dcnn_ctx* ctx, const dcnn_cache_append_args* p) {
    const char* what = "cache_append";
    if (!ctx || !p) return DCNN_EINVAL;
    HeadsArgs a{};
    dcnn_status st = check_cache(ctx, what, p->cache, &a.cache);
    if (st == DCNN_OK) st = check_rotation(ctx, what, p->rotation, p->cache.dim, &a.rotation);
    if (st == DCNN_OK) st = check_tokens(ctx, what, p->tokens, true, true, &a.tokens);
    if (st != DCNN_OK || p->tokens.list.rows == 0) return st;
    const int64_t rows = p->tokens.list.rows, c = (int64_t)p->cache.heads * p->cache.dim;
    if (rows * p->cache.heads > kMaxHeadRows) return fail(ctx, DCNN_EUNSUPPORTED, "%s: %lld rows of %d heads", what, (long long)rows, p->cache.heads);
    const size_t es = rows_dtype_size(p->cache.dtype);
    st = check_heads_matrix(ctx, what, "k", p->k_dev, p->ldk, c, es);
    if (st == DCNN_OK) st = check_heads_matrix(ctx, what, "v", p->v_dev, p->ldv, c, es);
    if (st == DCNN_OK) st = check_norm(ctx, what, p->k_norm, es);
    if (st != DCNN_OK) return st;
    a.job[0].in = p->k_dev, a.job[0].ld_in = p->ldk, a.job[0].heads = p->cache.heads;
    set_norm(p->k_norm, &a.job[0].norm, &a.job[0].eps, &a.job[0].w, &a.job[0].b);
    a.job[1].in = p->v_dev, a.job[1].ld_in = p->ldv, a.job[1].heads = p->cache.heads;
    const Bytes outs[] = {codes_bytes(p->cache), scales_bytes(p->cache)};
    const int64_t d = p->cache.dim * (int64_t)es;
    const Bytes ins[] = {matrix_bytes("k", p->k_dev, rows, p->ldk, c, es), matrix_bytes("v", p->v_dev, rows, p->ldv, c, es),
                         vector_bytes("a norm's weight", a.job[0].w, d), vector_bytes("a norm's bias", a.job[0].b, d), pages_bytes(p->cache),
                         idx_bytes(p->tokens), count_bytes(p->tokens), stream_bytes(p->tokens), pos_bytes(p->tokens), table_bytes(p->rotation)};
    st = check_apart(ctx, what, outs, ins);
    if (st != DCNN_OK) return st;
    return launch_heads(ctx, p->cache.dtype, p->cache.dim, kAppendHeads, a);
}

dcnn_status dcnn_cache_read(dcnn_ctx* ctx, const dcnn_cache_read_args* p) {
    const char* what = "cache_read";
    if (!ctx || !p) return DCNN_EINVAL;
    HeadsArgs a{};
    dcnn_status st = check_cache(ctx, what, p->cache, &a.cache);
    if (st == DCNN_OK) st = check_tokens(ctx, what, p->tokens, true, true, &a.tokens);
    if (st != DCNN_OK || p->tokens.list.rows == 0) return st;
    const int64_t rows = p->tokens.list.rows, c = (int64_t)p->cache.heads * p->cache.dim;
    if (rows * p->cache.heads > kMaxHeadRows) return fail(ctx, DCNN_EUNSUPPORTED, "%s: %lld rows of %d heads", what, (long long)rows, p->cache.heads);
    if (p->k_out_dev == nullptr && p->v_out_dev == nullptr) return fail(ctx, DCNN_EINVAL, "%s: neither keys nor values are wanted", what);
    const size_t es = rows_dtype_size(p->cache.dtype);
    st = check_ld(ctx, what, "k", p->k_out_dev, p->ldk, c, es);
    if (st == DCNN_OK) st = check_ld(ctx, what, "v", p->v_out_dev, p->ldv, c, es);
    if (st != DCNN_OK) return st;
    a.job[0].out = p->k_out_dev, a.job[0].ld_out = p->ldk, a.job[0].heads = p->k_out_dev != nullptr ? p->cache.heads : 0;
    a.job[1].out = p->v_out_dev, a.job[1].ld_out = p->ldv, a.job[1].heads = p->v_out_dev != nullptr ? p->cache.heads : 0;
    const Bytes outs[] = {matrix_bytes("k", p->k_out_dev, rows, p->ldk, c, es), matrix_bytes("v", p->v_out_dev, rows, p->ldv, c, es)};
    const Bytes ins[] = {codes_bytes(p->cache), scales_bytes(p->cache), pages_bytes(p->cache), idx_bytes(p->tokens), count_bytes(p->tokens),
                         stream_bytes(p->tokens), pos_bytes(p->tokens)};
    st = check_apart(ctx, what, outs, ins);
    if (st != DCNN_OK) return st;
    return launch_heads(ctx, p->cache.dtype, p->cache.dim, kReadHeads, a);
}

size_t dcnn_cache_scratch_bytes(int32_t dtype, int64_t rows, int32_t q_heads, int32_t heads, int32_t dim, int64_t streams, int64_t length) {
    if (!rows_float(dtype) || rows < 0 || rows > kRowsMax || heads < 1 || q_heads < 1 || q_heads % heads != 0 || !cache_dim(dim)) return 0;
    if (streams < 1 || streams > kRowsMax || length < 1 || length > kCacheMaxLength || rows * q_heads > kMaxHeadRows) return 0;
    const AttendPlan plan = attend_plan((int)rows_dtype_size(dtype), rows, q_heads, heads, dim, streams, length);
    return kPlanBytes + align_up((size_t)plan.parts * 2 * sizeof(float)) + align_up((size_t)plan.parts * (size_t)dim * sizeof(float));
}

dcnn_status dcnn_cache_attend(dcnn_ctx* ctx, const dcnn_cache_attend_args* p) {
    const char* what = "cache_attend";
    if (!ctx || !p) return DCNN_EINVAL;
    AttendArgs a{};
    dcnn_status st = check_cache(ctx, what, p->cache, &a.cache);
    if (st == DCNN_OK) st = check_tokens(ctx, what, p->tokens, true, p->causal != 0 || p->window != 0, &a.tokens);
    if (st != DCNN_OK) return st;
    if (p->q_heads < 1 || p->q_heads > 65536 || p->q_heads % p->cache.heads != 0)
        return fail(ctx, DCNN_EINVAL, "%s: %d heads of queries, %d of keys", what, p->q_heads, p->cache.heads);
    if (!(p->scale == p->scale) || p->scale - p->scale != 0.0f) return fail(ctx, DCNN_EINVAL, "%s: a scale that is no number", what);
    if (p->window < 0) return fail(ctx, DCNN_EINVAL, "%s: a window of %lld tokens", what, (long long)p->window);
    if (!aligned(p->lens_dev, 4)) return fail(ctx, DCNN_EINVAL, "%s: lens not 4-byte aligned", what);
    const int64_t rows = p->tokens.list.rows, c = (int64_t)p->q_heads * p->cache.dim;
    if (rows == 0) return DCNN_OK;
    if (rows * p->q_heads > kMaxHeadRows) return fail(ctx, DCNN_EUNSUPPORTED, "%s: %lld rows of %d heads", what, (long long)rows, p->q_heads);
    const size_t es = rows_dtype_size(p->cache.dtype);
    st = check_heads_matrix(ctx, what, "q", p->q_dev, p->ldq, c, es);
    if (st == DCNN_OK) st = check_heads_matrix(ctx, what, "y", p->y_dev, p->ldy, c, es);
    if (st != DCNN_OK) return st;
    const size_t need = dcnn_cache_scratch_bytes(p->cache.dtype, rows, p->q_heads, p->cache.heads, p->cache.dim, p->cache.streams, p->cache.length);
    if (p->scratch_bytes < need) return fail(ctx, DCNN_ENOMEM, "%s: scratch of %zu bytes, %zu needed", what, p->scratch_bytes, need);
    if (p->scratch_dev == nullptr || !aligned(p->scratch_dev, kAlign)) return fail(ctx, DCNN_EINVAL, "%s: scratch null or not 256-byte aligned", what);
    const Bytes outs[] = {matrix_bytes("y", p->y_dev, rows, p->ldy, c, es), vector_bytes("scratch", p->scratch_dev, (int64_t)need)};
    const Bytes ins[] = {matrix_bytes("q", p->q_dev, rows, p->ldq, c, es), codes_bytes(p->cache), scales_bytes(p->cache), pages_bytes(p->cache),
                         idx_bytes(p->tokens), count_bytes(p->tokens), stream_bytes(p->tokens), vector_bytes("positions", a.tokens.pos, p->tokens.list.map_rows * 4),
                         vector_bytes("lens", p->lens_dev, p->cache.streams * 4)};
    st = check_apart(ctx, what, outs, ins);
    if (st != DCNN_OK) return st;
    const AttendPlan plan = attend_plan((int)es, rows, p->q_heads, p->cache.heads, p->cache.dim, p->cache.streams, p->cache.length);
    a.q = p->q_dev, a.y = p->y_dev, a.ldq = p->ldq, a.ldy = p->ldy;
    a.group = p->q_heads / p->cache.heads, a.blocks = (int)cdiv(a.group, 16);
    // (a scale of zero: so small a number that any product with it is as good as zero, and what is masked, minus infinity, stays that)
    a.factor = __builtin_fabsf(p->scale) * 1.44269504088896341f, a.negate = p->scale < 0.0f;
    if (a.factor == 0.0f) a.factor = 0x1p-149f;
    if (a.factor > 3.4028234e38f) a.factor = 3.4028234e38f;    // (finite, for products of zero)
    a.causal = p->causal != 0, a.window = p->window < (int64_t)1 << 33 ? p->window : (int64_t)1 << 33;    // (positions are 32 bits)
    a.lens = p->lens_dev;
    a.by_group = make_fastdiv((uint32_t)a.group);
    a.splits = plan.splits;
    char* const scratch = static_cast<char*>(p->scratch_dev);
    a.plan = plan.tiles ? nullptr : reinterpret_cast<int*>(scratch);
    a.stat = reinterpret_cast<float*>(scratch + kPlanBytes);
    a.part = reinterpret_cast<float*>(scratch + kPlanBytes + align_up((size_t)plan.parts * 2 * sizeof(float)));
    return launch_attend(ctx, p->cache.dtype, p->cache.dim, plan, a);
}

}  // extern "C"
