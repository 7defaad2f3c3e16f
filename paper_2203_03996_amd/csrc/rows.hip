// C entry points of the row operators: checks of arguments, no kernels.
#include "rows.h"
#include "rows_check.h"

using namespace dcnn;

namespace {

constexpr int64_t kLdqMax = 1 << 22;       // 8-bit rows of a tile are addressed in 32 bits

dcnn_status check_q(dcnn_ctx* ctx, const char* what, const void* q, const void* scale, int64_t ld, int64_t c) {
    if (q == nullptr || scale == nullptr) return fail(ctx, DCNN_EINVAL, "%s: 8-bit rows need q and q_scale", what);
    if (!aligned(q, 16) || ld % 16 != 0) return fail(ctx, DCNN_EINVAL, "%s: 8-bit rows must start at multiples of 16 bytes (ldq %lld)", what, (long long)ld);
    if (ld > kLdqMax) return fail(ctx, DCNN_EUNSUPPORTED, "%s: 8-bit rows %lld bytes apart", what, (long long)ld);
    if (!aligned(scale, 4)) return fail(ctx, DCNN_EINVAL, "%s: q_scale not 4-byte aligned", what);
    return check_ld(ctx, what, "q", q, ld, c, 1);
}
// Scratch, which grows with the rows: the counts of workgroups that share a tile (at the same place whatever the sizes: they are zero between calls), their
// partial sums, then the 8-bit rows of a call that makes some: scales, rows
struct Scratch {
    int64_t ldq;
    size_t partial, scales, rows, bytes;
    Scratch(int64_t count, int64_t k, int64_t n) {
        ldq = (int64_t)align_up((size_t)k, 64);
        partial = align_up(kArrivedBytes);
        scales = partial + align_up(partial_bytes(count, k, n));
        rows = scales + align_up((size_t)count * sizeof(float));
        bytes = rows + align_up((size_t)count * (size_t)ldq);
    }
};

dcnn_status check_matmul(dcnn_ctx* ctx, const char* what, const dcnn_rows_matmul_args* p, int linear, MatmulArgs* m) {
    if (!rows_float(p->dtype)) return fail(ctx, DCNN_EDTYPE, "%s: dtype %d", what, p->dtype);
    if (p->act < DCNN_ACT_NONE || p->act > DCNN_ACT_RELU6) return fail(ctx, DCNN_EINVAL, "%s: activation %d", what, p->act);
    if (dcnn_rows_weights_bytes(p->k, p->n) == 0) return fail(ctx, DCNN_EINVAL, "%s: k %lld, n %lld", what, (long long)p->k, (long long)p->n);
    dcnn_status st = check_list(ctx, what, p->list);
    if (st != DCNN_OK) return st;
    if (p->list.rows == 0) return DCNN_OK;                     // (buffers of no rows may be null)
    if (p->packed_dev == nullptr || !aligned(p->packed_dev, kAlign)) return fail(ctx, DCNN_EINVAL, "%s: packed weights null or not 256-byte aligned", what);
    if (p->y_dev == nullptr) return fail(ctx, DCNN_EINVAL, "%s: y is null", what);
    const size_t es = rows_dtype_size(p->dtype);
    st = check_ld(ctx, what, "y", p->y_dev, p->ldy, p->n, es);
    if (st != DCNN_OK) return st;
    if (!aligned(p->bias_dev, es)) return fail(ctx, DCNN_EINVAL, "%s: bias is not aligned to its elements", what);
    const size_t need = dcnn_rows_scratch_bytes(p->list.rows, p->k, p->n, linear);
    if (p->scratch_bytes < need) return fail(ctx, DCNN_ENOMEM, "%s: scratch of %zu bytes, %zu needed", what, p->scratch_bytes, need);
    if (p->scratch_dev == nullptr || !aligned(p->scratch_dev, kAlign)) return fail(ctx, DCNN_EINVAL, "%s: scratch null or not 256-byte aligned", what);
    m->w = static_cast<const int8_t*>(p->packed_dev);
    m->w_scale = reinterpret_cast<const float*>(m->w + packed_scale_offset(p->k, p->n));
    m->bias = p->bias_dev;
    m->y = p->y_dev;
    m->count = p->list.count_dev;
    m->rows = (int)p->list.rows;
    m->n = (int)p->n;
    m->ldy = (int)p->ldy;
    m->kc = (int)cdiv(p->k, 16);
    m->kt = (int)(packed_k(p->k) / kPackK);
    m->act = p->act;
    char* scratch = static_cast<char*>(p->scratch_dev);
    m->arrived = reinterpret_cast<uint32_t*>(scratch);
    m->partial = reinterpret_cast<int32_t*>(scratch + Scratch(p->list.rows, p->k, p->n).partial);
    return DCNN_OK;
}

// ... y and scratch from what every product reads and from the rows (`ins`) of this one
template <int INS> dcnn_status check_product_apart(dcnn_ctx* ctx, const char* what, const dcnn_rows_matmul_args* p, int linear, const Bytes (&ins)[INS]) {
    const size_t es = rows_dtype_size(p->dtype);
    const Bytes outs[] = {matrix_bytes("y", p->y_dev, p->list.rows, p->ldy, p->n, es),
                          vector_bytes("scratch", p->scratch_dev, (int64_t)dcnn_rows_scratch_bytes(p->list.rows, p->k, p->n, linear))};
    const Bytes all[] = {vector_bytes("the packed weights", p->packed_dev, (int64_t)dcnn_rows_weights_bytes(p->k, p->n)), vector_bytes("bias", p->bias_dev, p->n * es),
                         vector_bytes("count", p->list.count_dev, 4)};
    const dcnn_status st = check_apart(ctx, what, outs, all);
    return st == DCNN_OK ? check_apart(ctx, what, outs, ins) : st;
}

}  // namespace

extern "C" {

dcnn_status dcnn_rows_norm(dcnn_ctx* ctx, const dcnn_rows_norm_args* p) {
    const char* what = "rows_norm";
    if (!ctx || !p) return DCNN_EINVAL;
    if (!rows_float(p->dtype)) return fail(ctx, DCNN_EDTYPE, "%s: dtype %d", what, p->dtype);
    if (p->c < 1) return fail(ctx, DCNN_EINVAL, "%s: %d channels", what, p->c);
    if (p->c > kRowsMaxC) return fail(ctx, DCNN_EUNSUPPORTED, "%s: %d channels, %d at most", what, p->c, kRowsMaxC);
    dcnn_status st = check_list(ctx, what, p->list);
    if (st == DCNN_OK) st = check_map(ctx, what, p->list);
    if (st != DCNN_OK || p->list.rows == 0) return st;         // (buffers of no rows may be null)
    if (p->x_dev == nullptr && p->h_dev == nullptr) return fail(ctx, DCNN_EINVAL, "%s: neither x nor h", what);
    if (p->y_dev == nullptr && p->z_dev == nullptr && p->q_dev == nullptr) return fail(ctx, DCNN_EINVAL, "%s: none of y, z, q is wanted", what);
    if (p->h_dev == nullptr && (p->y_dev != nullptr || p->gate_dev != nullptr || p->post.kind != DCNN_NORM_NONE))
        return fail(ctx, DCNN_EINVAL, "%s: y, a gate and a norm behind the block need h", what);
    if (p->scale != p->scale) return fail(ctx, DCNN_EINVAL, "%s: scale is NaN", what);
    if (p->gate_rows < 0 || p->gate_rows > kRowsMax) return fail(ctx, DCNN_EINVAL, "%s: gate_rows %lld", what, (long long)p->gate_rows);
    const size_t es = rows_dtype_size(p->dtype);
    st = check_norm(ctx, what, p->post, es);
    if (st == DCNN_OK) st = check_norm(ctx, what, p->pre, es);
    if (st == DCNN_OK) st = check_ld(ctx, what, "x", p->x_dev, p->ldx, p->c, es);
    if (st == DCNN_OK) st = check_ld(ctx, what, "h", p->h_dev, p->ldh, p->c, es);
    if (st == DCNN_OK) st = check_ld(ctx, what, "y", p->y_dev, p->ldy, p->c, es);
    if (st == DCNN_OK) st = check_ld(ctx, what, "z", p->z_dev, p->ldz, p->c, es);
    if (st == DCNN_OK) st = check_ld(ctx, what, "gate", p->gate_dev, p->gate_rows ? p->ldg : p->c, p->c, es);
    if (st == DCNN_OK && (p->q_dev != nullptr || p->q_scale_dev != nullptr)) st = check_q(ctx, what, p->q_dev, p->q_scale_dev, p->ldq, p->c);
    if (st != DCNN_OK) return st;
    const bool in_place = p->y_dev != nullptr && p->y_dev == p->x_dev;
    if (in_place && p->ldy != p->ldx && p->list.map_rows > 1)
        return fail(ctx, DCNN_ESHAPE, "%s: in place with leading dimensions %lld and %lld", what, (long long)p->ldx, (long long)p->ldy);

    NormArgs a;
    a.x = p->x_dev, a.h = p->h_dev, a.gate = p->gate_dev;
    a.y = p->y_dev, a.z = p->z_dev, a.q = p->q_dev, a.q_scale = p->q_scale_dev;
    a.idx = p->list.idx_dev, a.count = p->list.count_dev;
    a.rows = (int)p->list.rows, a.map_rows = (int)p->list.map_rows;
    a.ldx = (int)p->ldx, a.ldh = (int)p->ldh, a.ldg = (int)p->ldg, a.ldy = (int)p->ldy, a.ldz = (int)p->ldz, a.ldq = (int)p->ldq;
    a.c = p->c, a.scale = p->scale;
    set_norm(p->post, &a.post, &a.post_eps, &a.post_w, &a.post_b);
    set_norm(p->pre, &a.pre, &a.pre_eps, &a.pre_w, &a.pre_b);
    const int64_t rows = p->list.rows, map_rows = p->list.idx_dev != nullptr ? p->list.map_rows : rows, c = p->c;
    const Bytes outs[] = {matrix_bytes("y", p->y_dev, map_rows, p->ldy, c, es), matrix_bytes("z", p->z_dev, rows, p->ldz, c, es),
                          matrix_bytes("q", p->q_dev, rows, p->ldq, align_up((size_t)c, 16), 1), vector_bytes("q_scale", p->q_scale_dev, rows * 4)};
    const Bytes ins[] = {matrix_bytes("x", p->x_dev, map_rows, p->ldx, c, es), matrix_bytes("h", p->h_dev, rows, p->ldh, c, es),
                         matrix_bytes("the gate", p->gate_dev, p->gate_rows ? cdiv(map_rows, p->gate_rows) : 1, p->ldg, c, es),
                         vector_bytes("a norm's weight", a.post_w, c * es), vector_bytes("a norm's bias", a.post_b, c * es),
                         vector_bytes("a norm's weight", a.pre_w, c * es), vector_bytes("a norm's bias", a.pre_b, c * es),
                         vector_bytes("idx", a.idx, rows * 4), vector_bytes("count", a.count, 4)};
    st = check_apart(ctx, what, outs, ins, in_place ? &outs[0] : nullptr, &ins[0]);
    if (st != DCNN_OK) return st;
    a.gate_div = p->gate_rows ? make_fastdiv((uint32_t)p->gate_rows) : FastDiv{0, 0, 0};
    return launch_rows_norm(ctx, p->dtype, a);
}

size_t dcnn_rows_weights_bytes(int64_t k, int64_t n) {
    if (k < 1 || k > kRowsMaxK || n < 1 || n > kRowsMaxN) return 0;
    return align_up(packed_scale_offset(k, n) + (size_t)packed_n(n) * sizeof(float));
}

dcnn_status dcnn_rows_pack(dcnn_ctx* ctx, int32_t dtype, int64_t k, int64_t n, const void* w_dev, int64_t ldw, const float* scale_dev,
                           void* packed_dev, size_t packed_bytes) {
    const char* what = "rows_pack";
    if (!ctx) return DCNN_EINVAL;
    if (!rows_float(dtype) && dtype != DCNN_I8) return fail(ctx, DCNN_EDTYPE, "%s: dtype %d", what, dtype);
    const size_t need = dcnn_rows_weights_bytes(k, n);
    if (need == 0) return fail(ctx, DCNN_EINVAL, "%s: k %lld, n %lld", what, (long long)k, (long long)n);
    if (w_dev == nullptr || packed_dev == nullptr) return fail(ctx, DCNN_EINVAL, "%s: null weights", what);
    if ((scale_dev != nullptr) != (dtype == DCNN_I8)) return fail(ctx, DCNN_EINVAL, "%s: scales come with 8-bit weights and with no others", what);
    dcnn_status st = check_ld(ctx, what, "weights", w_dev, ldw, n, rows_dtype_size(dtype));
    if (st != DCNN_OK) return st;
    if (!aligned(packed_dev, kAlign) || !aligned(scale_dev, 4)) return fail(ctx, DCNN_EINVAL, "%s: misaligned buffer", what);
    if (packed_bytes < need) return fail(ctx, DCNN_ENOMEM, "%s: %zu bytes, %zu needed", what, packed_bytes, need);
    const Bytes outs[] = {vector_bytes("packed", packed_dev, (int64_t)need)};
    const Bytes ins[] = {matrix_bytes("the weights", w_dev, k, ldw, n, rows_dtype_size(dtype)), vector_bytes("scale", scale_dev, n * 4)};
    st = check_apart(ctx, what, outs, ins);
    if (st != DCNN_OK) return st;
    int8_t* packed = static_cast<int8_t*>(packed_dev);
    return launch_rows_pack(ctx, dtype, k, n, w_dev, ldw, scale_dev, packed, reinterpret_cast<float*>(packed + packed_scale_offset(k, n)));
}

size_t dcnn_rows_scratch_bytes(int64_t rows, int64_t k, int64_t n, int32_t linear) {
    if (rows < 0 || rows > kRowsMax || dcnn_rows_weights_bytes(k, n) == 0) return 0;
    const Scratch s(rows, k, n);
    return linear ? s.bytes : s.scales;
}

dcnn_status dcnn_rows_matmul(dcnn_ctx* ctx, const dcnn_rows_matmul_args* p) {
    const char* what = "rows_matmul";
    if (!ctx || !p) return DCNN_EINVAL;
    if (p->x_dev != nullptr || p->list.idx_dev != nullptr) return fail(ctx, DCNN_EINVAL, "%s: x and idx belong to rows_linear", what);
    MatmulArgs m;
    dcnn_status st = check_matmul(ctx, what, p, 0, &m);
    if (st == DCNN_OK && p->list.rows == 0) return st;
    if (st == DCNN_OK) st = check_q(ctx, what, p->q_dev, p->q_scale_dev, p->ldq, p->k);
    if (st != DCNN_OK) return st;
    const Bytes ins[] = {matrix_bytes("q", p->q_dev, p->list.rows, p->ldq, p->k, 1), vector_bytes("q_scale", p->q_scale_dev, p->list.rows * 4)};
    st = check_product_apart(ctx, what, p, 0, ins);
    if (st != DCNN_OK) return st;
    m.q = p->q_dev, m.q_scale = p->q_scale_dev, m.ldq = (int)p->ldq;
    return launch_rows_matmul(ctx, p->dtype, matmul_plan(p->list.rows, p->k, p->n, p->list.count_dev != nullptr), m);
}

dcnn_status dcnn_rows_linear(dcnn_ctx* ctx, const dcnn_rows_matmul_args* p) {
    const char* what = "rows_linear";
    if (!ctx || !p) return DCNN_EINVAL;
    if (p->q_dev != nullptr || p->q_scale_dev != nullptr) return fail(ctx, DCNN_EINVAL, "%s: q belongs to rows_matmul", what);
    if (p->k > kRowsMaxC) return fail(ctx, DCNN_EUNSUPPORTED, "%s: k %lld, %d at most", what, (long long)p->k, kRowsMaxC);
    MatmulArgs m;
    dcnn_status st = check_matmul(ctx, what, p, 1, &m);
    if (st == DCNN_OK) st = check_map(ctx, what, p->list);
    if (st == DCNN_OK && p->list.rows == 0) return st;
    if (st == DCNN_OK && p->x_dev == nullptr) st = fail(ctx, DCNN_EINVAL, "%s: x is null", what);
    if (st == DCNN_OK) st = check_ld(ctx, what, "x", p->x_dev, p->ldx, p->k, rows_dtype_size(p->dtype));
    if (st == DCNN_OK) st = check_norm(ctx, what, p->pre, rows_dtype_size(p->dtype));
    if (st != DCNN_OK) return st;

    char* scratch = static_cast<char*>(p->scratch_dev);
    NormArgs a{};
    a.x = p->x_dev, a.ldx = (int)p->ldx, a.c = (int)p->k, a.scale = 1.0f;
    a.idx = p->list.idx_dev, a.count = p->list.count_dev;
    a.rows = (int)p->list.rows, a.map_rows = (int)p->list.map_rows;
    const Scratch at(p->list.rows, p->k, p->n);
    a.q_scale = reinterpret_cast<float*>(scratch + at.scales);
    a.q = reinterpret_cast<int8_t*>(scratch + at.rows), a.ldq = (int)at.ldq;
    set_norm(p->pre, &a.pre, &a.pre_eps, &a.pre_w, &a.pre_b);
    const size_t es = rows_dtype_size(p->dtype);
    const Bytes ins[] = {matrix_bytes("x", p->x_dev, a.idx != nullptr ? a.map_rows : a.rows, p->ldx, p->k, es), vector_bytes("a norm's weight", a.pre_w, p->k * es),
                         vector_bytes("a norm's bias", a.pre_b, p->k * es), vector_bytes("idx", a.idx, p->list.rows * 4)};
    st = check_product_apart(ctx, what, p, 1, ins);
    if (st != DCNN_OK) return st;
    if (rows_linear_fuses(p->dtype, p->list.rows, p->k, p->n, p->list.count_dev != nullptr)) return launch_rows_linear_fused(ctx, p->dtype, a, m);
    st = launch_rows_norm(ctx, p->dtype, a);
    if (st != DCNN_OK) return st;
    m.q = a.q, m.q_scale = a.q_scale, m.ldq = a.ldq;
    return launch_rows_matmul(ctx, p->dtype, matmul_plan(p->list.rows, p->k, p->n, p->list.count_dev != nullptr), m);
}

}  // extern "C"
