// losses_api.hip -- the C ABI of the loss operators
// (include/deepreduce_losses.h): argument checks and workspace needs.
#include <cmath>

#include "deepreduce_losses.h"
#include "host.hpp"
#include "losses.hpp"

using namespace dr;
static_assert(TYPE_F32 == DR_TYPE_F32 && TYPE_BF16 == DR_TYPE_BF16 && TYPE_F16 == DR_TYPE_F16, "number types");
static_assert(INDEX_I32 == DR_INDEX_I32 && INDEX_I64 == DR_INDEX_I64, "index types");
static_assert(MAX_TOP == DR_MAX_TOP && MAX_TEACHER == DR_MAX_TEACHER && MAX_EXPERTS == DR_MAX_EXPERTS &&
                  STATS == DR_DISTILL_STATS,
              "limits of the header and the kernels");

namespace {

constexpr uint64_t MAX_ROWS = 1ull << 31;

bool shape_ok(uint64_t rows, uint64_t cols) { return rows < MAX_ROWS && cols >= 1 && cols < DR_MAX_COLS; }

dr_status check_matrix(const dr_logits *l, Matrix &m) {
    if (!l) return fail(DR_EINVAL, "logits descriptor is null");
    if (l->type > DR_TYPE_F16) return fail(DR_EINVAL, "unknown number type %u", l->type);
    if (!shape_ok(l->rows, l->cols))
        return fail(DR_EINVAL, "rows must be below 2^31 and cols in 1 .. 2^31 - 1 (%llu x %llu)",
                    (unsigned long long)l->rows, (unsigned long long)l->cols);
    if (l->row_stride < l->cols) return fail(DR_EINVAL, "row stride below cols");
    if (l->rows > 1 && l->row_stride > (UINT64_MAX / 8) / l->rows) return fail(DR_EINVAL, "row stride too large");
    if (!l->data && l->rows > 0) return fail(DR_EINVAL, "logits are null");
    if ((uintptr_t)l->data % type_bytes(l->type)) return fail(DR_EINVAL, "logits are not aligned to their type");
    m = {l->data, l->rows, l->row_stride, (uint32_t)l->cols, l->type};
    return DR_OK;
}

dr_status check_grad(const Matrix &m, const void *grad, uint64_t stride) {
    if (!grad && m.rows > 0) return fail(DR_EINVAL, "grad_out is null");
    if (stride < m.cols) return fail(DR_EINVAL, "gradient stride below cols");
    if (m.rows > 1 && stride > (UINT64_MAX / 8) / m.rows) return fail(DR_EINVAL, "gradient stride too large");
    if ((uintptr_t)grad % type_bytes(m.type)) return fail(DR_EINVAL, "grad_out is not aligned to its type");
    if (grad == m.p && m.rows > 1 && stride != m.stride)
        return fail(DR_EINVAL, "a gradient in place of the logits needs their stride");
    return DR_OK;
}

dr_status check_temperature(float t) {
    // its reciprocal times log2(e) is finite, too
    if (!std::isfinite(t) || !(t > 0.f) || !std::isfinite((float)(1.4426950408889634 / t)))
        return fail(DR_EINVAL, "temperature must be finite and above 0");
    return DR_OK;
}

dr_status check_index(const void *idx, uint64_t stride, uint32_t k, uint32_t type, const char *what) {
    if (type > DR_INDEX_I64) return fail(DR_EINVAL, "unknown index type %u", type);
    if (stride < k || stride > UINT64_MAX / 64 / MAX_ROWS) return fail(DR_EINVAL, "%s: stride out of range", what);
    if ((uintptr_t)idx % (type == DR_INDEX_I64 ? 8 : 4)) return fail(DR_EINVAL, "%s: not aligned to its type", what);
    return DR_OK;
}

dr_status check_teacher(const dr_teacher *t, const Matrix &m, Teacher &out) {
    if (!t) return fail(DR_EINVAL, "teacher descriptor is null");
    if (t->k < 1 || t->k > DR_MAX_TEACHER) return fail(DR_EINVAL, "k must be in 1 .. %u", DR_MAX_TEACHER);
    if (t->val_type > DR_TYPE_F16) return fail(DR_EINVAL, "unknown number type %u", t->val_type);
    if ((!t->idx || !t->val) && m.rows > 0) return fail(DR_EINVAL, "the teacher's columns or logits are null");
    dr_status st = check_index(t->idx, t->idx_stride, t->k, t->idx_type, "teacher's columns");
    if (st != DR_OK) return st;
    if (t->val_stride < t->k || t->val_stride > UINT64_MAX / 64 / MAX_ROWS)
        return fail(DR_EINVAL, "teacher's logits: stride out of range");
    if ((uintptr_t)t->val % type_bytes(t->val_type) || (uintptr_t)t->rest % 4)
        return fail(DR_EINVAL, "teacher's logits: not aligned to their type");
    out = {t->idx, t->val, t->rest, t->idx_stride, t->val_stride, t->k, t->idx_type, t->val_type};
    return DR_OK;
}

dr_status check_distill(const dr_logits *student_h, const dr_teacher *teacher_h, float temperature, Matrix &m,
                        Teacher &t) {
    dr_status st = check_matrix(student_h, m);
    if (st == DR_OK) st = check_teacher(teacher_h, m, t);
    if (st == DR_OK) st = check_temperature(temperature);
    if (st != DR_OK) return st;
    if (distill_threads(m) > MAX_THREADS) return fail(DR_EINVAL, "rows times cols too large for one call");
    return DR_OK;
}

dr_status check_routes(const dr_logits *router_h, const dr_routes *r, float coef, Matrix &m, Routes &out,
                       bool chosen) {
    dr_status st = check_matrix(router_h, m);
    if (st != DR_OK) return st;
    if (m.cols > DR_MAX_EXPERTS) return fail(DR_EINVAL, "more than %u experts", DR_MAX_EXPERTS);
    if (!r) return fail(DR_EINVAL, "routes descriptor is null");
    if (r->k < 1 || r->k > m.cols) return fail(DR_EINVAL, "k must be in 1 .. cols");
    if (m.rows * r->k >= MAX_ROWS) return fail(DR_EINVAL, "rows times k must be below 2^31");
    if (r->group_rows < 1 || r->group_rows >= MAX_ROWS) return fail(DR_EINVAL, "group_rows must be in 1 .. 2^31 - 1");
    if (!std::isfinite(coef)) return fail(DR_EINVAL, "coef is not finite");
    if (chosen) {
        if (!r->idx && m.rows > 0) return fail(DR_EINVAL, "the chosen experts are null");
        st = check_index(r->idx, r->idx_stride, r->k, r->idx_type, "chosen experts");
        if (st != DR_OK) return st;
    }
    out = {r->idx, r->row_mask, r->idx_stride, r->k, r->idx_type, (uint32_t)r->group_rows,
           (uint32_t)ceil_div(m.rows, r->group_rows)};
    if (balance_threads(m, out) > MAX_THREADS) return fail(DR_EINVAL, "too many groups for one call");
    return DR_OK;
}

dr_status ws_small(size_t need) {
    return fail(DR_EINVAL, "workspace too small or not 256-byte aligned (need %zu)", need);
}

}  // namespace

extern "C" {

size_t dr_losses_workspace_bytes(uint64_t rows, uint64_t cols, uint32_t k) {
    if (!shape_ok(rows, cols)) {
        fail(DR_EINVAL, "rows or cols out of range");
        return 0;
    }
    size_t n = 256;
    for (uint32_t type : {TYPE_F32, TYPE_BF16}) {
        if (k >= 1) n = std::max(n, plan_top(rows, cols, std::min(k, DR_MAX_TOP), type).bytes);
        n = std::max(n, distill_ws_bytes(rows, cols, type));
    }
    n = std::max(n, balance_ws_bytes(rows, std::min<uint64_t>(cols, DR_MAX_EXPERTS)));
    return align_up(n, 256);
}

dr_status dr_top_logits(const dr_logits *logits_h, uint32_t k, float temperature, int32_t *idx_out, float *val_out,
                        float *rest_out, void *ws, size_t ws_bytes, void *stream) {
    Matrix m;
    dr_status st = check_matrix(logits_h, m);
    if (st == DR_OK) st = check_temperature(temperature);
    if (st != DR_OK) return st;
    if (k < 1 || k > DR_MAX_TOP) return fail(DR_EINVAL, "k must be in 1 .. %u", DR_MAX_TOP);
    if ((!idx_out || !val_out) && m.rows > 0) return fail(DR_EINVAL, "null output pointer");
    const TopPlan p = plan_top(m.rows, m.cols, k, m.type);
    // the joins' blocks are no larger than the slices', and fewer
    if (m.rows * p.sl.n * p.threads > MAX_THREADS) return fail(DR_EINVAL, "rows times cols too large for one call");
    if (p.bytes && !ws_ok(ws, ws_bytes, p.bytes)) return ws_small(p.bytes);
    if (m.rows == 0) return DR_OK;
    const hipStream_t s = (hipStream_t)stream;
    trace_call(s);
    DR_HIP(launch_top(m, k, temperature, idx_out, val_out, rest_out, p, (uint8_t *)ws, s));
    return DR_OK;
}

dr_status dr_distill_forward(const dr_logits *student_h, const dr_teacher *teacher_h, float temperature,
                             const float *weight, float *loss_out, float *stats_out, void *ws, size_t ws_bytes,
                             void *stream) {
    Matrix m;
    Teacher t;
    dr_status st = check_distill(student_h, teacher_h, temperature, m, t);
    if (st != DR_OK) return st;
    if (!loss_out && m.rows > 0) return fail(DR_EINVAL, "loss_out is null");
    const size_t need = distill_ws_bytes(m.rows, m.cols, m.type);
    if (!ws_ok(ws, ws_bytes, need)) return ws_small(need);
    if (m.rows == 0) return DR_OK;
    const hipStream_t s = (hipStream_t)stream;
    trace_call(s);
    DR_HIP(launch_distill_forward(m, t, temperature, weight, loss_out, stats_out, (uint8_t *)ws, s));
    return DR_OK;
}

dr_status dr_distill_backward(const dr_logits *student_h, const dr_teacher *teacher_h, float temperature,
                              const float *weight, const float *upstream, uint64_t upstream_stride,
                              const float *stats, void *grad_out, uint64_t grad_stride, void *stream) {
    Matrix m;
    Teacher t;
    dr_status st = check_distill(student_h, teacher_h, temperature, m, t);
    if (st == DR_OK) st = check_grad(m, grad_out, grad_stride);
    if (st != DR_OK) return st;
    if (!stats && m.rows > 0) return fail(DR_EINVAL, "stats is null");
    if (upstream_stride > UINT64_MAX / 64 / MAX_ROWS) return fail(DR_EINVAL, "upstream stride out of range");
    if (m.rows == 0) return DR_OK;
    const hipStream_t s = (hipStream_t)stream;
    trace_call(s);
    DR_HIP(launch_distill_backward(m, t, temperature, weight, upstream, upstream_stride, stats, grad_out, grad_stride,
                                   s));
    return DR_OK;
}

dr_status dr_distill_step(const dr_logits *student_h, const dr_teacher *teacher_h, float temperature,
                          const float *weight, float *loss_out, void *grad_out, uint64_t grad_stride, void *ws,
                          size_t ws_bytes, void *stream) {
    Matrix m;
    Teacher t;
    dr_status st = check_distill(student_h, teacher_h, temperature, m, t);
    if (st == DR_OK) st = check_grad(m, grad_out, grad_stride);
    if (st != DR_OK) return st;
    if (!loss_out && m.rows > 0) return fail(DR_EINVAL, "loss_out is null");
    const size_t need = distill_ws_bytes(m.rows, m.cols, m.type);
    if (!ws_ok(ws, ws_bytes, need)) return ws_small(need);
    if (m.rows == 0) return DR_OK;
    const hipStream_t s = (hipStream_t)stream;
    trace_call(s);
    DR_HIP(launch_distill_step(m, t, temperature, weight, loss_out, grad_out, grad_stride, (uint8_t *)ws, s));
    return DR_OK;
}

dr_status dr_balance_forward(const dr_logits *router_h, const dr_routes *routes_h, float coef, int32_t *counts_out,
                             int32_t *rows_out, float *prob_out, float *loss_out, void *ws, size_t ws_bytes,
                             void *stream) {
    Matrix m;
    Routes r;
    dr_status st = check_routes(router_h, routes_h, coef, m, r, true);
    if (st != DR_OK) return st;
    if (!loss_out || ((!counts_out || !rows_out) && m.rows > 0)) return fail(DR_EINVAL, "null output pointer");
    const size_t need = balance_ws_bytes(m.rows, m.cols);
    if (!ws_ok(ws, ws_bytes, need)) return ws_small(need);
    const hipStream_t s = (hipStream_t)stream;
    trace_call(s);
    DR_HIP(launch_balance_forward(m, r, coef, counts_out, rows_out, prob_out, loss_out, (uint8_t *)ws, s));
    return DR_OK;
}

dr_status dr_balance_backward(const dr_logits *router_h, const dr_routes *routes_h, float coef, const int32_t *counts,
                              const int32_t *count_rows, const int32_t *rows_in, const float *upstream,
                              void *grad_out, uint64_t grad_stride, void *stream) {
    Matrix m;
    Routes r;
    dr_status st = check_routes(router_h, routes_h, coef, m, r, false);
    if (st == DR_OK) st = check_grad(m, grad_out, grad_stride);
    if (st != DR_OK) return st;
    if ((!counts || !count_rows || !rows_in) && m.rows > 0) return fail(DR_EINVAL, "null input pointer");
    if (m.rows == 0) return DR_OK;
    const hipStream_t s = (hipStream_t)stream;
    trace_call(s);
    DR_HIP(launch_balance_backward(m, r, coef, counts, count_rows, rows_in, upstream, grad_out, grad_stride, s));
    return DR_OK;
}

}  // extern "C"
