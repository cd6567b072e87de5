// C ABI of the mini-batch operators: argument checks and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <exception>
#include <string>
#include <utility>
#include <vector>

#include "w2v_ops.h"

using namespace w2v;

namespace {

hipStream_t as_stream(void *s) { return static_cast<hipStream_t>(s); }

bool aligned(const void *p, int64_t bytes) { return reinterpret_cast<uintptr_t>(p) % static_cast<uintptr_t>(bytes) == 0; }

int check_workspace(const void *ws, size_t have, size_t need) {
    if (have < need)
        return fail(W2V_E_WORKSPACE, "workspace_bytes " + std::to_string(have) + " < required " + std::to_string(need));
    if (need > 0 && !ws) return fail(W2V_E_ARG, "workspace is NULL");
    if (need > 0 && !aligned(ws, 256)) return fail(W2V_E_ARG, "workspace must be 256-byte aligned");
    return W2V_OK;
}

// Rows of `dim` elements at p (required where there are any), `stride` apart. Offsets are 64-bit element counts.
int check_rows(const void *p, int32_t type, int64_t rows, int64_t dim, int64_t stride, const std::string &name) {
    if (rows > 0 && !p) return fail(W2V_E_ARG, name + " is NULL");
    if (!aligned(p, type_bytes(type))) return fail(W2V_E_ARG, name + " is not aligned to its elements");
    if (rows > 1 && stride < dim) return fail(W2V_E_ARG, name + "'s stride must be >= its row length");
    if (rows > 1 && stride > (INT64_MAX >> 4) / rows) return fail(W2V_E_ARG, name + " is too large");
    return W2V_OK;
}

int check_floats(const void *p, const char *name, bool required) {
    if (required && !p) return fail(W2V_E_ARG, std::string(name) + " is NULL");
    if (!aligned(p, 4)) return fail(W2V_E_ARG, std::string(name) + " is not aligned to its elements");
    return W2V_OK;
}

int check_norm(int64_t rows, int32_t dim, int32_t type, int32_t w_type, const void *weight, const void *bias) {
    if (rows < 0) return fail(W2V_E_ARG, "rows must be >= 0");
    if (dim < 1 || dim > kNormMaxDim) return fail(W2V_E_ARG, "dim must be in 1.." + std::to_string(kNormMaxDim));
    if (!type_ok(type)) return fail(W2V_E_ARG, "type must be 0 (fp32), 1 (bf16) or 2 (fp16)");
    if (weight || bias) {
        if (w_type != W2V_F32 && w_type != type) return fail(W2V_E_ARG, "w_type must be fp32 or the rows' type");
        if (!aligned(weight, type_bytes(w_type)) || !aligned(bias, type_bytes(w_type)))
            return fail(W2V_E_ARG, "weight or bias is not aligned to its elements");
    }
    return W2V_OK;
}

int check_hs(const w2v_model *m, int32_t max_code_len) {
    if (!m) return fail(W2V_E_ARG, "model is NULL");
    if (m->V < 2) return fail(W2V_E_ARG, "V must be >= 2");
    if (m->dim < 1 || m->dim > 1024) return fail(W2V_E_ARG, "dim must be in 1..1024");
    if (m->row_stride < m->dim || m->row_stride % 4 != 0)
        return fail(W2V_E_ARG, "row_stride must be >= dim and a multiple of 4");
    if (max_code_len < 1 || max_code_len > 64) return fail(W2V_E_ARG, "max_code_len must be in 1..64");
    return W2V_OK;
}

int check_tensors(const w2v_adamw_tensor *t, int32_t n, int64_t n_moments) {
    using Span = std::pair<int64_t, int64_t>;
    std::vector<Span> moments, params;
    for (int32_t i = 0; i < n; ++i) {
        const w2v_adamw_tensor &x = t[i];
        const std::string name = "tensor " + std::to_string(i);
        if (!type_ok(x.param_type) || !type_ok(x.grad_type))
            return fail(W2V_E_ARG, name + ": a type must be 0 (fp32), 1 (bf16) or 2 (fp16)");
        if (x.rows < 0 || x.cols < 0 || (x.cols > 0 && x.rows > (int64_t(1) << 40) / x.cols))
            return fail(W2V_E_ARG, name + ": rows and cols must be >= 0, and at most 2^40 elements");
        const int64_t count = x.rows * x.cols;
        if (int rc = check_rows(x.param, x.param_type, count > 0 ? x.rows : 0, x.cols, x.param_stride, name + "'s param"))
            return rc;
        if (int rc = check_rows(x.grad, x.grad_type, count > 0 ? x.rows : 0, x.cols, x.grad_stride, name + "'s grad"))
            return rc;
        const bool packed = x.rows <= 1 || (x.param_stride == x.cols && x.grad_stride == x.cols);
        if (!packed && x.cols >= (int64_t(1) << 31))
            return fail(W2V_E_ARG, name + ": rows with gaps hold at most 2^31 - 1 elements");
        if (!std::isfinite(x.weight_decay)) return fail(W2V_E_ARG, name + ": weight_decay must be finite");
        const int64_t places = ceil_div(count, kMomentBlock) * kMomentBlock;
        if (x.moment_offset < 0 || x.moment_offset % kMomentBlock != 0 || x.moment_offset > n_moments - places)
            return fail(W2V_E_ARG, name + ": moment_offset must be a multiple of 256 with the tensor's blocks below n_moments");
        if (count == 0) continue;
        moments.emplace_back(x.moment_offset, x.moment_offset + places);
        const int64_t at = static_cast<int64_t>(reinterpret_cast<uintptr_t>(x.param));
        // rows with gaps may interleave with another tensor's; the first row may not lie in one all the same
        const bool one_span = x.rows <= 1 || x.param_stride == x.cols;
        params.emplace_back(at, at + (one_span ? count : x.cols) * type_bytes(x.param_type));
    }
    auto overlap = [](std::vector<Span> &s) {
        std::sort(s.begin(), s.end());
        for (size_t i = 1; i < s.size(); ++i)
            if (s[i].first < s[i - 1].second) return true;
        return false;
    };
    if (overlap(moments)) return fail(W2V_E_ARG, "two tensors' moments overlap");
    if (overlap(params)) return fail(W2V_E_ARG, "two tensors' parameters overlap");
    return W2V_OK;
}

// What both calls on batches read of their arguments.
int check_batch(const w2v_model *m, const int32_t *tokens, int64_t n_tokens, const w2v_params *p, const w2v_batch_params *b) {
    if (int rc = check_training_args(m, p)) return rc;
    if (p->arch != 1) return fail(W2V_E_ARG, "training in batches is CBOW (arch 1) only");
    if (p->sync_batch < 1 || p->sync_batch > (1 << 20)) return fail(W2V_E_ARG, "sync_batch must be in 1..2^20");
    if (n_tokens < 0 || (n_tokens > 0 && !tokens)) return fail(W2V_E_ARG, "bad tokens / n_tokens");
    if (ceil_div(n_tokens, p->doc_len) > (1 << 30))
        return fail(W2V_E_ARG, "too many documents for one call: split the stream (first_raw_index)");
    if (!b) return fail(W2V_E_ARG, "batch params is NULL");
    if (b->max_code_len < 1 || b->max_code_len > 64) return fail(W2V_E_ARG, "max_code_len must be in 1..64");
    if (!b->gain != !b->bias) return fail(W2V_E_ARG, "gain and bias come together");
    if (int rc = check_floats(b->gain, "gain", false)) return rc;
    if (int rc = check_floats(b->bias, "bias", false)) return rc;
    if (b->gain && (!(b->norm_eps >= 0.0f) || !std::isfinite(b->norm_eps)))
        return fail(W2V_E_ARG, "norm_eps must be >= 0 and finite");
    return W2V_OK;
}

bool batch_sizes_ok(const w2v_model *m, int64_t n_tokens, const w2v_params *p, const w2v_batch_params *b) {
    return m && p && b && m->V >= 2 && m->dim >= 1 && m->dim <= 1024 && n_tokens >= 0 && p->doc_len >= 1 && p->window >= 1 &&
           p->window <= 10 && p->sync_batch >= 1 && p->sync_batch <= (1 << 20) && b->max_code_len >= 1 &&
           b->max_code_len <= 64;
}

}  // namespace

extern "C" {

int w2v_layer_norm(const void *x, int32_t type, int64_t rows, int32_t dim, int64_t x_stride, const void *weight,
                   const void *bias, int32_t w_type, float eps, void *y, int64_t y_stride, float *mean, float *rstd,
                   void *hip_stream) {
    set_error("");
    if (int rc = check_norm(rows, dim, type, w_type, weight, bias)) return rc;
    if (!(eps >= 0.0f) || !std::isfinite(eps)) return fail(W2V_E_ARG, "eps must be >= 0 and finite");
    if (int rc = check_rows(x, type, rows, dim, x_stride, "x")) return rc;
    if (int rc = check_rows(y, type, rows, dim, y_stride, "y")) return rc;
    if (int rc = check_floats(mean, "mean", false)) return rc;
    if (int rc = check_floats(rstd, "rstd", false)) return rc;
    if (x == y && rows > 1 && x_stride != y_stride) return fail(W2V_E_ARG, "y may be x only with the same stride");
    NormArgs a{};
    a.x = x;
    a.rows = rows;
    a.dim = dim;
    a.type = type;
    a.w_type = w_type;
    a.x_stride = x_stride;
    a.out_stride = y_stride;
    a.w = weight;
    a.b = bias;
    a.eps = eps;
    a.out = y;
    a.mean = mean;
    a.rstd = rstd;
    return run_layer_norm(a, as_stream(hip_stream));
}

size_t w2v_layer_norm_backward_workspace_bytes(int64_t rows, int32_t dim) {
    return rows < 0 || dim < 1 || dim > kNormMaxDim ? 0 : norm_backward_bytes(rows, dim);
}

int w2v_layer_norm_backward(const void *dy, int64_t dy_stride, const void *x, int32_t type, int64_t rows, int32_t dim,
                            int64_t x_stride, const void *weight, int32_t w_type, const float *mean,
                            const float *rstd, void *dx, int64_t dx_stride, float *dweight, float *dbias,
                            void *workspace, size_t workspace_bytes, void *hip_stream) {
    set_error("");
    if (int rc = check_norm(rows, dim, type, w_type, weight, nullptr)) return rc;
    if (int rc = check_rows(dy, type, rows, dim, dy_stride, "dy")) return rc;
    if (int rc = check_rows(x, type, rows, dim, x_stride, "x")) return rc;
    if (int rc = check_rows(dx, type, rows, dim, dx_stride, "dx")) return rc;
    if (int rc = check_floats(mean, "mean", rows > 0)) return rc;
    if (int rc = check_floats(rstd, "rstd", rows > 0)) return rc;
    if (int rc = check_floats(dweight, "dweight", false)) return rc;
    if (int rc = check_floats(dbias, "dbias", false)) return rc;
    if (rows > 1 && ((dx == dy && dx_stride != dy_stride) || (dx == x && dx_stride != x_stride)))
        return fail(W2V_E_ARG, "dx may be dy or x only with the same stride");
    if (dweight || dbias)
        if (int rc = check_workspace(workspace, workspace_bytes, norm_backward_bytes(rows, dim))) return rc;
    NormArgs a{};
    a.x = x;
    a.dy = dy;
    a.rows = rows;
    a.dim = dim;
    a.type = type;
    a.w_type = w_type;
    a.x_stride = x_stride;
    a.dy_stride = dy_stride;
    a.out_stride = dx_stride;
    a.w = weight;
    a.out = dx;
    a.mean = const_cast<float *>(mean);
    a.rstd = const_cast<float *>(rstd);
    a.dw = dweight;
    a.db = dbias;
    return run_layer_norm_backward(a, workspace, as_stream(hip_stream));
}

size_t w2v_hs_loss_workspace_bytes(const w2v_model *m, int32_t max_code_len, int64_t rows) {
    if (!m || m->dim < 1 || max_code_len < 1 || max_code_len > 64 || rows < 0) return 0;
    return hs_loss_bytes(rows, m->dim, max_code_len);
}

int w2v_hs_loss(const w2v_model *m, int32_t max_code_len, const void *x, int32_t type, int64_t rows, int64_t x_stride,
                const int32_t *targets, const float *weights, float *loss, void *dx, int64_t dx_stride, float *dsyn1,
                int64_t dsyn1_stride, void *workspace, size_t workspace_bytes, void *hip_stream) {
    set_error("");
    if (int rc = check_hs(m, max_code_len)) return rc;
    if (!m->syn1 || !m->codelen || !m->code || !m->point_off || !m->points)
        return fail(W2V_E_ARG, "syn1 or a Huffman array is NULL");
    if (!aligned(m->syn1, 16)) return fail(W2V_E_ARG, "syn1 must be 16-byte aligned");
    if (!type_ok(type)) return fail(W2V_E_ARG, "type must be 0 (fp32), 1 (bf16) or 2 (fp16)");
    if (rows < 0) return fail(W2V_E_ARG, "rows must be >= 0");
    if (int rc = check_rows(x, type, rows, m->dim, x_stride, "x")) return rc;
    if (rows > 0 && !targets) return fail(W2V_E_ARG, "targets is NULL");
    if (!aligned(targets, 4)) return fail(W2V_E_ARG, "targets is not aligned to its elements");
    if (int rc = check_floats(weights, "weights", false)) return rc;
    if (int rc = check_floats(loss, "loss", false)) return rc;
    if (dx)
        if (int rc = check_rows(dx, type, rows, m->dim, dx_stride, "dx")) return rc;
    if (dx && dx == x) return fail(W2V_E_ARG, "dx may not be x");
    if (dsyn1) {
        if (int rc = check_rows(dsyn1, W2V_F32, m->V - 1, m->dim, dsyn1_stride, "dsyn1")) return rc;
        if (dsyn1 == m->syn1) return fail(W2V_E_ARG, "dsyn1 may not be syn1");
        if (int rc = check_workspace(workspace, workspace_bytes, hs_loss_bytes(rows, m->dim, max_code_len))) return rc;
    }
    HsLossArgs a{};
    a.V = m->V;
    a.dim = m->dim;
    a.stride = m->row_stride;
    a.longest = max_code_len;
    a.syn1 = m->syn1;
    a.codelen = m->codelen;
    a.code = m->code;
    a.point_off = m->point_off;
    a.points = m->points;
    a.x = x;
    a.type = type;
    a.rows = rows;
    a.x_stride = x_stride;
    a.targets = targets;
    a.weights = weights;
    a.loss = loss;
    a.dx = dx;
    a.dx_stride = dx_stride;
    a.dsyn1 = dsyn1;
    a.dsyn1_stride = dsyn1_stride;
    a.dsyn1_whole = dsyn1_stride == m->row_stride;
    return run_hs_loss(a, workspace, as_stream(hip_stream));
}

size_t w2v_adamw_plan_bytes(const w2v_adamw_tensor *tensors_host, int32_t n_tensors) {
    if (n_tensors < 0 || (n_tensors > 0 && !tensors_host)) return 0;
    for (int32_t i = 0; i < n_tensors; ++i)
        if (tensors_host[i].rows < 0 || tensors_host[i].cols < 0 ||
            (tensors_host[i].cols > 0 && tensors_host[i].rows > (int64_t(1) << 40) / tensors_host[i].cols))
            return 0;
    return adamw_plan_bytes(tensors_host, n_tensors);
}

int w2v_adamw_build_plan(const w2v_adamw_tensor *tensors_host, int32_t n_tensors, int64_t n_moments, void *plan,
                         size_t plan_bytes, int64_t *n_chunks_host, void *hip_stream) {
    set_error("");
    if (n_tensors < 0 || (n_tensors > 0 && !tensors_host)) return fail(W2V_E_ARG, "bad tensors_host / n_tensors");
    if (n_moments < 0 || n_moments % kMomentBlock != 0) return fail(W2V_E_ARG, "n_moments must be a multiple of 256");
    if (!n_chunks_host) return fail(W2V_E_ARG, "n_chunks_host is NULL");
    try {
        if (int rc = check_tensors(tensors_host, n_tensors, n_moments)) return rc;
        if (int rc = check_workspace(plan, plan_bytes, adamw_plan_bytes(tensors_host, n_tensors))) return rc;
        if (int rc = run_adamw_plan(tensors_host, n_tensors, plan, as_stream(hip_stream))) return rc;
    } catch (const std::exception &e) {   // host memory for the tables
        return fail(W2V_E_ARG, std::string("the plan's tables: ") + e.what());
    }
    *n_chunks_host = adamw_chunks(tensors_host, n_tensors);
    return W2V_OK;
}

int w2v_adamw_step(void *plan, int64_t n_chunks, int32_t bits, void *m, void *v, float *m_scale, float *v_scale,
                   const w2v_adamw_params *p, void *hip_stream) {
    set_error("");
    if (!p) return fail(W2V_E_ARG, "params is NULL");
    if (bits != 8 && bits != 32) return fail(W2V_E_ARG, "bits must be 8 or 32");
    if (n_chunks < 0) return fail(W2V_E_ARG, "n_chunks must be >= 0");
    if (!plan) return fail(W2V_E_ARG, "plan is NULL");
    if (!aligned(plan, 256)) return fail(W2V_E_ARG, "plan must be 256-byte aligned");
    if (n_chunks > 0 && (!m || !v)) return fail(W2V_E_ARG, "m or v is NULL");
    if (!aligned(m, 4) || !aligned(v, 4)) return fail(W2V_E_ARG, "m and v must be 4-byte aligned");
    if (bits == 8 && n_chunks > 0) {
        if (int rc = check_floats(m_scale, "m_scale", true)) return rc;
        if (int rc = check_floats(v_scale, "v_scale", true)) return rc;
    }
    if (!p->lr_device && !std::isfinite(p->lr)) return fail(W2V_E_ARG, "lr must be finite");
    if (!(p->beta1 >= 0.0 && p->beta1 < 1.0) || !(p->beta2 >= 0.0 && p->beta2 < 1.0))
        return fail(W2V_E_ARG, "beta1 and beta2 must be in [0, 1)");
    if (!(p->eps >= 0.0) || !std::isfinite(p->eps)) return fail(W2V_E_ARG, "eps must be >= 0 and finite");
    if (!p->step_device && p->step < 1) return fail(W2V_E_ARG, "step must be >= 1");
    if (!aligned(p->lr_device, 4) || !aligned(p->step_device, 8))
        return fail(W2V_E_ARG, "lr_device or step_device is not aligned to its type");
    return run_adamw_step(plan, n_chunks, bits, m, v, m_scale, v_scale, *p, as_stream(hip_stream));
}

int w2v_adamw_moments(const void *m, const void *v, const float *m_scale, const float *v_scale, int64_t n_moments,
                      float *m_out, float *v_out, void *hip_stream) {
    set_error("");
    if (n_moments < 0 || n_moments % kMomentBlock != 0) return fail(W2V_E_ARG, "n_moments must be a multiple of 256");
    if (n_moments > 0 && (!m || !v || !m_scale || !v_scale || !m_out || !v_out))
        return fail(W2V_E_ARG, "a required pointer is NULL");
    if (!aligned(m, 4) || !aligned(v, 4)) return fail(W2V_E_ARG, "m and v must be 4-byte aligned");
    return run_adamw_moments(m, v, m_scale, v_scale, n_moments, m_out, v_out, as_stream(hip_stream));
}

int64_t w2v_batch_n_moments(const w2v_model *m, const w2v_batch_params *bp) {
    return !m || !bp || m->V < 2 || m->dim < 1 || m->dim > 1024 ? 0 : batch_moments(m, bp);
}

size_t w2v_train_batch_workspace_bytes(const w2v_model *m, int64_t n_tokens, const w2v_params *p,
                                       const w2v_batch_params *bp) {
    return batch_sizes_ok(m, n_tokens, p, bp) ? batch_bytes(m, n_tokens, p, bp, true) : 0;
}

int w2v_train_batch_epoch(const w2v_model *m, const int32_t *tokens, int64_t n_tokens, const w2v_params *p,
                          const w2v_batch_params *bp, int64_t *stats, int64_t *steps_host, double *sum_ll_host,
                          int64_t *n_terms_host, void *workspace, size_t workspace_bytes, void *hip_stream) {
    set_error("");
    if (steps_host) *steps_host = 0;
    if (int rc = check_batch(m, tokens, n_tokens, p, bp)) return rc;
    if (bp->bits != 8 && bp->bits != 32) return fail(W2V_E_ARG, "bits must be 8 or 32");
    if (!bp->m || !bp->v || (bp->bits == 8 && (!bp->m_scale || !bp->v_scale))) return fail(W2V_E_ARG, "a moment is NULL");
    if (!aligned(bp->m, 4) || !aligned(bp->v, 4) || !aligned(bp->m_scale, 4) || !aligned(bp->v_scale, 4))
        return fail(W2V_E_ARG, "moments must be 4-byte aligned");
    if (!(bp->beta1 >= 0.0 && bp->beta1 < 1.0) || !(bp->beta2 >= 0.0 && bp->beta2 < 1.0))
        return fail(W2V_E_ARG, "beta1 and beta2 must be in [0, 1)");
    if (!(bp->eps >= 0.0) || !std::isfinite(bp->eps)) return fail(W2V_E_ARG, "eps must be >= 0 and finite");
    if (!std::isfinite(bp->weight_decay)) return fail(W2V_E_ARG, "weight_decay must be finite");
    if (bp->step0 < 0) return fail(W2V_E_ARG, "step0 must be >= 0");
    if (bp->gain && bp->gain == bp->bias) return fail(W2V_E_ARG, "gain and bias must differ");
    if (!steps_host) return fail(W2V_E_ARG, "steps_host is NULL");
    if (int rc = check_workspace(workspace, workspace_bytes, batch_bytes(m, n_tokens, p, bp, true))) return rc;
    try {
        return run_batches(m, tokens, n_tokens, p, bp, true, stats, steps_host, sum_ll_host, n_terms_host, workspace,
                           as_stream(hip_stream));
    } catch (const std::exception &e) {
        return fail(W2V_E_ARG, std::string("the plan's tables: ") + e.what());
    }
}

size_t w2v_batch_loglik_workspace_bytes(const w2v_model *m, int64_t n_tokens, const w2v_params *p,
                                        const w2v_batch_params *bp) {
    return batch_sizes_ok(m, n_tokens, p, bp) ? batch_bytes(m, n_tokens, p, bp, false) : 0;
}

int w2v_batch_loglik(const w2v_model *m, const int32_t *tokens, int64_t n_tokens, const w2v_params *p,
                     const w2v_batch_params *bp, double *sum_ll_host, int64_t *n_terms_host, void *workspace,
                     size_t workspace_bytes, void *hip_stream) {
    set_error("");
    if (int rc = check_batch(m, tokens, n_tokens, p, bp)) return rc;
    if (!sum_ll_host || !n_terms_host) return fail(W2V_E_ARG, "a required pointer is NULL");
    if (int rc = check_workspace(workspace, workspace_bytes, batch_bytes(m, n_tokens, p, bp, false))) return rc;
    return run_batches(m, tokens, n_tokens, p, bp, false, nullptr, nullptr, sum_ll_host, n_terms_host, workspace,
                       as_stream(hip_stream));
}

}  // extern "C"
