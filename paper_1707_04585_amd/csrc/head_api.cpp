// Host side of the classification head and of the log probabilities: validation, buffer layouts and the launches.
#include "api_common.h"
#include "matrix_overlap.h"

using namespace rvn;
using namespace rvn::api;

namespace {

int check_matrix(const char *name, const rvn_matrix *m, int64_t rows, int64_t cols, bool f32_only) {
    if (!m) return fail(RVN_ERR_NULL, "matrix %s is NULL", name);
    if (!m->ptr) return fail(RVN_ERR_NULL, "matrix %s has a NULL data pointer", name);
    const int dtype = enum_bits(m->dtype);
    if (dtype != RVN_F32 && (dtype != RVN_BF16 || f32_only)) return fail(RVN_ERR_DTYPE, "matrix %s: dtype %d is not supported", name, dtype);
    if (m->rows != rows || m->cols != cols)
        return fail(RVN_ERR_SHAPE, "matrix %s has shape [%lld,%lld], expected [%lld,%lld]", name, (long long)m->rows, (long long)m->cols,
                    (long long)rows, (long long)cols);
    const int size = dtype == RVN_F32 ? 4 : 2;
    if (m->ld < m->cols || m->ld > INT64_MAX / 8 / rows) return fail(RVN_ERR_STRIDE, "matrix %s: ld = %lld with %lld columns", name, (long long)m->ld, (long long)m->cols);
    if (reinterpret_cast<uintptr_t>(m->ptr) % size) return fail(RVN_ERR_STRIDE, "matrix %s: data pointer is not aligned to its elements", name);
    return RVN_OK;
}

size_t matrix_bytes(const rvn_matrix *m) {
    return (size_t)((m->rows - 1) * m->ld + m->cols) * (enum_bits(m->dtype) == RVN_F32 ? 4 : 2);
}

RowBlock rows_of(const rvn_matrix *m) {
    const int64_t size = enum_bits(m->dtype) == RVN_F32 ? 4 : 2;
    return RowBlock{(int64_t)reinterpret_cast<uintptr_t>(m->ptr), m->cols * size, m->ld * size, m->rows};
}

// ---- head --------------------------------------------------------------------------

int check_head(const rvn_head_desc *d, int64_t n, int64_t h, int64_t w) {
    if (!d) return fail(RVN_ERR_NULL, "descriptor is NULL");
    if (d->c <= 0 || d->c > 65535) return fail(RVN_ERR_SHAPE, "c = %d out of range [1, 65535]", d->c);
    if (d->classes <= 0 || d->classes > (1 << 20)) return fail(RVN_ERR_SHAPE, "classes = %d out of range [1, %d]", d->classes, 1 << 20);
    if (!(d->bn_eps > 0.f)) return fail(RVN_ERR_SHAPE, "bn_eps must be > 0");
    if (int rc = check_geo(n, h, w)) return rc;
    if (n > 65535) return fail(RVN_ERR_SHAPE, "n = %lld exceeds 65535", (long long)n);
    // (what the launches can count in tiles of 16 x 16, up to 512 threads each)
    if (n * d->c > (1LL << 30) || (int64_t)d->c * d->classes > 0x7fffffffLL)
        return fail(RVN_ERR_SHAPE, "n*c = %lld exceeds 2^30 or c*classes = %lld exceeds 2^31-1", (long long)(n * d->c), (long long)d->c * d->classes);
    return RVN_OK;
}

struct HeadPlan {
    size_t stats, pooled, count, xhat, saved;  // offsets in `saved`, and its size
    size_t d_pooled, ws;
};

HeadPlan make_head_plan(const rvn_head_desc &d, int64_t n) {
    HeadPlan p{};
    const size_t planes = (size_t)n * d.c * 4;
    size_t off = align_up(kStatsArrays * (size_t)d.c * 4);
    p.pooled = off;
    off = align_up(off + planes);
    p.count = off;
    off = align_up(off + planes);
    p.xhat = off;
    p.saved = align_up(off + planes);
    p.ws = align_up(planes);
    return p;
}

HeadSaved bind_saved(const HeadPlan &p, void *saved) {
    char *b = static_cast<char *>(saved);
    auto at = [&](size_t off) { return reinterpret_cast<float *>(b + off); };
    return HeadSaved{at(p.stats), at(p.pooled), at(p.count), at(p.xhat)};
}

int check_head_params(const rvn_head_params *p) {
    if (!p) return fail(RVN_ERR_NULL, "params is NULL");
    if (!p->bn_gamma || !p->bn_beta || !p->fc_w || !p->fc_b) return fail(RVN_ERR_NULL, "params has a NULL pointer");
    return RVN_OK;
}

// ---- log probabilities ---------------------------------------------------------------

int check_logits(const rvn_matrix *m, int64_t *rows, int64_t *classes) {
    if (!m) return fail(RVN_ERR_NULL, "matrix logits is NULL");
    if (m->rows <= 0 || m->rows > 0x7fffffffLL || m->cols <= 0 || m->cols > (1 << 30))
        return fail(RVN_ERR_SHAPE, "logits has %lld rows of %lld classes", (long long)m->rows, (long long)m->cols);
    *rows = m->rows;
    *classes = m->cols;
    return check_matrix("logits", m, m->rows, m->cols, false);
}

int check_top_k(int32_t top_k, int64_t classes) {
    if (top_k < 0 || top_k > RVN_MAX_TOP_K || top_k > classes)
        return fail(RVN_ERR_SHAPE, "top_k = %d out of range [0, min(%lld, %d)]", top_k, (long long)classes, RVN_MAX_TOP_K);
    return RVN_OK;
}

Logits logits_of(const rvn_matrix *m) { return Logits{m->ptr, enum_bits(m->dtype) == RVN_BF16, m->rows, m->ld, (int)m->cols}; }

}  // namespace

extern "C" {

int revnet_head_workspace_bytes(const rvn_head_desc *desc, int64_t n, int64_t h, int64_t w, size_t *saved_bytes, size_t *bwd_bytes) {
    if (int rc = check_head(desc, n, h, w)) return rc;
    const HeadPlan p = make_head_plan(*desc, n);
    if (saved_bytes) *saved_bytes = p.saved;
    if (bwd_bytes) *bwd_bytes = p.ws;
    return RVN_OK;
}

int revnet_head_fwd(const rvn_head_desc *desc, const rvn_tensor *x, const rvn_head_params *params, const rvn_matrix *logits,
                    void *saved, size_t saved_bytes, void *hip_stream) {
    if (!x) return fail(RVN_ERR_NULL, "tensor x is NULL");
    if (int rc = check_head(desc, x->n, x->h, x->w)) return rc;
    if (int rc = check_any_tensor("x", x, desc->c, x->n, x->h, x->w)) return rc;
    if (int rc = check_head_params(params)) return rc;
    if (int rc = check_matrix("logits", logits, x->n, desc->classes, true)) return rc;
    const HeadPlan p = make_head_plan(*desc, x->n);
    if (int rc = check_store("saved", saved, saved_bytes, p.saved)) return rc;
    if (overlaps_range(x, saved, p.saved)) return fail(RVN_ERR_ALIAS, "x overlaps saved");
    if (overlaps_range(x, logits->ptr, matrix_bytes(logits))) return fail(RVN_ERR_ALIAS, "x overlaps logits");
    if (ranges_overlap(logits->ptr, matrix_bytes(logits), saved, p.saved)) return fail(RVN_ERR_ALIAS, "logits overlaps saved");
    const HeadSaved s = bind_saved(p, saved);
    const Geo g{(int)x->n, (int)x->h, (int)x->w};
    Ctx cx;
    cx.stream = static_cast<hipStream_t>(hip_stream);
    head_pool(cx, view_of(x), desc->c, g, desc->bn_eps, params->bn_gamma, params->bn_beta, s);
    head_linear(cx, s.pooled, g.n, desc->c, desc->classes, params->fc_w, params->fc_b, static_cast<float *>(logits->ptr), logits->ld);
    return finish(cx);
}

int revnet_head_bwd(const rvn_head_desc *desc, const rvn_tensor *x, const void *saved, size_t saved_bytes, const rvn_matrix *d_logits,
                    const rvn_head_params *params, const rvn_tensor *dx, const rvn_head_grads *grads, int accumulate_wgrads, void *ws,
                    size_t ws_bytes, void *hip_stream) {
    if (!x) return fail(RVN_ERR_NULL, "tensor x is NULL");
    if (int rc = check_head(desc, x->n, x->h, x->w)) return rc;
    if (int rc = check_any_tensor("x", x, desc->c, x->n, x->h, x->w)) return rc;
    if (int rc = check_any_tensor("dx", dx, desc->c, x->n, x->h, x->w)) return rc;
    if (int rc = check_matrix("d_logits", d_logits, x->n, desc->classes, true)) return rc;
    if (int rc = check_head_params(params)) return rc;
    if (!grads) return fail(RVN_ERR_NULL, "grads is NULL");
    if (!grads->d_bn_gamma || !grads->d_bn_beta || !grads->d_fc_w || !grads->d_fc_b) return fail(RVN_ERR_NULL, "grads has a NULL pointer");
    const HeadPlan p = make_head_plan(*desc, x->n);
    if (int rc = check_store("saved", saved, saved_bytes, p.saved)) return rc;
    if (int rc = check_ws(ws, ws_bytes, p.ws)) return rc;
    if (overlaps(x, dx)) return fail(RVN_ERR_ALIAS, "x and dx overlap");
    const size_t dl_bytes = matrix_bytes(d_logits);
    if (overlaps_range(x, ws, p.ws) || overlaps_range(dx, ws, p.ws) || ranges_overlap(saved, p.saved, ws, p.ws) ||
        ranges_overlap(d_logits->ptr, dl_bytes, ws, p.ws))
        return fail(RVN_ERR_ALIAS, "a buffer overlaps the workspace");
    if (overlaps_range(dx, saved, p.saved) || overlaps_range(dx, d_logits->ptr, dl_bytes))
        return fail(RVN_ERR_ALIAS, "dx overlaps saved or d_logits");
    const HeadSaved s = bind_saved(p, const_cast<void *>(saved));  // (read only)
    const Geo g{(int)x->n, (int)x->h, (int)x->w};
    float *d_pooled = static_cast<float *>(ws);
    Ctx cx;
    cx.stream = static_cast<hipStream_t>(hip_stream);
    head_linear_bwd(cx, static_cast<const float *>(d_logits->ptr), d_logits->ld, s.pooled, g.n, desc->c, desc->classes, params->fc_w, d_pooled,
                    grads->d_fc_w, grads->d_fc_b, accumulate_wgrads != 0);
    head_pool_bwd(cx, view_of(x), desc->c, g, s, d_pooled, grads->d_bn_gamma, grads->d_bn_beta, accumulate_wgrads != 0, view_of(dx));
    return finish(cx);
}

int revnet_logprob_workspace_bytes(int64_t rows, int64_t classes, int32_t top_k, size_t *bytes) {
    if (rows <= 0 || rows > 0x7fffffffLL || classes <= 0 || classes > (1 << 30))
        return fail(RVN_ERR_SHAPE, "%lld rows of %lld classes", (long long)rows, (long long)classes);
    if (int rc = check_top_k(top_k, classes)) return rc;
    if (bytes) *bytes = logprob_scratch_bytes(rows, (int)classes, top_k);
    return RVN_OK;
}

int revnet_logprob_fwd(const rvn_matrix *logits, const int64_t *labels, int32_t top_k, float *logprob, float *entropy, float *lse,
                       int64_t *top_ids, float *top_logprob, void *ws, size_t ws_bytes, void *hip_stream) {
    int64_t rows, classes;
    if (int rc = check_logits(logits, &rows, &classes)) return rc;
    if (int rc = check_top_k(top_k, classes)) return rc;
    if (!labels != !logprob) return fail(RVN_ERR_NULL, "labels and logprob: both or neither");
    if ((top_k > 0) != (top_ids != nullptr) || (top_logprob && top_k == 0))
        return fail(RVN_ERR_NULL, "top_ids is needed with top_k > 0 and must be NULL, as top_logprob, with top_k = 0");
    if (!logprob && !entropy && !lse && !top_ids) return fail(RVN_ERR_NULL, "no output is asked for");
    const size_t need = logprob_scratch_bytes(rows, (int)classes, top_k);
    if (need) {
        if (int rc = check_ws(ws, ws_bytes, need)) return rc;
        if (ranges_overlap(logits->ptr, matrix_bytes(logits), ws, need)) return fail(RVN_ERR_ALIAS, "logits overlaps the workspace");
    }
    Ctx cx;
    cx.stream = static_cast<hipStream_t>(hip_stream);
    logprob_fwd(cx, logits_of(logits), labels, LogprobOut{logprob, entropy, lse, top_ids, top_logprob, top_k}, ws);
    return finish(cx);
}

int revnet_logprob_bwd(const rvn_matrix *logits, const int64_t *labels, const float *lse, const float *entropy, const float *d_logprob,
                       const float *d_entropy, float scale, const rvn_matrix *d_logits, void *hip_stream) {
    int64_t rows, classes;
    if (int rc = check_logits(logits, &rows, &classes)) return rc;
    if (int rc = check_matrix("d_logits", d_logits, rows, classes, false)) return rc;
    if (enum_bits(d_logits->dtype) != enum_bits(logits->dtype)) return fail(RVN_ERR_DTYPE, "logits and d_logits differ in dtype");
    if (!lse) return fail(RVN_ERR_NULL, "lse is NULL");
    if (!labels && !d_entropy) return fail(RVN_ERR_NULL, "neither labels nor d_entropy is given");
    if (d_logprob && !labels) return fail(RVN_ERR_NULL, "d_logprob without labels");
    if (d_entropy && !entropy) return fail(RVN_ERR_NULL, "d_entropy without entropy");
    const bool same = logits->ptr == d_logits->ptr && (logits->ld == d_logits->ld || rows == 1);
    if (!same && row_blocks_overlap(rows_of(logits), rows_of(d_logits)))
        return fail(RVN_ERR_ALIAS, "logits and d_logits overlap");
    Ctx cx;
    cx.stream = static_cast<hipStream_t>(hip_stream);
    logprob_bwd(cx, logits_of(logits), labels, lse, entropy, d_logprob, d_entropy, scale, d_logits->ptr, d_logits->ld);
    return finish(cx);
}

}  // extern "C"
