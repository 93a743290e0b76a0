// Host side of the 8-bit activation checkpoints: validation, the buffer's layout and the launches.
#include "api_common.h"

using namespace rvn;
using namespace rvn::api;

namespace {

int check_ckpt_shape(int64_t n, int64_t c, int64_t h, int64_t w) {
    if (c <= 0 || c > 65535) return fail(RVN_ERR_SHAPE, "c = %lld out of range [1, 65535]", (long long)c);
    if (int rc = check_geo(n, h, w)) return rc;
    return check_ckpt_extent(c, Geo{(int)n, (int)h, (int)w});
}

Ckpt ckpt_of(void *p, int c, const Geo &g) {
    char *b = static_cast<char *>(p);
    return Ckpt{reinterpret_cast<int8_t *>(b), reinterpret_cast<float *>(b + ckpt_codes_bytes(c, g))};
}

// A tensor of a checkpoint call: its own shape is the checkpoint's.
int check_ckpt_tensor(const char *name, const rvn_tensor *t, const void *ckpt, size_t have, int *c, Geo *g) {
    if (!t) return fail(RVN_ERR_NULL, "tensor %s is NULL", name);
    if (int rc = check_ckpt_shape(t->n, t->c, t->h, t->w)) return rc;
    if (int rc = check_any_tensor(name, t, t->c, t->n, t->h, t->w)) return rc;
    *c = (int)t->c;
    *g = Geo{(int)t->n, (int)t->h, (int)t->w};
    const size_t need = ckpt_bytes(*c, *g);
    if (int rc = check_store("ckpt", ckpt, have, need)) return rc;
    if (overlaps_range(t, ckpt, need)) return fail(RVN_ERR_ALIAS, "%s overlaps the checkpoint", name);
    return RVN_OK;
}

}  // namespace

extern "C" {

int revnet_ckpt_bytes(int64_t n, int64_t c, int64_t h, int64_t w, size_t *bytes) {
    if (int rc = check_ckpt_shape(n, c, h, w)) return rc;
    if (bytes) *bytes = ckpt_bytes((int)c, Geo{(int)n, (int)h, (int)w});
    return RVN_OK;
}

int revnet_ckpt_save(const rvn_tensor *x, const float *stats, void *ckpt, size_t have, void *hip_stream) {
    int c;
    Geo g;
    if (int rc = check_ckpt_tensor("x", x, ckpt, have, &c, &g)) return rc;
    Ctx cx;
    cx.stream = static_cast<hipStream_t>(hip_stream);
    const CkptTensor t{view_of(x), c, stats, ckpt_of(ckpt, c, g)};
    ckpt_save(cx, &t, 1, g);
    return finish(cx);
}

int revnet_ckpt_load(const void *ckpt, size_t have, const rvn_tensor *x, void *hip_stream) {
    int c;
    Geo g;
    if (int rc = check_ckpt_tensor("x", x, ckpt, have, &c, &g)) return rc;
    Ctx cx;
    cx.stream = static_cast<hipStream_t>(hip_stream);
    const CkptTensor t{view_of(x), c, nullptr, ckpt_of(const_cast<void *>(ckpt), c, g)};  // (the checkpoint is read only)
    ckpt_load(cx, &t, 1, g);
    return finish(cx);
}

int revnet_ckpt_bn_relu_workspace_bytes(int64_t n, int64_t c, int64_t h, int64_t w, size_t *bytes) {
    if (int rc = check_ckpt_shape(n, c, h, w)) return rc;
    if (bytes) *bytes = align_up(ckpt_bn_scratch_floats((int)c, Geo{(int)n, (int)h, (int)w}) * 4);
    return RVN_OK;
}

int revnet_ckpt_bn_relu_bwd(const void *ckpt, size_t have, const float *stats, const rvn_tensor *da, const rvn_tensor *skip,
                            const rvn_tensor *dx, float *d_gamma, float *d_beta, int accumulate, void *ws, size_t ws_bytes,
                            void *hip_stream) {
    int c;
    Geo g;
    if (int rc = check_ckpt_tensor("da", da, ckpt, have, &c, &g)) return rc;
    if (!stats) return fail(RVN_ERR_NULL, "stats is NULL");
    if (!d_gamma || !d_beta) return fail(RVN_ERR_NULL, "d_gamma or d_beta is NULL");
    if (int rc = check_any_tensor("dx", dx, c, g.n, g.h, g.w)) return rc;
    if (skip)
        if (int rc = check_any_tensor("skip", skip, c, g.n, g.h, g.w)) return rc;
    const size_t ckpt_need = ckpt_bytes(c, g), need = align_up(ckpt_bn_scratch_floats(c, g) * 4);
    if (int rc = check_ws(ws, ws_bytes, need)) return rc;
    const rvn_tensor *t[3] = {da, dx, skip};
    const char *nm[3] = {"da", "dx", "skip"};
    for (int i = 0; i < 3; ++i) {
        if (!t[i]) continue;
        if (overlaps_range(t[i], ckpt, ckpt_need)) return fail(RVN_ERR_ALIAS, "%s overlaps the checkpoint", nm[i]);
        if (overlaps_range(t[i], ws, need)) return fail(RVN_ERR_ALIAS, "%s overlaps the workspace", nm[i]);
        if (i != 1 && !same_tensor(t[i], dx) && overlaps(t[i], dx)) return fail(RVN_ERR_ALIAS, "%s and dx overlap", nm[i]);
    }
    if (ranges_overlap(ckpt, ckpt_need, ws, need)) return fail(RVN_ERR_ALIAS, "the checkpoint overlaps the workspace");
    Ctx cx;
    cx.stream = static_cast<hipStream_t>(hip_stream);
    const View kv = skip ? view_of(skip) : View{};
    ckpt_bn_relu_bwd(cx, ckpt_of(const_cast<void *>(ckpt), c, g), view_of(da), c, g, stats, static_cast<float *>(ws), d_gamma, d_beta,
                     accumulate != 0, skip ? &kv : nullptr, view_of(dx));
    return finish(cx);
}

}  // extern "C"
