// C ABI of the view refiner's operators (declared in include/mixrt.h): checks
// of their descriptors (pure host code) and the launches of the kernels in
// mixrt_norm.hip, mixrt_kept.hip and mixrt_rotary.hip on the context's stream.
#include "mixrt.h"

#include <cmath>

#include "mixrt_ctx.hpp"
#include "mixrt_refine.hpp"

namespace {

using mixrt::bind_device;
using mixrt::clear_err;
using mixrt::fail;
using mixrt::finish_launch;

constexpr int64_t kMaxElements = (int64_t)1 << 40;
constexpr int64_t kMaxStride = (int64_t)1 << 40;
constexpr int kMaxImages = 65535;
constexpr int kMaxHeads = 65535;
constexpr int kMaxHeadDim = 1024;

int elem_size(int dtype)
{
    return dtype == MIXRT_F32 ? 4 : dtype == MIXRT_F16 || dtype == MIXRT_BF16 ? 2 : 0;
}

bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

int check_dtype(mixrt_ctx *ctx, int dtype, const char *what)
{
    if (!elem_size(dtype))
        return fail(ctx, MIXRT_EUNSUPPORTED, "%s=%d (F32, F16 or BF16)", what, dtype);
    return MIXRT_OK;
}

int check_norm(mixrt_ctx *ctx, const mixrt_norm *d)
{
    if (!d) return fail(ctx, MIXRT_EINVAL, "norm is NULL");
    if (d->images < 0) return fail(ctx, MIXRT_EINVAL, "norm.images=%d", d->images);
    if (d->images > kMaxImages)
        return fail(ctx, MIXRT_EUNSUPPORTED, "norm.images=%d above %d", d->images, kMaxImages);
    if (d->channels < 1) return fail(ctx, MIXRT_EINVAL, "norm.channels=%d", d->channels);
    if (d->channels > MIXRT_MAX_CHANNELS)
        return fail(ctx, MIXRT_EUNSUPPORTED, "norm.channels=%d above %d", d->channels,
                    MIXRT_MAX_CHANNELS);
    if (d->pixels < 0) return fail(ctx, MIXRT_EINVAL, "norm.pixels=%lld", (long long)d->pixels);
    if (d->pixels >= kMaxElements / d->channels)
        return fail(ctx, MIXRT_EUNSUPPORTED, "norm: 2^40 elements or more per image");
    if (d->groups < 1 || d->channels % d->groups)
        return fail(ctx, MIXRT_EINVAL, "norm.groups=%d for %d channels", d->groups, d->channels);
    if (int rc = check_dtype(ctx, d->dtype, "norm.dtype")) return rc;
    if (d->act < MIXRT_ACT_NONE || d->act > MIXRT_ACT_GELU)
        return fail(ctx, MIXRT_EUNSUPPORTED, "norm.act=%d", d->act);
    if (!(d->eps >= 0.0f) || !std::isfinite(d->eps))
        return fail(ctx, MIXRT_EINVAL, "norm.eps=%g", d->eps);
    if (!aligned(d->gamma, 4) || !aligned(d->beta, 4))
        return fail(ctx, MIXRT_EINVAL, "norm.gamma or beta not 4-byte aligned");
    return MIXRT_OK;
}

// A map that the norm reads or, with out, writes: rows of an output must not
// overlap.  Strides are bounded so that no offset leaves 64 bits.
int check_map(mixrt_ctx *ctx, const mixrt_norm *d, const mixrt_map *m, const char *name, bool out)
{
    if (!m) return fail(ctx, MIXRT_EINVAL, "%s is NULL", name);
    if (d->images == 0 || d->pixels == 0) return MIXRT_OK;
    if (!m->data) return fail(ctx, MIXRT_EINVAL, "%s.data is NULL", name);
    if (!aligned(m->data, elem_size(d->dtype)))
        return fail(ctx, MIXRT_EINVAL, "%s.data not aligned to its element", name);
    if (m->pixel_stride < 0 || m->image_stride < 0 || m->pixel_stride >= kMaxStride ||
        m->image_stride >= kMaxStride ||
        (m->pixel_stride && d->pixels > kMaxElements / m->pixel_stride))
        return fail(ctx, MIXRT_EINVAL, "%s strides %lld, %lld", name, (long long)m->image_stride,
                    (long long)m->pixel_stride);
    if (!out) return MIXRT_OK;
    // disjoint rows: images apart from each other, or pixels of the images
    // interleaved with room for every image
    const int64_t C = d->channels, P = d->pixels, N = d->images;
    const int64_t image = (P - 1) * m->pixel_stride + C;
    const bool pixels = P == 1 || m->pixel_stride >= C;
    const bool apart = N == 1 || m->image_stride >= image;
    const bool between = N > 1 && m->image_stride >= C &&
                         (P == 1 || m->pixel_stride >= (N - 1) * m->image_stride + C);
    if (!((pixels && apart) || between))
        return fail(ctx, MIXRT_EINVAL, "%s: strides %lld, %lld make rows overlap", name,
                    (long long)m->image_stride, (long long)m->pixel_stride);
    return MIXRT_OK;
}

// An output in place of an input has the input's layout.
int check_in_place(mixrt_ctx *ctx, const mixrt_map *in, const mixrt_map *out, const char *names)
{
    if (in->data && in->data == out->data &&
        (in->pixel_stride != out->pixel_stride || in->image_stride != out->image_stride))
        return fail(ctx, MIXRT_EINVAL, "%s: the same data with other strides", names);
    return MIXRT_OK;
}

int check_kept(mixrt_ctx *ctx, const mixrt_kept *k, bool pointers)
{
    if (!k) return fail(ctx, MIXRT_EINVAL, "kept is NULL");
    if (k->rows < 0) return fail(ctx, MIXRT_EINVAL, "kept.rows=%lld", (long long)k->rows);
    if (k->channels < 1) return fail(ctx, MIXRT_EINVAL, "kept.channels=%d", k->channels);
    if (k->channels > MIXRT_MAX_CHANNELS)
        return fail(ctx, MIXRT_EUNSUPPORTED, "kept.channels=%d above %d", k->channels,
                    MIXRT_MAX_CHANNELS);
    if (k->rows >= kMaxElements / k->channels)
        return fail(ctx, MIXRT_EUNSUPPORTED, "kept: 2^40 elements or more");
    if (int rc = check_dtype(ctx, k->dtype, "kept.dtype")) return rc;
    if (pointers && k->rows > 0 && (!k->codes || !k->exps))
        return fail(ctx, MIXRT_EINVAL, "kept.codes or kept.exps is NULL");
    return MIXRT_OK;
}

// The kept form of a norm's x.
int check_norm_kept(mixrt_ctx *ctx, const mixrt_norm *d, const mixrt_kept *k)
{
    if (int rc = check_kept(ctx, k, true)) return rc;
    if (k->rows != d->images * d->pixels || k->channels != d->channels || k->dtype != d->dtype)
        return fail(ctx, MIXRT_EINVAL,
                    "kept of %lld rows, %d channels, dtype %d for a norm of %lld, %d, %d",
                    (long long)k->rows, k->channels, k->dtype,
                    (long long)(d->images * d->pixels), d->channels, d->dtype);
    return MIXRT_OK;
}

int check_workspace(mixrt_ctx *ctx, const void *ws, size_t have, size_t need)
{
    if (have < need)
        return fail(ctx, MIXRT_EINVAL, "workspace of %zu bytes, needs %zu", have, need);
    if (need && !ws) return fail(ctx, MIXRT_EINVAL, "workspace is NULL");
    if (!aligned(ws, 16)) return fail(ctx, MIXRT_EINVAL, "workspace not 16-byte aligned");
    return MIXRT_OK;
}

size_t norm_bytes(const mixrt_norm *d)
{
    return mixrt::norm_workspace(d->images, d->pixels, d->channels, d->groups, d->dtype);
}

mixrt::MapK map_k(const mixrt_map *m)
{
    return m ? mixrt::MapK{m->data, m->image_stride, m->pixel_stride}
             : mixrt::MapK{nullptr, 0, 0};
}

mixrt::NormLaunch norm_launch(const mixrt_norm *d, void *ws)
{
    mixrt::NormLaunch L{};
    L.N = d->images;
    L.C = d->channels;
    L.G = d->groups;
    L.dtype = d->dtype;
    L.act = d->act;
    L.P = d->pixels;
    L.eps = d->eps;
    L.gamma = d->gamma;
    L.beta = d->beta;
    L.ws = ws;
    return L;
}

// Rows of a packed or read-back array.
int check_rows(mixrt_ctx *ctx, const mixrt_kept *k, const void *p, int64_t stride, int dtype,
               const char *name, bool out, int width)
{
    if (k->rows == 0) return MIXRT_OK;
    if (!p) return fail(ctx, MIXRT_EINVAL, "%s is NULL", name);
    if (!aligned(p, elem_size(dtype)))
        return fail(ctx, MIXRT_EINVAL, "%s not aligned to its element", name);
    if (stride < 0 || stride >= kMaxStride || (stride && k->rows > kMaxElements / stride))
        return fail(ctx, MIXRT_EINVAL, "%s: row stride %lld", name, (long long)stride);
    if (out && k->rows > 1 && stride < width)
        return fail(ctx, MIXRT_EINVAL, "%s: row stride %lld makes rows overlap", name,
                    (long long)stride);
    return MIXRT_OK;
}

int check_outs(mixrt_ctx *ctx, int32_t outs)
{
    if (outs < 1) return fail(ctx, MIXRT_EINVAL, "outs=%d", outs);
    if (outs > MIXRT_MAX_CHANNELS)
        return fail(ctx, MIXRT_EUNSUPPORTED, "outs=%d above %d", outs, MIXRT_MAX_CHANNELS);
    return MIXRT_OK;
}

}  // namespace

extern "C" {

int mixrt_norm_workspace(const mixrt_norm *norm, size_t *bytes)
{
    clear_err(nullptr);
    if (!bytes) return fail(nullptr, MIXRT_EINVAL, "bytes is NULL");
    *bytes = 0;
    if (int rc = check_norm(nullptr, norm)) return rc;
    *bytes = norm_bytes(norm);
    return MIXRT_OK;
}

int mixrt_norm_forward(mixrt_ctx *ctx, const mixrt_norm *norm, const mixrt_map *x,
                       const mixrt_map *y, float *stats, const mixrt_kept *kept, void *workspace,
                       size_t workspace_bytes)
{
    if (!ctx) return fail(nullptr, MIXRT_EINVAL, "ctx is NULL");
    clear_err(ctx);
    int rc;
    if ((rc = check_norm(ctx, norm)) || (rc = check_map(ctx, norm, x, "x", false)) ||
        (rc = check_map(ctx, norm, y, "y", true)) || (rc = check_in_place(ctx, x, y, "x and y")))
        return rc;
    if (kept && (rc = check_norm_kept(ctx, norm, kept))) return rc;
    if (!aligned(stats, 8)) return fail(ctx, MIXRT_EINVAL, "stats not 8-byte aligned");
    if ((rc = check_workspace(ctx, workspace, workspace_bytes, norm_bytes(norm)))) return rc;
    if ((rc = bind_device(ctx))) return rc;
    mixrt::NormLaunch L = norm_launch(norm, workspace);
    L.x = map_k(x);
    L.y = map_k(y);
    L.stats = stats;
    L.codes = kept ? kept->codes : nullptr;
    L.exps = kept ? kept->exps : nullptr;
    return finish_launch(ctx, mixrt::launch_norm_forward(L, ctx->stream), "norm_forward");
}

int mixrt_norm_backward(mixrt_ctx *ctx, const mixrt_norm *norm, const mixrt_map *dy,
                        const mixrt_map *x, const mixrt_kept *kept, const float *stats,
                        const mixrt_map *dx, float *dgamma, float *dbeta, void *workspace,
                        size_t workspace_bytes)
{
    if (!ctx) return fail(nullptr, MIXRT_EINVAL, "ctx is NULL");
    clear_err(ctx);
    int rc;
    if ((rc = check_norm(ctx, norm)) || (rc = check_map(ctx, norm, dy, "dy", false))) return rc;
    if (!x == !kept) return fail(ctx, MIXRT_EINVAL, "one of x and kept has to be given");
    if (x && (rc = check_map(ctx, norm, x, "x", false))) return rc;
    if (kept && (rc = check_norm_kept(ctx, norm, kept))) return rc;
    if (dx && ((rc = check_map(ctx, norm, dx, "dx", true)) ||
               (rc = check_in_place(ctx, dy, dx, "dy and dx"))))
        return rc;
    if (x && dx && x->data && x->data == dx->data)
        return fail(ctx, MIXRT_EINVAL, "dx is x");
    if (norm->images > 0 && !stats) return fail(ctx, MIXRT_EINVAL, "stats is NULL");
    if (!aligned(stats, 8)) return fail(ctx, MIXRT_EINVAL, "stats not 8-byte aligned");
    if (!aligned(dgamma, 4) || !aligned(dbeta, 4))
        return fail(ctx, MIXRT_EINVAL, "dgamma or dbeta not 4-byte aligned");
    if ((rc = check_workspace(ctx, workspace, workspace_bytes, norm_bytes(norm)))) return rc;
    if ((rc = bind_device(ctx))) return rc;
    mixrt::NormLaunch L = norm_launch(norm, workspace);
    L.dy = map_k(dy);
    L.x = map_k(x);
    L.dx = map_k(dx);
    L.stats = (float *)stats;
    L.codes = kept ? kept->codes : nullptr;
    L.exps = kept ? kept->exps : nullptr;
    L.dgamma = dgamma;
    L.dbeta = dbeta;
    return finish_launch(ctx, mixrt::launch_norm_backward(L, ctx->stream), "norm_backward");
}

int mixrt_kept_pack(mixrt_ctx *ctx, const mixrt_kept *kept, const void *x, int64_t row_stride)
{
    if (!ctx) return fail(nullptr, MIXRT_EINVAL, "ctx is NULL");
    clear_err(ctx);
    int rc;
    if ((rc = check_kept(ctx, kept, true)) ||
        (rc = check_rows(ctx, kept, x, row_stride, kept->dtype, "x", false, kept->channels)))
        return rc;
    if ((rc = bind_device(ctx))) return rc;
    return finish_launch(ctx,
                         mixrt::launch_kept_pack(kept->dtype, kept->rows, kept->channels, x,
                                                 row_stride, kept->codes, kept->exps, ctx->stream),
                         "kept_pack");
}

int mixrt_kept_unpack(mixrt_ctx *ctx, const mixrt_kept *kept, int32_t out_dtype, void *out,
                      int64_t row_stride)
{
    if (!ctx) return fail(nullptr, MIXRT_EINVAL, "ctx is NULL");
    clear_err(ctx);
    int rc;
    if ((rc = check_kept(ctx, kept, true)) || (rc = check_dtype(ctx, out_dtype, "out_dtype")) ||
        (rc = check_rows(ctx, kept, out, row_stride, out_dtype, "out", true, kept->channels)))
        return rc;
    if ((rc = bind_device(ctx))) return rc;
    return finish_launch(ctx,
                         mixrt::launch_kept_unpack(out_dtype, kept->rows, kept->channels,
                                                   kept->codes, kept->exps, out, row_stride,
                                                   ctx->stream),
                         "kept_unpack");
}

int mixrt_linear_grad_workspace(const mixrt_kept *kept, int32_t outs, size_t *bytes)
{
    clear_err(nullptr);
    if (!bytes) return fail(nullptr, MIXRT_EINVAL, "bytes is NULL");
    *bytes = 0;
    int rc;
    if ((rc = check_kept(nullptr, kept, false)) || (rc = check_outs(nullptr, outs))) return rc;
    *bytes = mixrt::linear_grad_workspace(kept->rows, kept->channels, outs, kept->dtype);
    return MIXRT_OK;
}

int mixrt_linear_grad(mixrt_ctx *ctx, const mixrt_kept *kept, int32_t outs, const void *dy,
                      int64_t dy_stride, float *dw, float *db, void *workspace,
                      size_t workspace_bytes)
{
    if (!ctx) return fail(nullptr, MIXRT_EINVAL, "ctx is NULL");
    clear_err(ctx);
    int rc;
    if ((rc = check_kept(ctx, kept, true)) || (rc = check_outs(ctx, outs)) ||
        (rc = check_rows(ctx, kept, dy, dy_stride, kept->dtype, "dy", false, outs)))
        return rc;
    if (!dw) return fail(ctx, MIXRT_EINVAL, "dw is NULL");
    if (!aligned(dw, 4) || !aligned(db, 4))
        return fail(ctx, MIXRT_EINVAL, "dw or db not 4-byte aligned");
    if ((rc = check_workspace(ctx, workspace, workspace_bytes,
                              mixrt::linear_grad_workspace(kept->rows, kept->channels, outs,
                                                           kept->dtype))))
        return rc;
    if ((rc = bind_device(ctx))) return rc;
    return finish_launch(ctx,
                         mixrt::launch_linear_grad(kept->dtype, kept->rows, kept->channels, outs,
                                                   kept->codes, kept->exps, dy, dy_stride, dw, db,
                                                   workspace, ctx->stream),
                         "linear_grad");
}

int mixrt_rotary_apply(mixrt_ctx *ctx, const mixrt_rotary *r, const mixrt_heads *heads, int32_t n)
{
    if (!ctx) return fail(nullptr, MIXRT_EINVAL, "ctx is NULL");
    clear_err(ctx);
    int rc;
    if (!r) return fail(ctx, MIXRT_EINVAL, "rotary is NULL");
    if (r->tokens < 0) return fail(ctx, MIXRT_EINVAL, "rotary.tokens=%lld", (long long)r->tokens);
    if (r->tokens >= ((int64_t)1 << 31))
        return fail(ctx, MIXRT_EUNSUPPORTED, "rotary: 2^31 tokens or more");
    if (r->axes < 1 || r->axes > MIXRT_MAX_AXES)
        return fail(ctx, MIXRT_EUNSUPPORTED, "rotary.axes=%d outside 1..%d", r->axes,
                    MIXRT_MAX_AXES);
    if (r->layout != MIXRT_ROTARY_HALVES && r->layout != MIXRT_ROTARY_PAIRS)
        return fail(ctx, MIXRT_EUNSUPPORTED, "rotary.layout=%d", r->layout);
    if (r->pairs < 0) return fail(ctx, MIXRT_EINVAL, "rotary.pairs=%d", r->pairs);
    if (n < 1 || n > MIXRT_MAX_HEADS_ARRAYS)
        return fail(ctx, MIXRT_EINVAL, "n=%d outside 1..%d", n, MIXRT_MAX_HEADS_ARRAYS);
    if (!heads) return fail(ctx, MIXRT_EINVAL, "heads is NULL");
    if (r->pairs > 0 && r->tokens > 0) {
        if (!r->pos || !r->freq || !r->axis)
            return fail(ctx, MIXRT_EINVAL, "rotary.pos, freq or axis is NULL");
        if (!aligned(r->pos, 4) || !aligned(r->freq, 4))
            return fail(ctx, MIXRT_EINVAL, "rotary.pos or freq not 4-byte aligned");
    }
    mixrt::RotaryLaunch L{};
    L.tokens = r->tokens;
    L.axes = r->axes;
    L.pairs = r->pairs;
    L.layout = r->layout;
    L.dtype = heads[0].dtype;
    L.inverse = r->inverse != 0;
    L.pos = r->pos;
    L.freq = r->freq;
    L.axis = r->axis;
    if ((rc = check_dtype(ctx, L.dtype, "heads[0].dtype"))) return rc;
    for (int i = 0; i < n; ++i) {
        const mixrt_heads &h = heads[i];
        if (h.dtype != L.dtype)
            return fail(ctx, MIXRT_EINVAL, "heads[%d].dtype=%d beside %d", i, h.dtype, L.dtype);
        if (h.heads < 0 || h.heads > kMaxHeads)
            return fail(ctx, MIXRT_EUNSUPPORTED, "heads[%d].heads=%d outside 0..%d", i, h.heads,
                        kMaxHeads);
        if (h.head_dim < 1 || h.head_dim > kMaxHeadDim)
            return fail(ctx, MIXRT_EUNSUPPORTED, "heads[%d].head_dim=%d outside 1..%d", i,
                        h.head_dim, kMaxHeadDim);
        if (2 * r->pairs > h.head_dim)
            return fail(ctx, MIXRT_EINVAL, "heads[%d].head_dim=%d for %d pairs", i, h.head_dim,
                        r->pairs);
        if (h.heads == 0 || r->tokens == 0) continue;   // nothing of it is read or written
        if (!h.x || !h.out) return fail(ctx, MIXRT_EINVAL, "heads[%d].x or out is NULL", i);
        if (!aligned(h.x, elem_size(h.dtype)) || !aligned(h.out, elem_size(h.dtype)))
            return fail(ctx, MIXRT_EINVAL, "heads[%d].x or out not aligned to its element", i);
        const int64_t st[4] = {h.x_token_stride, h.x_head_stride, h.out_token_stride,
                               h.out_head_stride};
        for (int s = 0; s < 4; ++s)
            if (st[s] < 0 || st[s] >= kMaxStride ||
                (s % 2 == 0 && st[s] && r->tokens > kMaxElements / st[s]))
                return fail(ctx, MIXRT_EINVAL, "heads[%d]: stride %lld", i, (long long)st[s]);
        // the output's rows apart: heads inside a token, or tokens inside a head
        const int64_t D = h.head_dim, H = h.heads, T = r->tokens;
        const int64_t ot = h.out_token_stride, oh = h.out_head_stride;
        const bool inner = (H == 1 || oh >= D) && (T == 1 || ot >= (H - 1) * oh + D);
        const bool outer = (T == 1 || ot >= D) && (H == 1 || oh >= (T - 1) * ot + D);
        if (!inner && !outer)
            return fail(ctx, MIXRT_EINVAL, "heads[%d]: out strides %lld, %lld make rows overlap",
                        i, (long long)ot, (long long)oh);
        if (h.x == h.out && (h.x_token_stride != ot || h.x_head_stride != oh) && (T > 1 || H > 1))
            return fail(ctx, MIXRT_EINVAL, "heads[%d]: out is x with other strides", i);
        L.a[L.n++] = mixrt::HeadsK{h.heads, h.head_dim, h.x, h.out, h.x_token_stride,
                                   h.x_head_stride, ot, oh};
    }
    if ((rc = bind_device(ctx))) return rc;
    return finish_launch(ctx, mixrt::launch_rotary(L, ctx->stream), "rotary");
}

}  // extern "C"
