// esb_lm_api.cu -- the extern "C" entry points of the language-model
// operators: host-side argument validation and launches.  Declarations and
// contracts are in include/esb.h.
#include <cmath>
#include <cstdint>
#include <initializer_list>

#include <cuda_runtime.h>

#include "esb.h"
#include "esb_common.cuh"
#include "esb_internal.h"

using namespace esb;

namespace {

bool type_ok(int32_t t) { return t == ESB_F32 || t == ESB_F16 || t == ESB_BF16; }
bool group_ok(int64_t g) { return g >= 0 && g % 32 == 0; }
bool rounding_ok(int32_t r) { return r == ESB_ROUND_HALF_AWAY || r == ESB_ROUND_HALF_EVEN; }
int64_t groups_of(int64_t cols, int64_t g) { return g > 0 && g < cols ? (cols + g - 1) / g : 1; }
int64_t words_of(int64_t cols, int b) { return (cols + 32 / b - 1) / (32 / b); }
bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
// Rows of a type start on that type's boundary.
bool typed(const void* p, int32_t t) { return aligned(p, t == ESB_F32 ? 4 : 2); }
bool head_ok(int32_t d) { return d >= 8 && d <= 256 && d % 8 == 0; }
// A rotation that there may be, for tokens with these positions (or, not given,
// with those of their sequences).  A kernel reads row 0 for a position that the
// table lacks.
esb_status rotation_ok(const esb_rotation* r, int32_t head_dim, int64_t tokens, const int64_t* positions, bool given = true)
{
    if (!r || r->dim == 0) return ESB_OK;
    if (r->dim < 0 || r->dim % 2 != 0 || r->dim > head_dim) return ESB_ERR_UNSUPPORTED;
    if (!r->table || r->positions < 0 || r->ld < r->dim) return ESB_ERR_INVALID_ARG;
    if (tokens > 0 && (r->positions == 0 || (given && !positions))) return ESB_ERR_INVALID_ARG;
    return aligned(r->table, 4) && aligned(positions, 8) ? ESB_OK : ESB_ERR_ALIGN;
}
esb_status cache_ok(const esb_kv_cache* c)
{
    if (!c) return ESB_ERR_INVALID_ARG;
    for (const esb_format& f : {c->k_fmt, c->v_fmt})
        if (esb_format_check(f) != ESB_OK || f.b != 4 || !f.is_signed) return ESB_ERR_UNSUPPORTED;
    if (!head_ok(c->head_dim) || c->page_size <= 0 || c->page_size % 16 != 0) return ESB_ERR_UNSUPPORTED;
    if (c->pages < 0 || c->heads <= 0) return ESB_ERR_INVALID_ARG;
    const int64_t rows = (int64_t)c->heads * c->page_size;
    if (c->heads >= 1 << 23 || c->page_size > 1 << 24 || rows >= 1ll << 31 || c->pages > 1ll << 31 || c->page_ld >= 1ll << 34 ||
        c->page_lds >= 1ll << 32)
        return ESB_ERR_RANGE;
    if (c->pages > 0 && (!c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales)) return ESB_ERR_INVALID_ARG;
    if (c->pages > 1 && (c->page_ld < rows * esb_row_words(c->head_dim, 4) || c->page_lds < rows)) return ESB_ERR_INVALID_ARG;
    return aligned(c->k_codes, 16) && aligned(c->v_codes, 16) && (c->pages <= 1 || c->page_ld % 4 == 0) && aligned(c->k_scales, 4) &&
                   aligned(c->v_scales, 4) ? ESB_OK : ESB_ERR_ALIGN;
}
esb_status done(cudaError_t e) { return e == cudaSuccess ? ESB_OK : ESB_ERR_CUDA; }

}  // namespace

extern "C" {

esb_status esb_project_groups(const void* x, int32_t x_type, int64_t rows, int64_t cols, int64_t ldx, esb_format f,
                              int32_t rounding, int32_t rule, int64_t group, uint32_t* codes, int64_t ldc,
                              float* scales, int64_t lds, void* xq, int32_t xq_type, int64_t ldq, void* stream)
{
    if (esb_format_check(f) != ESB_OK || (f.b != 4 && f.b != 8) || !group_ok(group)) return ESB_ERR_UNSUPPORTED;
    if (!type_ok(x_type) || (xq && !type_ok(xq_type)) || !rounding_ok(rounding)) return ESB_ERR_INVALID_ARG;
    if (rule != ESB_SCALE_ABSMAX && rule != ESB_SCALE_DDA) return ESB_ERR_INVALID_ARG;
    if (rows < 0 || cols < 0 || ldx < cols || ldc < words_of(cols, f.b) || (xq && ldq < cols)) return ESB_ERR_INVALID_ARG;
    if (rows == 0 || cols == 0) return ESB_OK;
    if (!x || !codes || !scales || lds < groups_of(cols, group)) return ESB_ERR_INVALID_ARG;
    if (!typed(x, x_type) || !aligned(codes, 4) || !aligned(scales, 4) || (xq && !typed(xq, xq_type))) return ESB_ERR_ALIGN;
    double as = 0.0;
    if (rule == ESB_SCALE_DDA) {
        const esb_status s = esb_alpha_star(f.b, f.k, &as, nullptr);
        if (s != ESB_OK) return s;
    }
    return done(launch_project_groups(x, x_type, rows, cols, ldx, f, rounding, rule, group, as, codes, ldc, scales, lds,
                                      xq, xq_type, ldq, static_cast<cudaStream_t>(stream)));
}

esb_status esb_matvec_groups(int64_t M, int64_t N, int64_t K, const void* x, int32_t x_type, int64_t ldx,
                             const esb_coded* xc, const esb_coded* w, const float* bias, void* y, int32_t y_type,
                             int64_t ldy, void* stream)
{
    const bool coded = x_type == ESB_CODES;
    if ((!coded && !type_ok(x_type)) || !type_ok(y_type) || !w || (coded && !xc)) return ESB_ERR_INVALID_ARG;
    if (M < 0 || N < 0 || K < 0 || ldy < N) return ESB_ERR_INVALID_ARG;
    if (esb_format_check(w->fmt) != ESB_OK || w->fmt.b != 4 || !group_ok(w->group)) return ESB_ERR_UNSUPPORTED;
    if (K >= 1 << 18 || N > 1ll << 30) return ESB_ERR_RANGE;
    if (M == 0 || N == 0) return ESB_OK;
    if (!y || K == 0 || !w->codes || !w->scales || w->ld < words_of(K, 4) || w->lds < groups_of(K, w->group)) return ESB_ERR_INVALID_ARG;
    if (!aligned(w->codes, 16) || w->ld % 4 != 0 || !aligned(w->scales, 4) || !aligned(bias, 4) || !typed(y, y_type)) return ESB_ERR_ALIGN;
    if (coded) {
        if (esb_format_check(xc->fmt) != ESB_OK || xc->fmt.b != 8 || xc->fmt.k < 2 || !group_ok(xc->group)) return ESB_ERR_UNSUPPORTED;
        const int64_t gw = groups_of(K, w->group) == 1 ? 0 : w->group, gx = groups_of(K, xc->group) == 1 ? 0 : xc->group;
        if (gx && (!gw || gx % gw != 0)) return ESB_ERR_UNSUPPORTED;
        if (!xc->codes || !xc->scales || xc->ld < words_of(K, 8) || xc->lds < groups_of(K, xc->group)) return ESB_ERR_INVALID_ARG;
        if (!aligned(xc->codes, 4) || !aligned(xc->scales, 4)) return ESB_ERR_ALIGN;
    } else {
        if (!x || ldx < K) return ESB_ERR_INVALID_ARG;
        if (!typed(x, x_type)) return ESB_ERR_ALIGN;
    }
    return done(launch_matvec_groups(M, N, K, x, x_type, ldx, coded ? xc : nullptr, *w, bias, y, y_type, ldy,
                                     static_cast<cudaStream_t>(stream)));
}

esb_status esb_rmsnorm(int64_t rows, int64_t cols, const esb_norm* a, void* stream)
{
    if (!a || rows < 0 || cols < 0 || !(std::isfinite(a->eps) && a->eps >= 0.0f)) return ESB_ERR_INVALID_ARG;
    if (!type_ok(a->x_type) || (a->weight && !type_ok(a->w_type)) || ((a->y || a->yq) && !type_ok(a->y_type))) return ESB_ERR_INVALID_ARG;
    if (a->codes) {
        if (esb_format_check(a->fmt) != ESB_OK || a->fmt.b != 8 || !group_ok(a->group)) return ESB_ERR_UNSUPPORTED;
        if (!rounding_ok(a->rounding) || !a->scales || a->ldc < words_of(cols, 8) || a->lds < groups_of(cols, a->group)) return ESB_ERR_INVALID_ARG;
        if (!aligned(a->codes, 4) || !aligned(a->scales, 4)) return ESB_ERR_ALIGN;
    } else if (a->yq) {
        return ESB_ERR_INVALID_ARG;
    }
    if (rows == 0 || cols == 0) return ESB_OK;
    if (!a->x || a->ldx < cols || (a->residual && a->ldr < cols) || (a->h && a->ldh < cols) || (a->y && a->ldy < cols) ||
        (a->yq && a->ldq < cols))
        return ESB_ERR_INVALID_ARG;
    if (!typed(a->x, a->x_type) || !typed(a->residual, a->x_type) || !typed(a->h, a->x_type) || !aligned(a->rstd, 4) ||
        (a->weight && !typed(a->weight, a->w_type)) || (a->y && !typed(a->y, a->y_type)) || (a->yq && !typed(a->yq, a->y_type)))
        return ESB_ERR_ALIGN;
    return done(launch_rmsnorm(rows, cols, *a, static_cast<cudaStream_t>(stream)));
}

size_t esb_rmsnorm_backward_workspace_bytes(int64_t rows, int64_t cols)
{
    return rows > 0 && cols > 0 ? rmsnorm_grad_workspace_bytes(rows, cols) : 0;
}

esb_status esb_rmsnorm_backward(int64_t rows, int64_t cols, const esb_norm_grad* a, void* workspace, size_t workspace_bytes,
                                void* stream)
{
    if (!a || rows < 0 || cols < 0) return ESB_ERR_INVALID_ARG;
    if (!type_ok(a->x_type) || !type_ok(a->g_type) || (a->weight && !type_ok(a->w_type))) return ESB_ERR_INVALID_ARG;
    if (cols == 0 || (rows == 0 && !a->dweight)) return ESB_OK;
    if (rows == 0)   // no row adds to dweight
        return done(cudaMemsetAsync(a->dweight, 0, sizeof(float) * (size_t)cols, static_cast<cudaStream_t>(stream)));
    if (!a->dy || !a->h || !a->rstd || !a->dx || a->ldg < cols || a->ldh < cols || a->lddx < cols || (a->dh && a->lddh < cols))
        return ESB_ERR_INVALID_ARG;
    if (!typed(a->dy, a->g_type) || !typed(a->h, a->x_type) || !typed(a->dh, a->x_type) || !typed(a->dx, a->x_type) ||
        !aligned(a->rstd, 4) || !aligned(a->dweight, 4) || (a->weight && !typed(a->weight, a->w_type)))
        return ESB_ERR_ALIGN;
    if (a->dweight) {
        if (!workspace || workspace_bytes < rmsnorm_grad_workspace_bytes(rows, cols)) return ESB_ERR_INVALID_ARG;
        if (!aligned(workspace, 16)) return ESB_ERR_ALIGN;
    }
    return done(launch_rmsnorm_grad(rows, cols, *a, workspace, static_cast<cudaStream_t>(stream)));
}

esb_status esb_logprobs(const void* x, int32_t x_type, int64_t rows, int64_t cols, int64_t ldx, const int64_t* ids,
                        int32_t top, float* logp, float* entropy, float* lse, float* top_logp, int64_t* top_ids,
                        void* stream)
{
    if (!type_ok(x_type) || rows < 0 || cols < 0 || top < 0 || (logp && !ids)) return ESB_ERR_INVALID_ARG;
    if (top > ESB_MAX_TOP || cols >= 1ll << 31) return ESB_ERR_RANGE;
    if (rows == 0) return ESB_OK;
    if (cols == 0 || !x || ldx < cols || (top > 0 && (!top_logp || !top_ids))) return ESB_ERR_INVALID_ARG;
    if (!typed(x, x_type) || !aligned(ids, 8) || !aligned(top_ids, 8) || !aligned(logp, 4) || !aligned(entropy, 4) ||
        !aligned(lse, 4) || !aligned(top_logp, 4))
        return ESB_ERR_ALIGN;
    return done(launch_logprobs(x, x_type, rows, cols, ldx, ids, top, logp, entropy, lse, top_logp, top_ids,
                                static_cast<cudaStream_t>(stream)));
}

esb_status esb_logprobs_backward(const void* x, int32_t x_type, int64_t rows, int64_t cols, int64_t ldx,
                                 const int64_t* ids, const float* lse, const float* entropy, const float* dlogp,
                                 const float* dentropy, void* dx, int64_t lddx, void* stream)
{
    if (!type_ok(x_type) || rows < 0 || cols < 0 || (dlogp && !ids) || (dentropy && !entropy)) return ESB_ERR_INVALID_ARG;
    if (cols >= 1ll << 31) return ESB_ERR_RANGE;
    if (rows == 0 || cols == 0) return ESB_OK;
    if (!x || !lse || !dx || ldx < cols || lddx < cols) return ESB_ERR_INVALID_ARG;
    if (!typed(x, x_type) || !typed(dx, x_type) || !aligned(ids, 8) || !aligned(lse, 4) || !aligned(entropy, 4) ||
        !aligned(dlogp, 4) || !aligned(dentropy, 4))
        return ESB_ERR_ALIGN;
    return done(launch_logprobs_grad(x, x_type, rows, cols, ldx, ids, lse, entropy, dlogp, dentropy, dx, lddx,
                                     static_cast<cudaStream_t>(stream)));
}

esb_status esb_headnorm(int64_t tokens, const esb_head_norm* a, void* stream)
{
    if (!a || tokens < 0 || !(std::isfinite(a->eps) && a->eps >= 0.0f) || !type_ok(a->x_type)) return ESB_ERR_INVALID_ARG;
    if (!head_ok(a->head_dim)) return ESB_ERR_UNSUPPORTED;
    if (tokens >= 1ll << 31) return ESB_ERR_RANGE;
    const esb_status r = rotation_ok(&a->rotation, a->head_dim, tokens, a->positions);
    if (r != ESB_OK) return r;
    int64_t heads = 0;
    for (const esb_heads& h : a->part) {
        if (h.heads < 0) return ESB_ERR_INVALID_ARG;
        if (h.heads >= 1 << 23) return ESB_ERR_RANGE;
        heads += h.heads;
        if (h.heads == 0 || tokens == 0) continue;
        const int64_t cols = (int64_t)h.heads * a->head_dim;
        if (!h.x || !h.y || h.ldx < cols || h.ldy < cols || (h.weight && !type_ok(a->w_type))) return ESB_ERR_INVALID_ARG;
        if (!typed(h.x, a->x_type) || !typed(h.y, a->x_type) || !aligned(h.rstd, 4) || (h.weight && !typed(h.weight, a->w_type)))
            return ESB_ERR_ALIGN;
    }
    if (tokens == 0 || heads == 0) return ESB_OK;
    return done(launch_headnorm(tokens, *a, static_cast<cudaStream_t>(stream)));
}

size_t esb_headnorm_backward_workspace_bytes(int64_t tokens, int64_t heads, int32_t head_dim)
{
    return tokens > 0 && tokens < 1ll << 31 && heads > 0 && heads < 1 << 24 && head_ok(head_dim)
               ? headnorm_grad_workspace_bytes(tokens, heads, head_dim) : 0;
}

esb_status esb_headnorm_backward(int64_t tokens, const esb_head_norm_grad* a, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!a || tokens < 0 || !type_ok(a->x_type)) return ESB_ERR_INVALID_ARG;
    if (!head_ok(a->head_dim)) return ESB_ERR_UNSUPPORTED;
    if (tokens >= 1ll << 31) return ESB_ERR_RANGE;
    const esb_status r = rotation_ok(&a->rotation, a->head_dim, tokens, a->positions);
    if (r != ESB_OK) return r;
    int64_t heads = 0;
    bool sums = false;
    for (const esb_heads_grad& h : a->part) {
        if (h.heads < 0) return ESB_ERR_INVALID_ARG;
        if (h.heads >= 1 << 23) return ESB_ERR_RANGE;
        heads += h.heads;
        if (!aligned(h.dweight, 4)) return ESB_ERR_ALIGN;
        sums = sums || h.dweight;
        if (h.heads == 0 || tokens == 0) continue;
        const int64_t cols = (int64_t)h.heads * a->head_dim;
        if (!h.x || !h.dy || !h.dx || !h.rstd || h.ldx < cols || h.ldg < cols || h.lddx < cols || (h.weight && !type_ok(a->w_type)))
            return ESB_ERR_INVALID_ARG;
        if (!typed(h.x, a->x_type) || !typed(h.dy, a->x_type) || !typed(h.dx, a->x_type) || !aligned(h.rstd, 4) ||
            (h.weight && !typed(h.weight, a->w_type)))
            return ESB_ERR_ALIGN;
    }
    if (tokens == 0 || heads == 0) {    // nothing adds to the weights' gradients
        for (const esb_heads_grad& h : a->part)
            if (h.dweight) {
                const cudaError_t e = cudaMemsetAsync(h.dweight, 0, sizeof(float) * (size_t)a->head_dim, static_cast<cudaStream_t>(stream));
                if (e != cudaSuccess) return ESB_ERR_CUDA;
            }
        return ESB_OK;
    }
    if (sums) {
        if (!workspace || workspace_bytes < headnorm_grad_workspace_bytes(tokens, heads, a->head_dim)) return ESB_ERR_INVALID_ARG;
        if (!aligned(workspace, 16)) return ESB_ERR_ALIGN;
    }
    return done(launch_headnorm_grad(tokens, *a, workspace, static_cast<cudaStream_t>(stream)));
}

esb_status esb_cache_append(int64_t tokens, const esb_kv_cache* c, const esb_append* a, void* stream)
{
    if (!a || tokens < 0 || !type_ok(a->x_type) || ((a->kq || a->vq) && !type_ok(a->q_type)) || !rounding_ok(a->rounding) ||
        (a->rule != ESB_SCALE_ABSMAX && a->rule != ESB_SCALE_DDA))
        return ESB_ERR_INVALID_ARG;
    esb_status r = cache_ok(c);
    if (r != ESB_OK) return r;
    if (tokens >= 1ll << 31) return ESB_ERR_RANGE;
    r = rotation_ok(a->rotation, c->head_dim, tokens, a->positions);
    if (r != ESB_OK) return r;
    if (tokens == 0) return ESB_OK;
    const int64_t cols = (int64_t)c->heads * c->head_dim;
    if (!a->k || !a->v || !a->slots || a->ldk < cols || a->ldv < cols || (a->kq && a->ldkq < cols) || (a->vq && a->ldvq < cols))
        return ESB_ERR_INVALID_ARG;
    if (!typed(a->k, a->x_type) || !typed(a->v, a->x_type) || !aligned(a->slots, 8) || (a->kq && !typed(a->kq, a->q_type)) ||
        (a->vq && !typed(a->vq, a->q_type)))
        return ESB_ERR_ALIGN;
    double sk = 0.0, sv = 0.0;
    if (a->rule == ESB_SCALE_DDA) {
        r = esb_alpha_star(4, c->k_fmt.k, &sk, nullptr);
        if (r == ESB_OK) r = esb_alpha_star(4, c->v_fmt.k, &sv, nullptr);
        if (r != ESB_OK) return r;
    }
    return done(launch_cache_append(tokens, *c, *a, sk, sv, static_cast<cudaStream_t>(stream)));
}

size_t esb_cache_attention_workspace_bytes(int64_t tokens, int32_t seqs, int32_t q_heads, int32_t heads, int32_t head_dim, int32_t q_type)
{
    if (tokens <= 0 || tokens >= 1ll << 31 || seqs <= 0 || heads <= 0 || q_heads <= 0 || q_heads % heads != 0 || !head_ok(head_dim) || !type_ok(q_type))
        return 0;
    return attention_workspace_bytes(tokens, seqs, q_heads, heads, head_dim, q_type);
}

esb_status esb_cache_attention(int64_t tokens, const esb_kv_cache* c, const esb_attention* a, void* workspace, size_t workspace_bytes,
                               void* stream)
{
    if (!a || tokens < 0 || a->seqs < 0 || a->max_pages < 0 || a->window < 0 || !std::isfinite(a->scale) || !type_ok(a->q_type) ||
        !type_ok(a->out_type))
        return ESB_ERR_INVALID_ARG;
    esb_status r = cache_ok(c);
    if (r != ESB_OK) return r;
    if (a->q_heads <= 0 || a->q_heads % c->heads != 0) return ESB_ERR_UNSUPPORTED;
    if (tokens >= 1ll << 31 || a->q_heads >= 1 << 23 || (int64_t)a->max_pages * c->page_size > 1 << 30) return ESB_ERR_RANGE;
    if (tokens * (a->q_heads / c->heads) >= (1ll << 31) - 64) return ESB_ERR_RANGE;
    r = rotation_ok(a->rotation, c->head_dim, a->seqs > 0 ? tokens : 0, nullptr, false);
    if (r != ESB_OK) return r;
    if (tokens == 0 || a->seqs == 0) return ESB_OK;
    const int64_t cols = (int64_t)a->q_heads * c->head_dim;
    if (!a->q || !a->out || !a->lens || (!a->pages && a->max_pages > 0) || a->ldq < cols || a->ldo < cols || a->ld_pages < a->max_pages ||
        (!a->starts && tokens != a->seqs))
        return ESB_ERR_INVALID_ARG;
    if (!typed(a->q, a->q_type) || !typed(a->out, a->out_type) || !aligned(a->lse, 4) || !aligned(a->starts, 4) || !aligned(a->lens, 4) ||
        !aligned(a->pages, 4))
        return ESB_ERR_ALIGN;
    if (!workspace || workspace_bytes < attention_workspace_bytes(tokens, a->seqs, a->q_heads, c->heads, c->head_dim, a->q_type))
        return ESB_ERR_INVALID_ARG;
    if (!aligned(workspace, 16)) return ESB_ERR_ALIGN;
    return done(launch_attention(tokens, *c, *a, workspace, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
