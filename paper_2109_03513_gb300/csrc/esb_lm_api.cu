// esb_lm_api.cu -- the extern "C" entry points of the language-model
// operators: host-side argument validation and launches.  Declarations and
// contracts are in include/esb.h.
#include <cmath>
#include <cstdint>

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

}  // extern "C"
