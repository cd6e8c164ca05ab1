// C ABI of the residual step and the vocabulary loss: argument validation, workspace carving and launch sequencing.
#include "../../../include/stl.h"
#include "lm_kernels.h"

#include <cstdarg>
#include <cstdio>

namespace {

stl_status_t fail(stl_status_t st, const char *fmt, ...)
{
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(stl::error_text(), stl::kErrorText, fmt, ap);
    va_end(ap);
    return st;
}

#define LM_HIP(call, what)                                                                                                             \
    do {                                                                                                                               \
        const hipError_t e_ = (call);                                                                                                  \
        if (e_ != hipSuccess) return fail(STL_ERR_HIP, "%s: %s", what, hipGetErrorString(e_));                                         \
    } while (0)

template <typename... P>
bool any_misaligned(P... ptrs)
{
    return ((((uintptr_t)ptrs) & 15) || ...);
}

stl_status_t check_workspace(const char *fn, const void *ws, size_t ws_bytes, size_t need)
{
    if (need > 0 && (!ws || ws_bytes < need))
        return fail(STL_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, ws ? ws_bytes : (size_t)0);
    if (ws && ((uintptr_t)ws & 15)) return fail(STL_ERR_INVALID_ARG, "%s: workspace is not 16-byte aligned", fn);
    return STL_OK;
}

constexpr int kResidualFlags = STL_FLAG_POST_NORM | STL_FLAG_PRE_NORM | STL_FLAG_CENTER;
static_assert(STL_RESIDUAL_WIDEST == stl::lm::kResidualWidest, "documented width");

stl_status_t check_residual(const stl_residual_t *p, int flags, stl::lm::ResidualArgs *a)
{
    if (!p) return fail(STL_ERR_INVALID_ARG, "problem descriptor is NULL");
    if (p->dtype != STL_F32 && p->dtype != STL_BF16) return fail(STL_ERR_UNSUPPORTED, "unknown dtype %d", p->dtype);
    if (flags & ~kResidualFlags) return fail(STL_ERR_UNSUPPORTED, "unknown flag bits 0x%x", flags & ~kResidualFlags);
    if (p->rows < 0 || p->n < 1 || p->rows_per_gate < 1)
        return fail(STL_ERR_INVALID_ARG, "rows=%lld n=%lld rows_per_gate=%lld: rows may be 0, the others are positive", (long long)p->rows,
                    (long long)p->n, (long long)p->rows_per_gate);
    if (p->rows > STL_MAX_DIM) return fail(STL_ERR_INVALID_ARG, "more than %d rows", STL_MAX_DIM);
    if (p->n > STL_RESIDUAL_WIDEST) return fail(STL_ERR_UNSUPPORTED, "n=%lld: rows of at most %d elements are supported", (long long)p->n, STL_RESIDUAL_WIDEST);
    if (!(p->eps > 0.f)) return fail(STL_ERR_INVALID_ARG, "eps must be positive");
    *a = stl::lm::ResidualArgs{};
    a->rows = (int)p->rows, a->n = (int)p->n;
    a->per_gate = (int)(p->rows_per_gate < p->rows ? p->rows_per_gate : p->rows > 0 ? p->rows : 1);
    a->skip = p->skip, a->scale = p->scale, a->eps = p->eps;
    a->post = flags & STL_FLAG_POST_NORM, a->pre = flags & STL_FLAG_PRE_NORM, a->center = flags & STL_FLAG_CENTER;
    return STL_OK;
}

static_assert(STL_VOCAB_MOST_TOP == stl::lm::kMostTop, "documented count");

stl_status_t check_vocab(const stl_vocab_t *p, stl::lm::VocabArgs *a)
{
    if (!p) return fail(STL_ERR_INVALID_ARG, "problem descriptor is NULL");
    if (p->dtype != STL_F32 && p->dtype != STL_BF16) return fail(STL_ERR_UNSUPPORTED, "unknown dtype %d", p->dtype);
    if (p->rows < 0 || p->d < 1 || p->vocab < 1 || p->ntop < 0)
        return fail(STL_ERR_INVALID_ARG, "rows=%lld d=%lld vocab=%lld ntop=%lld: rows and ntop may be 0, the others are positive", (long long)p->rows,
                    (long long)p->d, (long long)p->vocab, (long long)p->ntop);
    if (p->rows > STL_MAX_DIM || p->d > STL_VOCAB_WIDEST || p->vocab > STL_VOCAB_MOST || p->ntop > STL_VOCAB_MOST_TOP)
        return fail(STL_ERR_INVALID_ARG, "more than %d rows, d=%d, vocab=%d or ntop=%d", STL_MAX_DIM, STL_VOCAB_WIDEST, STL_VOCAB_MOST, STL_VOCAB_MOST_TOP);
    if (p->ntop > 0 && !(p->temperature >= stl::lm::kLowestTau && p->temperature <= stl::lm::kHighestTau))
        return fail(STL_ERR_INVALID_ARG, "temperature %g outside [%g, %g]", (double)p->temperature, (double)stl::lm::kLowestTau, (double)stl::lm::kHighestTau);
    *a = stl::lm::VocabArgs{};
    a->rows = (int)p->rows, a->d = (int)p->d, a->vocab = (int)p->vocab, a->ntop = (int)p->ntop;
    a->tau = p->ntop > 0 ? p->temperature : 1.f;
    a->bf16 = p->dtype == STL_BF16;
    return STL_OK;
}

// what the forward and the backward call have in common
stl_status_t vocab_inputs(const char *fn, const stl_vocab_t *p, stl::lm::VocabArgs *a, const void *X, const void *W, const int64_t *label, const int64_t *top_id,
                          const float *top_logit, const float *label_loss, const float *top_loss)
{
    const stl_status_t st = check_vocab(p, a);
    if (st != STL_OK) return st;
    if (any_misaligned(X, W, label, top_id, top_logit, label_loss, top_loss)) return fail(STL_ERR_INVALID_ARG, "%s: a pointer is not 16-byte aligned", fn);
    if (a->rows > 0) {
        if (!X || !W) return fail(STL_ERR_INVALID_ARG, "%s: NULL pointer", fn);
        if (!label && a->ntop == 0) return fail(STL_ERR_INVALID_ARG, "%s: neither labels nor a teacher", fn);
        if (a->ntop > 0 && (!top_id || !top_logit)) return fail(STL_ERR_INVALID_ARG, "%s: ntop=%d without top_id or top_logit", fn, a->ntop);
    }
    if ((label_loss && !label && a->rows > 0) || (top_loss && a->ntop == 0)) return fail(STL_ERR_INVALID_ARG, "%s: the loss of a term that is not there", fn);
    a->X = X, a->W = W, a->label = label;
    if (a->ntop > 0) a->top_id = top_id, a->top_logit = top_logit;
    return STL_OK;
}

}  // namespace

extern "C" {

size_t stl_residual_norm_workspace_bytes(const stl_residual_t *prob, int flags)
{
    stl::lm::ResidualArgs a;
    if (check_residual(prob, flags, &a) != STL_OK) return 0;
    return stl::lm::residual_workspace_bytes(a.rows, a.n, a.per_gate);
}

stl_status_t stl_residual_norm_forward(const stl_residual_t *prob, const void *X, const void *H, const void *gate, const void *w_post,
                                       const void *b_post, const void *w_pre, const void *b_pre, void *Xout, void *Z, int flags, void *stream)
{
    stl::lm::ResidualArgs a;
    stl_status_t st = check_residual(prob, flags, &a);
    if (st != STL_OK) return st;
    if (any_misaligned(X, H, gate, w_post, b_post, w_pre, b_pre, Xout, Z))
        return fail(STL_ERR_INVALID_ARG, "residual_norm_forward: a pointer is not 16-byte aligned");
    if (a.rows == 0) return STL_OK;
    if (!X || !H || !Xout || (a.pre && !Z)) return fail(STL_ERR_INVALID_ARG, "residual_norm_forward: NULL pointer");
    a.X = X, a.H = H, a.gate = gate;
    if (a.post) a.w_post = w_post, a.b_post = b_post;
    if (a.pre) a.w_pre = w_pre, a.b_pre = b_pre;
    LM_HIP(stl::lm::launch_residual_forward(prob->dtype, a, Xout, Z, (hipStream_t)stream), "residual_norm_forward");
    return STL_OK;
}

stl_status_t stl_residual_norm_backward(const stl_residual_t *prob, const void *Xout, const void *H, const void *gate, const void *w_post,
                                        const void *b_post, const void *w_pre, const void *dXout, const void *dZ, void *dX, void *dH, float *dgate,
                                        float *dw_post, float *db_post, float *dw_pre, float *db_pre, int accumulate, void *ws, size_t ws_bytes,
                                        int flags, void *stream)
{
    stl::lm::ResidualArgs a;
    stl_status_t st = check_residual(prob, flags, &a);
    if (st != STL_OK) return st;
    if (any_misaligned(Xout, H, gate, w_post, b_post, w_pre, dXout, dZ, dX, dH, dgate, dw_post, db_post, dw_pre, db_pre))
        return fail(STL_ERR_INVALID_ARG, "residual_norm_backward: a pointer is not 16-byte aligned");
    if (accumulate != 0 && accumulate != 1) return fail(STL_ERR_INVALID_ARG, "residual_norm_backward: accumulate must be 0 or 1");
    if ((dgate && !gate) || ((dw_post || db_post) && !a.post) || ((dw_pre || db_pre) && !a.pre))
        return fail(STL_ERR_INVALID_ARG, "residual_norm_backward: the gradient of a gate or norm that the step does not have");
    hipStream_t s = (hipStream_t)stream;
    if (a.rows == 0) {
        // sums over no rows; there is no row of a gate either
        float *outs[4] = {dw_post, db_post, dw_pre, db_pre};
        for (float *o : outs)
            if (o && !accumulate) LM_HIP(stl::lm::launch_zero_elements(false, o, (size_t)a.n, s), "residual_norm_backward/no rows");
        return STL_OK;
    }
    if ((a.pre && !Xout) || (!H && (a.post || dgate))) return fail(STL_ERR_INVALID_ARG, "residual_norm_backward: NULL pointer");
    st = check_workspace("residual_norm_backward", ws, ws_bytes, stl::lm::residual_workspace_bytes(a.rows, a.n, a.per_gate));
    if (st != STL_OK) return st;
    a.X = Xout, a.H = H, a.gate = gate;
    if (a.post) a.w_post = w_post, a.b_post = b_post;
    if (a.pre) a.w_pre = w_pre;
    const stl::lm::ResidualGrads g{dXout, a.pre ? dZ : nullptr, dX, dH, dgate, dw_post, db_post, dw_pre, db_pre, accumulate};
    LM_HIP(stl::lm::launch_residual_backward(prob->dtype, a, g, ws, s), "residual_norm_backward");
    return STL_OK;
}

size_t stl_vocab_loss_workspace_bytes(const stl_vocab_t *prob, int op)
{
    stl::lm::VocabArgs a;
    if (check_vocab(prob, &a) != STL_OK) return 0;
    if (op != STL_OP_FORWARD && op != STL_OP_BACKWARD) {
        fail(STL_ERR_INVALID_ARG, "vocab_loss_workspace_bytes: op is STL_OP_FORWARD or STL_OP_BACKWARD");
        return 0;
    }
    return stl::lm::vocab_workspace_bytes(a, op == STL_OP_BACKWARD);
}

stl_status_t stl_vocab_loss_forward(const stl_vocab_t *prob, const void *X, const void *W, const int64_t *label, const int64_t *top_id,
                                    const float *top_logit, float *label_loss, float *top_loss, void *ws, size_t ws_bytes, void *stream)
{
    stl::lm::VocabArgs a;
    stl_status_t st = vocab_inputs("vocab_loss_forward", prob, &a, X, W, label, top_id, top_logit, label_loss, top_loss);
    if (st != STL_OK || a.rows == 0) return st;
    if (!label_loss && !top_loss) return fail(STL_ERR_INVALID_ARG, "vocab_loss_forward: no output");
    st = check_workspace("vocab_loss_forward", ws, ws_bytes, stl::lm::vocab_workspace_bytes(a, false));
    if (st != STL_OK) return st;
    LM_HIP(stl::lm::launch_vocab_loss(a, nullptr, label_loss, top_loss, ws, (hipStream_t)stream), "vocab_loss_forward");
    return STL_OK;
}

stl_status_t stl_vocab_loss_backward(const stl_vocab_t *prob, const void *X, const void *W, const int64_t *label, const int64_t *top_id,
                                     const float *top_logit, const float *dlabel, const float *dtop, float *label_loss, float *top_loss, void *dX,
                                     void *dW, void *ws, size_t ws_bytes, void *stream)
{
    stl::lm::VocabArgs a;
    stl_status_t st = vocab_inputs("vocab_loss_backward", prob, &a, X, W, label, top_id, top_logit, label_loss, top_loss);
    if (st != STL_OK) return st;
    if (any_misaligned(dlabel, dtop, dX, dW)) return fail(STL_ERR_INVALID_ARG, "vocab_loss_backward: a pointer is not 16-byte aligned");
    hipStream_t s = (hipStream_t)stream;
    if (a.rows == 0) {
        // a sum over no rows
        if (dW) LM_HIP(stl::lm::launch_zero_elements(a.bf16, dW, (size_t)a.vocab * a.d, s), "vocab_loss_backward/no rows");
        return STL_OK;
    }
    if (!dX && !dW) return fail(STL_ERR_INVALID_ARG, "vocab_loss_backward: neither dX nor dW");
    if (!(dlabel && label) && !(dtop && a.ntop > 0)) return fail(STL_ERR_INVALID_ARG, "vocab_loss_backward: no upstream gradient of a term that is there");
    st = check_workspace("vocab_loss_backward", ws, ws_bytes, stl::lm::vocab_workspace_bytes(a, true));
    if (st != STL_OK) return st;
    const stl::lm::VocabGrads g{dlabel, dtop, dX, dW};
    LM_HIP(stl::lm::launch_vocab_loss(a, &g, label_loss, top_loss, ws, s), "vocab_loss_backward");
    return STL_OK;
}

}  // extern "C"
