// C ABI of the embedding, the norms and rotation of queries and keys, and attention with decay: argument validation and launch sequencing.
#include "../../include/stl.h"
#include "seq_kernels.h"
#include "../csrc/lm/lm_kernels.h"

#include <cmath>
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

#define SEQ_HIP(call, what)                                                                                                            \
    do {                                                                                                                               \
        const hipError_t e_ = (call);                                                                                                  \
        if (e_ != hipSuccess) return fail(STL_ERR_HIP, "%s: %s", what, hipGetErrorString(e_));                                         \
    } while (0)

template <typename... P>
bool any_misaligned(P... ptrs)
{
    return ((((uintptr_t)ptrs) & 15) || ...);
}
template <typename... P>
bool any_off_element(int dtype, P... ptrs)
{
    return ((((uintptr_t)ptrs) & (dtype == STL_BF16 ? 1 : 3)) || ...);
}

stl_status_t check_workspace(const char *fn, const void *ws, size_t ws_bytes, size_t need)
{
    if (need > 0 && (!ws || ws_bytes < need))
        return fail(STL_ERR_WORKSPACE, "%s: workspace of %zu bytes needed, %zu given", fn, need, ws ? ws_bytes : (size_t)0);
    if (ws && ((uintptr_t)ws & 15)) return fail(STL_ERR_INVALID_ARG, "%s: workspace is not 16-byte aligned", fn);
    return STL_OK;
}

stl_status_t check_dtype(int dtype)
{
    return dtype == STL_F32 || dtype == STL_BF16 ? STL_OK : fail(STL_ERR_UNSUPPORTED, "unknown dtype %d", dtype);
}

stl_status_t check_embed(const stl_embed_t *p, stl::seq::EmbedArgs *a)
{
    if (!p) return fail(STL_ERR_INVALID_ARG, "problem descriptor is NULL");
    if (check_dtype(p->dtype) != STL_OK) return STL_ERR_UNSUPPORTED;
    if (p->rows < 0 || p->d < 1 || p->vocab < 1)
        return fail(STL_ERR_INVALID_ARG, "rows=%lld d=%lld vocab=%lld: rows may be 0, the others are positive", (long long)p->rows, (long long)p->d, (long long)p->vocab);
    if (p->rows > STL_MAX_DIM || p->d > STL_VOCAB_WIDEST || p->vocab > STL_VOCAB_MOST)
        return fail(STL_ERR_INVALID_ARG, "more than %d rows, d=%d or vocab=%d", STL_MAX_DIM, STL_VOCAB_WIDEST, STL_VOCAB_MOST);
    *a = stl::seq::EmbedArgs{(int)p->rows, (int)p->d, (int)p->vocab, p->scale};
    return STL_OK;
}

static_assert(STL_HEAD_WIDEST == stl::seq::kHeadWidest && STL_DECAY_WIDEST == stl::seq::kDecayWidest, "documented widths");
constexpr int kMostHeads = 65536;

stl_status_t check_head(const stl_head_norm_t *p, int flags, stl::seq::HeadArgs *a)
{
    if (!p) return fail(STL_ERR_INVALID_ARG, "problem descriptor is NULL");
    if (check_dtype(p->dtype) != STL_OK) return STL_ERR_UNSUPPORTED;
    if (flags & ~(STL_FLAG_PRE_NORM | STL_FLAG_ADJACENT)) return fail(STL_ERR_UNSUPPORTED, "unknown flag bits 0x%x", flags & ~(STL_FLAG_PRE_NORM | STL_FLAG_ADJACENT));
    if (p->rows < 0 || p->rows > STL_MAX_DIM || p->heads < 1 || p->heads > kMostHeads || p->kv_heads < 0 || p->kv_heads > kMostHeads || p->d < 1)
        return fail(STL_ERR_INVALID_ARG, "rows=%lld heads=%lld kv_heads=%lld d=%lld: up to %d rows, 1 to %d heads, up to as many of keys, d positive", (long long)p->rows,
                    (long long)p->heads, (long long)p->kv_heads, (long long)p->d, STL_MAX_DIM, kMostHeads);
    if (p->d > STL_HEAD_WIDEST) return fail(STL_ERR_UNSUPPORTED, "d=%lld: heads of at most %d elements are supported", (long long)p->d, STL_HEAD_WIDEST);
    if (p->rot < 0 || p->rot > p->d || p->rot % 2) return fail(STL_ERR_INVALID_ARG, "rot=%lld: even, 0 to d", (long long)p->rot);
    if (!(p->base > 0.f) || !(p->eps > 0.f) || std::isinf(p->base)) return fail(STL_ERR_INVALID_ARG, "base and eps must be positive");
    const int64_t wide[2] = {p->heads * p->d, p->kv_heads * p->d}, ld[4] = {p->ld_q, p->ld_k, p->ld_qout, p->ld_kout};
    for (int i = 0; i < 4; ++i)
        if (wide[i & 1] > 0 && (ld[i] < wide[i & 1] || ld[i] > (int64_t)1 << 40))
            return fail(STL_ERR_INVALID_ARG, "%lld elements from row to row, rows have %lld", (long long)ld[i], (long long)wide[i & 1]);
    *a = stl::seq::HeadArgs{};
    a->rows = (int)p->rows, a->heads[0] = (int)p->heads, a->heads[1] = (int)p->kv_heads, a->d = (int)p->d, a->rot = (int)p->rot;
    a->ld_in[0] = (size_t)p->ld_q, a->ld_in[1] = (size_t)p->ld_k, a->ld_out[0] = (size_t)p->ld_qout, a->ld_out[1] = (size_t)p->ld_kout;
    a->eps = p->eps, a->log2_base = std::log2((double)p->base);
    a->norm = flags & STL_FLAG_PRE_NORM, a->adjacent = flags & STL_FLAG_ADJACENT;
    return STL_OK;
}

stl_status_t head_inputs(const char *fn, const stl_head_norm_t *p, const void *Q, const void *K, const void *w_q, const void *w_k, const int64_t *position,
                         stl::seq::HeadArgs *a)
{
    if (any_off_element(p->dtype, Q, K)) return fail(STL_ERR_INVALID_ARG, "%s: a pointer is not aligned to an element", fn);
    if (any_misaligned(w_q, w_k, position)) return fail(STL_ERR_INVALID_ARG, "%s: a pointer is not 16-byte aligned", fn);
    a->in[0] = Q, a->in[1] = K, a->position = position;
    if (!position) a->rot = 0;
    if (a->norm) a->w[0] = w_q, a->w[1] = w_k;
    return STL_OK;
}

stl_status_t check_decay(const stl_decay_attention_t *p, stl::seq::DecayArgs *a)
{
    if (!p) return fail(STL_ERR_INVALID_ARG, "problem descriptor is NULL");
    if (check_dtype(p->dtype) != STL_OK) return STL_ERR_UNSUPPORTED;
    if (p->rows < 0 || p->rows > STL_MAX_DIM || p->sequences < 1 || p->length < 0 || p->length > STL_MAX_DIM)
        return fail(STL_ERR_INVALID_ARG, "rows=%lld sequences=%lld length=%lld: up to %d rows and tokens, at least one sequence", (long long)p->rows,
                    (long long)p->sequences, (long long)p->length, STL_MAX_DIM);
    if (p->heads < 1 || p->kv_heads < 1 || p->heads % p->kv_heads) return fail(STL_ERR_INVALID_ARG, "heads=%lld kv_heads=%lld: kv_heads divides heads",
                                                                               (long long)p->heads, (long long)p->kv_heads);
    if (p->sequences > 4194304 || p->heads > 4194304 / p->sequences) return fail(STL_ERR_INVALID_ARG, "more than 4194304 heads of all sequences");
    if (p->dk < 1 || p->dv < 1) return fail(STL_ERR_INVALID_ARG, "dk=%lld dv=%lld: positive", (long long)p->dk, (long long)p->dv);
    if (p->dk > STL_DECAY_WIDEST || p->dv > STL_DECAY_WIDEST)
        return fail(STL_ERR_UNSUPPORTED, "dk=%lld dv=%lld: heads of at most %d elements are supported", (long long)p->dk, (long long)p->dv, STL_DECAY_WIDEST);
    const int64_t wide[4] = {p->heads * p->dk, p->kv_heads * p->dk, p->kv_heads * p->dv, p->heads * p->dv}, ld[4] = {p->ld_q, p->ld_k, p->ld_v, p->ld_o};
    for (int i = 0; i < 4; ++i)
        if (ld[i] < wide[i] || ld[i] > (int64_t)1 << 40)
            return fail(STL_ERR_INVALID_ARG, "%lld elements from row to row, rows have %lld", (long long)ld[i], (long long)wide[i]);
    if (!std::isfinite(p->scale) || p->scale == 0.f || !std::isfinite(1.f / p->scale)) return fail(STL_ERR_INVALID_ARG, "scale %g: finite and not 0", (double)p->scale);
    *a = stl::seq::DecayArgs{};
    a->rows = (int)p->rows, a->sequences = (int)p->sequences, a->length = (int)p->length, a->heads = (int)p->heads, a->kv_heads = (int)p->kv_heads;
    a->dk = (int)p->dk, a->dv = (int)p->dv;
    a->ld_q = (size_t)p->ld_q, a->ld_k = (size_t)p->ld_k, a->ld_v = (size_t)p->ld_v, a->ld_o = (size_t)p->ld_o;
    a->scale = p->scale;
    return STL_OK;
}

// which rows the tokens have
stl_status_t decay_rows(const char *fn, const stl_decay_attention_t *p, const int64_t *offset, stl::seq::DecayArgs *a)
{
    a->offset = offset;
    if (offset) {
        if (a->length > a->rows) a->length = a->rows;
        return STL_OK;
    }
    if (p->length == 0) return STL_OK;
    // (distances that no two tokens have are not looked at)
    const int64_t seq_step = p->sequences > 1 ? p->seq_step : 0, token_step = p->length > 1 ? p->token_step : 0;
    if (seq_step < 0 || token_step < 0 || seq_step > p->rows || token_step > p->rows)
        return fail(STL_ERR_INVALID_ARG, "%s: seq_step=%lld token_step=%lld with %lld rows", fn, (long long)p->seq_step, (long long)p->token_step, (long long)p->rows);
    const int64_t tokens = (p->length - 1) * token_step, seqs = (p->sequences - 1) * seq_step;
    if (tokens + seqs >= p->rows) return fail(STL_ERR_INVALID_ARG, "%s: the last token lies in row %lld of %lld", fn, (long long)(tokens + seqs), (long long)p->rows);
    const bool one_by_one = (p->sequences == 1 || seq_step > tokens) && (p->length == 1 || token_step > 0);
    const bool side_by_side = (p->length == 1 || token_step > seqs) && (p->sequences == 1 || seq_step > 0);
    if (!one_by_one && !side_by_side) return fail(STL_ERR_INVALID_ARG, "%s: two tokens share a row", fn);
    a->seq_step = (int)seq_step, a->token_step = (int)token_step;
    return STL_OK;
}

stl_status_t decay_inputs(const char *fn, const stl_decay_attention_t *p, const void *Q, const void *K, const void *V, const float *log_decay, const int64_t *offset,
                          const float *state_in, stl::seq::DecayArgs *a)
{
    stl_status_t st = check_decay(p, a);
    if (st != STL_OK) return st;
    if (any_off_element(p->dtype, Q, K, V)) return fail(STL_ERR_INVALID_ARG, "%s: a pointer is not aligned to an element", fn);
    if (any_misaligned(log_decay, offset, state_in)) return fail(STL_ERR_INVALID_ARG, "%s: a pointer is not 16-byte aligned", fn);
    st = decay_rows(fn, p, offset, a);
    if (st != STL_OK) return st;
    if (a->length > 0 && (!Q || !K || !V)) return fail(STL_ERR_INVALID_ARG, "%s: NULL pointer", fn);
    a->Q = Q, a->K = K, a->V = V, a->log_decay = log_decay, a->state = state_in;
    return STL_OK;
}

}  // namespace

extern "C" {

size_t stl_embed_workspace_bytes(const stl_embed_t *prob)
{
    stl::seq::EmbedArgs a;
    return check_embed(prob, &a) == STL_OK ? stl::seq::embed_plan(a).bytes : 0;
}

stl_status_t stl_embed_forward(const stl_embed_t *prob, const int64_t *token, const void *W, void *X, void *stream)
{
    stl::seq::EmbedArgs a;
    const stl_status_t st = check_embed(prob, &a);
    if (st != STL_OK) return st;
    if (any_misaligned(token, W, X)) return fail(STL_ERR_INVALID_ARG, "embed_forward: a pointer is not 16-byte aligned");
    if (a.rows == 0) return STL_OK;
    if (!token || !W || !X) return fail(STL_ERR_INVALID_ARG, "embed_forward: NULL pointer");
    SEQ_HIP(stl::seq::launch_embed_forward(prob->dtype, a, token, W, X, (hipStream_t)stream), "embed_forward");
    return STL_OK;
}

stl_status_t stl_embed_backward(const stl_embed_t *prob, const int64_t *token, const void *dX, void *dW, int accumulate, void *ws, size_t ws_bytes, void *stream)
{
    stl::seq::EmbedArgs a;
    stl_status_t st = check_embed(prob, &a);
    if (st != STL_OK) return st;
    if (any_misaligned(token, dX, dW)) return fail(STL_ERR_INVALID_ARG, "embed_backward: a pointer is not 16-byte aligned");
    if (accumulate != 0 && accumulate != 1) return fail(STL_ERR_INVALID_ARG, "embed_backward: accumulate must be 0 or 1");
    if (!dW) return fail(STL_ERR_INVALID_ARG, "embed_backward: NULL pointer");
    hipStream_t s = (hipStream_t)stream;
    if (a.rows == 0) {
        if (!accumulate) SEQ_HIP(stl::lm::launch_zero_elements(prob->dtype == STL_BF16, dW, (size_t)a.vocab * a.d, s), "embed_backward/no rows");
        return STL_OK;
    }
    if (!token || !dX) return fail(STL_ERR_INVALID_ARG, "embed_backward: NULL pointer");
    st = check_workspace("embed_backward", ws, ws_bytes, stl::seq::embed_plan(a).bytes);
    if (st != STL_OK) return st;
    SEQ_HIP(stl::seq::launch_embed_backward(prob->dtype, a, token, dX, dW, accumulate, ws, s), "embed_backward");
    return STL_OK;
}

size_t stl_head_norm_workspace_bytes(const stl_head_norm_t *prob, int flags)
{
    stl::seq::HeadArgs a;
    if (check_head(prob, flags, &a) != STL_OK) return 0;
    return stl::seq::head_workspace_bytes(a);
}

stl_status_t stl_head_norm_forward(const stl_head_norm_t *prob, const void *Q, const void *K, const void *w_q, const void *w_k, const int64_t *position,
                                   void *Qout, void *Kout, int flags, void *stream)
{
    stl::seq::HeadArgs a;
    stl_status_t st = check_head(prob, flags, &a);
    if (st != STL_OK) return st;
    st = head_inputs("head_norm_forward", prob, Q, K, w_q, w_k, position, &a);
    if (st != STL_OK) return st;
    if (any_off_element(prob->dtype, Qout, Kout)) return fail(STL_ERR_INVALID_ARG, "head_norm_forward: a pointer is not aligned to an element");
    if (a.rows == 0) return STL_OK;
    if (!Q || !Qout || (a.heads[1] && (!K || !Kout))) return fail(STL_ERR_INVALID_ARG, "head_norm_forward: NULL pointer");
    void *const out[2] = {Qout, Kout};
    SEQ_HIP(stl::seq::launch_head_forward(prob->dtype, a, out, (hipStream_t)stream), "head_norm_forward");
    return STL_OK;
}

stl_status_t stl_head_norm_backward(const stl_head_norm_t *prob, const void *Q, const void *K, const void *w_q, const void *w_k, const int64_t *position,
                                    const void *dQout, const void *dKout, void *dQ, void *dK, float *dw_q, float *dw_k, int accumulate, void *ws,
                                    size_t ws_bytes, int flags, void *stream)
{
    stl::seq::HeadArgs a;
    stl_status_t st = check_head(prob, flags, &a);
    if (st != STL_OK) return st;
    st = head_inputs("head_norm_backward", prob, Q, K, w_q, w_k, position, &a);
    if (st != STL_OK) return st;
    if (any_off_element(prob->dtype, dQout, dKout, dQ, dK)) return fail(STL_ERR_INVALID_ARG, "head_norm_backward: a pointer is not aligned to an element");
    if (any_misaligned(dw_q, dw_k)) return fail(STL_ERR_INVALID_ARG, "head_norm_backward: a pointer is not 16-byte aligned");
    if (accumulate != 0 && accumulate != 1) return fail(STL_ERR_INVALID_ARG, "head_norm_backward: accumulate must be 0 or 1");
    if ((dw_q || dw_k) && !a.norm) return fail(STL_ERR_INVALID_ARG, "head_norm_backward: the gradient of a norm that there is not");
    if (a.heads[1] == 0 && (dK || dw_k)) return fail(STL_ERR_INVALID_ARG, "head_norm_backward: the gradient of keys that there are not");
    hipStream_t s = (hipStream_t)stream;
    if (a.rows == 0) {
        float *outs[2] = {dw_q, dw_k};
        for (float *o : outs)
            if (o && !accumulate) SEQ_HIP(stl::lm::launch_zero_elements(false, o, (size_t)a.d, s), "head_norm_backward/no rows");
        return STL_OK;
    }
    if (a.norm && (((dQ || dw_q) && !Q) || ((dK || dw_k) && !K))) return fail(STL_ERR_INVALID_ARG, "head_norm_backward: NULL pointer");
    if (!dQ && !dK && !dw_q && !dw_k) return fail(STL_ERR_INVALID_ARG, "head_norm_backward: no output");
    st = check_workspace("head_norm_backward", ws, ws_bytes, stl::seq::head_workspace_bytes(a));
    if (st != STL_OK) return st;
    const stl::seq::HeadGrads g{{dQout, dKout}, {dQ, dK}, {dw_q, dw_k}, accumulate};
    SEQ_HIP(stl::seq::launch_head_backward(prob->dtype, a, g, ws, s), "head_norm_backward");
    return STL_OK;
}

size_t stl_decay_attention_workspace_bytes(const stl_decay_attention_t *prob, int op)
{
    stl::seq::DecayArgs a;
    if (check_decay(prob, &a) != STL_OK) return 0;
    if (op != STL_OP_FORWARD && op != STL_OP_BACKWARD) {
        fail(STL_ERR_INVALID_ARG, "decay_attention_workspace_bytes: op is STL_OP_FORWARD or STL_OP_BACKWARD");
        return 0;
    }
    return stl::seq::decay_workspace_bytes(prob->dtype, a, op == STL_OP_BACKWARD);
}

stl_status_t stl_decay_attention_forward(const stl_decay_attention_t *prob, const void *Q, const void *K, const void *V, const float *log_decay,
                                         const int64_t *offset, const float *state_in, void *O, float *state_out, void *ws, size_t ws_bytes, void *stream)
{
    stl::seq::DecayArgs a;
    stl_status_t st = decay_inputs("decay_attention_forward", prob, Q, K, V, log_decay, offset, state_in, &a);
    if (st != STL_OK) return st;
    if (any_off_element(prob->dtype, O)) return fail(STL_ERR_INVALID_ARG, "decay_attention_forward: a pointer is not aligned to an element");
    if (any_misaligned(state_out)) return fail(STL_ERR_INVALID_ARG, "decay_attention_forward: a pointer is not 16-byte aligned");
    if (!O && a.length > 0) return fail(STL_ERR_INVALID_ARG, "decay_attention_forward: NULL pointer");
    if (a.length == 0 && !state_out) return STL_OK;
    st = check_workspace("decay_attention_forward", ws, ws_bytes, stl::seq::decay_workspace_bytes(prob->dtype, a, false));
    if (st != STL_OK) return st;
    SEQ_HIP(stl::seq::launch_decay_forward(prob->dtype, a, O, state_out, ws, (hipStream_t)stream), "decay_attention_forward");
    return STL_OK;
}

stl_status_t stl_decay_attention_backward(const stl_decay_attention_t *prob, const void *Q, const void *K, const void *V, const float *log_decay,
                                          const int64_t *offset, const float *state_in, const void *dO, const float *dstate_out, void *dQ, void *dK, void *dV,
                                          float *dstate_in, void *ws, size_t ws_bytes, void *stream)
{
    stl::seq::DecayArgs a;
    stl_status_t st = decay_inputs("decay_attention_backward", prob, Q, K, V, log_decay, offset, state_in, &a);
    if (st != STL_OK) return st;
    if (any_off_element(prob->dtype, dO, dQ, dK, dV)) return fail(STL_ERR_INVALID_ARG, "decay_attention_backward: a pointer is not aligned to an element");
    if (any_misaligned(dstate_out, dstate_in)) return fail(STL_ERR_INVALID_ARG, "decay_attention_backward: a pointer is not 16-byte aligned");
    if (!dO && a.length > 0) return fail(STL_ERR_INVALID_ARG, "decay_attention_backward: NULL pointer");
    if (!dQ && !dK && !dV && !dstate_in) return fail(STL_ERR_INVALID_ARG, "decay_attention_backward: no output");
    if (dstate_in && (dstate_in == dstate_out || dstate_in == state_in)) return fail(STL_ERR_INVALID_ARG, "decay_attention_backward: an output is an input");
    if (a.length == 0 && !dstate_in) return STL_OK;
    st = check_workspace("decay_attention_backward", ws, ws_bytes, stl::seq::decay_workspace_bytes(prob->dtype, a, true));
    if (st != STL_OK) return st;
    const stl::seq::DecayGrads g{dO, dstate_out, dQ, dK, dV, dstate_in};
    SEQ_HIP(stl::seq::launch_decay_backward(prob->dtype, a, g, ws, (hipStream_t)stream), "decay_attention_backward");
    return STL_OK;
}

}  // extern "C"
