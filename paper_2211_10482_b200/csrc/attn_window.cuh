// Arguments of the window attention's prompt and gradient.
#pragma once
#include "attn_tc.cuh"

namespace st {
namespace attn {

struct WindowArgs {
    Table q, k, v;
    const int *q_offsets, *k_offsets;
    int nseq, nq, nk, group, d, window, sinks;
    float scale;
    bf16 *out;
    float *lse;
    unsigned *status;
    int heads;
};

inline WindowArgs window_args(const st_tokens *t, const void *q, const void *k, const void *v, const int *qo, const int *ko, int64_t window,
                              int64_t sinks, float scale, void *ws)
{
    WindowArgs a = {};
    a.q = {(const bf16 *)q, stride_of(t->nq, t->q_row), stride_of(t->heads, t->q_head)};
    a.k = {(const bf16 *)k, stride_of(t->nk, t->k_row), stride_of(t->kv_heads, t->k_head)};
    a.v = {(const bf16 *)v, stride_of(t->nk, t->v_row), stride_of(t->kv_heads, t->v_head)};
    a.q_offsets = qo;
    a.k_offsets = ko;
    a.nseq = (int)t->nseq;
    a.nq = (int)t->nq;
    a.nk = (int)t->nk;
    a.heads = (int)t->heads;
    a.group = (int)(t->heads / t->kv_heads);
    a.d = (int)t->d;
    a.window = clamp_int(window);
    a.sinks = clamp_int(sinks);
    a.scale = scale;
    a.status = (unsigned *)ws;
    return a;
}

inline st_status check_window(const st_tokens *t, const int32_t *qo, const int32_t *ko, int64_t window, int64_t sinks, float scale)
{
    const st_status rc = check_tokens(t);
    if (rc != ST_OK) return rc;
    if (t->d != t->dv || window < 1 || sinks < 0) return ST_ERR_SHAPE;
    if (!(scale > 0.f && scale < INFINITY)) return ST_ERR_UNSUPPORTED;
    if (!qo != !ko) return ST_ERR_NULL;
    if (!qo && t->nseq != 1) return ST_ERR_NULL;
    return ST_OK;
}

}  // namespace attn
}  // namespace st
