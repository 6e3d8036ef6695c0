// st_attn_decay_step: one thread per column of a state.
#include "attn_common.cuh"

namespace st {
namespace attn {

__global__ void decay_step_kernel(const bf16 *q, const bf16 *k, const bf16 *v, const float *log_decay, float *state, float scale,
                                  bf16 *out, int heads, int dk, int dv)
{
    pdl_wait();
    pdl_trigger();
    const int64_t bh = (int64_t)blockIdx.y * heads + blockIdx.x;
    const int e = threadIdx.x;
    if (e >= dv) return;
    const float decay = expf(log_decay[blockIdx.x]), z = __bfloat162float(v[bh * dv + e]);
    float o = 0.f;
    for (int i = 0; i < dk; ++i) {
        float &s = state[(bh * dk + i) * dv + e];
        s = decay * s + __bfloat162float(k[bh * dk + i]) * z;
        o += __bfloat162float(q[bh * dk + i]) * s;
    }
    out[bh * dv + e] = __float2bfloat16(scale * o);
}

}  // namespace attn
}  // namespace st

using namespace st;
using namespace st::attn;

extern "C" st_status st_attn_decay_step(const st_tokens *t, const void *q, const void *k, const void *v, const float *log_decay,
                             float *state, float scale, void *out, void *stream)
{
    const st_status rc = check_tokens(t);
    if (rc != ST_OK) return rc;
    if (t->nq != t->nk || t->heads != t->kv_heads || t->nseq != t->nq) return ST_ERR_SHAPE;
    if (!q || !k || !v || !log_decay || !state || !out) return ST_ERR_NULL;
    if (t->nq > 65535) return ST_ERR_UNSUPPORTED;
    for (const void *p : {q, k, v, (const void *)log_decay, (const void *)state, (const void *)out})
        if (!aligned16(p)) return ST_ERR_ALIGN;
    return launch(decay_step_kernel, dim3((unsigned)t->heads, (unsigned)t->nq), 128, 0, (cudaStream_t)stream, (const bf16 *)q, (const bf16 *)k, (const bf16 *)v,
                  log_decay, state, scale, (bf16 *)out, (int)t->heads, (int)t->d, (int)t->dv);
}
