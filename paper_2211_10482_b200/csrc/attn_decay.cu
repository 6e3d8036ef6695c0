// st_attn_decay, its gradient and its step: one block per (sequence, head), token after token.
#include "attn_common.cuh"

namespace st {
namespace attn {

// S = [first step: 1 or e^a] S + in_scale y[t] (x) z[t];  out[t] = out_scale x[t].S, forwards or backwards in time
struct FadeArgs {
    Table x, y, z;
    int dx, dz;                       // extent of x and y, extent of z and out
    const float *log_decay;
    const int *offsets;
    int nseq, n, heads;
    const float *init;                // [nseq, heads, dx, dz] or, transposed, [nseq, heads, dz, dx]
    float *last;
    int transposed, backwards, decay_last;   // decay_last: one more factor e^a on `last`
    float in_scale, out_scale;
    bf16 *out;
    unsigned *status;
};

__global__ void fade_kernel(const FadeArgs a)
{
    __shared__ float xs[128], ys[128];
    pdl_wait();
    pdl_trigger();
    const int b = blockIdx.x, h = blockIdx.y, e = threadIdx.x;
    if (a.status && b == 0 && h == 0) {
        const int all = __syncthreads_and(offsets_fine(a.offsets, a.nseq, a.n, threadIdx.x, blockDim.x));
        if (threadIdx.x == 0) {
            a.status[kWsStatusWord] = all ? 0u : (unsigned)ST_ERR_DEV_BOUNDS;
            a.status[kWsDetailWord] = 0u;
        }
    }
    const Rows r = rows_of(a.offsets, b, a.n);
    const float decay = expf(a.log_decay[h]);
    const int64_t base = ((int64_t)b * a.heads + h) * a.dx * a.dz;
    float s[128];
    for (int i = 0; i < 128; ++i) {
        const bool in = a.init && i < a.dx && e < a.dz;
        s[i] = in ? a.init[base + (a.transposed ? (int64_t)e * a.dx + i : (int64_t)i * a.dz + e)] : 0.f;
    }
    for (int j = 0; j < r.len; ++j) {
        const int64_t row = r.first + (a.backwards ? r.len - 1 - j : j);
        __syncthreads();
        if (e < a.dx) {
            xs[e] = __bfloat162float(a.x.p[row * a.x.row + h * a.x.head + e]);
            ys[e] = __bfloat162float(a.y.p[row * a.y.row + h * a.y.head + e]);
        }
        __syncthreads();
        if (e >= a.dz) continue;
        const float z = a.in_scale * __bfloat162float(a.z.p[row * a.z.row + h * a.z.head + e]);
        const float f = a.backwards && j == 0 ? 1.f : decay;
        float o = 0.f;
        for (int i = 0; i < 128; ++i) {
            if (i < a.dx) {
                s[i] = f * s[i] + ys[i] * z;
                o += xs[i] * s[i];
            }
        }
        if (a.out) a.out[(row * a.heads + h) * a.dz + e] = __float2bfloat16(a.out_scale * o);
    }
    if (a.last && e < a.dz)
        for (int i = 0; i < 128; ++i)
            if (i < a.dx) a.last[base + (a.transposed ? (int64_t)e * a.dx + i : (int64_t)i * a.dz + e)] = a.decay_last && r.len ? decay * s[i] : s[i];
}

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

size_t attn_decay_workspace(int64_t n, int64_t nseq, int64_t heads, int64_t d)
{
    if (n <= 0 || nseq <= 0 || heads <= 0 || d <= 0 || d > 128) return 0;
    return kWsHeaderBytes;
}

}  // namespace st

using namespace st;
using namespace st::attn;

static st_status check_decay(const st_tokens *t, const int32_t *offsets)
{
    const st_status rc = check_tokens(t);
    if (rc != ST_OK) return rc;
    if (t->nq != t->nk || t->heads != t->kv_heads) return ST_ERR_SHAPE;
    return !offsets && t->nseq != 1 ? ST_ERR_NULL : ST_OK;
}

static FadeArgs fade_args(const st_tokens *t, const float *log_decay, const int32_t *offsets)
{
    FadeArgs a = {};
    a.log_decay = log_decay;
    a.offsets = offsets;
    a.nseq = (int)t->nseq;
    a.n = (int)t->nq;
    a.heads = (int)t->heads;
    a.in_scale = a.out_scale = 1.f;
    return a;
}

extern "C" {

st_status st_attn_decay(const st_tokens *t, const void *q, const void *k, const void *v, const float *log_decay,
                        const int32_t *offsets, const float *state_in, float scale, void *out, float *state_out,
                        void *ws, size_t ws_bytes, void *stream)
{
    const st_status rc = check_decay(t, offsets);
    if (rc != ST_OK) return rc;
    if (!q || !k || !v || !log_decay || !out) return ST_ERR_NULL;
    for (const void *p : {q, k, v, (const void *)log_decay, (const void *)offsets, (const void *)state_in, (const void *)out, (const void *)state_out})
        if (!aligned16(p)) return ST_ERR_ALIGN;
    if (!ws || ws_bytes < attn_decay_workspace(t->nq, t->nseq, t->heads, t->d > t->dv ? t->d : t->dv)) return ST_ERR_WORKSPACE;
    if (!aligned256(ws)) return ST_ERR_ALIGN;
    FadeArgs a = fade_args(t, log_decay, offsets);
    a.x = {(const bf16 *)q, t->q_row, t->q_head};
    a.y = {(const bf16 *)k, t->k_row, t->k_head};
    a.z = {(const bf16 *)v, t->v_row, t->v_head};
    a.dx = (int)t->d;
    a.dz = (int)t->dv;
    a.init = state_in;
    a.last = state_out;
    a.out_scale = scale;
    a.out = (bf16 *)out;
    a.status = (unsigned *)ws;
    return launch(fade_kernel, dim3(a.nseq, a.heads), 128, 0, (cudaStream_t)stream, a);
}

st_status st_attn_decay_grad(const st_tokens *t, const void *q, const void *k, const void *v, const float *log_decay,
                             const void *dout, const int32_t *offsets, const float *state_in, const float *dstate_out,
                             float scale, void *dq, void *dk, void *dv, float *dstate_in, void *ws, size_t ws_bytes,
                             void *stream)
{
    st_status rc = check_decay(t, offsets);
    if (rc != ST_OK) return rc;
    if (!q || !k || !v || !log_decay || !dout || !dq || !dk || !dv) return ST_ERR_NULL;
    for (const void *p : {q, k, v, (const void *)log_decay, dout, (const void *)offsets, (const void *)state_in, (const void *)dstate_out,
                          (const void *)dq, (const void *)dk, (const void *)dv, (const void *)dstate_in})
        if (!aligned16(p)) return ST_ERR_ALIGN;
    if (!ws || ws_bytes < attn_decay_workspace(t->nq, t->nseq, t->heads, t->d > t->dv ? t->d : t->dv)) return ST_ERR_WORKSPACE;
    if (!aligned256(ws)) return ST_ERR_ALIGN;
    const Table Q = {(const bf16 *)q, t->q_row, t->q_head}, K = {(const bf16 *)k, t->k_row, t->k_head}, V = {(const bf16 *)v, t->v_row, t->v_head},
                O = {(const bf16 *)dout, t->heads * t->dv, t->dv};
    cudaStream_t s = (cudaStream_t)stream;
    // dq[t] = scale sum e^{a(t-s)} (dout[t].v[s]) k[s]
    FadeArgs a = fade_args(t, log_decay, offsets);
    a.x = O; a.y = V; a.z = K;
    a.dx = (int)t->dv;
    a.dz = (int)t->d;
    a.init = state_in;
    a.transposed = 1;
    a.out_scale = scale;
    a.out = (bf16 *)dq;
    a.status = (unsigned *)ws;
    if ((rc = launch(fade_kernel, dim3(a.nseq, a.heads), 128, 0, s, a)) != ST_OK) return rc;
    // dk[s] = sum e^{a(t-s)} (v[s].dout[t]) scale q[t], backwards
    a.x = V; a.y = O; a.z = Q;
    a.init = dstate_out;
    a.backwards = 1;
    a.in_scale = scale;
    a.out_scale = 1.f;
    a.out = (bf16 *)dk;
    a.status = nullptr;
    if ((rc = launch(fade_kernel, dim3(a.nseq, a.heads), 128, 0, s, a)) != ST_OK) return rc;
    // dv[s] = sum e^{a(t-s)} (k[s].q[t]) scale dout[t], backwards
    a.x = K; a.y = Q; a.z = O;
    a.dx = (int)t->d;
    a.dz = (int)t->dv;
    a.transposed = 0;
    a.last = dstate_in;
    a.decay_last = 1;
    a.out = (bf16 *)dv;
    return launch(fade_kernel, dim3(a.nseq, a.heads), 128, 0, s, a);
}

st_status st_attn_decay_step(const st_tokens *t, const void *q, const void *k, const void *v, const float *log_decay,
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

}  // extern "C"
