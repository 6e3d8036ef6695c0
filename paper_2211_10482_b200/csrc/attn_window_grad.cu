// st_attn_window_grad: one warp per (query, head) for dq and per (key, key head) for dk and dv, the formulas as they stand.
#include "attn_window.cuh"

namespace st {
namespace attn {

__device__ __forceinline__ int sequence_of(const int *offsets, int nseq, int row, int n)
{
    if (!offsets) return row < n ? 0 : -1;
    for (int b = 0; b < nseq; ++b) {
        const Rows r = rows_of(offsets, b, n);
        if (row >= r.first && row < r.first + r.len) return b;
    }
    return -1;
}

__device__ __forceinline__ float dot(const bf16 *a, const bf16 *b, int d)
{
    float s = 0.f;
    for (int i = 0; i < d; ++i) s += __bfloat162float(a[i]) * __bfloat162float(b[i]);
    return s;
}

struct WindowGradArgs {
    WindowArgs w;
    const bf16 *o, *dout;
    bf16 *dq, *dk, *dv;
};

// dq: one warp per (query, head)
__global__ void window_dq_kernel(const WindowGradArgs g)
{
    const WindowArgs &a = g.w;
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0 && blockIdx.y == 0) {
        const bool fine = offsets_fine(a.q_offsets, a.nseq, a.nq, threadIdx.x, blockDim.x) && offsets_fine(a.k_offsets, a.nseq, a.nk, threadIdx.x, blockDim.x);
        const int all = __syncthreads_and(fine);
        if (threadIdx.x == 0) {
            a.status[kWsStatusWord] = all ? 0u : (unsigned)ST_ERR_DEV_BOUNDS;
            a.status[kWsDetailWord] = 0u;
        }
    }
    const int row = blockIdx.x * 4 + threadIdx.x / 32, lane = threadIdx.x & 31, h = blockIdx.y;
    if (row >= a.nq) return;
    const int b = sequence_of(a.q_offsets, a.nseq, row, a.nq);
    if (b < 0) return;
    const Rows rq = rows_of(a.q_offsets, b, a.nq), rk = rows_of(a.k_offsets, b, a.nk);
    const int t = row - rq.first + rk.len - rq.len;
    const int64_t at = ((int64_t)row * a.heads + h) * a.d;
    const bf16 *q = a.q.p + row * a.q.row + h * a.q.head;
    const float delta = dot(g.o + at, g.dout + at, a.d), lse = a.lse[(int64_t)row * a.heads + h];
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s <= t; ++s) {
        if (!(s > t - a.window || s < a.sinks)) continue;
        const bf16 *k = a.k.p + (rk.first + s) * a.k.row + (h / a.group) * a.k.head, *v = a.v.p + (rk.first + s) * a.v.row + (h / a.group) * a.v.head;
        float x = 0.f, dp = 0.f;
        for (int i = lane; i < a.d; i += 32) {
            x += __bfloat162float(q[i]) * __bfloat162float(k[i]);
            dp += __bfloat162float(g.dout[at + i]) * __bfloat162float(v[i]);
        }
        for (int o = 16; o; o >>= 1) {
            x += __shfl_xor_sync(~0u, x, o);
            dp += __shfl_xor_sync(~0u, dp, o);
        }
        const float ds = expf(a.scale * x - lse) * (dp - delta) * a.scale;
        for (int c = 0; c < 4; ++c)
            if (lane + 32 * c < a.d) acc[c] += ds * __bfloat162float(k[lane + 32 * c]);
    }
    for (int c = 0; c < 4; ++c)
        if (lane + 32 * c < a.d) g.dq[at + lane + 32 * c] = __float2bfloat16(acc[c]);
}

// dk, dv: one warp per (key, key head)
__global__ void window_dkv_kernel(const WindowGradArgs g)
{
    const WindowArgs &a = g.w;
    pdl_wait();
    pdl_trigger();
    const int row = blockIdx.x * 4 + threadIdx.x / 32, lane = threadIdx.x & 31, hk = blockIdx.y;
    if (row >= a.nk) return;
    const int b = sequence_of(a.k_offsets, a.nseq, row, a.nk);
    if (b < 0) return;
    const Rows rq = rows_of(a.q_offsets, b, a.nq), rk = rows_of(a.k_offsets, b, a.nk);
    const int s = row - rk.first;
    const bf16 *k = a.k.p + row * a.k.row + hk * a.k.head, *v = a.v.p + row * a.v.row + hk * a.v.head;
    float dk[4] = {0.f, 0.f, 0.f, 0.f}, dv[4] = {0.f, 0.f, 0.f, 0.f};
    for (int i = 0; i < rq.len; ++i) {
        const int t = i + rk.len - rq.len;
        if (!(s <= t && (s > t - a.window || s < a.sinks))) continue;
        for (int h = hk * a.group; h < (hk + 1) * a.group; ++h) {
            const int qr = rq.first + i;
            const int64_t at = ((int64_t)qr * a.heads + h) * a.d;
            const bf16 *q = a.q.p + qr * a.q.row + h * a.q.head;
            float x = 0.f, dp = 0.f, delta = 0.f;
            for (int c = lane; c < a.d; c += 32) {
                x += __bfloat162float(q[c]) * __bfloat162float(k[c]);
                dp += __bfloat162float(g.dout[at + c]) * __bfloat162float(v[c]);
                delta += __bfloat162float(g.dout[at + c]) * __bfloat162float(g.o[at + c]);
            }
            for (int o = 16; o; o >>= 1) {
                x += __shfl_xor_sync(~0u, x, o);
                dp += __shfl_xor_sync(~0u, dp, o);
                delta += __shfl_xor_sync(~0u, delta, o);
            }
            const float p = expf(a.scale * x - a.lse[(int64_t)qr * a.heads + h]), ds = p * (dp - delta) * a.scale;
            for (int c = 0; c < 4; ++c)
                if (lane + 32 * c < a.d) {
                    dk[c] += ds * __bfloat162float(q[lane + 32 * c]);
                    dv[c] += p * __bfloat162float(g.dout[at + lane + 32 * c]);
                }
        }
    }
    const int64_t at = ((int64_t)row * (a.heads / a.group) + hk) * a.d;
    for (int c = 0; c < 4; ++c)
        if (lane + 32 * c < a.d) {
            g.dk[at + lane + 32 * c] = __float2bfloat16(dk[c]);
            g.dv[at + lane + 32 * c] = __float2bfloat16(dv[c]);
        }
}

}  // namespace attn

size_t attn_window_grad_workspace(int64_t nq, int64_t heads)
{
    if (nq <= 0 || heads <= 0 || nq > (1 << 30) || heads > 65535) return 0;
    return kWsHeaderBytes + (size_t)nq * heads * sizeof(float);
}

}  // namespace st

using namespace st;
using namespace st::attn;

extern "C" st_status st_attn_window_grad(const st_tokens *tokens, const void *q, const void *k, const void *v, const void *out,
                              const float *lse, const void *dout, const int32_t *q_offsets, const int32_t *k_offsets,
                              int64_t window, int64_t sinks, float scale, void *dq, void *dk, void *dv, void *ws,
                              size_t ws_bytes, void *stream)
{
    st_status rc = check_window(tokens, q_offsets, k_offsets, window, sinks, scale);
    if (rc != ST_OK) return rc;
    if (!q || !k || !v || !out || !lse || !dout || !dq || !dk || !dv) return ST_ERR_NULL;
    for (const void *p : {q, k, v, out, (const void *)lse, dout, (const void *)dq, (const void *)dk, (const void *)dv, (const void *)q_offsets, (const void *)k_offsets})
        if (!aligned16(p)) return ST_ERR_ALIGN;
    if (!ws || ws_bytes < attn_window_grad_workspace(tokens->nq, tokens->heads)) return ST_ERR_WORKSPACE;
    if (!aligned256(ws)) return ST_ERR_ALIGN;
    WindowGradArgs g = {};
    g.w = window_args(tokens, q, k, v, q_offsets, k_offsets, window, sinks, scale, ws);
    g.w.lse = const_cast<float *>(lse);
    g.o = (const bf16 *)out;
    g.dout = (const bf16 *)dout;
    g.dq = (bf16 *)dq;
    g.dk = (bf16 *)dk;
    g.dv = (bf16 *)dv;
    rc = launch(window_dq_kernel, dim3((g.w.nq + 3) / 4, g.w.heads), 128, 0, (cudaStream_t)stream, g);
    if (rc != ST_OK) return rc;
    return launch(window_dkv_kernel, dim3((g.w.nk + 3) / 4, g.w.heads / g.w.group), 128, 0, (cudaStream_t)stream, g);
}
