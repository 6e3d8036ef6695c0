// st_attn_window: one warp per (query, head), the formula as it stands.
#include "attn_common.cuh"

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

__global__ void window_kernel(const WindowArgs a)
{
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
    const bf16 *q = a.q.p + row * a.q.row + h * a.q.head;
    float most = -INFINITY, sum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 <= t; s0 += 32) {
        if (s0 + 31 <= t - a.window && s0 >= a.sinks) continue;
        const int s = s0 + lane;
        const bool seen = s <= t && (s > t - a.window || s < a.sinks);
        float x = -INFINITY;
        if (seen) x = a.scale * dot(q, a.k.p + (rk.first + s) * a.k.row + (h / a.group) * a.k.head, a.d);
        float m = x;
        for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, o));
        m = fmaxf(m, most);
        if (m == -INFINITY) continue;
        const float old = expf(most - m), p = expf(x - m);
        float ps = p;
        for (int o = 16; o; o >>= 1) ps += __shfl_xor_sync(~0u, ps, o);
        sum = sum * old + ps;
        most = m;
        for (int c = 0; c < 4; ++c) acc[c] *= old;
        for (int j = 0; j < 32; ++j) {
            const float pj = __shfl_sync(~0u, p, j);
            if (pj == 0.f) continue;
            const bf16 *v = a.v.p + (rk.first + s0 + j) * a.v.row + (h / a.group) * a.v.head;
            for (int c = 0; c < 4; ++c)
                if (lane + 32 * c < a.d) acc[c] += pj * __bfloat162float(v[lane + 32 * c]);
        }
    }
    const float inv = sum > 0.f ? 1.f / sum : 0.f;
    for (int c = 0; c < 4; ++c)
        if (lane + 32 * c < a.d) a.out[((int64_t)row * a.heads + h) * a.d + lane + 32 * c] = __float2bfloat16(acc[c] * inv);
    if (lane == 0) a.lse[(int64_t)row * a.heads + h] = sum > 0.f ? most + logf(sum) : -INFINITY;
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

struct StepArgs {
    const bf16 *q, *k, *v;
    bf16 *k_pages, *v_pages;
    const int *table, *lens;
    int nseq, heads, group, d, pages, page, cols, window, sinks;
    int64_t page_stride, token_stride, head_stride;
    float scale;
    bf16 *out;
    unsigned *status;
};

__global__ void window_step_kernel(const StepArgs a)
{
    pdl_wait();
    pdl_trigger();
    const int h = blockIdx.x, b = blockIdx.y, lane = threadIdx.x, hk = h / a.group, hkn = a.heads / a.group;
    if (h == 0 && b == 0) {
        bool fine = true;
        for (int i = 0; i < a.nseq; ++i) {
            const int n = a.lens[i];
            fine = fine && n >= 0 && (int64_t)n <= (int64_t)a.cols * a.page;
            for (int c = lane; c < min(a.cols, (n + a.page - 1) / a.page); c += 32) fine = fine && (unsigned)a.table[(int64_t)i * a.cols + c] < (unsigned)a.pages;
        }
        fine = __all_sync(~0u, fine);
        if (lane == 0) {
            a.status[kWsStatusWord] = fine ? 0u : (unsigned)ST_ERR_DEV_BOUNDS;
            a.status[kWsDetailWord] = 0u;
        }
    }
    const int len = (int)min((int64_t)max(a.lens[b], 0), (int64_t)a.cols * a.page), t = len - 1;
    const bf16 *q = a.q + ((int64_t)b * a.heads + h) * a.d;
    const bf16 *kn = a.k + ((int64_t)b * hkn + hk) * a.d, *vn = a.v + ((int64_t)b * hkn + hk) * a.d;
    float most = -INFINITY, sum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s <= t; ++s) {
        if (!(s > t - a.window || s < a.sinks)) continue;
        const int p = a.table[(int64_t)b * a.cols + s / a.page];
        if ((unsigned)p >= (unsigned)a.pages) continue;
        const int64_t at = p * a.page_stride + (s % a.page) * a.token_stride + hk * a.head_stride;
        const bf16 *k = s == t ? kn : a.k_pages + at, *v = s == t ? vn : a.v_pages + at;
        if (s == t && h % a.group == 0)
            for (int c = lane; c < a.d; c += 32) {
                a.k_pages[at + c] = kn[c];
                a.v_pages[at + c] = vn[c];
            }
        float x = 0.f;
        for (int c = lane; c < a.d; c += 32) x += __bfloat162float(q[c]) * __bfloat162float(k[c]);
        for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
        x *= a.scale;
        const float m = fmaxf(most, x), old = expf(most - m), w = expf(x - m);
        sum = sum * old + w;
        most = m;
        for (int c = 0; c < 4; ++c)
            if (lane + 32 * c < a.d) acc[c] = acc[c] * old + w * __bfloat162float(v[lane + 32 * c]);
    }
    for (int c = 0; c < 4; ++c)
        if (lane + 32 * c < a.d) a.out[((int64_t)b * a.heads + h) * a.d + lane + 32 * c] = __float2bfloat16(sum > 0.f ? acc[c] / sum : 0.f);
}

static WindowArgs window_args(const st_tokens *t, const void *q, const void *k, const void *v, const int *qo, const int *ko, int64_t window,
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

}  // namespace attn

size_t attn_window_grad_workspace(int64_t nq, int64_t heads)
{
    if (nq <= 0 || heads <= 0 || nq > (1 << 30) || heads > 65535) return 0;
    return kWsHeaderBytes + (size_t)nq * heads * sizeof(float);
}

}  // namespace st

using namespace st;
using namespace st::attn;

static st_status check_window(const st_tokens *t, const int32_t *qo, const int32_t *ko, int64_t window, int64_t sinks, float scale)
{
    const st_status rc = check_tokens(t);
    if (rc != ST_OK) return rc;
    if (t->d != t->dv || window < 1 || sinks < 0) return ST_ERR_SHAPE;
    if (!(scale > 0.f && scale < INFINITY)) return ST_ERR_UNSUPPORTED;
    if (!qo != !ko) return ST_ERR_NULL;
    if (!qo && t->nseq != 1) return ST_ERR_NULL;
    return ST_OK;
}

extern "C" {

st_status st_attn_window(const st_tokens *tokens, const void *q, const void *k, const void *v, const int32_t *q_offsets,
                         const int32_t *k_offsets, int64_t window, int64_t sinks, float scale, void *out, float *lse,
                         void *ws, size_t ws_bytes, void *stream)
{
    st_status rc = check_window(tokens, q_offsets, k_offsets, window, sinks, scale);
    if (rc != ST_OK) return rc;
    if (!q || !k || !v || !out || !lse) return ST_ERR_NULL;
    for (const void *p : {q, k, v, (const void *)out, (const void *)lse, (const void *)q_offsets, (const void *)k_offsets})
        if (!aligned16(p)) return ST_ERR_ALIGN;
    if (!ws || ws_bytes < kWsHeaderBytes) return ST_ERR_WORKSPACE;
    if (!aligned256(ws)) return ST_ERR_ALIGN;
    WindowArgs a = window_args(tokens, q, k, v, q_offsets, k_offsets, window, sinks, scale, ws);
    a.out = (bf16 *)out;
    a.lse = lse;
    return launch(window_kernel, dim3((a.nq + 3) / 4, a.heads), 128, 0, (cudaStream_t)stream, a);
}

st_status st_attn_window_grad(const st_tokens *tokens, const void *q, const void *k, const void *v, const void *out,
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

st_status st_attn_window_step(const st_cache *c, const void *q, const void *k, const void *v, void *k_pages,
                              void *v_pages, const int32_t *table, const int32_t *lens, int64_t window, int64_t sinks,
                              float scale, void *out, void *ws, size_t ws_bytes, void *stream)
{
    if (!c) return ST_ERR_NULL;
    if (c->dtype != ST_BF16) return ST_ERR_DTYPE;
    if (c->reserved != 0 || c->nseq <= 0 || c->heads <= 0 || c->kv_heads <= 0 || c->d <= 0 || c->pages <= 0 || c->page <= 0 || c->table_cols <= 0 ||
        c->heads % c->kv_heads != 0 || window < 1 || sinks < 0)
        return ST_ERR_SHAPE;
    if (c->nseq > 65535 || c->heads > 65535 || c->d % 8 != 0 || c->d > 128 || c->pages > (1 << 30) || c->page > (1 << 30) || c->table_cols > (1 << 30))
        return ST_ERR_UNSUPPORTED;
    if (!stride_ok(c->pages, c->page_stride, c->d) || !stride_ok(c->page, c->token_stride, c->d) || !stride_ok(c->kv_heads, c->head_stride, c->d))
        return ST_ERR_SHAPE;
    if ((c->pages > 1 && c->page_stride % 8 != 0) || (c->page > 1 && c->token_stride % 8 != 0) || (c->kv_heads > 1 && c->head_stride % 8 != 0))
        return ST_ERR_ALIGN;
    if (!(scale > 0.f && scale < INFINITY)) return ST_ERR_UNSUPPORTED;
    if (!q || !k || !v || !k_pages || !v_pages || !table || !lens || !out) return ST_ERR_NULL;
    for (const void *p : {q, k, v, (const void *)k_pages, (const void *)v_pages, (const void *)table, (const void *)lens, (const void *)out})
        if (!aligned16(p)) return ST_ERR_ALIGN;
    if (!ws || ws_bytes < kWsHeaderBytes) return ST_ERR_WORKSPACE;
    if (!aligned256(ws)) return ST_ERR_ALIGN;
    StepArgs a = {};
    a.q = (const bf16 *)q;
    a.k = (const bf16 *)k;
    a.v = (const bf16 *)v;
    a.k_pages = (bf16 *)k_pages;
    a.v_pages = (bf16 *)v_pages;
    a.table = table;
    a.lens = lens;
    a.nseq = (int)c->nseq;
    a.heads = (int)c->heads;
    a.group = (int)(c->heads / c->kv_heads);
    a.d = (int)c->d;
    a.pages = (int)c->pages;
    a.page = (int)c->page;
    a.cols = (int)c->table_cols;
    a.window = clamp_int(window);
    a.sinks = clamp_int(sinks);
    a.page_stride = stride_of(c->pages, c->page_stride);
    a.token_stride = stride_of(c->page, c->token_stride);
    a.head_stride = stride_of(c->kv_heads, c->head_stride);
    a.scale = scale;
    a.out = (bf16 *)out;
    a.status = (unsigned *)ws;
    return launch(window_step_kernel, dim3(a.heads, a.nseq), 32, 0, (cudaStream_t)stream, a);
}

}  // extern "C"
