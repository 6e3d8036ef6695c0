// st_attn_window_step: one warp per (sequence, head), key after key.
#include "attn_common.cuh"

namespace st {
namespace attn {

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

}  // namespace attn
}  // namespace st

using namespace st;
using namespace st::attn;

extern "C" st_status st_attn_window_step(const st_cache *c, const void *q, const void *k, const void *v, void *k_pages,
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
