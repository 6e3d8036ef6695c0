// A cache in cells: where a token's row lies, and what its cells stand for.
#pragma once
#include "attn_common.cuh"

namespace st {
namespace attn {

constexpr int GROUP = 32;                  // columns of ST_I4 that share a step and a lowest value
constexpr float FEWEST_SCALE = 7.888609052210118e-31f;     // 2^-100: below it a scale is 0, so that neither it nor its reciprocal leaves fp32's normal numbers

struct Cells {
    unsigned char *k, *v;
    uint32_t *k_scales, *v_scales;
    const int *table, *lens;
    int64_t page_stride, token_stride, head_stride, scale_page, scale_token, scale_head;
    int nseq, kv_heads, d, pages, page, cols;
    unsigned page_magic;                   // floor((2^32 - 1) / page): __umulhi with it is s / page or one less, s below 2^31
};

inline int64_t row_bytes(int dtype, int64_t d) { return dtype == ST_BF16 ? 2 * d : dtype == ST_I8 ? d : d / 2; }
inline int64_t row_scales(int dtype, int64_t d) { return dtype == ST_BF16 ? 0 : dtype == ST_I8 ? 1 : (d + GROUP - 1) / GROUP; }

// How far behind the first row the last one begins, each in the units of the strides.
constexpr __int128 MOST_BYTES = (__int128)1 << 61;
inline __int128 cells_extent(int64_t pages, int64_t page_stride, int64_t page, int64_t token_stride, int64_t heads, int64_t head_stride)
{
    return (__int128)(pages - 1) * page_stride + (__int128)(page - 1) * token_stride + (__int128)(heads - 1) * head_stride;
}

inline st_status check_cells(const st_cells *c, const void *k_pages, const void *v_pages, const void *k_scales, const void *v_scales, const void *table,
                             const void *lens)
{
    if (!c) return ST_ERR_NULL;
    if (c->dtype != ST_BF16 && c->dtype != ST_I8 && c->dtype != ST_I4) return ST_ERR_DTYPE;
    if (c->reserved != 0 || c->nseq <= 0 || c->heads <= 0 || c->kv_heads <= 0 || c->d <= 0 || c->pages <= 0 || c->page <= 0 || c->table_cols <= 0 || c->heads % c->kv_heads != 0)
        return ST_ERR_SHAPE;
    if (c->nseq > (1 << 20) || c->heads > 65535 || c->d % (c->dtype == ST_I4 ? 16 : 8) != 0 || c->d > 128 || c->pages > (1 << 30) || c->page > (1 << 30) ||
        c->table_cols > (1 << 30) || c->page * c->table_cols > (1 << 30))          // tokens of a sequence
        return ST_ERR_UNSUPPORTED;
    const int64_t bytes = row_bytes(c->dtype, c->d), scales = row_scales(c->dtype, c->d), unit = c->dtype == ST_BF16 ? 16 : 8;
    if (!stride_ok(c->pages, c->page_stride, bytes) || !stride_ok(c->page, c->token_stride, bytes) || !stride_ok(c->kv_heads, c->head_stride, bytes)) return ST_ERR_SHAPE;
    if (scales && (!stride_ok(c->pages, c->scale_page, scales) || !stride_ok(c->page, c->scale_token, scales) || !stride_ok(c->kv_heads, c->scale_head, scales))) return ST_ERR_SHAPE;
    for (const int64_t s : {c->page_stride, c->token_stride, c->head_stride, c->scale_page, c->scale_token, c->scale_head})
        if (s > ((int64_t)1 << 38)) return ST_ERR_UNSUPPORTED;         // half of what a tensor map's stride may be
    if (cells_extent(c->pages, c->page_stride, c->page, c->token_stride, c->kv_heads, c->head_stride) > MOST_BYTES ||
        (scales && 4 * cells_extent(c->pages, c->scale_page, c->page, c->scale_token, c->kv_heads, c->scale_head) > MOST_BYTES))
        return ST_ERR_UNSUPPORTED;
    if ((c->pages > 1 && c->page_stride % unit != 0) || (c->page > 1 && c->token_stride % unit != 0) || (c->kv_heads > 1 && c->head_stride % unit != 0)) return ST_ERR_ALIGN;
    if (!k_pages || !v_pages || !table || !lens || (scales && (!k_scales || !v_scales))) return ST_ERR_NULL;
    if (!scales && (k_scales || v_scales)) return ST_ERR_SHAPE;
    for (const void *p : {k_pages, v_pages, k_scales, v_scales})
        if (!aligned16(p)) return ST_ERR_ALIGN;
    return aligned4(table) && aligned4(lens) ? ST_OK : ST_ERR_ALIGN;
}

inline Cells cells_of(const st_cells *c, const void *k_pages, const void *v_pages, const void *k_scales, const void *v_scales, const int32_t *table, const int32_t *lens)
{
    Cells r = {};
    r.k = (unsigned char *)k_pages;
    r.v = (unsigned char *)v_pages;
    r.k_scales = (uint32_t *)k_scales;
    r.v_scales = (uint32_t *)v_scales;
    r.table = table;
    r.lens = lens;
    // the stride of an extent of one is never used
    r.page_stride = c->pages == 1 ? 0 : c->page_stride;
    r.token_stride = c->page == 1 ? 0 : c->token_stride;
    r.head_stride = c->kv_heads == 1 ? 0 : c->head_stride;
    r.scale_page = c->pages == 1 ? 0 : c->scale_page;
    r.scale_token = c->page == 1 ? 0 : c->scale_token;
    r.scale_head = c->kv_heads == 1 ? 0 : c->scale_head;
    r.nseq = (int)c->nseq;
    r.kv_heads = (int)c->kv_heads;
    r.d = (int)c->d;
    r.pages = (int)c->pages;
    r.page = (int)c->page;
    r.cols = (int)c->table_cols;
    r.page_magic = 0xFFFFFFFFu / (unsigned)c->page;
    return r;
}

// The bytes between a cache's first and last: a result within them may lie over a row.  Pages of keys and of values may interleave.
inline bool meets_cells(const st_cells *c, const void *pages, const void *scales, const void *p, int64_t bytes)
{
    const Cells r = cells_of(c, pages, pages, scales, scales, nullptr, nullptr);
    const int64_t n = (c->pages - 1) * r.page_stride + (c->page - 1) * r.token_stride + (c->kv_heads - 1) * r.head_stride + row_bytes(c->dtype, c->d);
    const int64_t m = 4 * ((c->pages - 1) * r.scale_page + (c->page - 1) * r.scale_token + (c->kv_heads - 1) * r.scale_head + row_scales(c->dtype, c->d));
    return arrays_meet(pages, n, p, bytes) || (scales && arrays_meet(scales, m, p, bytes));
}

#if defined(__CUDACC__)

// Tokens of a sequence, as far as its row of a table goes.
__device__ __forceinline__ int length_of(int told, int cols, int page) { return (int)min((int64_t)max(told, 0), (int64_t)cols * page); }

// Place s of a sequence: page `col` of its row of the table, token `slot` of the page.
struct Place {
    int col, slot;
};
__device__ __forceinline__ Place place_of(int s, int page, unsigned magic)
{
    const int p = (int)__umulhi((unsigned)s, magic), q = s - p * page >= page ? p + 1 : p;
    return {q, s - q * page};
}

#endif

}  // namespace attn
}  // namespace st
