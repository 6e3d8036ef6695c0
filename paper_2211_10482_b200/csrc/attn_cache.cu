// st_attn_cache_write and st_attn_cache_read: rows of keys and values into the pages of a cache and back, as they are or quantised.
//
// Bound by memory: a row is read once and written once.  16 lanes own a row, 8 of its columns each.  A block has T tokens and C of their 2 kv_heads
// rows; first each group of 16 lanes finds a token's place (which sequence: a search in the offsets, 16 at a time; then its length, its page), while
// the rows to be written are on their way.
#include "attn_cells.cuh"

namespace st {
namespace attn {

struct CacheArgs {
    Cells c;
    const bf16 *k, *v;                     // write: rows with strides
    int64_t k_row, k_head, v_row, v_head;
    bf16 *k_out, *v_out;                   // read: contiguous rows
    const int *offsets;
    unsigned *status;
    int n, tokens, cols, col_tiles;        // of a tile
};

namespace cells {
constexpr int THREADS = 256, LANES = 16, GROUPS = THREADS / LANES, ROWS = 4;
}

// The sequence whose rows `row` is among (the last one that begins at or before it); by 16 lanes, all 32 of a warp at once.
__device__ __forceinline__ int sequence_of(const int *offsets, int nseq, int row)
{
    const int lane = threadIdx.x & 15, shift = threadIdx.x & 16;
    int lo = 0;
    for (int span = nseq, step; span > 1; span = step) {
        step = (span + 15) / 16;
        const int at = lo + (lane + 1) * step;
        const bool before = lane < 15 && at < min(lo + span, nseq) && offsets[at] <= row;
        lo += __popc(__ballot_sync(~0u, before) >> shift & 0xFFFFu) * step;
    }
    return lo;
}

// Where a token's rows lie: cells in bytes, scales in units of 4 bytes; cells < 0: nowhere (NO_ROW: it is a row of no sequence).
constexpr int64_t NOWHERE = -1, NO_ROW = -2;
struct Spot {
    int64_t cells, scales;
};
__device__ __forceinline__ Spot spot_of(const CacheArgs &a, int row, bool there)
{
    const Cells &c = a.c;
    int b, first = 0, last = a.n;
    if (!a.offsets) {
        b = c.nseq == 1 ? 0 : row;
        if (c.nseq > 1) first = row, last = row + 1;
    } else {
        b = sequence_of(a.offsets, c.nseq, row);
        const Rows r = rows_of(a.offsets, b, a.n);
        first = r.first;
        last = r.first + r.len;
    }
    if (!there || row < first || row >= last) return {NO_ROW, 0};
    const int64_t at = (int64_t)c.lens[b] - (last - row);
    if (at < 0 || at >= (int64_t)c.cols * c.page) {
        a.status[kWsStatusWord] = (unsigned)ST_ERR_DEV_BOUNDS;
        return {NOWHERE, 0};
    }
    const Place p = place_of((int)at, c.page, c.page_magic);
    const int page = c.table[(int64_t)b * c.cols + p.col];
    if ((unsigned)page >= (unsigned)c.pages) {
        a.status[kWsStatusWord] = (unsigned)ST_ERR_DEV_BOUNDS;
        return {NOWHERE, 0};
    }
    return {page * c.page_stride + p.slot * c.token_stride, page * c.scale_page + p.slot * c.scale_token};
}

__global__ void clear_status_kernel(unsigned *status)
{
    pdl_trigger();
    pdl_wait();
    status[kWsStatusWord] = 0u;
    status[kWsDetailWord] = 0u;
}
st_status clear_status(unsigned *status, cudaStream_t stream) { return launch(clear_status_kernel, dim3(1), 1, 0, stream, status); }

__device__ __forceinline__ void report_offsets(const CacheArgs &a)
{
    if (blockIdx.x == 0 && !offsets_fine(a.offsets, a.c.nseq, a.n, threadIdx.x, cells::THREADS)) a.status[kWsStatusWord] = (unsigned)ST_ERR_DEV_BOUNDS;
}

template <int DTYPE>
__global__ void __launch_bounds__(cells::THREADS) cache_write_kernel(const CacheArgs a)
{
    using namespace cells;
    __shared__ Spot spots[GROUPS * ROWS];
    const int group = threadIdx.x / LANES, lane = threadIdx.x % LANES, e0 = lane * 8, width = 2 * a.c.kv_heads;
    const bool inside = e0 < a.c.d;
    pdl_wait();
    pdl_trigger();
    report_offsets(a);
    const int t0 = blockIdx.x / a.col_tiles * a.tokens, c0 = blockIdx.x % a.col_tiles * a.cols;
    const int nt = min(a.tokens, a.n - t0), nc = min(a.cols, width - c0);
    uint4 u[ROWS];
    int token[ROWS], col[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        const int row = group + j * GROUPS;
        token[j] = row / a.cols;
        col[j] = c0 + row - token[j] * a.cols;
        if (token[j] >= nt || col[j] >= c0 + nc) token[j] = -1;
        const bool is_k = col[j] < a.c.kv_heads;
        const int64_t t = t0 + token[j];
        const bf16 *src = is_k ? a.k + t * a.k_row + col[j] * a.k_head : a.v + t * a.v_row + (col[j] - a.c.kv_heads) * a.v_head;
        u[j] = token[j] >= 0 && inside ? *reinterpret_cast<const uint4 *>(src + e0) : make_uint4(0u, 0u, 0u, 0u);
    }
    for (int t = group; t < (nt + 1) / 2 * 2; t += GROUPS) {           // both halves of a warp take part in the search
        const Spot s = spot_of(a, t0 + t, t < nt);
        if (lane == 0 && t < nt) spots[t] = s;
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        const Spot at = token[j] >= 0 ? spots[token[j]] : Spot{NOWHERE, 0};
        const bool is_k = col[j] < a.c.kv_heads;
        const int h = is_k ? col[j] : col[j] - a.c.kv_heads;
        const bool put = at.cells >= 0 && inside;
        unsigned char *dst = (is_k ? a.c.k : a.c.v) + at.cells + h * a.c.head_stride;
        uint32_t *scales = (is_k ? a.c.k_scales : a.c.v_scales) + at.scales + h * a.c.scale_head;
        if (DTYPE == ST_BF16) {
            if (put) *reinterpret_cast<uint4 *>(dst + e0 * 2) = u[j];
            continue;
        }
        float x[8];
        unpack8(u[j], x);
        if (DTYPE == ST_I8) {
            // largest magnitude by its bits, among which NaN and infinity are the largest
            unsigned top = 0;
#pragma unroll
            for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7FFFFFFFu);
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(~0u, top, o));
            const float most = __uint_as_float(top);
            const bool fine = top < 0x7F800000u, some = fine && most >= FEWEST_SCALE;
            const float scale = !fine ? __uint_as_float(0x7FC00000u) : some ? __fdiv_rn(most, 127.f) : 0.f, inv = some ? __fdiv_rn(127.f, most) : 0.f;
            uint32_t w[2] = {0u, 0u};
            if (some)
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e / 4] |= (uint32_t)(__float2int_rn(__fmul_rn(x[e], inv)) & 0xFF) << (8 * (e % 4));
            if (put) *reinterpret_cast<uint2 *>(dst + e0) = make_uint2(w[0], w[1]);
            if (put && lane == 0) *scales = __float_as_uint(scale);
        } else {
            float lo = INFINITY, hi = -INFINITY;
            bool fine = true;
            if (inside)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    lo = fminf(lo, x[e]);
                    hi = fmaxf(hi, x[e]);
                    fine = fine && fabsf(x[e]) < INFINITY;
                }
            unsigned bad = !fine;
#pragma unroll
            for (int o = 1; o < GROUP / 8; o <<= 1) {
                lo = fminf(lo, __shfl_xor_sync(~0u, lo, o));
                hi = fmaxf(hi, __shfl_xor_sync(~0u, hi, o));
                bad |= __shfl_xor_sync(~0u, bad, o);
            }
            const float told = __bfloat162float(__float2bfloat16(__fdiv_rn(hi - lo, 15.f)));
            fine = !bad && told < INFINITY;
            const bool some = fine && told >= FEWEST_SCALE;
            const float step = some ? told : 0.f, inv = some ? __fdiv_rn(1.f, step) : 0.f;
            uint32_t w = 0u;
            if (some)
#pragma unroll
                for (int e = 0; e < 8; ++e) w |= (uint32_t)min(max(__float2int_rn(__fmul_rn(__fsub_rn(x[e], lo), inv)), 0), 15) << (4 * e);
            if (put) *reinterpret_cast<uint32_t *>(dst + e0 / 2) = w;
            if (put && lane % (GROUP / 8) == 0)
                scales[e0 / GROUP] = fine ? __float_as_uint(step) >> 16 | (__float_as_uint(lo) & 0xFFFF0000u) : 0x7FC07FC0u;
        }
    }
}

template <int DTYPE>
__global__ void __launch_bounds__(cells::THREADS) cache_read_kernel(const CacheArgs a)
{
    using namespace cells;
    __shared__ Spot spots[GROUPS * ROWS];
    const int group = threadIdx.x / LANES, lane = threadIdx.x % LANES, e0 = lane * 8, width = 2 * a.c.kv_heads;
    const bool inside = e0 < a.c.d;
    pdl_wait();
    pdl_trigger();
    report_offsets(a);
    const int t0 = blockIdx.x / a.col_tiles * a.tokens, c0 = blockIdx.x % a.col_tiles * a.cols;
    const int nt = min(a.tokens, a.n - t0), nc = min(a.cols, width - c0);
    for (int t = group; t < (nt + 1) / 2 * 2; t += GROUPS) {           // both halves of a warp take part in the search
        const Spot s = spot_of(a, t0 + t, t < nt);
        if (lane == 0 && t < nt) spots[t] = s;
    }
    __syncthreads();
    uint4 u[ROWS];
    uint32_t scale[ROWS];
    bf16 *dst[ROWS];
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        const int row = group + j * GROUPS, token = row / a.cols, col = c0 + row - token * a.cols;
        const bool is_k = col < a.c.kv_heads;
        const int h = is_k ? col : col - a.c.kv_heads;
        const Spot at = token < nt && col < c0 + nc ? spots[token] : Spot{NO_ROW, 0};
        const bool put = at.cells != NO_ROW && inside, get = put && at.cells >= 0;
        dst[j] = put ? (is_k ? a.k_out : a.v_out) + ((int64_t)(t0 + token) * a.c.kv_heads + h) * a.c.d + e0 : nullptr;
        const unsigned char *src = (is_k ? a.c.k : a.c.v) + at.cells + h * a.c.head_stride;
        u[j] = make_uint4(0u, 0u, 0u, 0u);
        scale[j] = 0u;
        if (!get) continue;
        if (DTYPE == ST_BF16) u[j] = *reinterpret_cast<const uint4 *>(src + e0 * 2);
        if (DTYPE == ST_I8) {
            const uint2 x = *reinterpret_cast<const uint2 *>(src + e0);
            u[j].x = x.x;
            u[j].y = x.y;
        }
        if (DTYPE == ST_I4) u[j].x = *reinterpret_cast<const uint32_t *>(src + e0 / 2);
        if (DTYPE != ST_BF16) scale[j] = ((is_k ? a.c.k_scales : a.c.v_scales) + at.scales + h * a.c.scale_head)[DTYPE == ST_I4 ? e0 / GROUP : 0];
    }
#pragma unroll
    for (int j = 0; j < ROWS; ++j) {
        if (!dst[j]) continue;
        if (DTYPE != ST_BF16) {
            const uint32_t in[2] = {u[j].x, u[j].y};
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (DTYPE == ST_I8) x[e] = __uint_as_float(scale[j]) * (float)(int)(signed char)(in[e / 4] >> (8 * (e % 4)));
                else x[e] = fmaf(__uint_as_float(scale[j] << 16), (float)(in[0] >> (4 * e) & 15u), __uint_as_float(scale[j] & 0xFFFF0000u));
            }
            u[j] = pack8(x);
       }
        *reinterpret_cast<uint4 *>(dst[j]) = u[j];
    }
}

static st_status run_cache(CacheArgs &a, int dtype, bool write, cudaStream_t stream)
{
    using namespace cells;
    const int width = 2 * a.c.kv_heads;
    a.cols = width < GROUPS * ROWS ? width : GROUPS * ROWS;
    a.tokens = GROUPS * ROWS / a.cols;
    a.col_tiles = (width + a.cols - 1) / a.cols;
    const int64_t grid = ((int64_t)a.n + a.tokens - 1) / a.tokens * a.col_tiles;
    if (grid > INT32_MAX) return ST_ERR_UNSUPPORTED;
    const st_status rc = clear_status(a.status, stream);
    if (rc != ST_OK) return rc;
    void (*kernel)(CacheArgs) = nullptr;
    if (write) kernel = dtype == ST_BF16 ? cache_write_kernel<ST_BF16> : dtype == ST_I8 ? cache_write_kernel<ST_I8> : cache_write_kernel<ST_I4>;
    else kernel = dtype == ST_BF16 ? cache_read_kernel<ST_BF16> : dtype == ST_I8 ? cache_read_kernel<ST_I8> : cache_read_kernel<ST_I4>;
    return launch(kernel, dim3((unsigned)grid), THREADS, 0, stream, a);
}

static st_status check_rows_of(const st_cells *c, int64_t n, const int32_t *offsets, const void *ws, size_t ws_bytes)
{
    if (n <= 0 || (!offsets && c->nseq != 1 && c->nseq != n)) return ST_ERR_SHAPE;
    if (n > (1 << 29)) return ST_ERR_UNSUPPORTED;
    if (!aligned4(offsets)) return ST_ERR_ALIGN;
    if (!ws || ws_bytes < kWsHeaderBytes) return ST_ERR_WORKSPACE;
    return aligned256(ws) ? ST_OK : ST_ERR_ALIGN;
}

}  // namespace attn
}  // namespace st

using namespace st;
using namespace st::attn;

extern "C" st_status st_attn_cache_write(const st_cells *c, const st_tokens *t, const void *k, const void *v, const int32_t *table, const int32_t *lens,
                                         const int32_t *offsets, void *k_pages, void *v_pages, void *k_scales, void *v_scales, void *ws, size_t ws_bytes,
                                         void *stream)
{
    st_status rc = check_cells(c, k_pages, v_pages, k_scales, v_scales, table, lens);
    if (rc != ST_OK) return rc;
    if (!t || !k || !v) return ST_ERR_NULL;
    st_tokens rows = *t;                   // as a table without queries
    rows.nseq = c->nseq;
    rows.nq = rows.nk;
    rows.heads = rows.kv_heads;
    rows.q_row = rows.k_row;
    rows.q_head = rows.k_head;
    if ((rc = check_tokens(&rows)) != ST_OK) return rc;
    if (rows.kv_heads != c->kv_heads || rows.d != c->d || rows.dv != c->d) return ST_ERR_SHAPE;
    if ((rc = check_rows_of(c, rows.nk, offsets, ws, ws_bytes)) != ST_OK) return rc;
    if (!aligned16(k) || !aligned16(v)) return ST_ERR_ALIGN;
    for (const Operand &o : {k_of(&rows, k), v_of(&rows, v)}) {
        const int64_t bytes = 2 * ((o.rows - 1) * o.row + (o.heads - 1) * o.head + o.cols);
        if (meets_cells(c, k_pages, k_scales, o.p, bytes) || meets_cells(c, v_pages, v_scales, o.p, bytes)) return ST_ERR_UNSUPPORTED;
    }
    CacheArgs a = {};
    a.c = cells_of(c, k_pages, v_pages, k_scales, v_scales, table, lens);
    a.k = (const bf16 *)k;
    a.v = (const bf16 *)v;
    a.k_row = stride_of(rows.nk, rows.k_row);
    a.k_head = stride_of(rows.kv_heads, rows.k_head);
    a.v_row = stride_of(rows.nk, rows.v_row);
    a.v_head = stride_of(rows.kv_heads, rows.v_head);
    a.offsets = offsets;
    a.status = (unsigned *)ws;
    a.n = (int)rows.nk;
    return run_cache(a, c->dtype, true, (cudaStream_t)stream);
}

extern "C" st_status st_attn_cache_read(const st_cells *c, int64_t n, const void *k_pages, const void *v_pages, const void *k_scales, const void *v_scales,
                                        const int32_t *table, const int32_t *lens, const int32_t *offsets, void *k, void *v, void *ws, size_t ws_bytes,
                                        void *stream)
{
    st_status rc = check_cells(c, k_pages, v_pages, k_scales, v_scales, table, lens);
    if (rc != ST_OK) return rc;
    if (!k || !v) return ST_ERR_NULL;
    if ((rc = check_rows_of(c, n, offsets, ws, ws_bytes)) != ST_OK) return rc;
    if (!aligned16(k) || !aligned16(v)) return ST_ERR_ALIGN;
    const int64_t bytes = n * c->kv_heads * c->d * 2;
    if (arrays_meet(k, bytes, v, bytes)) return ST_ERR_UNSUPPORTED;
    for (const void *p : {(const void *)k, (const void *)v})
        if (meets_cells(c, k_pages, k_scales, p, bytes) || meets_cells(c, v_pages, v_scales, p, bytes)) return ST_ERR_UNSUPPORTED;
    CacheArgs a = {};
    a.c = cells_of(c, k_pages, v_pages, k_scales, v_scales, table, lens);
    a.k_out = (bf16 *)k;
    a.v_out = (bf16 *)v;
    a.offsets = offsets;
    a.status = (unsigned *)ws;
    a.n = (int)n;
    return run_cache(a, c->dtype, false, (cudaStream_t)stream);
}
