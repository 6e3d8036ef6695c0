// st_attn_cache_write and st_attn_cache_read: rows of keys and values into the pages of a cache and back, as they are or quantised.
//
// Bound by memory: a row is read once and written once.  16 lanes (8 up to 64 columns) own a row, 8 of its columns each.  A warp takes a run of tokens, of each
// the keys or the values of some heads (to read, with those of the token after on their way): the sequence that a token belongs to, its length and its page are
// looked up where the run begins, a sequence ends or a page does, and the next page's number while the one before is in use.
// 8 key heads of 128, pages of 64: 12 prompts at 8 bits, 17000 tokens, written in 23 us and read back in 20.5 (with a look-up and divisions of its own for each row 62
// together), 4.6 and 5.1 TB/s: issue slots 70 %, conversions and places.  25000 tokens of 4 bits 36.6 us (3.6 TB/s, divisions and two extremes for 32 columns) and
// 27.5 (4.9); 27000 of 16 bits 37.9 (5.8 TB/s) and 38.7.
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
    int n, run, chunks;                    // tokens; of a warp's run; pieces of a token's keys, and as many of its values, that warps share
};

namespace cells {
constexpr int WARPS = 4, ROWS = 4;         // of a block; rows of each group of lanes of a token
}

// A warp's way along a run of tokens: where its rows lie, cells in bytes, scales in units of 4 bytes.
struct Run {
    int first, last;                       // rows of the sequence that the token is in; none: empty
    int b, col, slot, page, next_page;     // the sequence, its page, its place in it
    __device__ __forceinline__ int page_at(const Cells &c, int i) const { return i < c.cols ? c.table[(int64_t)b * c.cols + i] : -1; }
    // The token of row `row`, wherever the one before was.
    __device__ __forceinline__ void find(const CacheArgs &a, int row)
    {
        const Cells &c = a.c;
        b = 0, first = 0, last = a.n;
        if (!a.offsets) {
            if (c.nseq > 1) b = row, first = row, last = row + 1;
        } else {
            // the last sequence that begins at or before the row
            const int lane = threadIdx.x & 31;
            for (int span = c.nseq, step; span > 1; span = step) {
                step = (span + 31) / 32;
                const int at = b + (lane + 1) * step;
                const bool before = lane < 31 && at < min(b + span, c.nseq) && a.offsets[at] <= row;
                b += __popc(__ballot_sync(~0u, before)) * step;
            }
            const Rows r = rows_of(a.offsets, b, a.n);
            first = r.first;
            last = r.first + r.len;
        }
        if (row < first || row >= last) {                  // a row of no sequence
            first = last = 0;
            return;
        }
        const int64_t at = (int64_t)c.lens[b] - (last - row);
        page = next_page = -1;
        slot = 0;
        col = at < 0 ? -1 : c.cols;                        // before the first place, or behind the last
        if (at >= 0 && at < (int64_t)c.cols * c.page) {
            const Place p = place_of((int)at, c.page, c.page_magic);
            col = p.col;
            slot = p.slot;
            page = page_at(c, col);
            next_page = page_at(c, col + 1);
        }
    }
    // On to the row behind it.
    __device__ __forceinline__ void on(const CacheArgs &a, int row)
    {
        if (row >= last || col < 0) {                      // the next sequence, or still no place
            find(a, row);
        } else if (++slot == a.c.page) {
            slot = 0;
            page = next_page;
            next_page = page_at(a.c, ++col + 1);
        }
    }
    // Whether it is a row of a sequence; then whether it has a place, which is reported where not.
    __device__ __forceinline__ bool row() const { return last > first; }
    __device__ __forceinline__ bool place(const CacheArgs &a) const
    {
        const bool there = col >= 0 && (unsigned)page < (unsigned)a.c.pages;
        if (!there) a.status[kWsStatusWord] = (unsigned)ST_ERR_DEV_BOUNDS;
        return there;
    }
    __device__ __forceinline__ int64_t cells(const Cells &c) const { return page * c.page_stride + slot * c.token_stride; }
    __device__ __forceinline__ int64_t scales(const Cells &c) const { return page * c.scale_page + slot * c.scale_token; }
};

__device__ __forceinline__ void report_offsets(const CacheArgs &a)
{
    if (blockIdx.x == 0 && !offsets_fine(a.offsets, a.c.nseq, a.n, threadIdx.x, cells::WARPS * 32)) a.status[kWsStatusWord] = (unsigned)ST_ERR_DEV_BOUNDS;
}

__global__ void clear_status_kernel(unsigned *status)
{
    pdl_trigger();
    pdl_wait();
    status[kWsStatusWord] = 0u;
    status[kWsDetailWord] = 0u;
}
// The status is cleared ahead of the warps that may report: within one kernel no block is known to run before another.
static st_status clear_status(unsigned *status, cudaStream_t stream) { return launch(clear_status_kernel, dim3(1), 1, 0, stream, status); }

// What a warp does: tokens t0 .. t1 - 1, of each the keys or the values of heads h0 + j GROUPS + sub, j below ROWS; bit j of `has`: this lane's group has that one.
template <int LANES>
struct Item {
    int t0, t1, h0, sub, lane, e0;
    bool values, inside;
    unsigned has;
    __device__ __forceinline__ explicit Item(const CacheArgs &a)
    {
        using namespace cells;
        constexpr int GROUPS = 32 / LANES;
        const int item = blockIdx.x * WARPS + (threadIdx.x >> 5), piece = item % (2 * a.chunks);
        t0 = item / (2 * a.chunks) * a.run;
        t1 = min(t0 + a.run, a.n);
        values = piece >= a.chunks;
        h0 = (values ? piece - a.chunks : piece) * GROUPS * ROWS;
        lane = threadIdx.x % LANES;
        sub = (threadIdx.x & 31) / LANES;
        e0 = lane * 8;
        inside = e0 < a.c.d;
        has = 0;
#pragma unroll
        for (int j = 0; j < ROWS; ++j)
            if (h0 + j * GROUPS + sub < a.c.kv_heads) has |= 1u << j;
    }
};

// What a row that is quantised needs besides is made for all rows of a token at once, by another lane for each: a division for every row would be
// one for every lane of it.
template <int DTYPE, int LANES>
__global__ void __launch_bounds__(cells::WARPS * 32) cache_write_kernel(const CacheArgs a)
{
    using namespace cells;
    constexpr int GROUPS = 32 / LANES;
    pdl_wait();
    pdl_trigger();
    report_offsets(a);
    const Item<LANES> it(a);
    if (it.t0 >= it.t1) return;
    const int lane = it.lane;
    const int64_t row = it.values ? a.v_row : a.k_row, head = it.values ? a.v_head : a.k_head;
    const bf16 *from = (it.values ? a.v : a.k) + it.t0 * row + (it.h0 + it.sub) * head + it.e0;
    unsigned char *to = (it.values ? a.c.v : a.c.k) + (it.h0 + it.sub) * a.c.head_stride + (DTYPE == ST_BF16 ? it.e0 * 2 : DTYPE == ST_I8 ? it.e0 : it.e0 / 2);
    // ST_I8: lane j has the scale of its group's row j; ST_I4: lane j of four, that of the four's columns in row j
    const int own = lane % ROWS;
    uint32_t *to_scale = (it.values ? a.c.v_scales : a.c.k_scales) + (it.h0 + own * GROUPS + it.sub) * a.c.scale_head + (DTYPE == ST_I4 ? lane / 4 : 0);
    const bool has_scale = (it.has >> own & 1u) && (DTYPE == ST_I8 ? lane < ROWS : lane / 4 * GROUP < a.c.d);
    Run run;
    for (int t = it.t0; t < it.t1; ++t, from += row) {
        uint4 u[ROWS];
#pragma unroll
        for (int j = 0; j < ROWS; ++j)
            u[j] = (it.has >> j & 1u) && it.inside ? *reinterpret_cast<const uint4 *>(from + j * GROUPS * head) : make_uint4(0u, 0u, 0u, 0u);
        if (t == it.t0) run.find(a, t);
        else run.on(a, t);
        if (!run.row() || !run.place(a)) continue;
        unsigned char *dst = to + run.cells(a.c);
        float inv = 0.f, low[ROWS];
        if (DTYPE == ST_I8) {
            // largest magnitudes by their bits, among which NaN and infinity are the largest
            unsigned mine = 0;
#pragma unroll
            for (int j = 0; j < ROWS; ++j) {
                unsigned top = __vmaxu2(__vmaxu2(u[j].x & 0x7FFF7FFFu, u[j].y & 0x7FFF7FFFu), __vmaxu2(u[j].z & 0x7FFF7FFFu, u[j].w & 0x7FFF7FFFu));
#pragma unroll
                for (int o = LANES / 2; o > 0; o >>= 1) top = __vmaxu2(top, __shfl_xor_sync(~0u, top, o));
                if (own == j) mine = top;
            }
            mine = max(mine << 16, mine & 0xFFFF0000u);
            const float most = __uint_as_float(mine);
            const bool fine = mine < 0x7F800000u, some = fine && most >= FEWEST_SCALE;
            inv = some ? __fdiv_rn(127.f, most) : 0.f;
            if (has_scale) to_scale[run.scales(a.c)] = !fine ? 0x7FC00000u : some ? __float_as_uint(__fdiv_rn(most, 127.f)) : 0u;
        } else if (DTYPE == ST_I4) {
            float range = 0.f, base = 0.f;
            unsigned wrong = 0u;
#pragma unroll
            for (int j = 0; j < ROWS; ++j) {
                float x[8], lo = INFINITY, hi = -INFINITY;
                unpack8(u[j], x);
                unsigned bad = 0;
                if (it.inside) {
                    const unsigned top = __vmaxu2(__vmaxu2(u[j].x & 0x7FFF7FFFu, u[j].y & 0x7FFF7FFFu), __vmaxu2(u[j].z & 0x7FFF7FFFu, u[j].w & 0x7FFF7FFFu));
                    bad = max(top << 16, top & 0xFFFF0000u) >= 0x7F800000u;
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        lo = fminf(lo, x[e]);
                        hi = fmaxf(hi, x[e]);
                    }
                }
#pragma unroll
                for (int o = 1; o < GROUP / 8; o <<= 1) {
                    lo = fminf(lo, __shfl_xor_sync(~0u, lo, o));
                    hi = fmaxf(hi, __shfl_xor_sync(~0u, hi, o));
                    bad |= __shfl_xor_sync(~0u, bad, o);
                }
                low[j] = lo;
                if (own == j) range = hi - lo, base = lo, wrong = bad;
            }
            const float told = __bfloat162float(__float2bfloat16(__fdiv_rn(range, 15.f)));
            const bool fine = !wrong && told < INFINITY, some = fine && told >= FEWEST_SCALE;
            const float step = some ? told : 0.f;
            inv = some ? __fdiv_rn(1.f, step) : 0.f;
            if (has_scale) to_scale[run.scales(a.c)] = fine ? __float_as_uint(step) >> 16 | (__float_as_uint(base) & 0xFFFF0000u) : 0x7FC07FC0u;
        }
        constexpr float WHOLE = 12582912.f;                // 1.5 2^23 added rounds to a whole number, to nearest even, and leaves it in the low bits
#pragma unroll
        for (int j = 0; j < ROWS; ++j, dst += GROUPS * a.c.head_stride) {
            const bool put = (it.has >> j & 1u) && it.inside;
            if (DTYPE == ST_BF16) {
                if (put) *reinterpret_cast<uint4 *>(dst) = u[j];
                continue;
            }
            const float f = __shfl_sync(~0u, inv, DTYPE == ST_I8 ? it.sub * LANES + j : (threadIdx.x & 28) + j);
            float x[8];
            unpack8(u[j], x);
            uint32_t b[8];                                 // one by one: of a packed product and a packed sum ptxas makes one operation that rounds once
#pragma unroll
            for (int e = 0; e < 8; ++e) b[e] = __float_as_uint(__fadd_rn(__fmul_rn(DTYPE == ST_I4 ? __fsub_rn(x[e], low[j]) : x[e], f), WHOLE));
            if (DTYPE == ST_I8) {
                const uint32_t w0 = __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410);
                const uint32_t w1 = __byte_perm(__byte_perm(b[4], b[5], 0x0040), __byte_perm(b[6], b[7], 0x0040), 0x5410);
                if (put) *reinterpret_cast<uint2 *>(dst) = f == 0.f ? make_uint2(0u, 0u) : make_uint2(w0, w1);
            } else {
                // whole numbers n from 0 to 15 as 0x4B400000 + n: sixteens of them in 32 bits, less what their upper bits add up to
                uint32_t w = b[7];
#pragma unroll
                for (int e = 6; e >= 0; --e) w = w * 16u + b[e];
                if (put) *reinterpret_cast<uint32_t *>(dst) = f == 0.f ? 0u : w - 0x4B400000u * 0x11111111u;
            }
        }
    }
}

template <int DTYPE, int LANES>
__global__ void __launch_bounds__(cells::WARPS * 32) cache_read_kernel(const CacheArgs a)
{
    using namespace cells;
    constexpr int GROUPS = 32 / LANES;
    pdl_wait();
    pdl_trigger();
    report_offsets(a);
    const Item<LANES> it(a);
    if (it.t0 >= it.t1) return;
    const unsigned char *from = (it.values ? a.c.v : a.c.k) + (it.h0 + it.sub) * a.c.head_stride + (DTYPE == ST_BF16 ? it.e0 * 2 : DTYPE == ST_I8 ? it.e0 : it.e0 / 2);
    const uint32_t *from_scale = (it.values ? a.c.v_scales : a.c.k_scales) + (it.h0 + it.sub) * a.c.scale_head + (DTYPE == ST_I4 ? it.e0 / GROUP : 0);
    const int64_t row = (int64_t)a.c.kv_heads * a.c.d;
    bf16 *to = (it.values ? a.v_out : a.k_out) + it.t0 * row + (it.h0 + it.sub) * a.c.d + it.e0;
    const unsigned has = it.inside ? it.has : 0u;
    Run run;
    uint4 next[ROWS];                                      // of the token after
    uint32_t next_scale[ROWS];
    bool next_row = false, next_there = false;             // whether it is a row of a sequence, and has a place
    auto load = [&](int t) {
        next_row = false;
        if (t >= it.t1) return;
        if (t == it.t0) run.find(a, t);
        else run.on(a, t);
        next_row = run.row();
        next_there = next_row && run.place(a);
        if (!next_there) return;
        const unsigned char *src = from + run.cells(a.c);
        const uint32_t *src_scale = from_scale + run.scales(a.c);
#pragma unroll
        for (int j = 0; j < ROWS; ++j, src += GROUPS * a.c.head_stride, src_scale += GROUPS * a.c.scale_head) {
            if (!(has >> j & 1u)) continue;
            if (DTYPE == ST_BF16) next[j] = *reinterpret_cast<const uint4 *>(src);
            if (DTYPE == ST_I8) {
                const uint2 x = *reinterpret_cast<const uint2 *>(src);
                next[j].x = x.x;
                next[j].y = x.y;
            }
            if (DTYPE == ST_I4) next[j].x = *reinterpret_cast<const uint32_t *>(src);
            if (DTYPE != ST_BF16) next_scale[j] = *src_scale;
        }
    };
    load(it.t0);
    for (int t = it.t0; t < it.t1; ++t, to += row) {
        const bool is_row = next_row, there = next_there;
        uint4 u[ROWS];
        uint32_t scale[ROWS];
#pragma unroll
        for (int j = 0; j < ROWS; ++j) {
            u[j] = next[j];
            scale[j] = next_scale[j];
        }
        load(t + 1);
        if (!is_row) continue;
        if (!there) {
#pragma unroll
            for (int j = 0; j < ROWS; ++j)
                if (has >> j & 1u) *reinterpret_cast<uint4 *>(to + j * GROUPS * a.c.d) = make_uint4(0u, 0u, 0u, 0u);
            continue;
        }
        bf16 *dst = to;
#pragma unroll
        for (int j = 0; j < ROWS; ++j, dst += GROUPS * a.c.d) {
            if (!(has >> j & 1u)) continue;
            if (DTYPE == ST_I8) {
                // whole numbers n from 0 on as 2^23 + n, less 2^23 and the 128 that was added to a signed byte
                const uint32_t in[2] = {u[j].x ^ 0x80808080u, u[j].y ^ 0x80808080u};
                const Pair f = pair(scale[j], scale[j]), less = pair(-8388736.f, -8388736.f);
                Pair x[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t w = in[e / 2], pick = 0x7540u + 2 * (e % 2);
                    x[e] = mul(f, add(pair(__byte_perm(w, 0x4B000000u, pick), __byte_perm(w, 0x4B000000u, pick + 1)), less));
                }
                u[j] = pack8(x);
            } else if (DTYPE == ST_I4) {
                // cells i and i + 4 side by side in bf16: 0x43 beside c is 128 + c; then lo + step c, rounded once
                const uint32_t step = __byte_perm(scale[j], 0u, 0x1010), lo = __byte_perm(scale[j], 0u, 0x3232);
                uint32_t r[4];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    asm("{\n\t.reg .b32 c;\n\t"
                        "sub.rn.bf16x2 c, %1, %2;\n\t"
                        "fma.rn.bf16x2 %0, %3, c, %4;\n\t}"
                        : "=r"(r[i])
                        : "r"((u[j].x >> (4 * i) & 0x000F000Fu) | 0x43004300u), "r"(0x43004300u), "r"(step), "r"(lo));
                u[j] = make_uint4(__byte_perm(r[0], r[1], 0x5410), __byte_perm(r[2], r[3], 0x5410), __byte_perm(r[0], r[1], 0x7632), __byte_perm(r[2], r[3], 0x7632));
            }
            *reinterpret_cast<uint4 *>(dst) = u[j];
        }
    }
}

// Runs as long as leave 64 warps to every SM, and no longer than 16 tokens.
static st_status run_cache(CacheArgs &a, int dtype, bool write, cudaStream_t stream)
{
    using namespace cells;
    const bool small = a.c.d <= 64;
    const int heads = (small ? 4 : 2) * ROWS;
    a.chunks = (a.c.kv_heads + heads - 1) / heads;
    const int64_t runs = (int64_t)a.n * 2 * a.chunks / (sm_count_or_default() * 64);
    a.run = (int)(runs < 1 ? 1 : runs > 16 ? 16 : runs);
    const int64_t items = ((int64_t)a.n + a.run - 1) / a.run * 2 * a.chunks, grid = (items + WARPS - 1) / WARPS;
    if (items > INT32_MAX - WARPS) return ST_ERR_UNSUPPORTED;
    const st_status rc = clear_status(a.status, stream);
    if (rc != ST_OK) return rc;
    void (*kernel)(CacheArgs) = nullptr;
    if (write && small) kernel = dtype == ST_BF16 ? cache_write_kernel<ST_BF16, 8> : dtype == ST_I8 ? cache_write_kernel<ST_I8, 8> : cache_write_kernel<ST_I4, 8>;
    else if (write) kernel = dtype == ST_BF16 ? cache_write_kernel<ST_BF16, 16> : dtype == ST_I8 ? cache_write_kernel<ST_I8, 16> : cache_write_kernel<ST_I4, 16>;
    else if (small) kernel = dtype == ST_BF16 ? cache_read_kernel<ST_BF16, 8> : dtype == ST_I8 ? cache_read_kernel<ST_I8, 8> : cache_read_kernel<ST_I4, 8>;
    else kernel = dtype == ST_BF16 ? cache_read_kernel<ST_BF16, 16> : dtype == ST_I8 ? cache_read_kernel<ST_I8, 16> : cache_read_kernel<ST_I4, 16>;
    return launch(kernel, dim3((unsigned)grid), WARPS * 32, 0, stream, a);
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
        if (meets_cells(c, k_pages, k_scales, p, bytes) || meets_cells(c, v_pages, v_scales, p, bytes) || arrays_meet(p, bytes, table, c->nseq * c->table_cols * 4) ||
            arrays_meet(p, bytes, lens, c->nseq * 4) || arrays_meet(p, bytes, offsets, (c->nseq + 1) * 4))
            return ST_ERR_UNSUPPORTED;
    CacheArgs a = {};
    a.c = cells_of(c, k_pages, v_pages, k_scales, v_scales, table, lens);
    a.k_out = (bf16 *)k;
    a.v_out = (bf16 *)v;
    a.offsets = offsets;
    a.status = (unsigned *)ws;
    a.n = (int)n;
    return run_cache(a, c->dtype, false, (cudaStream_t)stream);
}
