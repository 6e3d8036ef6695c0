// What the attention calls share: checks of their arguments, and where the tokens of a sequence lie.
#pragma once
#include <cuda_bf16.h>
#include "attn_index.cuh"
#include "st_common.cuh"

namespace st {
namespace attn {

typedef __nv_bfloat16 bf16;

// A table of tokens: rows, heads within a row.
struct Table {
    const bf16 *p;
    int64_t row, head;        // strides in elements
};

inline bool stride_ok(int64_t extent, int64_t stride, int64_t least)
{
    return extent == 1 || stride >= least;
}

inline st_status check_tokens(const st_tokens *t)
{
    if (!t) return ST_ERR_NULL;
    if (t->dtype != ST_BF16) return ST_ERR_DTYPE;
    if (t->reserved != 0 || t->nseq <= 0 || t->nq <= 0 || t->nk <= 0 || t->heads <= 0 || t->kv_heads <= 0 || t->d <= 0 || t->dv <= 0)
        return ST_ERR_SHAPE;
    if (t->heads % t->kv_heads != 0) return ST_ERR_SHAPE;
    // rows and sequences are counted in 32 bits, with room for a position less a window less a position; heads are a grid's second extent
    if (t->nq > (1 << 29) || t->nk > (1 << 29) || t->nseq > (1 << 20) || t->heads > 65535) return ST_ERR_UNSUPPORTED;
    if (t->d % 8 != 0 || t->dv % 8 != 0 || t->d > 128 || t->dv > 128) return ST_ERR_UNSUPPORTED;
    const bool fits = stride_ok(t->nq, t->q_row, t->d) && stride_ok(t->heads, t->q_head, t->d) && stride_ok(t->nk, t->k_row, t->d) &&
                      stride_ok(t->kv_heads, t->k_head, t->d) && stride_ok(t->nk, t->v_row, t->dv) && stride_ok(t->kv_heads, t->v_head, t->dv);
    if (!fits) return ST_ERR_SHAPE;
    // 2^38 elements: half of what a tensor map's stride may be
    for (const int64_t s : {t->q_row, t->q_head, t->k_row, t->k_head, t->v_row, t->v_head})
        if (s > ((int64_t)1 << 38)) return ST_ERR_UNSUPPORTED;
    const bool even = (t->nq == 1 || t->q_row % 8 == 0) && (t->heads == 1 || t->q_head % 8 == 0) && (t->nk == 1 || t->k_row % 8 == 0) &&
                      (t->kv_heads == 1 || t->k_head % 8 == 0) && (t->nk == 1 || t->v_row % 8 == 0) && (t->kv_heads == 1 || t->v_head % 8 == 0);
    return even ? ST_OK : ST_ERR_ALIGN;
}

// The stride of an extent of one is never used; whatever was passed, it is a legal one.
inline int64_t stride_of(int64_t extent, int64_t stride) { return extent == 1 ? 128 : stride; }

// The tables of a call, for the check of its results: a result may not lie over an operand that is still read when it is written.
struct Operand {
    const void *p;
    int64_t rows, heads, cols, row, head;
    // whether `bytes` bytes of results at `to` lie over it; in_place: they may take its place as a whole, if it is contiguous
    bool under(const void *to, int64_t bytes, bool in_place = false) const
    {
        const bool whole = to == p && bytes == rows * heads * cols * 2 && (heads == 1 || head == cols) && (rows == 1 || row == heads * cols);
        return !(in_place && whole) && overlap((uint64_t)p, rows, heads, cols * 2, row * 2, head * 2, (uint64_t)to, bytes);
    }
};
inline Operand q_of(const st_tokens *t, const void *q) { return {q, t->nq, t->heads, t->d, stride_of(t->nq, t->q_row), stride_of(t->heads, t->q_head)}; }
inline Operand k_of(const st_tokens *t, const void *k) { return {k, t->nk, t->kv_heads, t->d, stride_of(t->nk, t->k_row), stride_of(t->kv_heads, t->k_head)}; }
inline Operand v_of(const st_tokens *t, const void *v) { return {v, t->nk, t->kv_heads, t->dv, stride_of(t->nk, t->v_row), stride_of(t->kv_heads, t->v_head)}; }
inline Operand dense_of(const void *p, int64_t rows, int64_t heads, int64_t cols) { return {p, rows, heads, cols, heads * cols, cols}; }
// Two arrays without gaps; none where one is missing.
inline bool arrays_meet(const void *a, int64_t a_bytes, const void *b, int64_t b_bytes)
{
    return a && b && (uint64_t)a < (uint64_t)b + b_bytes && (uint64_t)b < (uint64_t)a + a_bytes;
}

// A window or a number of first columns: the whole of the longest sequence is as far as it goes.
inline int clamp_int(int64_t x, int most = 1 << 29) { return x > most ? most : (int)x; }

#if defined(__CUDACC__)

// Two fp32 at a time.
struct Pair {
    uint64_t v;
};
__device__ __forceinline__ Pair pair(float lo, float hi)
{
    Pair r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r.v) : "f"(lo), "f"(hi));
    return r;
}
__device__ __forceinline__ Pair pair(uint32_t lo, uint32_t hi) { return pair(__uint_as_float(lo), __uint_as_float(hi)); }
__device__ __forceinline__ float2 split(Pair a)
{
    float2 r;
    asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(a.v));
    return r;
}
__device__ __forceinline__ Pair mul(Pair a, Pair b)
{
    Pair r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair add(Pair a, Pair b)
{
    Pair r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r.v) : "l"(a.v), "l"(b.v));
    return r;
}
__device__ __forceinline__ Pair fma(Pair a, Pair b, Pair c)
{
    Pair r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r.v) : "l"(a.v), "l"(b.v), "l"(c.v));
    return r;
}

// Eight bf16 as floats and back, rounded once.
__device__ __forceinline__ void unpack8(const uint4 &u, float (&x)[8])
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(w[i] << 16);
        x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ uint4 pack8(const float (&x)[8])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

__device__ __forceinline__ void unpack8(const uint4 &u, Pair (&x)[4])
{
    x[0] = pair(u.x << 16, u.x & 0xFFFF0000u);
    x[1] = pair(u.y << 16, u.y & 0xFFFF0000u);
    x[2] = pair(u.z << 16, u.z & 0xFFFF0000u);
    x[3] = pair(u.w << 16, u.w & 0xFFFF0000u);
}
__device__ __forceinline__ uint4 pack8(const Pair (&x)[4])
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = split(x[i]);
        const __nv_bfloat162 b = __floats2bfloat162_rn(f.x, f.y);
        w[i] = *reinterpret_cast<const uint32_t *>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Rows [first, first + len) of sequence b, cut to the table.
struct Rows {
    int first, len;
};
__device__ __forceinline__ Rows rows_of(const int *offsets, int b, int n)
{
    if (!offsets) return {0, n};
    const int lo = min(max(offsets[b], 0), n), hi = min(max(offsets[b + 1], lo), n);
    return {lo, hi - lo};
}

// Status of a call by what its offsets are; the threads of one block look them all over.
__device__ __forceinline__ bool offsets_fine(const int *offsets, int nseq, int n, int tid, int threads)
{
    bool fine = true;
    if (offsets)
        for (int b = tid; b < nseq; b += threads) {
            const int lo = offsets[b], hi = offsets[b + 1];
            fine = fine && lo >= 0 && hi >= lo && hi <= n;
        }
    return fine;
}

#endif

}  // namespace attn
}  // namespace st
