// Building blocks of the tensor-core attention kernels: tiles of 128 tokens in shared memory and tensor memory, and which
// tiles of keys a tile of queries sees.
#pragma once
#include "attn_common.cuh"
#include "tc_common.cuh"

namespace st {
namespace attn {

constexpr int TILE_LOG = 7, TILE = 1 << TILE_LOG;                     // tokens of a tile
constexpr int SLAB = TILE * 128;              // bytes of 64 columns of a tile: rows of 128 bytes, 128-byte swizzle
constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// A table as a tensor map {column, head, row}, boxes of 64 columns x 1 head x `rows` rows; what lies outside reads as zero.
inline bool make_tmap_table(CUtensorMap *m, const Table &t, int64_t rows, int64_t heads, int64_t cols, uint32_t box_rows = TILE)
{
    const tc::EncodeTiledFn fn = tc::encode_tiled_fn();
    if (!fn) return false;
    cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)heads, (cuuint64_t)rows};
    cuuint64_t strides[2] = {(cuuint64_t)t.head * 2, (cuuint64_t)t.row * 2};
    cuuint32_t box[3] = {64, 1, box_rows}, estr[3] = {1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<bf16 *>(t.p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

#if defined(__CUDACC__)

__device__ __forceinline__ void tma_load_3d(void *dst, const CUtensorMap *m, uint64_t *bar, int x, int y, int z)
{
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
        ::"r"(tc::smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(m)), "r"(tc::smem_u32(bar)), "r"(x), "r"(y), "r"(z)
        : "memory");
}

// 128 rows from `row` of one head, COLS columns, as slabs of 64 columns; the copy's bytes are counted on `bar`.
template <int COLS>
__device__ __forceinline__ void load_tile(unsigned char *dst, const CUtensorMap *m, uint64_t *bar, int head, int row)
{
#pragma unroll
    for (int c = 0; c < COLS / 64; ++c) tma_load_3d(dst + c * SLAB, m, bar, c * 64, head, row);
}

// The other way: what lies outside the table is not written.  Needs a proxy fence by the writers of the shared memory first.
__device__ __forceinline__ void tma_store_3d(const CUtensorMap *m, const void *src, int x, int y, int z)
{
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%2, %3, %4}], [%1];"
                 ::"l"(reinterpret_cast<uint64_t>(m)), "r"(tc::smem_u32(src)), "r"(x), "r"(y), "r"(z)
                 : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void tma_store_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void tma_store_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// The same copies as far as L2.
__device__ __forceinline__ void prefetch_3d(const CUtensorMap *m, int x, int y, int z)
{
    asm volatile("cp.async.bulk.prefetch.tensor.3d.L2.global [%0, {%1, %2, %3}];" ::"l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y), "r"(z) : "memory");
}
template <int COLS>
__device__ __forceinline__ void prefetch_tile(const CUtensorMap *m, int head, int row)
{
#pragma unroll
    for (int c = 0; c < COLS / 64; ++c) prefetch_3d(m, c * 64, head, row);
}

// Products are issued by one lane (`lead`) of a warp whose lanes all run the loop around them: what the instruction takes is the same
// for the whole warp and stays in uniform registers.  Inside a branch that one lane took alone every operand was moved there first, at
// some 90 cycles an instruction beside busy warps.
__device__ __forceinline__ void mma_ss(bool lead, uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"((uint32_t)add), "r"((uint32_t)lead)
        : "memory");
}
// The A operand from tensor memory: 128 lanes, two bf16 of consecutive k to a column.
__device__ __forceinline__ void mma_ts(bool lead, uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, bool add)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"((uint32_t)add), "r"((uint32_t)lead)
        : "memory");
}
__device__ __forceinline__ void commit(bool lead, uint64_t *bar)
{
    asm volatile(
        "{\n\t.reg .pred q;\n\t"
        "setp.ne.b32 q, %1, 0;\n\t"
        "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}"
        ::"r"(tc::smem_u32(bar)), "r"((uint32_t)lead)
        : "memory");
}

// D[128, N] = A B^T over COLS columns of two K-major tiles (rows of A are lanes of D, rows of B are columns of D).
template <int COLS>
__device__ __forceinline__ void mma_rows(bool lead, uint32_t d_tmem, const unsigned char *A, const unsigned char *B, uint32_t idesc)
{
    const uint64_t a = tc::make_smem_desc(tc::smem_u32(A), 16, 1024), b = tc::make_smem_desc(tc::smem_u32(B), 16, 1024);
#pragma unroll
    for (int k = 0; k < COLS / 16; ++k) {
        const uint64_t off = (uint64_t)(((k >> 2) * SLAB + (k & 3) * 32) >> 4);
        mma_ss(lead, d_tmem, a + off, b + off, idesc, k > 0);
    }
}

// D[128, N] (+)= A B over tokens 16 K0 .. 16 K1 of a tile: A[128, 128 tokens] bf16 in tensor memory, its second 64 tokens HALF columns behind
// the first, B a tile whose rows are the tokens.
template <int HALF = 32, int K0 = 0, int K1 = TILE / 16>
__device__ __forceinline__ void mma_tokens(bool lead, uint32_t d_tmem, uint32_t a_tmem, const unsigned char *B, uint32_t idesc, bool add)
{
    const uint64_t b = tc::make_smem_desc(tc::smem_u32(B), SLAB, 1024);
#pragma unroll
    for (int k = K0; k < K1; ++k) mma_ts(lead, d_tmem, a_tmem + (k >> 2) * HALF + (k & 3) * 8, b + (uint64_t)(k * 2048 >> 4), idesc, add || k > 0);
}

// A wait of a whole warp: all lanes see the phase over, or none goes on.
template <typename... Args>
__device__ __forceinline__ bool warp_wait(uint64_t *bar, uint32_t parity, Args... args)
{
    return __all_sync(~0u, tc::mbar_wait(bar, parity, args...));
}

__device__ __forceinline__ void tmem_st_32x16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
          "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float y;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
    return y;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

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
__device__ __forceinline__ uint32_t pack_bf16(Pair a)
{
    const float2 f = split(a);
    return pack_bf16(f.x, f.y);
}

// Tile number `index` of the tiles of `rows` tokens that the sequences are cut into, by a whole warp; at least `least` tiles to a
// sequence.  seq = -1: there is none.
struct TileOf {
    int seq, tile;
};
__device__ __forceinline__ TileOf tile_of(const int *offsets, int nseq, int n, int rows, int index, int lane, int least = 0)
{
    if (!offsets) return {index < (n - 1) / rows + 1 ? 0 : -1, index};
    for (int b0 = 0; b0 < nseq; b0 += 32) {
        const int b = b0 + lane;
        const int mine = b < nseq ? max((rows_of(offsets, b, n).len - 1 + rows) / rows, least) : 0;
        int sum = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(~0u, sum, o);
            if (lane >= o) sum += x;
        }
        const unsigned behind = __ballot_sync(~0u, index < sum);
        if (behind) {
            const int l = __ffs(behind) - 1;
            return {b0 + l, index - __shfl_sync(~0u, sum - mine, l)};
        }
        index -= __shfl_sync(~0u, sum, 31);
    }
    return {-1, 0};
}

// Which pairs of positions the window and the first columns leave.
struct Mask {
    int window, sinks;
    // whether any of the queries t0..t1 sees any of the keys s0..s1, or each of them every one
    __device__ __forceinline__ bool any(int t0, int t1, int s0, int s1) const { return s0 <= t1 && (s1 > t0 - window || s0 < sinks) && t1 >= t0; }
    __device__ __forceinline__ bool all(int t0, int t1, int s0, int s1) const { return s1 <= t0 && (s0 > t1 - window || s1 < sinks); }
};

// Which of 32 columns, of which the first is `first` columns into a tile that begins at key s0, the query at position t sees: bit c, column c.
struct RowMask {
    int hi, lo, sinks;                         // columns of the tile: at most hi, and at least lo or below sinks
    __device__ __forceinline__ RowMask(const Mask &m, int t, int s0) : hi(t - s0), lo(t - m.window + 1 - s0), sinks(m.sinks - s0) {}
    __device__ __forceinline__ explicit RowMask(int last) : hi(last), lo(0), sinks(0) {}            // columns up to `last`
    static __device__ __forceinline__ unsigned below(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1u; }
    __device__ __forceinline__ unsigned of(int first) const { return below(hi + 1 - first) & (~below(lo - first) | below(sinks - first)); }
};
// The tiles of keys that the queries at positions t0..t1 see: `first` with the first columns in front of the band, cut at `sinks`, and `band` from
// key `origin` on.  The band's tiles begin where it does, not at multiples of 128: 128 queries with a window of 512 meet five of them wherever
// they stand, and not six (prompts of up to 2111 tokens behind 40, 16 heads: with the piece of the first columns 145 -> 132 us).
struct KeyTiles {
    static constexpr int PIECE = 32;
    int first, band, origin, sinks;
    __device__ __forceinline__ int count() const { return first + band; }
    __device__ __forceinline__ int key(int i) const { return i < first ? i * TILE : origin + (i - first) * TILE; }
    // a few first columns alone in the first tile: only so many columns of it are multiplied
    __device__ __forceinline__ bool piece(int i) const { return i == 0 && first == 1 && sinks <= PIECE; }
    // Rows [unseen, used) of the last tile of first columns are multiplied by weights of 0 and seen by nobody: an older part of a cache, which may
    // hold anything.  Where there are any they are cleared, by the warp that copies: in the loop of the one that issues the products the stores took
    // 15 % (32768 tokens, window 4096), in a warp of their own 3 %, here 1 %.
    __device__ __forceinline__ int unseen() const { return sinks - (first - 1) * TILE; }
    __device__ __forceinline__ int used() const { return piece(first - 1) ? PIECE : TILE; }
    __device__ __forceinline__ int cleared() const { return first > 0 && unseen() < used() ? first - 1 : -1; }      // that tile, or -1
    // whether each of the queries t0..t1 sees all of tile i, and which columns of it the one at t sees
    __device__ __forceinline__ bool all(const Mask &m, int t0, int t1, int i) const
    {
        return i < first ? (i + 1) * TILE <= sinks : m.all(t0, t1, key(i), key(i) + TILE - 1);
    }
    __device__ __forceinline__ RowMask row_mask(const Mask &m, int t, int i) const
    {
        RowMask r(m, t, key(i));
        if (i < first) r = RowMask(sinks - 1 - i * TILE);
        return r;
    }
};
__device__ __forceinline__ KeyTiles key_tiles(const Mask &m, int t0, int t1)
{
    KeyTiles k;
    k.origin = max(0, t0 - m.window + 1);
    k.band = t1 < k.origin ? 0 : (t1 - k.origin) / TILE + 1;
    k.sinks = k.band ? min(m.sinks, k.origin) : 0;
    k.first = (k.sinks + TILE - 1) / TILE;
    return k;
}

// The same for a key at position s and the 32 queries from position t0 + first: s <= t, and t < s + window or s < sinks.
struct ColumnMask {
    int lo, hi;
    bool sink;
    __device__ __forceinline__ ColumnMask(const Mask &m, int s, int t0) : lo(s - t0), hi(s + m.window - 1 - t0), sink(s < m.sinks) {}
    __device__ __forceinline__ unsigned of(int first) const
    {
        return ~RowMask::below(lo - first) & (sink ? ~0u : RowMask::below(hi + 1 - first));
    }
};

// Values of the columns whose bit is not set become 0.
template <int N>
__device__ __forceinline__ void keep(Pair (&v)[N], unsigned bits)
{
#pragma unroll
    for (int e = 0; e < N; ++e) {
        const float2 x = split(v[e]);
        v[e] = pair(bits >> (2 * e) & 1u ? x.x : 0.f, bits >> (2 * e + 1) & 1u ? x.y : 0.f);
    }
}

// A thread's row of an accumulator (128 lanes, COLS columns), scaled, as bf16 rows of a table from `row` on.  `rows`: shared memory of a tile that no
// product reads any more.  A warp's 32 rows leave in one copy for each 64 columns, those at a sequence's end (`live` of the warp's are left) one
// by one; rows up to `skip` not at all.  To be waited for with tma_store_wait by lane 0.
template <int COLS>
__device__ __forceinline__ void store_rows(uint32_t taddr, unsigned char *rows, const CUtensorMap *map, bf16 *table, int64_t stride, int cols, int row, int head,
                                           int r, int live, int skip, float scale, bool zero)
{
    const int lane = r & 31, wr = r - lane, r8 = r & 7;
    const bool all = live >= 32 && skip <= 0;
    const Pair f = pair(scale, scale);
#pragma unroll 1
    for (int j = 0; j < COLS / 16; ++j) {
        uint32_t o[16];
        tc::tmem_ld_32x16(taddr + j * 16, o);
        tc::tmem_ld_wait();
        unsigned char *at = rows + (j / 4) * SLAB + r * 128;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            uint32_t u[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) u[k] = zero ? 0u : pack_bf16(mul(pair(o[e * 8 + 2 * k], o[e * 8 + 2 * k + 1]), f));
            *reinterpret_cast<uint4 *>(at + (((j % 4) * 2 + e) ^ r8) * 16) = make_uint4(u[0], u[1], u[2], u[3]);
        }
        if (all && j % 4 == 3) {
            tc::fence_proxy_async();
            __syncwarp();
            if (lane == 0) tma_store_3d(map, rows + (j / 4) * SLAB + wr * 128, j / 4 * 64, head, row);
        }
    }
    __syncwarp();
    if (!all)
        for (int k = max(skip, 0); k < min(live, 32); ++k)
            if (lane * 8 < cols && lane < COLS / 8)
                *reinterpret_cast<uint4 *>(table + (int64_t)(row + k) * stride + head * cols + lane * 8) =
                    *reinterpret_cast<const uint4 *>(rows + (lane / 8) * SLAB + (wr + k) * 128 + (((lane & 7) ^ (k & 7)) << 4));
}

// Rows [from, to) of a tile in shared memory, whatever they are, become zero; by a whole warp, before the tensor cores read the tile.
template <int COLS>
__device__ __forceinline__ void clear_rows(unsigned char *tile, int from, int to, int lane)
{
    from = max(from, 0);
    to = min(to, TILE);
    if (from >= to) return;
#pragma unroll
    for (int c = 0; c < COLS / 64; ++c)
        for (int i = from * 8 + lane; i < to * 8; i += 32) *reinterpret_cast<uint4 *>(tile + c * SLAB + i * 16) = make_uint4(0u, 0u, 0u, 0u);
    tc::fence_proxy_async();
    __syncwarp();
}

#endif

}  // namespace attn
}  // namespace st
