// st_attn_cache_step: one token of every sequence against a cache in cells, which holds it already; and the own tokens of st_attn_shared_step.
//
// Bound by the cells' bytes: every visible row of K and V is read once for all query heads that share it.  The division of work is that of
// st_attn_window_step: a cluster of blocks owns one key head of one sequence and 16 of its query heads, its warps take tiles of 16 or 32 visible keys in
// turn through rings of their own (cp.async, page numbers one tile further ahead), and multiply with mma.sync, of whose 16 rows a group of heads fills some.
//
// Cells meet the tensor cores as whole numbers in bf16, which holds all of them exactly: 8 bits by their bits (128 + low seven bits, less 128 or 256),
// 4 bits likewise (128 + c, less 128).  Scales come in afterwards, where they are one number for a key (ST_I8: a score times its key's scale, a weight
// times its value's) or for 32 columns (ST_I4: partial scores of 32 columns, x += step acc + lo sum(q); a set of weights for each 32 columns, and what lo
// brings beside it, sum(w lo)).  The order of a fragment's columns is free as long as both operands agree, so that no byte has to change its lane:
// a lane's four bytes of K are four or eight consecutive columns, of which the queries' fragments take the same ones.
#include "attn_cells_step.cuh"
#include "tc_common.cuh"

namespace st {
namespace attn {

namespace cstep {
constexpr int HEADS = 16, MAX_SPLITS = 16;
constexpr int FEWEST = 2;                  // tiles of a warp, where keys are split further
template <int DTYPE, int DP, int WARPS, int STAGES> struct Shape {
    static constexpr int KEYS = DTYPE == ST_BF16 ? 16 : 32;                        // of a tile
    static constexpr int ROW = DTYPE == ST_BF16 ? 2 * DP : DTYPE == ST_I8 ? DP : DP / 2;       // bytes
    static constexpr int SCALES = DTYPE == ST_BF16 ? 0 : DTYPE == ST_I8 ? 1 : DP / GROUP;      // of a row, 4 bytes each
    static constexpr int PIECES = ROW / 16;
    static constexpr int TILE = KEYS * ROW, STAGE = 2 * (TILE + KEYS * SCALES * 4), RING = STAGES * STAGE;
    static constexpr size_t SMEM = (size_t)WARPS * RING + (2 * WARPS + 2 + MAX_SPLITS + MAX_PARTS) * HEADS * sizeof(float) + WARPS * KEYS * sizeof(int64_t) + 32;
    static_assert(HEADS * DP * 4 <= RING, "a warp's output takes the place of its ring");
    // 16-byte pieces of a tile lie so that eight rows of one piece fall on different banks
    static __device__ __forceinline__ int swizzle(int row) { return ROW >= 128 ? row & 7 : ROW == 64 ? row >> 1 & 3 : row >> 2 & 1; }
};
}  // namespace cstep

template <int BYTES>
__device__ __forceinline__ void copy_async(uint32_t dst, const void *src, bool there)
{
    if (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(dst), "l"(src), "n"(BYTES), "r"(there ? BYTES : 0) : "memory");
}
__device__ __forceinline__ void load4x8x8(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void load2x8x8(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x2.shared.b16 {%0, %1}, [%2];" : "=r"(r[0]), "=r"(r[1]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void load4x8x8_trans(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float load_cluster(uint32_t addr)
{
    float x;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(addr) : "memory");
    return x;
}
__device__ __forceinline__ float exp2_fast(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pair_bf16(float lo, float hi)
{
    const __nv_bfloat162 w = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&w);
}
__device__ __forceinline__ uint32_t minus_bf16(uint32_t a, uint32_t b)
{
    const __nv_bfloat162 w = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&a), *reinterpret_cast<const __nv_bfloat162 *>(&b));
    return *reinterpret_cast<const uint32_t *>(&w);
}
// Two signed bytes of w as bf16, those that `which` picks: 0x43 beside a byte b is 128 + b up to 127, so its low seven bits are taken as that, less
// 128, or less 256 (0x4380) where its sign bit is set.
__device__ __forceinline__ uint32_t bytes_bf16(uint32_t w, uint32_t which)
{
    const uint32_t x = __byte_perm(w, 0x43434343u, which);
    return minus_bf16(x & 0xFF7FFF7Fu, x & 0xFF80FF80u);
}
// Nibbles i and i + 4 of w.
__device__ __forceinline__ uint32_t nibbles_bf16(uint32_t w, int i) { return minus_bf16((w >> (4 * i) & 0x000F000Fu) | 0x43004300u, 0x43004300u); }
__device__ __forceinline__ float low_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_bf16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// WIDE: rows and scales may be copied in 16-byte pieces
template <int DTYPE, int DP, int WARPS, int STAGES, bool WIDE>
__global__ void __launch_bounds__(WARPS * 32) cells_step_kernel(const CellsStepArgs a)
{
    using namespace cstep;
    using S = Shape<DTYPE, DP, WARPS, STAGES>;
    constexpr int KEYS = S::KEYS, ROW = S::ROW, PIECES = S::PIECES, NB = KEYS / 8, GROUPS = DP / GROUP;
    extern __shared__ __align__(128) unsigned char smem[];
    float *most_w = (float *)(smem + WARPS * S::RING), *sum_w = most_w + WARPS * HEADS, *most_b = sum_w + WARPS * HEADS, *sum_b = most_b + HEADS;
    float *share = sum_b + HEADS;                          // weight of every block's part, over the sum: [block][head]
    float *part_share = share + MAX_SPLITS * HEADS;        // likewise of every part of the prefix
    int64_t *offsets = (int64_t *)(part_share + MAX_PARTS * HEADS);
    int *flags = (int *)(offsets + WARPS * KEYS);          // [0]: something to report, [1]: this block has a visible key
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = lane & 3;
    const int splits = gridDim.x, split = blockIdx.x, chunks = (a.group + HEADS - 1) / HEADS, b = blockIdx.z;
    const int hk = blockIdx.y / chunks, g0 = blockIdx.y % chunks * HEADS, g = min(a.group - g0, HEADS);
    const Cells &cs = a.c;

    if (threadIdx.x < 2) flags[threadIdx.x] = 0;
    // Parts of a prefix come from the kernel before this one, which lets this one begin only when all before itself is there: they alone are waited for.
    if (!a.part_count) pdl_wait();
    pdl_trigger();
    __syncthreads();
    const int told = cs.lens[b], len = length_of(told, cs.cols, cs.page);
    if (told != len && threadIdx.x == 0) flags[0] = 1;
    // visible keys: [0, first) and [lo, len)
    const int lo = max(0, len - a.window), first = min(a.sinks, lo), keys = first + len - lo, tiles = (keys + KEYS - 1) / KEYS;
    const unsigned char *kc = cs.k + hk * cs.head_stride, *vc = cs.v + hk * cs.head_stride;
    const uint32_t *ks = cs.k_scales + hk * cs.scale_head, *vs = cs.v_scales + hk * cs.scale_head;
    const uint32_t ring = tc::smem_u32(smem + warp * S::RING);
    const int step = splits * WARPS, tile0 = split * WARPS + warp;
    const int64_t head0 = hk * a.group + g0;

    // The queries as fragments: row = head; which columns a lane has is what its bytes of K are.
    uint32_t q[DP / 16][4];
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = lane / 4 + (i & 1) * 8, j = i >> 1;
            const int c0 = DTYPE == ST_BF16 ? k * 16 + quad * 2 + j * 8 : DTYPE == ST_I8 ? k * 16 + quad * 4 + j * 2 : (k / 2) * 32 + quad * 8 + (k & 1) * 2 + j;
            const int c1 = DTYPE == ST_I4 ? c0 + 4 : c0 + 1;
            const unsigned short *at = reinterpret_cast<const unsigned short *>(a.q + b * a.q_row + (head0 + row) * a.q_head);
            q[k][i] = row < g ? (c0 < cs.d ? (uint32_t)at[c0] : 0u) | (c1 < cs.d ? (uint32_t)at[c1] << 16 : 0u) : 0u;
        }
    // ST_I4: sums of 32 columns of the queries, for the two heads of this lane
    float qsum[2][GROUPS];
    if (DTYPE == ST_I4)
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int p = 0; p < GROUPS; ++p) {
                float s = 0.f;
#pragma unroll
                for (int k = 2 * p; k < 2 * p + 2; ++k) s += low_bf16(q[k][i]) + high_bf16(q[k][i]) + low_bf16(q[k][i + 2]) + high_bf16(q[k][i + 2]);
                s += __shfl_xor_sync(~0u, s, 1);
                qsum[i][p] = s + __shfl_xor_sync(~0u, s, 2);
            }

    // Lane r finds row r of a tile: its page (-1: none, or outside the cache), then its place in the pages, which goes where all lanes that copy a
    // piece of the row see it.
    auto page_of = [&](int tile, int &slot) -> int {
        const int u = tile * KEYS + (lane & (KEYS - 1)), s = u < first ? u : lo + u - first;
        slot = 0;
        if (u >= keys) return -1;
        const Place p = place_of(s, cs.page, cs.page_magic);
        slot = p.slot;
        const int page = cs.table[(int64_t)b * cs.cols + p.col];
        if ((unsigned)page < (unsigned)cs.pages) return page;
        flags[0] = 1;
        return -1;
    };
    int64_t *at = offsets + warp * KEYS;
    const int piece = lane % PIECES, row0 = lane / PIECES;
    const int left = DTYPE == ST_BF16 ? 2 * cs.d - piece * 16 : DTYPE == ST_I8 ? cs.d - piece * 16 : cs.d / 2 - piece * 16;     // bytes of the row from this piece on
    constexpr int ROWS = 32 / PIECES;                      // rows that a warp copies at a time
    // bit r: row r of the tile is there.  What is not there is zeros.
    auto fetch = [&](int tile, int stage, int page, int slot) -> unsigned {
        const unsigned there = __ballot_sync(~0u, page >= 0 && lane < KEYS);
        if (tile < tiles) {
            const uint32_t dst = ring + stage * S::STAGE;
            __syncwarp();
            if (lane < KEYS) at[lane] = page >= 0 ? page * cs.page_stride + slot * cs.token_stride : 0;
            if (DTYPE != ST_BF16) {
                const int64_t from = page >= 0 ? page * cs.scale_page + slot * cs.scale_token : 0;
                const uint32_t o = dst + 2 * S::TILE + lane * S::SCALES * 4;
                const int n = (cs.d + GROUP - 1) / GROUP;
                if (DTYPE == ST_I8) {
                    copy_async<4>(o, ks + from, page >= 0);
                    copy_async<4>(o + KEYS * 4, vs + from, page >= 0);
                } else if (WIDE && DP == 128) {
                    copy_async<16>(o, ks + from, page >= 0);
                    copy_async<16>(o + KEYS * S::SCALES * 4, vs + from, page >= 0);
                } else {
#pragma unroll
                    for (int p = 0; p < S::SCALES; ++p) {
                        const int at_p = p < n ? p : 0;
                        copy_async<4>(o + p * 4, ks + from + at_p, page >= 0 && p < n);
                        copy_async<4>(o + KEYS * S::SCALES * 4 + p * 4, vs + from + at_p, page >= 0 && p < n);
                    }
                }
            }
            __syncwarp();
#pragma unroll
            for (int i = 0; i < KEYS / ROWS; ++i) {
                const int row = row0 + i * ROWS;
                const bool in = there >> row & 1;
                const int64_t from = at[row] + (left > 0 ? piece * 16 : 0);
                const uint32_t o = dst + row * ROW + ((piece ^ S::swizzle(row)) << 4);
                if (WIDE) {
                    copy_async<16>(o, kc + from, in && left > 0);
                    copy_async<16>(o + S::TILE, vc + from, in && left > 0);
                } else {
                    const int next = left > 8 ? 8 : 0;
                    copy_async<8>(o, kc + from, in && left > 0);
                    copy_async<8>(o + 8, kc + from + next, in && left > 8);
                    copy_async<8>(o + S::TILE, vc + from, in && left > 0);
                    copy_async<8>(o + S::TILE + 8, vc + from + next, in && left > 8);
                }
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        return there;
    };

    const float c = a.scale * 1.4426950408889634f;
    float o[DP / 8][4], most[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
    float low[2][GROUPS];                                  // ST_I4: what the values' lowest numbers bring to 32 columns
#pragma unroll
    for (int n = 0; n < DP / 8; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][i] = 0.f;
#pragma unroll
    for (int p = 0; p < GROUPS; ++p) low[0][p] = low[1][p] = 0.f;

    auto attend = [&](int stage, unsigned there) {
        const uint32_t K = ring + stage * S::STAGE, V = K + S::TILE;
        const uint32_t *kscale = reinterpret_cast<const uint32_t *>(smem + warp * S::RING + stage * S::STAGE + 2 * S::TILE), *vscale = kscale + KEYS * S::SCALES;
        float x[NB][4];
#pragma unroll
        for (int n = 0; n < NB; ++n) {
#pragma unroll
            for (int i = 0; i < 4; ++i) x[n][i] = 0.f;
            const int row = n * 8 + (lane & 7);
            if (DTYPE == ST_BF16) {
#pragma unroll
                for (int k = 0; k < DP / 32; ++k) {
                    uint32_t f[4];                         // 8 keys, 32 columns
                    load4x8x8(f, K + row * ROW + (((k * 4 + lane / 8) ^ S::swizzle(row)) << 4));
                    mma(x[n], q[2 * k], f[0], f[1]);
                    mma(x[n], q[2 * k + 1], f[2], f[3]);
                }
            } else if (DTYPE == ST_I8) {
#pragma unroll
                for (int k = 0; k < DP / 64; ++k) {
                    uint32_t f[4];                         // 8 keys, 64 columns
                    load4x8x8(f, K + row * ROW + (((k * 4 + lane / 8) ^ S::swizzle(row)) << 4));
#pragma unroll
                    for (int m = 0; m < 4; ++m) mma(x[n], q[4 * k + m], bytes_bf16(f[m], 0x4140u), bytes_bf16(f[m], 0x4342u));
                }
                const float2 s = *reinterpret_cast<const float2 *>(kscale + n * 8 + quad * 2);
                x[n][0] *= s.x;
                x[n][1] *= s.y;
                x[n][2] *= s.x;
                x[n][3] *= s.y;
            } else {
                uint32_t f[4];                             // 8 keys, all columns
                const uint32_t from = K + row * ROW + (((lane / 8 % PIECES) ^ S::swizzle(row)) << 4);
                if (DP == 128) load4x8x8(f, from);
                else load2x8x8(f, from);
#pragma unroll
                for (int p = 0; p < GROUPS; ++p) {
                    float y[4] = {0.f, 0.f, 0.f, 0.f};
                    mma(y, q[2 * p], nibbles_bf16(f[p], 0), nibbles_bf16(f[p], 1));
                    mma(y, q[2 * p + 1], nibbles_bf16(f[p], 2), nibbles_bf16(f[p], 3));
                    const uint32_t s0 = kscale[(n * 8 + quad * 2) * S::SCALES + p], s1 = kscale[(n * 8 + quad * 2 + 1) * S::SCALES + p];
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        x[n][2 * i] = fmaf(low_bf16(s0), y[2 * i], fmaf(high_bf16(s0), qsum[i][p], x[n][2 * i]));
                        x[n][2 * i + 1] = fmaf(low_bf16(s1), y[2 * i + 1], fmaf(high_bf16(s1), qsum[i][p], x[n][2 * i + 1]));
                    }
                }
            }
        }
        if (there != (KEYS == 32 ? ~0u : 0xFFFFu))
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!(there >> (n * 8 + quad * 2 + (i & 1)) & 1)) x[n][i] = -INFINITY;
        float top[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            top[i] = fmaxf(x[0][2 * i], x[0][2 * i + 1]);
#pragma unroll
            for (int n = 1; n < NB; ++n) top[i] = fmaxf(top[i], fmaxf(x[n][2 * i], x[n][2 * i + 1]));
            top[i] = fmaxf(top[i], __shfl_xor_sync(~0u, top[i], 1));
            top[i] = fmaxf(top[i], __shfl_xor_sync(~0u, top[i], 2));
        }
        // as long as no weight passes 2^8 the reference stays: any reference gives the same quotient
        if (__any_sync(~0u, c * (top[0] - most[0]) > 8.f || c * (top[1] - most[1]) > 8.f)) {
            float f[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float now = fmaxf(most[i], top[i]);
                f[i] = now == -INFINITY ? 1.f : exp2f(c * (most[i] - now));
                most[i] = now;
                sum[i] *= f[i];
                if (DTYPE == ST_I4)
#pragma unroll
                    for (int p = 0; p < GROUPS; ++p) low[i][p] *= f[i];
            }
#pragma unroll
            for (int n = 0; n < DP / 8; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[n][i] *= f[i >> 1];
        }
        const float ref[2] = {most[0] == -INFINITY ? 0.f : c * most[0], most[1] == -INFINITY ? 0.f : c * most[1]};
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                x[n][i] = exp2_fast(fmaf(c, x[n][i], -ref[i >> 1]));
                sum[i >> 1] += x[n][i];
            }
        // weights, times their values' scales, rounded once for the product with V
#pragma unroll
        for (int h = 0; h < KEYS / 16; ++h) {
            const int row = h * 16 + (lane & 15);
            if (DTYPE == ST_BF16) {
                const uint32_t p[4] = {pair_bf16(x[2 * h][0], x[2 * h][1]), pair_bf16(x[2 * h][2], x[2 * h][3]), pair_bf16(x[2 * h + 1][0], x[2 * h + 1][1]),
                                       pair_bf16(x[2 * h + 1][2], x[2 * h + 1][3])};
#pragma unroll
                for (int n = 0; n < DP / 16; ++n) {
                    uint32_t f[4];                         // 16 keys, 16 columns
                    load4x8x8_trans(f, V + row * ROW + (((n * 2 + lane / 16) ^ S::swizzle(row)) << 4));
                    mma(o[2 * n], p, f[0], f[1]);
                    mma(o[2 * n + 1], p, f[2], f[3]);
                }
            } else if (DTYPE == ST_I8) {
                uint32_t p[4];
#pragma unroll
                for (int n = 0; n < 2; ++n) {
                    const float2 s = *reinterpret_cast<const float2 *>(vscale + (2 * h + n) * 8 + quad * 2);
                    const float *y = x[2 * h + n];
                    p[2 * n] = pair_bf16(y[0] * s.x, y[1] * s.y);
                    p[2 * n + 1] = pair_bf16(y[2] * s.x, y[3] * s.y);
                }
#pragma unroll
                for (int n = 0; n < DP / 32; ++n) {
                    uint32_t f[4];                         // 16 keys, 32 columns: even columns in one product, odd ones in another
                    load4x8x8_trans(f, V + row * ROW + (((n * 2 + lane / 16) ^ S::swizzle(row)) << 4));
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        mma(o[4 * n + 2 * m], p, bytes_bf16(f[2 * m], 0x4240u), bytes_bf16(f[2 * m + 1], 0x4240u));
                        mma(o[4 * n + 2 * m + 1], p, bytes_bf16(f[2 * m], 0x4341u), bytes_bf16(f[2 * m + 1], 0x4341u));
                    }
                }
            } else {
#pragma unroll
                for (int n = 0; n < DP / 64; ++n) {
                    uint32_t f[4];                         // 16 keys, 64 columns
                    load4x8x8_trans(f, V + row * ROW + (((n * 2 + lane / 16) ^ S::swizzle(row)) << 4));
#pragma unroll
                    for (int m = 0; m < 2; ++m) {
                        const int group = 2 * n + m;
                        uint32_t p[4];
#pragma unroll
                        for (int e = 0; e < 2; ++e) {
                            const int key = (2 * h + e) * 8 + quad * 2;
                            const uint32_t s0 = vscale[key * S::SCALES + group], s1 = vscale[(key + 1) * S::SCALES + group];
                            const float *y = x[2 * h + e];
                            p[2 * e] = pair_bf16(y[0] * low_bf16(s0), y[1] * low_bf16(s1));
                            p[2 * e + 1] = pair_bf16(y[2] * low_bf16(s0), y[3] * low_bf16(s1));
                            low[0][group] = fmaf(y[0], high_bf16(s0), fmaf(y[1], high_bf16(s1), low[0][group]));
                            low[1][group] = fmaf(y[2], high_bf16(s0), fmaf(y[3], high_bf16(s1), low[1][group]));
                        }
#pragma unroll
                        for (int i = 0; i < 4; ++i) mma(o[4 * group + i], p, nibbles_bf16(f[2 * m], i), nibbles_bf16(f[2 * m + 1], i));
                    }
                }
            }
        }
    };
    unsigned there[STAGES], any = 0;
    int slot, page = page_of(tile0, slot);
#pragma unroll
    for (int s = 0; s < STAGES - 1; ++s) {
        const int p = page, l = slot;
        page = page_of(tile0 + (s + 1) * step, slot);
        there[s] = fetch(tile0 + s * step, s, p, l);
    }
    int stage = 0;
    for (int tile = tile0; tile < tiles; tile += step) {
        const int p = page, l = slot;
        page = page_of(tile + STAGES * step, slot);
        there[STAGES - 1] = fetch(tile + (STAGES - 1) * step, stage == 0 ? STAGES - 1 : stage - 1, p, l);      // the stage before was read by all lanes
        asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
        __syncwarp();
        any |= there[0];
        attend(stage, there[0]);
        __syncwarp();
#pragma unroll
        for (int s = 0; s + 1 < STAGES; ++s) there[s] = there[s + 1];
        if (++stage == STAGES) stage = 0;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();
    if (any && lane == 0) flags[1] = 1;

    // join the warps: each leaves its output where its ring was
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        sum[i] += __shfl_xor_sync(~0u, sum[i], 1);
        sum[i] += __shfl_xor_sync(~0u, sum[i], 2);
        if (DTYPE == ST_I4)
#pragma unroll
            for (int p = 0; p < GROUPS; ++p) {
                low[i][p] += __shfl_xor_sync(~0u, low[i][p], 1);
                low[i][p] += __shfl_xor_sync(~0u, low[i][p], 2);
            }
        if (quad == 0) {
            most_w[warp * HEADS + i * 8 + lane / 4] = most[i];
            sum_w[warp * HEADS + i * 8 + lane / 4] = sum[i];
        }
        // the columns of a product's results, as the values' cells lay
        float *mine = (float *)(smem + warp * S::RING) + (lane / 4 + i * 8) * DP;
        if (DTYPE == ST_BF16)
#pragma unroll
            for (int n = 0; n < DP / 8; ++n) *reinterpret_cast<float2 *>(mine + n * 8 + quad * 2) = make_float2(o[n][2 * i], o[n][2 * i + 1]);
        if (DTYPE == ST_I8)
#pragma unroll
            for (int n = 0; n < DP / 16; ++n)
                *reinterpret_cast<float4 *>(mine + n * 16 + quad * 4) = make_float4(o[2 * n][2 * i], o[2 * n + 1][2 * i], o[2 * n][2 * i + 1], o[2 * n + 1][2 * i + 1]);
        if (DTYPE == ST_I4)
#pragma unroll
            for (int n = 0; n < DP / 32; ++n)
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    *reinterpret_cast<float4 *>(mine + n * 32 + quad * 8 + e * 4) =
                        make_float4(o[4 * n][2 * i + e] + low[i][n], o[4 * n + 1][2 * i + e] + low[i][n], o[4 * n + 2][2 * i + e] + low[i][n],
                                    o[4 * n + 3][2 * i + e] + low[i][n]);
    }
    __syncthreads();
    // weight of a part whose largest score is m, where the largest of all is `all`
    auto weight = [&](float m, float all) { return m == -INFINITY ? 0.f : exp2f(c * (m - all)); };
    if (threadIdx.x < HEADS) {
        float all = -INFINITY, s = 0.f, w[WARPS];
#pragma unroll
        for (int i = 0; i < WARPS; ++i) all = fmaxf(all, most_w[i * HEADS + threadIdx.x]);
#pragma unroll
        for (int i = 0; i < WARPS; ++i) {
            w[i] = weight(most_w[i * HEADS + threadIdx.x], all);
            s += sum_w[i * HEADS + threadIdx.x] * w[i];
        }
#pragma unroll
        for (int i = 0; i < WARPS; ++i) most_w[i * HEADS + threadIdx.x] = w[i];
        most_b[threadIdx.x] = all;
        // a sum of 0 says that there is no key; where there are, of scores -inf all, it is 1, of weight 0
        sum_b[threadIdx.x] = all == -INFINITY && flags[1] && s == 0.f ? 1.f : s;
    }
    __syncthreads();
    float *block = (float *)smem;                          // the first warp's place
    for (int e = 4 * threadIdx.x; e < g * DP; e += 4 * WARPS * 32) {
        float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int i = 0; i < WARPS; ++i) {
            const float w = most_w[i * HEADS + e / DP];
            const float4 x = *reinterpret_cast<const float4 *>(smem + i * S::RING + e * 4);
            s = make_float4(fmaf(w, x.x, s.x), fmaf(w, x.y, s.y), fmaf(w, x.z, s.z), fmaf(w, x.w, s.w));
        }
        *reinterpret_cast<float4 *>(block + e) = s;
    }
    if (splits > 1) tc::cluster_sync_all();
    else __syncthreads();
    // then the blocks, and the prefix's parts: their shares first, each read once, then every block its piece of the output
    int parts = 0;
    const int rows = cs.nseq * a.group;
    const int64_t part_row = (int64_t)hk * rows + b * a.group + g0, part_rows = (int64_t)(a.heads / a.group) * rows;
    if (a.part_count) {
        pdl_wait();
        parts = min(a.part_count[b], MAX_PARTS);
    }
    if (threadIdx.x < HEADS) {
        float m[MAX_SPLITS], l[MAX_SPLITS], all = -INFINITY, s = 0.f;
        bool seen = false;
#pragma unroll
        for (int r = 0; r < MAX_SPLITS; ++r) {
            m[r] = -INFINITY;
            l[r] = 0.f;
            if (r < splits) {
                m[r] = splits > 1 ? load_cluster(tc::map_to_cta(tc::smem_u32(most_b + threadIdx.x), r)) : most_b[threadIdx.x];
                l[r] = splits > 1 ? load_cluster(tc::map_to_cta(tc::smem_u32(sum_b + threadIdx.x), r)) : sum_b[threadIdx.x];
            }
            all = fmaxf(all, m[r]);
            seen = seen || l[r] != 0.f;
        }
        const int n = threadIdx.x < g ? parts : 0;
        for (int r = 0; r < n; ++r) all = fmaxf(all, a.part_most[r * part_rows + part_row + threadIdx.x]);
#pragma unroll
        for (int r = 0; r < MAX_SPLITS; ++r) {
            m[r] = weight(m[r], all);
            s = fmaf(m[r], l[r], s);
        }
        for (int r = 0; r < n; ++r) {
            const float w = weight(a.part_most[r * part_rows + part_row + threadIdx.x], all), x = a.part_sum[r * part_rows + part_row + threadIdx.x];
            part_share[r * HEADS + threadIdx.x] = w;
            s = fmaf(w, x, s);
            seen = seen || x != 0.f;
        }
        const float inv = seen ? 1.f / s : 0.f;            // a sum of 0 (all scores are -inf) or NaN gives NaN
#pragma unroll
        for (int r = 0; r < MAX_SPLITS; ++r) share[r * HEADS + threadIdx.x] = m[r] * inv;
        for (int r = 0; r < n; ++r) part_share[r * HEADS + threadIdx.x] *= inv;
    }
    __syncthreads();
    // four columns to a thread, heads next to one another as they lie in the parts
    for (int e = split * WARPS * 32 + threadIdx.x; e < g * (DP / 4); e += splits * WARPS * 32) {
        const int row = e % g, quad4 = e / g, col = quad4 * 4;
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
        auto more = [&](float w, const float4 &x) { y = make_float4(fmaf(w, x.x, y.x), fmaf(w, x.y, y.y), fmaf(w, x.z, y.z), fmaf(w, x.w, y.w)); };
        if (splits == 1) {
            more(share[row], *reinterpret_cast<const float4 *>(block + row * DP + col));
        } else {
#pragma unroll 8
            for (int r = 0; r < splits; ++r) {
                const uint32_t at = tc::map_to_cta(tc::smem_u32(block + row * DP + col), r);
                float4 x;
                asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(at) : "memory");
                more(share[r * HEADS + row], x);
            }
        }
#pragma unroll 4
        for (int r = 0; r < parts; ++r) {
            const int64_t unit = (int64_t)r * (a.heads / a.group) + hk;
            const float w = part_share[r * HEADS + row];
            // a part without a finite score was not written, and one whose sum is NaN says so by its share
            if (w != 0.f) more(w, *reinterpret_cast<const float4 *>(a.part + ((unit * (DP / 4) + quad4) * rows + b * a.group + g0 + row) * 4));
        }
        if (col < cs.d)
            *reinterpret_cast<uint2 *>(a.out + ((int64_t)b * a.heads + head0 + row) * cs.d + col) = make_uint2(pair_bf16(y.x, y.y), pair_bf16(y.z, y.w));
    }
    if (splits > 1) tc::cluster_sync_all();                // no block ends while another reads its shared memory
    if (flags[0] && threadIdx.x == 0) atomicExch(a.status + kWsStatusWord, (unsigned)ST_ERR_DEV_BOUNDS);
}

__global__ void clear_status_kernel(unsigned *status, int *counts, int n)
{
    pdl_trigger();
    pdl_wait();
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < 2) status[i == 0 ? kWsStatusWord : kWsDetailWord] = 0u;
    if (i < n) counts[i] = 0;
}

st_status clear_status(unsigned *status, int *counts, int n, cudaStream_t stream)
{
    return launch(clear_status_kernel, dim3((unsigned)(n / 256 + 1)), n > 32 ? 256 : 32, 0, stream, status, counts, n);
}

template <int DTYPE, int DP, int WARPS, int STAGES, bool WIDE>
static st_status launch_cells(const CellsStepArgs &a, int splits, cudaStream_t stream)
{
    const auto kernel = cells_step_kernel<DTYPE, DP, WARPS, STAGES, WIDE>;
    const size_t smem = cstep::Shape<DTYPE, DP, WARPS, STAGES>::SMEM;
    if (!ensure_dynamic_smem(kernel, smem) || !allow_large_clusters(kernel)) return ST_ERR_CUDA;
    const int chunks = (a.group + cstep::HEADS - 1) / cstep::HEADS;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)splits, (unsigned)(a.heads / a.group * chunks), (unsigned)a.c.nseq);
    cfg.blockDim = dim3(WARPS * 32);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = stream;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = (unsigned)splits;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = splits > 1 ? 2 : 1;
    if (cudaLaunchKernelEx(&cfg, kernel, a) != cudaSuccess) {
        (void)cudaGetLastError();
        return ST_ERR_CUDA;
    }
    return ST_OK;
}

// Where heads and sequences are few the keys are split over a cluster of up to 16 blocks.
template <int DTYPE, int DP, bool WIDE>
static st_status run_cells(const CellsStepArgs &a, cudaStream_t stream)
{
    using S = cstep::Shape<DTYPE, DP, 4, 2>;
    const int64_t most = (int64_t)a.c.cols * a.c.page, visible = most < (int64_t)a.window + a.sinks ? most : (int64_t)a.window + a.sinks;
    const int64_t blocks = (int64_t)a.c.nseq * (a.heads / a.group) * ((a.group + cstep::HEADS - 1) / cstep::HEADS);
    const int64_t sms = sm_count_or_default(), tiles = (visible + S::KEYS - 1) / S::KEYS;
    int n = 1;
    while (n < cstep::MAX_SPLITS && blocks * n < 3 * sms && tiles > (int64_t)2 * n * 4 * cstep::FEWEST) n *= 2;
    return launch_cells<DTYPE, DP, 4, 2, WIDE>(a, n, stream);
}

st_status run_cells_step(const CellsStepArgs &a, int dtype, cudaStream_t stream)
{
    const bool small = a.c.d <= 64;
    const int64_t row = row_bytes(dtype, a.c.d);
    bool wide = row % 16 == 0 && a.c.page_stride % 16 == 0 && a.c.token_stride % 16 == 0 && a.c.head_stride % 16 == 0;
    if (dtype == ST_BF16) return small ? run_cells<ST_BF16, 64, true>(a, stream) : run_cells<ST_BF16, 128, true>(a, stream);
    if (dtype == ST_I8) {
        if (small) return wide ? run_cells<ST_I8, 64, true>(a, stream) : run_cells<ST_I8, 64, false>(a, stream);
        return wide ? run_cells<ST_I8, 128, true>(a, stream) : run_cells<ST_I8, 128, false>(a, stream);
    }
    if (!small) wide = wide && a.c.d > 96 && a.c.scale_page % 4 == 0 && a.c.scale_token % 4 == 0 && a.c.scale_head % 4 == 0;
    if (small) return wide ? run_cells<ST_I4, 64, true>(a, stream) : run_cells<ST_I4, 64, false>(a, stream);
    return wide ? run_cells<ST_I4, 128, true>(a, stream) : run_cells<ST_I4, 128, false>(a, stream);
}

st_status check_step(const st_cells *c, const void *q, int64_t q_row, int64_t q_head, float scale, const void *out)
{
    if (c->nseq > 65535) return ST_ERR_UNSUPPORTED;
    if (!q || !out) return ST_ERR_NULL;
    if (!stride_ok(c->nseq, q_row, c->d) || !stride_ok(c->heads, q_head, c->d)) return ST_ERR_SHAPE;
    if (q_row > ((int64_t)1 << 38) || q_head > ((int64_t)1 << 38) || !(scale > 0.f && scale < INFINITY)) return ST_ERR_UNSUPPORTED;
    if ((c->nseq > 1 && q_row % 8 != 0) || (c->heads > 1 && q_head % 8 != 0) || !aligned16(q) || !aligned16(out)) return ST_ERR_ALIGN;
    return ST_OK;
}

CellsStepArgs step_args(const st_cells *c, const void *q, int64_t q_row, int64_t q_head, const void *k_pages, const void *v_pages, const void *k_scales,
                        const void *v_scales, const int32_t *table, const int32_t *lens, float scale, void *out, void *ws)
{
    CellsStepArgs a = {};
    a.c = cells_of(c, k_pages, v_pages, k_scales, v_scales, table, lens);
    a.q = (const bf16 *)q;
    a.q_row = stride_of(c->nseq, q_row);
    a.q_head = stride_of(c->heads, q_head);
    a.heads = (int)c->heads;
    a.group = (int)(c->heads / c->kv_heads);
    a.window = 1 << 30;
    a.scale = scale;
    a.out = (bf16 *)out;
    a.status = (unsigned *)ws;
    return a;
}

}  // namespace attn
}  // namespace st

using namespace st;
using namespace st::attn;

extern "C" st_status st_attn_cache_step(const st_cells *c, const void *q, int64_t q_row, int64_t q_head, const void *k_pages, const void *v_pages,
                                        const void *k_scales, const void *v_scales, const int32_t *table, const int32_t *lens, int64_t window,
                                        int64_t sinks, float scale, void *out, void *ws, size_t ws_bytes, void *stream)
{
    st_status rc = check_cells(c, k_pages, v_pages, k_scales, v_scales, table, lens);
    if (rc != ST_OK) return rc;
    if (window < 1 || sinks < 0) return ST_ERR_SHAPE;
    if ((rc = check_step(c, q, q_row, q_head, scale, out)) != ST_OK) return rc;
    if (!ws || ws_bytes < kWsHeaderBytes) return ST_ERR_WORKSPACE;
    if (!aligned256(ws)) return ST_ERR_ALIGN;
    CellsStepArgs a = step_args(c, q, q_row, q_head, k_pages, v_pages, k_scales, v_scales, table, lens, scale, out, ws);
    a.window = clamp_int(window, 1 << 30);
    a.sinks = clamp_int(sinks, 1 << 30);
    const int64_t bytes = c->nseq * c->heads * c->d * 2;
    // blocks that share 16 heads or fewer read their queries before any of them writes
    const Operand Q = {q, c->nseq, c->heads, c->d, a.q_row, a.q_head};
    if (Q.under(out, bytes, true) || meets_cells(c, k_pages, k_scales, out, bytes) || meets_cells(c, v_pages, v_scales, out, bytes) ||
        arrays_meet(out, bytes, table, c->nseq * c->table_cols * 4) || arrays_meet(out, bytes, lens, c->nseq * 4))
        return ST_ERR_UNSUPPORTED;
    if ((rc = clear_status(a.status, nullptr, 0, (cudaStream_t)stream)) != ST_OK) return rc;
    return run_cells_step(a, c->dtype, (cudaStream_t)stream);
}
