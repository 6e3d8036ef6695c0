// st_attn_cache_step: one token of every sequence against a cache in cells, which holds it already; and the own tokens of st_attn_shared_step.
//
// Bound by the cells' bytes: every visible row of K and V is read once for all query heads that share it.  The work is a line of units (one key head of one
// sequence with 8 or 16 of its query heads), each as long as its tiles of 16 or 32 visible keys and what a unit costs beside them, and every warp takes an equal
// piece of that line, however long the sequences are: a small kernel ahead sums up their tiles, and one behind joins the units that warps share.  (Clusters of
// blocks that split each unit alike waited for the longest sequences, and blocks whose warps shared units waited for each other at every end of a short
// one: 64 sequences of up to 6000 tokens 125 and 134 us.)  A warp's page numbers are two tiles ahead and its rows one, in a ring of its own (cp.async), over
// the ends of units; no barrier of a block lies anywhere.  It multiplies with mma.sync, keys and the values' columns as the 16 rows of a product and
// heads as its 8 columns:  S^T = K Q^T,  O^T = V^T P^T.  (Heads as rows would leave half of a product, of the scores in registers and of the sums empty
// up to 8 heads.)  Weights go from the first product's layout to the second's by transposing 8 x 8 matrices of bf16 within the warp.
//
// Cells meet the tensor cores as whole numbers in fp16 or bf16, which hold all of them exactly, made from their bits (0x64 beside a byte u is 1024 + u in
// fp16, 0x43 beside a nibble is 128 + it in bf16).  fp16 takes less, where the other operand fits: the queries, each head's times the power
// of two that brings its largest number to 2^8, which leaves all of bf16's digits down to 2^-22 of that; weights times the scales of bytes, in units that follow the largest.  Scales
// come in afterwards, where they are one number for a key (ST_I8: a score times its key's scale, a weight times its value's) or for 32 columns (ST_I4: partial
// scores of 32 columns, x += step acc, and what lo brings beside them, lo sum(q), by one product more; a set of weights for each 32 columns, and sum(w lo)).
// The order of a fragment's columns is free as long as both operands agree, so that no byte has to change its lane: a lane's four bytes of K are four or eight
// consecutive columns, of which the queries' fragments take the same ones.
//
// What bounds it now (64 sequences of up to 6000 tokens, 32 heads on 8 key heads of 128): of 8 bits 84 us for 377 MB; instructions, some 890 for a tile of 32 keys, are
// issued in 59 % of the cycles by twelve warps of an SM.  Of 4 bits 83 us for 189 MB, some 1160 instructions for a tile.  One sequence, window 8192: 18.3 us, five
// dependent steps (lay-out, pages, rows, pieces, joins) of some 3 us each.
#include "attn_cells_step.cuh"
#include "tc_common.cuh"
#include <cuda_fp16.h>

namespace st {
namespace attn {

namespace cstep {
constexpr int WARPS = 4, MOST_HEADS = 32;                  // warps of a block; blocks on an SM times heads of a unit
// What a unit costs a warp beside its tiles, in tiles: its queries, its results.  64 sequences of up to 6000 tokens with a cost of 1, 3 and 6: of 8 bits 88, 86 and 83 us,
// of 4 bits 83, 83 and 85.5, of 16 bits 153, 151.5 and 148; 96 sequences of up to 100 tokens 19.8, 18.9 and 19.0.
constexpr int UNIT_COST = 3;
// The shortest piece of the line that is worth a warp, in tiles.  With 1, 3 and 8: one sequence behind a window of 8192 keys 19.9, 18.4 and 22.9 us, four of up to 3000
// tokens 17.2, 19.5 and 29.3, 96 of up to 100 tokens 17.4, 18.9 and 22.6; longer batches take the same.
constexpr int LEAST = 3;
template <int DTYPE, int DP, int HN> struct Shape {
    static constexpr int HEADS = 8 * HN;                                           // of a unit
    static constexpr int BLOCKS = HN == 2 ? 2 : 3;                                 // on an SM, as registers and shared memory leave room for
    // Tiles in a ring.  Of 4 bits, whose tiles are half as large, three (64 sequences of up to 6000 tokens 83 us; two 99; two and a fourth block on the SM,
    // for which registers are few, 88); of 8 bits three leave room for two blocks only (117 us, with two 86).
    static constexpr int STAGES = DTYPE == ST_I4 ? 3 : 2;
    static constexpr int KEYS = DTYPE == ST_BF16 ? 16 : 32;                        // of a tile
    static constexpr int ROW = DTYPE == ST_BF16 ? 2 * DP : DTYPE == ST_I8 ? DP : DP / 2;       // bytes
    static constexpr int SCALES = DTYPE == ST_BF16 ? 0 : DTYPE == ST_I8 ? 1 : DP / GROUP;      // of a row, 4 bytes each
    static constexpr int PIECES = ROW / 16;
    static constexpr int TILE = KEYS * ROW, STAGE = 2 * (TILE + KEYS * SCALES * 4), RING = STAGES * STAGE;
    static constexpr size_t SMEM = (size_t)WARPS * (RING + KEYS * sizeof(int64_t));
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
__device__ __forceinline__ void load4x8x8_trans(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_half(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// The same without a sum before it.
__device__ __forceinline__ void mma_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
__device__ __forceinline__ void mma_half_first(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
        : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
// An 8 x 8 matrix of bf16, two to a lane, transposed.
__device__ __forceinline__ uint32_t transposed(uint32_t x)
{
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
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
// Two bytes of w as fp16, those that `which` picks; w holds them with 128 added (sign bits flipped).  0x64 beside u is 1024 + u.
__device__ __forceinline__ uint32_t bytes_half(uint32_t w, uint32_t which)
{
    uint32_t r;
    asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(__byte_perm(w, 0x64646464u, which)), "r"(0xE480E480u));
    return r;
}
// Nibbles i and i + 4 of w.
__device__ __forceinline__ uint32_t nibbles_bf16(uint32_t w, int i) { return minus_bf16((w >> (4 * i) & 0x000F000Fu) | 0x43004300u, 0x43004300u); }
// The same in fp16, where 0x64 above 16 u is 1024 + 16 u: odd ones need no shift.
__device__ __forceinline__ uint32_t nibbles_half(uint32_t w, int i)
{
    const uint32_t v = i >= 2 ? w >> 8 : w;
    uint32_t r;
    if (i & 1) asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"((v & 0x00F000F0u) | 0x64006400u), "r"(0x2C002C00u), "r"(0xD400D400u));
    else asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"((v & 0x000F000Fu) | 0x64006400u), "r"(0xE400E400u));
    return r;
}
__device__ __forceinline__ float low_bf16(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float high_bf16(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }

// ST_I4's scales of a row
__device__ __forceinline__ void scales_of(uint32_t (&s)[4], const uint32_t *from)
{
    const uint4 x = *reinterpret_cast<const uint4 *>(from);
    s[0] = x.x, s[1] = x.y, s[2] = x.z, s[3] = x.w;
}
__device__ __forceinline__ void scales_of(uint32_t (&s)[2], const uint32_t *from)
{
    const uint2 x = *reinterpret_cast<const uint2 *>(from);
    s[0] = x.x, s[1] = x.y;
}

// 1 / x of a power of two between 2^-126 and 2^126
__device__ __forceinline__ float inverse_of(float x) { return __uint_as_float((254u << 23) - __float_as_uint(x)); }
// Weight of a part whose largest score is m, where the largest of all is `all`.
__device__ __forceinline__ float weight_of(float m, float all, float c) { return m == -INFINITY ? 0.f : exp2f(c * (m - all)); }

// A sequence's visible keys: [0, first) and [lo, len).
struct Visible {
    int lo, first, keys;
    __device__ __forceinline__ Visible(const CellsStepArgs &a, int told)
    {
        const int len = length_of(told, a.c.cols, a.c.page);
        lo = max(0, len - a.window);
        first = min(a.sinks, lo);
        keys = first + len - lo;
    }
};
__host__ __device__ __forceinline__ int length_on_line(int tiles) { return tiles ? tiles + cstep::UNIT_COST : 0; }
// Warps that take pieces of a line of that length, the beginning of one's piece, and the one whose piece a place is in.
__device__ __forceinline__ int workers_of(int64_t total, int most) { return (int)min((int64_t)most, (total + cstep::LEAST - 1) / cstep::LEAST); }
__device__ __forceinline__ int64_t piece_of(int64_t total, int workers, int i) { return total * i / workers; }
__device__ __forceinline__ int worker_at(int64_t total, int workers, int64_t at) { return (int)(((at + 1) * workers - 1) / total); }

// The sequence that place `at` of the line is in: the last one that begins at or before it.  By a whole warp.
__device__ __forceinline__ int sequence_at(const int64_t *starts, int nseq, int64_t at)
{
    const int lane = threadIdx.x & 31;
    int lo = 0;
    for (int span = nseq, step; span > 1; span = step) {
        step = (span + 31) / 32;
        const int i = lo + (lane + 1) * step;
        const bool before = lane < 31 && i < min(lo + span, nseq) && starts[i] <= at;
        lo += __popc(__ballot_sync(~0u, before)) * step;
    }
    return lo;
}

// A team's way along its piece of the line, unit by unit (of each of the team's heads).
template <int KEYS>
struct Walk {
    int64_t left;                          // of the piece, behind the unit
    int b, unit, within;                   // the unit; places of its part of the line that are other warps'
    int told_next;                         // length of the sequence behind it, read ahead
    Visible see;
    int tiles, tile, last;                 // of the unit; the piece of it that is this warp's
    __device__ __forceinline__ Walk(const CellsStepArgs &a, int b_, int64_t within_b, int64_t left_) : left(left_), b(b_), see(a, a.c.lens[b_])
    {
        told_next = b + 1 < a.c.nseq ? a.c.lens[b + 1] : 0;
        tiles = (see.keys + KEYS - 1) / KEYS;
        const int length = max(length_on_line(tiles), 1);
        unit = (int)(within_b / length) - 1;
        within = (int)(within_b - (int64_t)(unit + 1) * length);
    }
    // On to the next unit with tiles for this warp; false: there is none.
    __device__ __forceinline__ bool next(const CellsStepArgs &a)
    {
        while (left > 0) {
            ++unit;
            while (unit == a.units / a.team || tiles == 0) {
                unit = 0;
                if (++b >= a.c.nseq) return false;
                see = Visible(a, told_next);
                told_next = b + 1 < a.c.nseq ? a.c.lens[b + 1] : 0;
                tiles = (see.keys + KEYS - 1) / KEYS;
            }
            const int take = (int)min(left, (int64_t)(length_on_line(tiles) - within));
            tile = max(0, within - cstep::UNIT_COST);
            last = within + take - cstep::UNIT_COST;
            within = 0;
            left -= take;
            if (last > tile) return true;
        }
        return false;
    }
};

// WIDE: rows and scales may be copied in 16-byte pieces, not in ones of 8 and 4 (64 sequences of 8 bits: rows of 80 bytes 76 us, of 72 bytes 101)
template <int DTYPE, int DP, int HN, bool WIDE>
__global__ void __launch_bounds__(cstep::WARPS * 32, (cstep::Shape<DTYPE, DP, HN>::BLOCKS)) cells_step_kernel(const CellsStepArgs a)
{
    using namespace cstep;
    using S = Shape<DTYPE, DP, HN>;
    constexpr int STAGES = S::STAGES, KEYS = S::KEYS, ROW = S::ROW, PIECES = S::PIECES, NK = KEYS / 16, GROUPS = DP / GROUP, HEADS = S::HEADS;
    extern __shared__ __align__(128) unsigned char smem[];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, quad = lane & 3;
    const int chunks = (a.group + HEADS - 1) / HEADS;
    const Cells &cs = a.c;
    const float c = a.scale * 1.4426950408889634f;
    unsigned char *mine = smem + warp * S::RING;
    const uint32_t ring = tc::smem_u32(mine);
    int64_t *at = (int64_t *)(smem + WARPS * S::RING) + warp * KEYS;

    // Behind a prefix's kernel too: that one's wait makes what was written before it visible to its own blocks, and says nothing of this one's.
    pdl_wait();
    pdl_trigger();
    const int64_t total = a.starts[cs.nseq];
    // few pieces go to as many SMs as there are
    const int teams = workers_of(total, a.slots / a.team), team = warp / a.team * gridDim.x + blockIdx.x, head_of_team = warp % a.team, worker = team * a.team + head_of_team;
    if (team < teams) {
        const int64_t begin = piece_of(total, teams, team), left = piece_of(total, teams, team + 1) - begin;
        const int b0 = sequence_at(a.starts, cs.nseq, begin);
        Walk<KEYS> ahead(a, b0, begin - a.starts[b0], left), here = ahead;
        bool more = ahead.next(a), bad = false;

        // Lane r finds row r of the tile after: where it lies in the pages of keys (those of values lie alike), and its scales; -1: nowhere.
        int64_t cell = -1, scale = 0;
        bool coming = false;                               // there is a tile whose places these are
        auto look = [&] {
            cell = -1;
            coming = more;
            if (!more) return;
            const int u = ahead.tile * KEYS + (lane & (KEYS - 1)), s = u < ahead.see.first ? u : ahead.see.lo + u - ahead.see.first;
            if (u < ahead.see.keys) {
                const Place p = place_of(s, cs.page, cs.page_magic);
                const int page = cs.table[(int64_t)ahead.b * cs.cols + p.col], hk = (ahead.unit * a.team + head_of_team) / chunks;
                if ((unsigned)page < (unsigned)cs.pages) {
                    cell = page * cs.page_stride + p.slot * cs.token_stride + hk * cs.head_stride;
                    scale = page * cs.scale_page + p.slot * cs.scale_token + hk * cs.scale_head;
                } else {
                    bad = true;
                }
            }
            if (++ahead.tile == ahead.last) more = ahead.next(a);
        };
        const int piece = lane % PIECES, row0 = lane / PIECES;
        const int bytes = DTYPE == ST_BF16 ? 2 * cs.d - piece * 16 : DTYPE == ST_I8 ? cs.d - piece * 16 : cs.d / 2 - piece * 16;   // of the row from this piece on
        constexpr int ROWS = 32 / PIECES;                  // rows that a warp copies at a time
        constexpr unsigned ALL = KEYS == 32 ? ~0u : 0xFFFFu;
        // Copies the tile whose places were found.  Bit r: row r is there; what is not there is zeros.
        auto fetch = [&](int stage) -> unsigned {
            const unsigned there = __ballot_sync(~0u, cell >= 0 && lane < KEYS);
            if (coming) {
                const uint32_t dst = ring + stage * S::STAGE;
                __syncwarp();
                if (lane < KEYS) at[lane] = max(cell, (int64_t)0);
                if (DTYPE != ST_BF16) {
                    const bool in = cell >= 0;
                    const uint32_t *ks = cs.k_scales + (in ? scale : 0), *vs = cs.v_scales + (in ? scale : 0);
                    const uint32_t o = dst + 2 * S::TILE + lane * S::SCALES * 4;
                    const int n = (cs.d + GROUP - 1) / GROUP;
                    if (DTYPE == ST_I8) {
                        copy_async<4>(o, ks, in);
                        copy_async<4>(o + KEYS * 4, vs, in);
                    } else if (WIDE && DP == 128) {
                        copy_async<16>(o, ks, in);
                        copy_async<16>(o + KEYS * S::SCALES * 4, vs, in);
                    } else {
#pragma unroll
                        for (int p = 0; p < S::SCALES; ++p) {
                            const int at_p = p < n ? p : 0;
                            copy_async<4>(o + p * 4, ks + at_p, in && p < n);
                            copy_async<4>(o + KEYS * S::SCALES * 4 + p * 4, vs + at_p, in && p < n);
                        }
                    }
                }
                __syncwarp();
                if (WIDE && there == ALL && bytes > 0) {
                    const unsigned char *k = cs.k + piece * 16, *v = cs.v + piece * 16;
#pragma unroll
                    for (int i = 0; i < KEYS / ROWS; ++i) {
                        const int row = row0 + i * ROWS;
                        const int64_t from = at[row];
                        const uint32_t o = dst + row * ROW + ((piece ^ S::swizzle(row)) << 4);
                        copy_async<16>(o, k + from, true);
                        copy_async<16>(o + S::TILE, v + from, true);
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < KEYS / ROWS; ++i) {
                        const int row = row0 + i * ROWS;
                        const bool in = (there >> row & 1) && bytes > 0;
                        const int64_t from = at[row] + (bytes > 0 ? piece * 16 : 0);
                        const uint32_t o = dst + row * ROW + ((piece ^ S::swizzle(row)) << 4);
                        if (WIDE) {
                            copy_async<16>(o, cs.k + from, in);
                            copy_async<16>(o + S::TILE, cs.v + from, in);
                        } else {
                            const int next = bytes > 8 ? 8 : 0;
                            copy_async<8>(o, cs.k + from, in);
                            copy_async<8>(o + 8, cs.k + from + next, in && bytes > 8);
                            copy_async<8>(o + S::TILE, cs.v + from, in);
                            copy_async<8>(o + S::TILE + 8, cs.v + from + next, in && bytes > 8);
                        }
                    }
                }
            }
            asm volatile("cp.async.commit_group;" ::: "memory");
            return there;
        };
        unsigned there[STAGES];
        look();
#pragma unroll
        for (int s = 0; s < STAGES - 1; ++s) {
            there[s] = fetch(s);
            look();
        }
        int stage = 0;
        while (here.next(a)) {
            const int unit = here.unit * a.team + head_of_team, hk = unit / chunks, g0 = unit % chunks * HEADS, g = min(a.group - g0, HEADS);
            const int64_t head0 = hk * a.group + g0;
            // The queries as fragments: column = head lane / 4; which rows (columns of q) a lane has is what its bytes of K are.
            uint32_t q[DP / 16][HN][2];
#pragma unroll
            for (int n = 0; n < HN; ++n) {
                const int head = n * 8 + lane / 4;
                const unsigned short *from = reinterpret_cast<const unsigned short *>(a.q + here.b * a.q_row + (head0 + head) * a.q_head);
#pragma unroll
                for (int k = 0; k < DP / 16; ++k)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        const int col = DTYPE == ST_BF16 ? k * 16 + quad * 2 + j * 8 : DTYPE == ST_I8 ? k * 16 + quad * 4 + j * 2 : (k / 2) * 32 + quad * 8 + (k & 1) * 2 + j;
                        q[k][n][j] = 0u;
                        if (head < g && col < cs.d)        // rows are whole eights of columns
                            q[k][n][j] = DTYPE == ST_I4 ? (uint32_t)from[col] | (uint32_t)from[col + 4] << 16 : *reinterpret_cast<const uint32_t *>(from + col);
                    }
            }
            // ST_I8, ST_I4: as fp16, times a power of two; unit[n][i] is what scores are in, for the two heads of this lane's scores
            float unit_c[HN][2], unit_of[HN][2];
#pragma unroll
            for (int n = 0; n < HN; ++n) {
                float in = 1.f;
                if (DTYPE != ST_BF16) {
                    unsigned top = 0;
#pragma unroll
                    for (int k = 0; k < DP / 16; ++k)
#pragma unroll
                        for (int j = 0; j < 2; ++j) top = max(top, max(q[k][n][j] & 0x7FFFu, q[k][n][j] >> 16 & 0x7FFFu));
                    top = max(top, __shfl_xor_sync(~0u, top, 1));
                    top = max(top, __shfl_xor_sync(~0u, top, 2));
                    const int exponent = top >> 7;         // of the largest, with 127 added
                    const float f = __uint_as_float((unsigned)min(262 - exponent, 254) << 23);
                    in = exp2f((float)(127 - min(262 - exponent, 254)));
#pragma unroll
                    for (int k = 0; k < DP / 16; ++k)
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const __half2 two = __floats2half2_rn(low_bf16(q[k][n][j]) * f, high_bf16(q[k][n][j]) * f);
                            q[k][n][j] = *reinterpret_cast<const uint32_t *>(&two);
                        }
                }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    unit_of[n][i] = DTYPE != ST_BF16 ? __shfl_sync(~0u, in, (2 * quad + i) * 4) : 1.f;
                    // above 0 whatever the scale: 0 times a score of -inf would be no number (2^-149 times any score moves a weight by 2^-21 of it at most)
                    unit_c[n][i] = DTYPE != ST_BF16 ? fmaxf(c * unit_of[n][i], 1.4e-45f) : c;
                }
            }
            // ST_I4: sums of 32 columns of the queries, which meet a key's lowest numbers in a product of their own: rows 0 to 3 of it (32 columns each) are the
            // sums' first 8 bits, 4 to 7 the next 8 and 8 to 11 the last 8.
            uint32_t qsum[HN][2];
            if (DTYPE == ST_I4)
#pragma unroll
                for (int n = 0; n < HN; ++n) {
                    float s[4], part[4];
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        s[p] = 0.f;
                        if (p < GROUPS)
#pragma unroll
                            for (int k = 2 * p; k < 2 * p + 2; ++k)
#pragma unroll
                                for (int j = 0; j < 2; ++j) {
                                    const float2 two = __half22float2(*reinterpret_cast<const __half2 *>(&q[k][n][j]));
                                    s[p] += two.x + two.y;
                                }
                        s[p] += __shfl_xor_sync(~0u, s[p], 1);
                        s[p] += __shfl_xor_sync(~0u, s[p], 2);
                    }
                    qsum[n][0] = qsum[n][1] = 0u;
#pragma unroll
                    for (int i = 0; i < 3; ++i) {
#pragma unroll
                        for (int p = 0; p < 4; ++p) {
                            part[p] = __bfloat162float(__float2bfloat16(s[p]));
                            s[p] -= part[p];
                        }
                        if (quad / 2 == (i & 1)) qsum[n][i / 2] = quad & 1 ? pair_bf16(part[2], part[3]) : pair_bf16(part[0], part[1]);
                    }
                }
            // o: rows are columns of the values, columns heads 2 quad and 2 quad + 1
            float o[DP / 16][HN][4], most[HN][2], sum[HN][2];
            // ST_I8: weights times their values' scales are multiplied as fp16, times the power of two unit_w that leaves the largest of a head's between 1 and
            // 2^15; high: that largest one, when unit_w was set
            float unit_w[HN][2], high[HN][2];
            float low[HN][2][GROUPS];                      // ST_I4: what the values' lowest numbers bring to 32 columns
            unsigned any = 0;                              // whether a key of this piece is there
#pragma unroll
            for (int n = 0; n < HN; ++n) {
#pragma unroll
                for (int k = 0; k < DP / 16; ++k)
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[k][n][i] = 0.f;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    most[n][i] = -INFINITY;
                    sum[n][i] = 0.f;
                    unit_w[n][i] = 1.f;
                    high[n][i] = 0.f;
#pragma unroll
                    for (int p = 0; p < GROUPS; ++p) low[n][i][p] = 0.f;
                }
            }
            auto attend = [&](int stage, unsigned there) {
                const uint32_t K = ring + stage * S::STAGE, V = K + S::TILE;
                const uint32_t *kscale = reinterpret_cast<const uint32_t *>(mine + stage * S::STAGE + 2 * S::TILE) + lane / 4 * S::SCALES, *vscale = kscale + KEYS * S::SCALES;
                float x[NK][HN][4];                                // keys lane / 4 (and 8 more) of 16, heads 2 quad and 2 quad + 1
#pragma unroll
                for (int h = 0; h < NK; ++h) {
#pragma unroll
                    for (int n = 0; n < HN; ++n)
#pragma unroll
                        for (int i = 0; i < 4; ++i) x[h][n][i] = 0.f;
                    const int row = h * 16 + (lane & 15);
                    const uint32_t at_row = K + row * ROW;
                    if (DTYPE == ST_BF16) {
#pragma unroll
                        for (int k = 0; k < DP / 16; ++k) {
                            uint32_t f[4];                         // 16 keys, 16 columns
                            load4x8x8(f, at_row + (((k * 2 + lane / 16) ^ S::swizzle(row)) << 4));
#pragma unroll
                            for (int n = 0; n < HN; ++n) mma(x[h][n], f, q[k][n][0], q[k][n][1]);
                        }
                    } else if (DTYPE == ST_I8) {
#pragma unroll
                        for (int k = 0; k < DP / 32; ++k) {
                            uint32_t f[4];                         // 16 keys, 32 columns
                            load4x8x8(f, at_row + (((k * 2 + lane / 16) ^ S::swizzle(row)) << 4));
#pragma unroll
                            for (int m = 0; m < 4; ++m) f[m] ^= 0x80808080u;
#pragma unroll
                            for (int m = 0; m < 2; ++m) {
                                const uint32_t c[4] = {bytes_half(f[2 * m], 0x4140u), bytes_half(f[2 * m + 1], 0x4140u), bytes_half(f[2 * m], 0x4342u), bytes_half(f[2 * m + 1], 0x4342u)};
#pragma unroll
                                for (int n = 0; n < HN; ++n) mma_half(x[h][n], c, q[2 * k + m][n][0], q[2 * k + m][n][1]);
                            }
                        }
                        const float s0 = __uint_as_float(kscale[h * 16]), s1 = __uint_as_float(kscale[h * 16 + 8]);
#pragma unroll
                        for (int n = 0; n < HN; ++n) {
                            x[h][n][0] *= s0;
                            x[h][n][1] *= s0;
                            x[h][n][2] *= s1;
                            x[h][n][3] *= s1;
                        }
                    } else {
                        // scales of 32 columns each, of keys lane / 4 and 8 more
                        uint32_t s0[GROUPS], s1[GROUPS];
                        scales_of(s0, kscale + h * 16 * S::SCALES);
                        scales_of(s1, kscale + (h * 16 + 8) * S::SCALES);
                        const bool second = GROUPS == 4 && quad & 1;
                        const uint32_t lo0 = __byte_perm(second ? s0[GROUPS - 2] : s0[0], second ? s0[GROUPS - 1] : s0[1], 0x7632);
                        const uint32_t lo1 = __byte_perm(second ? s1[GROUPS - 2] : s1[0], second ? s1[GROUPS - 1] : s1[1], 0x7632);
                        const uint32_t lows[4] = {lo0, lo1, lo0, lo1};
#pragma unroll
                        for (int n = 0; n < HN; ++n) mma_first(x[h][n], lows, qsum[n][0], qsum[n][1]);
#pragma unroll
                        for (int k = 0; k < DP / 64; ++k) {
                            uint32_t f[4];                         // 16 keys, 64 columns
                            load4x8x8(f, at_row + (((k * 2 + lane / 16) ^ S::swizzle(row)) << 4));
#pragma unroll
                            for (int m = 0; m < 2; ++m) {
                                const int p = 2 * k + m;
                                float y[HN][4];
#pragma unroll
                                for (int j = 0; j < 2; ++j) {
                                    const uint32_t c[4] = {nibbles_half(f[2 * m], 2 * j), nibbles_half(f[2 * m + 1], 2 * j), nibbles_half(f[2 * m], 2 * j + 1), nibbles_half(f[2 * m + 1], 2 * j + 1)};
#pragma unroll
                                    for (int n = 0; n < HN; ++n) {
                                        if (j == 0) mma_half_first(y[n], c, q[2 * p][n][0], q[2 * p][n][1]);
                                        else mma_half(y[n], c, q[2 * p + 1][n][0], q[2 * p + 1][n][1]);
                                    }
                                }
#pragma unroll
                                for (int n = 0; n < HN; ++n)
#pragma unroll
                                    for (int i = 0; i < 2; ++i) {
                                        x[h][n][i] = fmaf(low_bf16(s0[p]), y[n][i], x[h][n][i]);
                                        x[h][n][2 + i] = fmaf(low_bf16(s1[p]), y[n][2 + i], x[h][n][2 + i]);
                                    }
                            }
                        }
                    }
                }
                if (there != ALL) {
                    const unsigned mine = there >> (lane / 4);
#pragma unroll
                    for (int h = 0; h < NK; ++h)
#pragma unroll
                        for (int n = 0; n < HN; ++n)
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (!(mine >> (h * 16 + i / 2 * 8) & 1u)) x[h][n][i] = -INFINITY;
                }
                float top[HN][2];
                bool moves = false;
#pragma unroll
                for (int n = 0; n < HN; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float m = fmaxf(x[0][n][i], x[0][n][2 + i]);
#pragma unroll
                        for (int h = 1; h < NK; ++h) m = fmaxf(m, fmaxf(x[h][n][i], x[h][n][2 + i]));
#pragma unroll
                        for (int e = 4; e < 32; e <<= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, e));
                        top[n][i] = m;
                        moves = moves || unit_c[n][i] * (m - most[n][i]) > 8.f;
                    }
                // as long as no weight passes 2^8 the reference stays: any reference gives the same quotient
                const bool moved = __any_sync(~0u, moves);
                if (moved) {
#pragma unroll
                    for (int n = 0; n < HN; ++n)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float now = fmaxf(most[n][i], top[n][i]), f = now == -INFINITY ? 1.f : exp2f(unit_c[n][i] * (most[n][i] - now));
                            most[n][i] = now;
                            sum[n][i] *= f;
                            high[n][i] *= f;
                            if (DTYPE == ST_I4)
#pragma unroll
                                for (int p = 0; p < GROUPS; ++p) low[n][i][p] *= f;
#pragma unroll
                            for (int k = 0; k < DP / 16; ++k) {
                                o[k][n][i] *= f;
                                o[k][n][2 + i] *= f;
                            }
                        }
                }
                // Weights as fragments: heads lane / 4, keys 2 quad and 2 quad + 1 (and 8 more); those of ST_I4 are made for each 32 columns below.  Rounded to one bf16
                // number, a weight would add as much error to a result as the result's own rounding (0.0025 in the root mean square, not 0.0017; of 4 bits, where step
                // sum(w c) and sum(w lo) cancel, up to 0.0042): two of them beside bf16 values and nibbles, and one in fp16 beside bytes, 2^-12 of it or,
                // below 2^-14, 2^-25 of the largest (64 sequences of 8 bits 89 us with two bf16 numbers there, 88 so; of 4 bits 75 with one, 83 with two, where one
                // in fp16 would want a unit for each 32 columns).
                uint32_t p[NK][HN][2], rest[NK][HN][2];
#pragma unroll
                for (int h = 0; h < NK; ++h) {
                    const float s0 = DTYPE == ST_I8 ? __uint_as_float(vscale[h * 16]) : 1.f, s1 = DTYPE == ST_I8 ? __uint_as_float(vscale[h * 16 + 8]) : 1.f;
#pragma unroll
                    for (int n = 0; n < HN; ++n) {
                        float *y = x[h][n];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            y[i] = exp2_fast(fmaf(unit_c[n][i & 1], y[i], most[n][i & 1] == -INFINITY ? 0.f : -unit_c[n][i & 1] * most[n][i & 1]));
                            sum[n][i & 1] += y[i];
                        }
                        if (DTYPE == ST_BF16) {
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const uint32_t whole = pair_bf16(y[2 * i], y[2 * i + 1]);
                                p[h][n][i] = transposed(whole);
                                rest[h][n][i] = transposed(pair_bf16(y[2 * i] - low_bf16(whole), y[2 * i + 1] - high_bf16(whole)));
                            }
                        } else if (DTYPE == ST_I8) {
#pragma unroll
                            for (int i = 0; i < 4; ++i) y[i] *= i < 2 ? s0 : s1;
                        }
                    }
                }
                if (DTYPE == ST_I8) {
                    float all[HN][2];
                    bool over = moved;                     // the first tile among them
#pragma unroll
                    for (int n = 0; n < HN; ++n)
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            float m = fmaxf(x[0][n][i], x[0][n][2 + i]);
#pragma unroll
                            for (int h = 1; h < NK; ++h) m = fmaxf(m, fmaxf(x[h][n][i], x[h][n][2 + i]));
                            all[n][i] = m;
                            over = over || m * unit_w[n][i] > 32768.f;
                        }
                    if (__any_sync(~0u, over)) {
#pragma unroll
                        for (int n = 0; n < HN; ++n)
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                float m = all[n][i];
#pragma unroll
                                for (int e = 4; e < 32; e <<= 1) m = fmaxf(m, __shfl_xor_sync(~0u, m, e));
                                high[n][i] = fmaxf(high[n][i], m);
                                const int exponent = __float_as_uint(high[n][i]) >> 23;            // 255: not finite, and so is the result
                                const float now = exponent == 255 ? unit_w[n][i] : __uint_as_float((unsigned)min(max(254 - exponent, 1), 253) << 23);
                                const float f = fminf(now * inverse_of(unit_w[n][i]), 8.5e37f);    // finite, also where it meets sums of nothing
                                unit_w[n][i] = now;
#pragma unroll
                                for (int k = 0; k < DP / 16; ++k) {
                                    o[k][n][i] *= f;
                                    o[k][n][2 + i] *= f;
                                }
                            }
                    }
#pragma unroll
                    for (int h = 0; h < NK; ++h)
#pragma unroll
                        for (int n = 0; n < HN; ++n)
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const __half2 two = __floats2half2_rn(x[h][n][2 * i] * unit_w[n][0], x[h][n][2 * i + 1] * unit_w[n][1]);
                                p[h][n][i] = transposed(*reinterpret_cast<const uint32_t *>(&two));
                            }
                }
#pragma unroll
                for (int h = 0; h < NK; ++h) {
                    const int row = h * 16 + (lane & 15);
                    const uint32_t at_row = V + row * ROW;
                    if (DTYPE == ST_BF16) {
#pragma unroll
                        for (int k = 0; k < DP / 16; ++k) {
                            uint32_t f[4];                         // 16 keys, 16 columns: columns 0..7 of keys 0..7 and 8..15, then 8..15
                            load4x8x8_trans(f, at_row + (((k * 2 + lane / 16) ^ S::swizzle(row)) << 4));
                            const uint32_t c[4] = {f[0], f[2], f[1], f[3]};
#pragma unroll
                            for (int n = 0; n < HN; ++n) {
                                mma(o[k][n], c, p[h][n][0], p[h][n][1]);
                                mma(o[k][n], c, rest[h][n][0], rest[h][n][1]);
                            }
                        }
                    } else if (DTYPE == ST_I8) {
#pragma unroll
                        for (int k = 0; k < DP / 32; ++k) {
                            uint32_t f[4];                         // 16 keys, 32 columns: of 16, even ones are rows 0..7 of a product and odd ones rows 8..15
                            load4x8x8_trans(f, at_row + (((k * 2 + lane / 16) ^ S::swizzle(row)) << 4));
#pragma unroll
                            for (int m = 0; m < 4; ++m) f[m] ^= 0x80808080u;
#pragma unroll
                            for (int m = 0; m < 2; ++m) {
                                const uint32_t c[4] = {bytes_half(f[2 * m], 0x4240u), bytes_half(f[2 * m], 0x4341u), bytes_half(f[2 * m + 1], 0x4240u), bytes_half(f[2 * m + 1], 0x4341u)};
#pragma unroll
                                for (int n = 0; n < HN; ++n) mma_half(o[2 * k + m][n], c, p[h][n][0], p[h][n][1]);
                            }
                        }
                    } else {
                        uint32_t v0[GROUPS], v1[GROUPS];
                        scales_of(v0, vscale + h * 16 * S::SCALES);
                        scales_of(v1, vscale + (h * 16 + 8) * S::SCALES);
#pragma unroll
                        for (int k = 0; k < DP / 64; ++k) {
                            uint32_t f[4];                         // 16 keys, 64 columns: of four neighbours, two are rows 0..7 and 8..15 of one product, two of the next
                            load4x8x8_trans(f, at_row + (((k * 2 + lane / 16) ^ S::swizzle(row)) << 4));
#pragma unroll
                            for (int m = 0; m < 2; ++m) {
                                const int group = 2 * k + m;
                                const uint32_t s0 = v0[group], s1 = v1[group];
                                uint32_t w[HN][2], more[HN][2];
#pragma unroll
                                for (int n = 0; n < HN; ++n) {
                                    const float *y = x[h][n];
#pragma unroll
                                    for (int i = 0; i < 2; ++i) {
                                        const float step = low_bf16(i ? s1 : s0), w0 = y[2 * i] * step, w1 = y[2 * i + 1] * step;
                                        const uint32_t whole = pair_bf16(w0, w1);
                                        w[n][i] = transposed(whole);
                                        more[n][i] = transposed(pair_bf16(w0 - low_bf16(whole), w1 - high_bf16(whole)));
                                    }
#pragma unroll
                                    for (int i = 0; i < 2; ++i) low[n][i][group] = fmaf(y[i], high_bf16(s0), fmaf(y[2 + i], high_bf16(s1), low[n][i][group]));
                                }
#pragma unroll
                                for (int j = 0; j < 2; ++j) {
                                    const uint32_t c[4] = {nibbles_bf16(f[2 * m], 2 * j), nibbles_bf16(f[2 * m], 2 * j + 1), nibbles_bf16(f[2 * m + 1], 2 * j), nibbles_bf16(f[2 * m + 1], 2 * j + 1)};
#pragma unroll
                                    for (int n = 0; n < HN; ++n) {
                                        mma(o[2 * group + j][n], c, w[n][0], w[n][1]);
                                        mma(o[2 * group + j][n], c, more[n][0], more[n][1]);
                                    }
                                }
                            }
                        }
                    }
                }
            };
            for (int tile = here.tile; tile < here.last; ++tile) {
                there[STAGES - 1] = fetch(stage == 0 ? STAGES - 1 : stage - 1);              // the stage before was read by all lanes
                look();
                asm volatile("cp.async.wait_group %0;" ::"n"(STAGES - 1) : "memory");
                __syncwarp();
                any |= there[0];
                attend(stage, there[0]);
                __syncwarp();
#pragma unroll
                for (int s = 0; s + 1 < STAGES; ++s) there[s] = there[s + 1];
                if (++stage == STAGES) stage = 0;
            }

            if (DTYPE == ST_I8)
#pragma unroll
                for (int n = 0; n < HN; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i)
#pragma unroll
                        for (int k = 0; k < DP / 16; ++k) {
                            o[k][n][i] *= inverse_of(unit_w[n][i]);
                            o[k][n][2 + i] *= inverse_of(unit_w[n][i]);
                        }

            // A whole unit's output is done; with a prefix it goes to where the prefix's parts lie, a piece to where pieces are joined.
            const bool whole = here.tile == 0 && here.last == here.tiles, done = whole && !a.part_count;
            const int64_t slot = ((int64_t)worker * 2 + (here.tile > 0 ? 0 : 1)) * HEADS;
            const int64_t rows = (int64_t)cs.nseq * a.group, part = (int64_t)a.own_part * (a.heads / a.group) + hk, id = (int64_t)here.b * a.group + g0;
#pragma unroll
            for (int n = 0; n < HN; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) {
#pragma unroll
                    for (int e = 4; e < 32; e <<= 1) {
                        sum[n][i] += __shfl_xor_sync(~0u, sum[n][i], e);
                        if (DTYPE == ST_I4)
#pragma unroll
                            for (int p = 0; p < GROUPS; ++p) low[n][i][p] += __shfl_xor_sync(~0u, low[n][i][p], e);
                    }
                    const int head = n * 8 + 2 * quad + i, r = lane / 4;
                    if (head >= g) continue;
                    // a sum of 0 says that there is no key; where there are, of scores -inf all, it is 1, of weight 0
                    const bool least = most[n][i] == -INFINITY && any != 0u && sum[n][i] == 0.f;
                    if (!done && r == 0) {
                        (whole ? a.part_most + part * rows + id : a.slot_most + slot)[head] = most[n][i] * unit_of[n][i];
                        (whole ? a.part_sum + part * rows + id : a.slot_sum + slot)[head] = least ? 1.f : sum[n][i];
                    }
                    const float f = !done ? 1.f : any ? (least ? NAN : 1.f / sum[n][i]) : 0.f;
                    bf16 *out = a.out + ((int64_t)here.b * a.heads + head0 + head) * cs.d;
                    float *values = a.slot + (slot + head) * DP;
                    // four columns from `col` on of the output, or of where it goes to be joined
                    auto put4 = [&](int col, float x, float y, float z, float w) {
                        if (!done) *reinterpret_cast<float4 *>(whole ? a.part + ((part * (DP / 4) + col / 4) * rows + id + head) * 4 : values + col) = make_float4(x, y, z, w);
                        else if (col < cs.d) *reinterpret_cast<uint2 *>(out + col) = make_uint2(pair_bf16(x * f, y * f), pair_bf16(z * f, w * f));
                    };
                    auto put2 = [&](int col, float x, float y) {
                        if (!done) *reinterpret_cast<float2 *>(whole ? a.part + ((part * (DP / 4) + col / 4) * rows + id + head) * 4 + col % 4 : values + col) = make_float2(x, y);
                        else if (col < cs.d) *reinterpret_cast<uint32_t *>(out + col) = pair_bf16(x * f, y * f);
                    };
                    auto put1 = [&](int col, float x) {
                        if (!done) (whole ? a.part + ((part * (DP / 4) + col / 4) * rows + id + head) * 4 + col % 4 : values + col)[0] = x;
                        else if (col < cs.d) out[col] = __float2bfloat16(x * f);
                    };
                    // the rows of a product's results, as the values' cells lay
                    if (DTYPE == ST_BF16)
#pragma unroll
                        for (int k = 0; k < DP / 16; ++k) {
                            put1(k * 16 + r, o[k][n][i]);
                            put1(k * 16 + r + 8, o[k][n][2 + i]);
                        }
                    if (DTYPE == ST_I8)
#pragma unroll
                        for (int k = 0; k < DP / 16; ++k) put2(k * 16 + r * 2, o[k][n][i], o[k][n][2 + i]);
                    if (DTYPE == ST_I4)
#pragma unroll
                        for (int k = 0; k < GROUPS; ++k)
                            put4(k * 32 + r * 4, o[2 * k][n][i] + low[n][i][k], o[2 * k][n][2 + i] + low[n][i][k], o[2 * k + 1][n][i] + low[n][i][k],
                                 o[2 * k + 1][n][2 + i] + low[n][i][k]);
                }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        if (__any_sync(~0u, bad) && lane == 0) atomicExch(a.status + kWsStatusWord, (unsigned)ST_ERR_DEV_BOUNDS);
    }
}

// Units that several warps had pieces of, and all of them where prefixes have parts; what has no visible key is 0.  A block to a unit, or to a quarter of its
// columns where units are few, four columns of a head to a thread, and several threads for the same columns where there are pieces enough: each goes through its pieces and parts once, with the largest score and
// the sum of those so far, a few on their way at a time.
namespace cstep {
constexpr int JOIN = 512;                  // threads at most
}
// BATCH pieces on their way at a time: 8 of them where there are pieces alone (one sequence of 8192 keys 19.2 us, with 4 20.6), 4 beside a prefix's parts, where
// the registers of 8 leave an SM one block (8 sequences behind one prefix 21.6 and 24.9 us).
template <int DP, int BATCH>
__global__ void __launch_bounds__(cstep::JOIN) cells_join_kernel(const CellsStepArgs a, int unit_heads, int keys_of_tile, int quarters)
{
    using namespace cstep;
    __shared__ float4 joined[JOIN];
    __shared__ float most_j[JOIN], sum_j[JOIN];
    const Cells &cs = a.c;
    const int chunks = (a.group + unit_heads - 1) / unit_heads, unit = blockIdx.x / quarters, b = blockIdx.y;
    const int hk = unit / chunks, g0 = unit % chunks * unit_heads, g = min(a.group - g0, unit_heads);
    const float c = a.scale * 1.4426950408889634f;
    pdl_wait();
    pdl_trigger();
    const int64_t total = a.starts[cs.nseq], start = a.starts[b];
    const int prefix = a.part_count ? min(a.part_count[b], a.own_part) : 0, tiles = (Visible(a, cs.lens[b]).keys + keys_of_tile - 1) / keys_of_tile;
    int t0 = 0, pieces = 0;                                // the teams whose pieces its first tile and its last are in
    if (tiles) {
        const int teams = workers_of(total, a.slots / a.team);
        const int64_t from = start + (int64_t)(unit / a.team) * length_on_line(tiles) + UNIT_COST;
        t0 = worker_at(total, teams, from);
        pieces = worker_at(total, teams, from + tiles - 1) - t0 + 1;
    }
    if (pieces == 1 && !a.part_count) return;
    // a unit that one warp had the whole of is among the parts
    const int n = pieces == 1 ? 0 : pieces, parts = prefix + (pieces == 1), threads = blockDim.x;
    const int64_t rows = (int64_t)cs.nseq * a.group, id = (int64_t)b * a.group + g0;
    auto slot_of = [&](int i) { return ((int64_t)((t0 + i) * a.team + unit % a.team) * 2 + (i == 0 ? 1 : 0)) * unit_heads; };
    auto part_of = [&](int i) { return (int64_t)(i < prefix ? i : a.own_part) * (a.heads / a.group) + hk; };
    // heads next to one another, as they lie in the parts
    const int quads = DP / 4 / quarters, quad0 = blockIdx.x % quarters * quads, items = g * quads, slices = max(1, threads / items), slice = slices > 1 ? threadIdx.x / items : 0;
    for (int e0 = 0; e0 < items; e0 += threads) {
        const int e = slices > 1 ? threadIdx.x % items : e0 + threadIdx.x, row = e % g, quad4 = quad0 + e / g;
        const bool busy = slice < slices && e < items;
        float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
        float all = -INFINITY, s = 0.f;
        bool seen = false;
        auto more = [&](float m, float l, const float4 &x) {
            const float now = fmaxf(all, m), f = weight_of(all, now, c), w = weight_of(m, now, c);
            y = make_float4(fmaf(w, x.x, y.x * f), fmaf(w, x.y, y.y * f), fmaf(w, x.z, y.z * f), fmaf(w, x.w, y.w * f));
            s = fmaf(w, l, s * f);
            all = now;
            seen = seen || l != 0.f;
        };
        // the pieces from this slice on, then the parts; what there is no more of is what has no key
        auto go = [&](int count, auto most, auto sum, auto values) {
            for (int i0 = slice; i0 < count; i0 += BATCH * slices) {
                float m[BATCH], l[BATCH];
                float4 x[BATCH];
#pragma unroll
                for (int u = 0; u < BATCH; ++u) {
                    const int i = i0 + u * slices;
                    m[u] = -INFINITY;
                    l[u] = 0.f;
                    x[u] = make_float4(0.f, 0.f, 0.f, 0.f);
                    if (i >= count) continue;
                    m[u] = *most(i);
                    l[u] = *sum(i);
                    x[u] = *reinterpret_cast<const float4 *>(values(i));
                }
#pragma unroll
                for (int u = 0; u < BATCH; ++u)
                    if (i0 + u * slices < count) more(m[u], l[u], x[u]);
            }
        };
        if (busy) {
            go(n, [&](int i) { return a.slot_most + slot_of(i) + row; }, [&](int i) { return a.slot_sum + slot_of(i) + row; },
               [&](int i) { return a.slot + (slot_of(i) + row) * DP + quad4 * 4; });
            go(parts, [&](int i) { return a.part_most + part_of(i) * rows + id + row; }, [&](int i) { return a.part_sum + part_of(i) * rows + id + row; },
               [&](int i) { return a.part + ((part_of(i) * (DP / 4) + quad4) * rows + id + row) * 4; });
        }
        if (slices > 1) {
            joined[threadIdx.x] = y;
            most_j[threadIdx.x] = all;
            sum_j[threadIdx.x] = seen && s == 0.f ? (all == -INFINITY ? 1.f : 0.f) : s;
            __syncthreads();
            if (busy && slice == 0)
                for (int i = 1; i < slices; ++i) more(most_j[i * items + e], sum_j[i * items + e], joined[i * items + e]);
        }
        if (busy && slice == 0 && quad4 * 4 < cs.d) {
            // no visible key: 0; otherwise a sum of 0 (all scores are -inf) or NaN gives NaN
            const float f = seen ? (s == 0.f ? NAN : 1.f / s) : 0.f;
            *reinterpret_cast<uint2 *>(a.out + ((int64_t)b * a.heads + hk * a.group + g0 + row) * cs.d + quad4 * 4) =
                make_uint2(pair_bf16(y.x * f, y.y * f), pair_bf16(y.z * f, y.w * f));
        }
    }
}

// Sums up the tiles of all sequences; one block, so that it may clear the status and then report lengths that the tables do not hold.  With groups of sequences it
// takes the largest offset so far for each group's beginning: groups of offsets that decrease would have sequences in common, whose parts two blocks write.
__global__ void __launch_bounds__(1024) cells_plan_kernel(const CellsStepArgs a, int keys_of_tile)
{
    __shared__ int64_t sums[32];
    __shared__ int64_t before;
    __shared__ int mosts[32], most_before;
    pdl_trigger();
    pdl_wait();
    const Cells &cs = a.c;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    bool fine = true;
    if (threadIdx.x == 0) before = 0, most_before = 0;
    const int ends = a.group_offsets ? a.groups + 1 : 0;
    for (int i0 = 0; i0 < max(cs.nseq, ends); i0 += blockDim.x) {
        const int i = i0 + threadIdx.x, told_group = i < ends ? a.group_offsets[i] : 0;
        int64_t mine = 0;
        if (i < cs.nseq) {
            const int told = cs.lens[i];
            fine = fine && told == length_of(told, cs.cols, cs.page);
            mine = (int64_t)length_on_line((Visible(a, told).keys + keys_of_tile - 1) / keys_of_tile) * (a.units / a.team);
            if (a.part_count) a.part_count[i] = 0;
        }
        int64_t sum = mine;
        int most = min(max(told_group, 0), cs.nseq);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int64_t x = __shfl_up_sync(~0u, sum, o);
            if (lane >= o) sum += x;
            if (ends) most = max(most, __shfl_up_sync(~0u, most, o));          // of lanes without one before them, their own
        }
        if (lane == 31) sums[warp] = sum, mosts[warp] = most;
        __syncthreads();
        if (warp == 0) {
            int64_t s = lane < warps ? sums[lane] : 0;
            int m = lane < warps ? mosts[lane] : 0;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const int64_t x = __shfl_up_sync(~0u, s, o);
                if (lane >= o) s += x;
                m = max(m, __shfl_up_sync(~0u, m, o));
            }
            sums[lane] = s;
            mosts[lane] = m;
        }
        __syncthreads();
        const int64_t at = before + (warp ? sums[warp - 1] : 0) + sum;
        if (i < cs.nseq) a.starts[i + 1] = at;
        most = max(most, max(most_before, warp ? mosts[warp - 1] : 0));
        if (i < ends) {
            a.group_cuts[i] = most;
            fine = fine && told_group == most;
        }
        __syncthreads();
        if (threadIdx.x == blockDim.x - 1) before = at, most_before = most;
        __syncthreads();
    }
    fine = __syncthreads_and(fine);
    if (threadIdx.x == 0) {
        a.starts[0] = 0;
        a.status[kWsStatusWord] = fine ? 0u : (unsigned)ST_ERR_DEV_BOUNDS;
        a.status[kWsDetailWord] = 0u;
    }
}

StepPlan step_plan(int64_t nseq, size_t from)
{
    StepPlan p;
    const size_t rows = (size_t)sm_count_or_default() * cstep::MOST_HEADS * cstep::WARPS * 2;
    p.starts = round_up(from, 256);
    p.most = round_up(p.starts + (nseq + 1) * sizeof(int64_t), 256);
    p.sum = p.most + rows * sizeof(float);
    p.values = p.sum + rows * sizeof(float);
    p.bytes = p.values + rows * 128 * sizeof(float);
    return p;
}

void place_step(CellsStepArgs &a, const StepPlan &p, void *ws)
{
    char *at = (char *)ws;
    a.starts = (int64_t *)(at + p.starts);
    a.slot_most = (float *)(at + p.most);
    a.slot_sum = (float *)(at + p.sum);
    a.slot = (float *)(at + p.values);
}

size_t attn_step_workspace(int64_t nseq) { return nseq > 0 && nseq <= 65535 ? step_plan(nseq, kWsHeaderBytes).bytes : 0; }

// Query heads of a unit: up to 8 of them take half of the products of 16.  64 sequences with 16 heads to a key head, as one unit of 16 and as two of 8, which
// read the cells twice: of 16 bits 139 and 159 us, of 8 bits 93 and 112, of 4 bits 123 and 155.
static int unit_heads(const CellsStepArgs &a) { return a.group <= 8 ? 8 : 16; }
static int tile_keys(int dtype) { return dtype == ST_BF16 ? 16 : 32; }

st_status plan_step(CellsStepArgs &a, int dtype, cudaStream_t stream)
{
    a.units = a.heads / a.group * ((a.group + unit_heads(a) - 1) / unit_heads(a));
    a.team = a.units % 4 == 0 ? 4 : a.units % 2 == 0 ? 2 : 1;
    return launch(cells_plan_kernel, dim3(1), a.c.nseq > 256 ? 1024 : 256, 0, stream, a, tile_keys(dtype));
}

template <int DTYPE, int DP, int HN, bool WIDE>
static st_status run_heads(CellsStepArgs a, unsigned what, cudaStream_t stream)
{
    using S = cstep::Shape<DTYPE, DP, HN>;
    static_assert(S::BLOCKS * S::HEADS <= cstep::MOST_HEADS && S::KEYS == (DTYPE == ST_BF16 ? 16 : 32), "as the workspace and the plan have it");
    if (!ensure_dynamic_smem(cells_step_kernel<DTYPE, DP, HN, WIDE>, S::SMEM)) return ST_ERR_CUDA;
    const int blocks = sm_count_or_default() * S::BLOCKS;
    a.slots = blocks * cstep::WARPS;
    if (what & STEP_UNITS) {
        const st_status rc = launch(cells_step_kernel<DTYPE, DP, HN, WIDE>, dim3((unsigned)blocks), cstep::WARPS * 32, S::SMEM, stream, a);
        if (rc != ST_OK) return rc;
    }
    if (!(what & STEP_JOIN)) return ST_OK;
    // few units may have many pieces each
    const bool few = (int64_t)a.units * a.c.nseq < 2 * sm_count_or_default();
    const int quarters = few ? 4 : 1;
    return launch(a.part_count ? cells_join_kernel<DP, 4> : cells_join_kernel<DP, 8>, dim3((unsigned)(a.units * quarters), (unsigned)a.c.nseq), few ? 512 : 128, 0, stream, a,
                  S::HEADS, S::KEYS, quarters);
}

template <int DTYPE, int DP, bool WIDE>
static st_status run_cells(const CellsStepArgs &a, unsigned what, cudaStream_t stream)
{
    return unit_heads(a) == 8 ? run_heads<DTYPE, DP, 1, WIDE>(a, what, stream) : run_heads<DTYPE, DP, 2, WIDE>(a, what, stream);
}

st_status run_cells_step(const CellsStepArgs &a, int dtype, unsigned what, cudaStream_t stream)
{
    const bool small = a.c.d <= 64;
    const int64_t row = row_bytes(dtype, a.c.d);
    bool wide = row % 16 == 0 && a.c.page_stride % 16 == 0 && a.c.token_stride % 16 == 0 && a.c.head_stride % 16 == 0;
    if (dtype == ST_BF16) return small ? run_cells<ST_BF16, 64, true>(a, what, stream) : run_cells<ST_BF16, 128, true>(a, what, stream);
    if (dtype == ST_I8) {
        if (small) return wide ? run_cells<ST_I8, 64, true>(a, what, stream) : run_cells<ST_I8, 64, false>(a, what, stream);
        return wide ? run_cells<ST_I8, 128, true>(a, what, stream) : run_cells<ST_I8, 128, false>(a, what, stream);
    }
    if (!small) wide = wide && a.c.d > 96 && a.c.scale_page % 4 == 0 && a.c.scale_token % 4 == 0 && a.c.scale_head % 4 == 0;
    if (small) return wide ? run_cells<ST_I4, 64, true>(a, what, stream) : run_cells<ST_I4, 64, false>(a, what, stream);
    return wide ? run_cells<ST_I4, 128, true>(a, what, stream) : run_cells<ST_I4, 128, false>(a, what, stream);
}

st_status check_step(const st_cells *c, const void *q, int64_t q_row, int64_t q_head, float scale, const void *out)
{
    if (c->nseq > 65535) return ST_ERR_UNSUPPORTED;
    if (!q || !out) return ST_ERR_NULL;
    if (!stride_ok(c->nseq, q_row, c->d) || !stride_ok(c->heads, q_head, c->d)) return ST_ERR_SHAPE;
    if (q_row > ((int64_t)1 << 38) || q_head > ((int64_t)1 << 38) || !(scale > 0.f && scale < INFINITY)) return ST_ERR_UNSUPPORTED;
    if ((c->nseq > 1 && q_row % 8 != 0) || (c->heads > 1 && q_head % 8 != 0) || !aligned16(q) || !aligned16(out)) return ST_ERR_ALIGN;
    // a place on the line of work times the number of warps stays below 2^63
    if (c->nseq * c->heads * (c->page * c->table_cols / 16 + cstep::UNIT_COST + 1) > ((int64_t)1 << 50)) return ST_ERR_UNSUPPORTED;
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
    const StepPlan plan = step_plan(c->nseq, kWsHeaderBytes);
    if (!ws || ws_bytes < plan.bytes) return ST_ERR_WORKSPACE;
    if (!aligned256(ws)) return ST_ERR_ALIGN;
    CellsStepArgs a = step_args(c, q, q_row, q_head, k_pages, v_pages, k_scales, v_scales, table, lens, scale, out, ws);
    a.window = clamp_int(window, 1 << 30);
    a.sinks = clamp_int(sinks, 1 << 30);
    const int64_t bytes = c->nseq * c->heads * c->d * 2;
    // a unit's output is written when all that reads its queries is done
    const Operand Q = {q, c->nseq, c->heads, c->d, a.q_row, a.q_head};
    if (Q.under(out, bytes, true) || meets_cells(c, k_pages, k_scales, out, bytes) || meets_cells(c, v_pages, v_scales, out, bytes) ||
        arrays_meet(out, bytes, table, c->nseq * c->table_cols * 4) || arrays_meet(out, bytes, lens, c->nseq * 4))
        return ST_ERR_UNSUPPORTED;
    place_step(a, plan, ws);
    if ((rc = plan_step(a, c->dtype, (cudaStream_t)stream)) != ST_OK) return rc;
    return run_cells_step(a, c->dtype, STEP_UNITS | STEP_JOIN, (cudaStream_t)stream);
}
