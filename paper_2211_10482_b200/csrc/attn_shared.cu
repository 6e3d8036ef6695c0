// st_attn_shared_step: one token of every sequence over a prefix that its group of sequences shares, then over its own tokens.
//
// Two kernels, between one that lays out the work and one that joins.  The first is the single-token kernel over each sequence's own keys.  The second
// takes all queries of a group that read one key head as the rows of a matrix, up to 256 of them, and makes
//     S = Q K^T  (tcgen05, fp32 in tensor memory);   P = exp2(c S - c m)  (two threads per row);   O += P V
// over a range of the prefix's keys, as st_attn_window does for a tile of a prompt; it leaves (m, l, O) as a part, and the pieces of the own keys are joined
// with the parts.  A row of the prefix is so read once for 256 queries, not once for every sequence.  (The prefix's blocks, which fill their SMs, are set up
// while the own tokens' last ones run; the other way round nothing of the second kernel is under way when the first ends: 116 and 112.6 us for 128 sequences.)
//
// Pages whose length divides a tile of 128 keys, or is a multiple of it, come by TMA, a box to a page: one warp looks the pages up and asks for them.  A page
// that is not there is a box outside the tensor and so zeros; values behind the last key are cleared.  Pages of other lengths are gathered by cp.async
// into the swizzled tiles that the tensor cores read, by one or two warps for each stage, which copy, see the copies done, make them visible to the tensor
// cores' proxy and hand the tile over.  (128 sequences behind two prefixes, the whole call: with pages of 64 122 us, with pages of 100, which are gathered, 157.)
// Either way a bit of a mask says which keys have a place.
//
// Weights meet the values as two bf16 numbers each, P and behind it in tensor memory what is left of P, in place of the scores: two products where one would do, and
// none of the error that one would add (0.0022 and 0.0023 in the root mean square of the two cases below, where a result's own rounding is 0.0017).  128 sequences behind two prefixes
// 113.3 to 122.2 us, 8 samples of one prompt 30.8 to 31.6.  (Splitting weights by cutting bits off instead of rounding takes as long: 122.8.)
//
// A tile of keys takes some 4900 cycles where it meets two tiles of rows, whose six products of 128 x 128 x 128 take 512 each: one tile's weights (scores from
// tensor memory, maxima, an exchange with the other half's thread, 64 exponentials) are made while the other one's products run, and in turns, as without them both tiles
// wanted the exponentials at once and the tensor cores then (with one number to a weight 107.4 us for 114.9; with one thread to a row and no turns 112;
// with weights handed over in quarters 113.5).
//
// Which part of which prefix a block takes is decided on the device, where the lengths are: key tiles of a part are as many as give no more parts than there
// are blocks in one turn on the SMs.
#include "attn_cells_step.cuh"
#include "attn_tc.cuh"

namespace st {
namespace attn {

struct SharedArgs {
    CellsStepArgs step;
    const int *prefix_table, *prefix_lens;
    int groups, prefix_cols;
    int seqs;                              // of a tile of rows
    int slots, most_parts;                 // blocks, parts of a prefix
    float *part_most, *part_sum, *part;
};

namespace shared {
// TILES of 128 rows; with one there is room for a third stage of keys and values, whose bytes bound few rows, and for a second warp to copy each
template <int DP, int TILES, bool BOXES> struct Shape {
    static constexpr int STAGES = TILES == 1 ? 3 : 2;
    static constexpr int TILE_BYTES = DP / 64 * SLAB;
    static constexpr int SOFTMAX = 8 * TILES, ISSUE = SOFTMAX, COPY = ISSUE + TILES, COPIERS = BOXES ? 1 : 2 / TILES, WARPS = COPY + (BOXES ? 1 : COPIERS * STAGES), THREADS = WARPS * 32;
    static constexpr int TMEM = TILES == 1 ? 256 : 512;            // columns: S of every tile, O of every tile
    static constexpr size_t SMEM = 1024 + (size_t)TILE_BYTES * (TILES + 2 * STAGES) + 512 + TILES * 2 * TILE * sizeof(float);
};
constexpr int MOST_ROWS = 256;
}  // namespace shared

// A cache's pages as a tensor map {column, head, token, page}, boxes of 64 columns of one head's `rows` tokens of one page.
static bool make_tmap_pages(CUtensorMap *m, const unsigned char *p, const Cells &c, uint32_t rows)
{
    const tc::EncodeTiledFn fn = tc::encode_tiled_fn();
    if (!fn) return false;
    // the stride of an extent of one is never used: whatever was passed, it is a legal one
    auto stride = [](int64_t s) { return (cuuint64_t)(s ? s : 256); };
    cuuint64_t dims[4] = {(cuuint64_t)c.d, (cuuint64_t)c.kv_heads, (cuuint64_t)c.page, (cuuint64_t)c.pages};
    cuuint64_t strides[3] = {stride(c.head_stride), stride(c.token_stride), stride(c.page_stride)};
    cuuint32_t box[4] = {64, 1, rows, 1}, estr[4] = {1, 1, 1, 1};
    return fn(m, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<unsigned char *>(p), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
              CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
__device__ __forceinline__ void tma_load_4d(void *dst, const CUtensorMap *m, uint64_t *bar, int x, int y, int z, int w)
{
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
        ::"r"(tc::smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(m)), "r"(tc::smem_u32(bar)), "r"(x), "r"(y), "r"(z), "r"(w)
        : "memory");
}

__device__ __forceinline__ void copy_row(uint32_t dst, const void *src, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}

// Key tiles of a group's prefix, tiles of its rows, and what a key tile costs with one of these: 8 where the 256 rows are two products, else 7.  Nothing hangs on the
// exact ratio (128 sequences 122 us with 4 to 3 and 9 to 8 too; with none 131), nor at 64 columns, where none is as good (95.8 and 95.3 us).
struct GroupOf {
    Rows seqs;
    int tiles, keys, cost;
    __device__ __forceinline__ int parts(int work) const { return (keys * cost + work - 1) / work; }
};
__device__ __forceinline__ GroupOf group_of(const SharedArgs &a, int i)
{
    if (i >= a.groups) return {{0, 0}, 0, 0, 7};
    const Rows r = rows_of(a.step.group_cuts, i, a.step.c.nseq);
    const int len = length_of(a.prefix_lens[i], a.prefix_cols, a.step.c.page);
    return {r, (r.len + a.seqs - 1) / a.seqs, (len + TILE - 1) / TILE, (int64_t)r.len * a.step.group > TILE ? 8 : 7};
}

// Part `part` of `parts` of a tile of rows; none: group -1.
struct PartOf {
    int group, tile, part, parts;
};
// By a whole warp: the least work in a part that needs no more parts than there are blocks, and no more of one prefix than there is room for, 32 candidates at
// a time (6000 cycles with the loads ahead of it; one after the other 5500 to 10000); then what block `index` of one key head does.
__device__ __forceinline__ PartOf part_of(const SharedArgs &a, int index, int kv_heads, int lane)
{
    const GroupOf mine = group_of(a, lane);                // all there is, up to 32 groups
    const int chunks = (a.groups + 31) / 32;
    auto chunk = [&](int i) { return i == 0 ? mine : group_of(a, i * 32 + lane); };
    int most = 0, least = 1;
    for (int i = 0; i < chunks; ++i) {
        const GroupOf g = chunk(i);
        if (g.tiles) {
            most = max(most, g.keys * g.cost);
            least = max(least, (g.keys + a.most_parts - 1) / a.most_parts * g.cost);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
        most = max(most, __shfl_xor_sync(~0u, most, o));
        least = max(least, __shfl_xor_sync(~0u, least, o));
    }
    if (most == 0) return {-1, 0, 0, 0};
    const int room = max(a.slots / kv_heads, 1);
    int lo = min(least, most), hi = most;                  // at `most` every tile of rows is one part, for which there is room
    while (lo < hi) {
        const int step = (hi - lo + 31) / 32, mid = min(lo + lane * step, hi);
        int64_t parts = 0;
        for (int i = 0; i < chunks; ++i) {
            const GroupOf g = chunk(i);
            const int work = g.keys * g.cost, n = min(32, a.groups - i * 32);
            for (int l = 0; l < n; ++l) parts += (int64_t)__shfl_sync(~0u, g.tiles, l) * ((__shfl_sync(~0u, work, l) + mid - 1) / mid);
        }
        const unsigned fits = __ballot_sync(~0u, parts <= room || mid == hi);
        if (!fits) {                                       // the last candidate is short of hi
            lo = lo + 31 * step + 1;
        } else {
            const int l = __ffs(fits) - 1;
            hi = min(lo + l * step, hi);
            if (l > 0) lo = lo + (l - 1) * step + 1;
        }
    }
    for (int i = 0; i < chunks; ++i) {
        const GroupOf g = chunk(i);
        const int parts = g.parts(lo), here = g.tiles * parts;
        int sum = here;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(~0u, sum, o);
            if (lane >= o) sum += x;
        }
        const unsigned behind = __ballot_sync(~0u, index < sum);
        if (behind) {
            const int l = __ffs(behind) - 1, rest = index - __shfl_sync(~0u, sum - here, l), n = __shfl_sync(~0u, parts, l);
            return {i * 32 + l, rest / n, rest % n, n};
        }
        index -= __shfl_sync(~0u, sum, 31);
    }
    return {-1, 0, 0, 0};
}

template <int DP, int TILES, bool BOXES>
__global__ void __launch_bounds__((shared::Shape<DP, TILES, BOXES>::THREADS), 1)
shared_prefix_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const SharedArgs a)
{
    using namespace tc;
    using S = shared::Shape<DP, TILES, BOXES>;
    constexpr int STAGES = S::STAGES, SLOTS = 2 * STAGES, PIECES = DP / 8, COPIERS = S::COPIERS;
    extern __shared__ unsigned char raw[];
    unsigned char *smem = align_smem(raw);
    unsigned char *Q = smem, *K = Q + TILES * S::TILE_BYTES, *V = K + STAGES * S::TILE_BYTES;
    // bit k of word [k / 32] of a tile: key k has a place.  Tile i's words are written again for tile i + SLOTS, whose keys are copied after the values of tile
    // i + STAGES, and these after the product with tile i's weights: the words have been read, and no wait on their barrier can meet a phase too far.
    uint32_t *valid = (uint32_t *)(V + STAGES * S::TILE_BYTES);        // [SLOTS][4]
    uint64_t *bars = (uint64_t *)(valid + SLOTS * 4);
    uint64_t *k_full = bars, *k_empty = k_full + STAGES, *v_full = k_empty + STAGES, *v_empty = v_full + STAGES, *q_full = v_empty + STAGES,
             *s_full = q_full + TILES, *p_full = s_full + TILES, *o_full = p_full + 2 * TILES, *valid_full = o_full + TILES, *copied = valid_full + SLOTS, *turn = copied + 1;
    uint32_t *tmem_slot = (uint32_t *)(turn + 4 * TILES);
    float *halves = (float *)(valid + 512 / 4);            // [TILES][2][128]: what the halves of the rows have to tell one another
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1), *met = abort_flag + 1;         // met: a page outside the cache
    const Cells &cs = a.step.c;
    const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
    const int group = a.step.group, kv_heads = cs.kv_heads, hk = blockIdx.x % kv_heads;

    if (BOXES && warp == S::COPY && lane < 2) prefetch_tmap(lane ? &vmap : &kmap);
    pdl_wait();
    pdl_trigger();
    if (blockIdx.x == 0) {
        bool fine = true;
        for (int i = threadIdx.x; i < a.groups; i += S::THREADS)
            fine = fine && a.prefix_lens[i] == length_of(a.prefix_lens[i], a.prefix_cols, cs.page);
        if (!fine) atomicExch(a.step.status + kWsStatusWord, (unsigned)ST_ERR_DEV_BOUNDS);
    }
    const PartOf at = part_of(a, blockIdx.x / kv_heads, kv_heads, lane);
    if (at.group < 0) return;
    const GroupOf mine = group_of(a, at.group);
    const int b0 = mine.seqs.first + at.tile * a.seqs, seqs = min(a.seqs, mine.seqs.len - at.tile * a.seqs), rows = seqs * group;
    const int len = length_of(a.prefix_lens[at.group], a.prefix_cols, cs.page);
    const int first = (int)((int64_t)mine.keys * at.part / at.parts), n = (int)((int64_t)mine.keys * (at.part + 1) / at.parts) - first;      // key tiles
    const int active = TILES == 2 && rows > TILE ? 2 : 1;  // tiles of rows that there are

    // The queries' rows, 16 (8) lanes to a row, on their way while the rest is set up; what is no row is zeros.
    constexpr int LOADS = PIECES / 2;                      // of a lane: 16 rows of PIECES pieces to a warp
    uint4 queries[LOADS];
    if (warp < S::SOFTMAX && warp / 8 < active)
#pragma unroll
        for (int j = 0; j < LOADS; ++j) {
            const int piece = lane % PIECES, id = warp * 16 + lane / PIECES + j * (32 / PIECES), b = id / group;
            const bf16 *from = a.step.q + (b0 + b) * a.step.q_row + (hk * group + id - b * group) * a.step.q_head + piece * 8;
            queries[j] = id < rows && piece * 8 < cs.d ? *reinterpret_cast<const uint4 *>(from) : make_uint4(0u, 0u, 0u, 0u);
        }

    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(&k_full[s], COPIERS);
            mbar_init(&v_full[s], COPIERS);
            mbar_init(&k_empty[s], active);
            mbar_init(&v_empty[s], active);
        }
        for (int s = 0; s < SLOTS; ++s) mbar_init(&valid_full[s], COPIERS);
        mbar_init(copied, 1);
        for (int w = 0; w < TILES; ++w) {
            mbar_init(&q_full[w], 8);
            mbar_init(&s_full[w], 1);
            mbar_init(&o_full[w], 1);
            mbar_init(&p_full[2 * w], 4);
            mbar_init(&p_full[2 * w + 1], 4);
            for (int i = 0; i < 4; ++i) mbar_init(&turn[4 * w + i], 2);
        }
        *abort_flag = 0;
        *met = 0;
        fence_barrier_init();
    }
    if (warp == S::ISSUE) {
        tmem_alloc(tmem_slot, S::TMEM);
        tmem_relinquish();
    }
    if (hk == 0 && at.part == 0)
        for (int i = threadIdx.x; i < seqs; i += S::THREADS) a.step.part_count[b0 + i] = at.parts;
    // BOXES: a lane to a box, `box` keys of one page; a page that is not there is one behind the last.  The first tile's are looked up during the set-up.
    const int *table = a.prefix_table + (int64_t)at.group * a.prefix_cols;
    const int box = min(cs.page, TILE), boxes = TILE / box;
    int next_page = 0, next_slot = 0;
    bool missing = false;
    auto look = [&](int i) {
        const int key = (first + i) * TILE + lane * box;
        next_page = cs.pages;
        next_slot = 0;
        if (i >= n || lane >= boxes || key >= len) return;
        const Place p = place_of(key, cs.page, cs.page_magic);
        const int page = table[p.col];
        next_slot = p.slot;
        missing = (unsigned)page >= (unsigned)cs.pages;
        if (!missing) next_page = page;
    };
    if (BOXES && warp == S::COPY) look(0);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(~0u, *tmem_slot, 0);

    if (BOXES && warp == S::COPY) {
        bool ok = true;
        for (int i = 0; i < n && ok; ++i) {
            const int page = next_page, in_page = next_slot;
            if (missing) *met = 1;                         // said before the tile's rows are asked for
            const int s = i % STAGES, use = i / STAGES, slot = (use & 1) * STAGES + s;
            const uint32_t parity = (uint32_t)((use + 1) & 1);
            // bits of this lane's word: 32 keys, which may be several boxes or a part of one
            unsigned word = 0;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const bool there = __shfl_sync(~0u, page, (w * 32 + lane) / box) < cs.pages && (first + i) * TILE + w * 32 + lane < len;
                const unsigned bits = __ballot_sync(~0u, there);
                if (lane == w) word = bits;
            }
            const int left = len - (first + i) * TILE;     // keys from here on
            const bool edge = left < TILE;
            ok = warp_wait(&k_empty[s], parity, abort_flag, a.step.status, 1);
            if (!ok) break;
            if (lane < 4) valid[slot * 4 + lane] = word;
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(&valid_full[slot]);
                mbar_expect_tx(&k_full[s], S::TILE_BYTES);
            }
            __syncwarp();
            auto ask = [&](unsigned char *tile, const CUtensorMap *map, uint64_t *bar) {
                if (lane < boxes)
#pragma unroll
                    for (int c = 0; c < DP / 64; ++c) tma_load_4d(tile + c * SLAB + lane * box * 128, map, bar, c * 64, hk, in_page, page);
            };
            ask(K + s * S::TILE_BYTES, &kmap, &k_full[s]);
            look(i + 1);
            ok = warp_wait(&v_empty[s], parity, abort_flag, a.step.status, 2);
            if (!ok) break;
            uint64_t *bar = edge ? copied : &v_full[s];
            if (lane == 0) mbar_expect_tx(bar, S::TILE_BYTES);
            __syncwarp();
            ask(V + s * S::TILE_BYTES, &vmap, bar);
            if (edge) {                                    // the last tile: what lies behind the last key may be anything
                ok = warp_wait(copied, 0, abort_flag, a.step.status, 11);
                if (!ok) break;
                clear_rows<DP>(V + s * S::TILE_BYTES, left, TILE, lane);
                if (lane == 0) mbar_arrive(&v_full[s]);
            }
        }
    } else if (!BOXES && warp >= S::COPY) {
        // each copies 128 / COPIERS keys of a stage; 16 (8) lanes to a row
        constexpr int KEYS = TILE / COPIERS, WORDS = KEYS / 32;
        const int s = (warp - S::COPY) / COPIERS, half = (warp - S::COPY) % COPIERS;
        const unsigned char *kc = cs.k + hk * cs.head_stride, *vc = cs.v + hk * cs.head_stride;
        const int piece = lane % PIECES, row0 = lane / PIECES;
        constexpr int ROWS = 32 / PIECES;                  // rows that a warp copies at a time
        const bool inside = piece * 8 < cs.d;
        const uint32_t to = (uint32_t)(piece / 8 * SLAB + half * KEYS * 128);
        bool ok = true;
        int64_t next[WORDS];                               // places of this lane's keys of the tile after
        auto place = [&](int i) {
#pragma unroll
            for (int e = 0; e < WORDS; ++e) {
                const int key = (first + i) * TILE + half * KEYS + e * 32 + lane;
                next[e] = -1;
                if (i >= n || key >= len) continue;
                const Place p = place_of(key, cs.page, cs.page_magic);
                const int page = table[p.col];
                if ((unsigned)page < (unsigned)cs.pages) next[e] = page * cs.page_stride + p.slot * cs.token_stride;
                else *met = 1;
            }
        };
        place(s);
        for (int i = s, use = 0; i < n && ok; i += STAGES, ++use) {
            int64_t from[WORDS];
            unsigned there[WORDS];
#pragma unroll
            for (int e = 0; e < WORDS; ++e) {
                from[e] = next[e];
                there[e] = __ballot_sync(~0u, from[e] >= 0);
            }
            const uint32_t parity = (uint32_t)((use + 1) & 1);
            auto copy = [&](uint32_t tile, const unsigned char *src) {
#pragma unroll
                for (int e = 0; e < WORDS; ++e)
#pragma unroll 4
                    for (int r = 0; r < 32; r += ROWS) {
                        const int row = e * 32 + r + row0;
                        const int64_t o = __shfl_sync(~0u, from[e], r + row0);
                        copy_row(tile + to + row * 128 + (((piece & 7) ^ (row & 7)) << 4), src + (o < 0 ? 0 : o) + (inside ? piece * 16 : 0), o >= 0 && inside);
                    }
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
            ok = warp_wait(&k_empty[s], parity, abort_flag, a.step.status, 1);
            if (!ok) break;
            const int slot = (use & 1) * STAGES + s;
#pragma unroll
            for (int e = 0; e < WORDS; ++e)
                if (lane == 0) valid[slot * 4 + half * WORDS + e] = there[e];
            if (lane == 0) mbar_arrive(&valid_full[slot]);
            copy(smem_u32(K + s * S::TILE_BYTES), kc);
            ok = warp_wait(&v_empty[s], parity, abort_flag, a.step.status, 2);
            if (!ok) break;
            copy(smem_u32(V + s * S::TILE_BYTES), vc);
            place(i + STAGES);
            asm volatile("cp.async.wait_group 1;" ::: "memory");
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(&k_full[s]);
            asm volatile("cp.async.wait_group 0;" ::: "memory");
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(&v_full[s]);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
    } else if (warp >= S::ISSUE && warp < S::COPY) {
        // A tile of rows has a warp that issues its products: the scores of a tile of keys follow the product with the values of the one before, whose weights
        // they overwrite (products are carried out in the order of their issue).
        const int w = warp - S::ISSUE;
        if (w < active) {
            const bool lead = elect_one();
            const uint32_t s_idesc = make_idesc(1, 0, 0, TILE, TILE), o_idesc = make_idesc(1, 0, 1, TILE, DP);
            const uint32_t s_col = tmem + w * TILE, o_col = tmem + TILES * TILE + w * DP;
            const unsigned char *rows_at = Q + w * S::TILE_BYTES;
            bool ok = warp_wait(&q_full[w], 0, abort_flag, a.step.status, 3);
            for (int i = 0; i <= n && ok; ++i) {
                if (i > 0) {
                    const int s = (i - 1) % STAGES;
                    const uint32_t parity = (uint32_t)((i - 1) / STAGES & 1), done = (uint32_t)((i - 1) & 1);
                    ok = warp_wait(&v_full[s], parity, abort_flag, a.step.status, 4);
                    if (ok) ok = warp_wait(&p_full[2 * w], done, abort_flag, a.step.status, 5);
                    if (!ok) break;
                    tc_fence_after();
                    mma_tokens<32, 0, 4>(lead, o_col, s_col, V + s * S::TILE_BYTES, o_idesc, i > 1);
                    mma_tokens<32, 0, 4>(lead, o_col, s_col + 64, V + s * S::TILE_BYTES, o_idesc, true);
                    ok = warp_wait(&p_full[2 * w + 1], done, abort_flag, a.step.status, 6);
                    if (!ok) break;
                    tc_fence_after();
                    mma_tokens<32, 4, 8>(lead, o_col, s_col, V + s * S::TILE_BYTES, o_idesc, true);
                    mma_tokens<32, 4, 8>(lead, o_col, s_col + 64, V + s * S::TILE_BYTES, o_idesc, true);
                    commit(lead, &v_empty[s]);
                }
                if (i == n) break;
                const int s = i % STAGES;
                ok = warp_wait(&k_full[s], (uint32_t)(i / STAGES & 1), abort_flag, a.step.status, 7);
                if (!ok) break;
                tc_fence_after();
                mma_rows<DP>(lead, s_col, rows_at, K + s * S::TILE_BYTES, s_idesc);
                commit(lead, &s_full[w]);
                commit(lead, &k_empty[s]);
            }
            if (ok) commit(lead, &o_full[w]);
            __syncwarp();
        }
    } else if (warp / 8 < active) {
        // Two threads to a row of scores, half of a tile's keys each, in warps on one scheduler.
        const int w = warp >> 3, half = warp >> 2 & 1, r = (warp & 3) * 32 + lane;                 // this thread's row of the tile
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, s_addr = tmem + lanes + w * TILE, o_addr = tmem + lanes + TILES * TILE + w * DP;
        float *mine_told = halves + (w * 2 + half) * TILE + r;
        const float *other_told = halves + (w * 2 + (half ^ 1)) * TILE + r;
        // What the other thread of the row tells.  It is read before that thread's weights are handed over, and written again after their product.  Both come here
        // as often whatever fails: the barrier of the two warps has no limit of its own.
        auto exchange = [&](float x) {
            *mine_told = x;
            tc_fence_before();
            asm volatile("bar.sync %0, 64;" ::"r"(1 + 4 * w + (warp & 3)) : "memory");
            tc_fence_after();
            return *(volatile const float *)other_told;
        };
        {
            unsigned char *to = Q + w * S::TILE_BYTES;
            const int piece = lane % PIECES;
#pragma unroll
            for (int j = 0; j < LOADS; ++j) {
                const int row = (warp & 7) * 16 + lane / PIECES + j * (32 / PIECES);
                *reinterpret_cast<uint4 *>(to + piece / 8 * SLAB + row * 128 + (((piece & 7) ^ (row & 7)) << 4)) = queries[j];
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) mbar_arrive(&q_full[w]);
        }
        const float c = a.step.scale * LOG2E;
        float m = -INFINITY, l = 0.f;
        bool ok = true, seen = false;
        for (int i = 0; i < n; ++i) {
            if (ok) ok = warp_wait(&s_full[w], (uint32_t)(i & 1), abort_flag, a.step.status, 8);
            // the bits are looked at behind the last key, and once a page was met that is not there (which is said before its rows are asked for)
            const int slot = (i / STAGES & 1) * STAGES + i % STAGES;
            const bool holes = (first + i + 1) * TILE > len || *met;
            if (ok && holes) ok = warp_wait(&valid_full[slot], (uint32_t)(i / SLOTS & 1), abort_flag, a.step.status, 9);
            if (!ok) {
                exchange(0.f);
                continue;
            }
            tc_fence_after();
            uint4 bits = make_uint4(~0u, ~0u, ~0u, ~0u);
            if (holes) bits = *reinterpret_cast<const uint4 *>(valid + slot * 4);
            const bool cut = (bits.x & bits.y & bits.z & bits.w) != ~0u;
            seen = seen || (bits.x | bits.y | bits.z | bits.w) != 0u;
            uint32_t x[2][32];
#pragma unroll
            for (int j = 0; j < 2; ++j) tmem_ld_32x32(s_addr + half * 64 + j * 32, x[j]);
            tmem_ld_wait();
            if (cut) {
                const uint32_t word[2] = {half ? bits.z : bits.x, half ? bits.w : bits.y};
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (!(word[j] >> e & 1u)) x[j][e] = __float_as_uint(-INFINITY);
            }
            float most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int e = 0; e < 32; e += 2) most[e / 2 & 3] = max3(most[e / 2 & 3], __uint_as_float(x[j][e]), __uint_as_float(x[j][e + 1]));
            float top = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
            top = fmaxf(top, exchange(top));               // both have their scores: weights may overwrite them
            // the reference moves: 8 is the factor 2^8 that P may exceed 1 by
            if (__any_sync(~0u, c * (top - m) > 8.f)) {
                const float now = fmaxf(top, m), f = now == -INFINITY ? 1.f : ex2(c * (m - now));
                m = now;
                l *= f;
                if (i > 0 && half == 0) {                  // whose weights are waited for first
#pragma unroll 1
                    for (int j = 0; j < DP / 16; ++j) {
                        uint32_t o[16];
                        tmem_ld_32x16(o_addr + j * 16, o);
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                        tmem_st_32x16(o_addr + j * 16, o);
                    }
                }
            }
            const float mc = m == -INFINITY ? 0.f : -m * c;
            const Pair cc = pair(c, c), mm = pair(mc, mc), minus = pair(-1.f, -1.f);
            Pair sum[2] = {pair(0.f, 0.f), pair(0.f, 0.f)};
            if (active == 2) {                             // one tile of rows after the other: the products of one go on under the weights of the other
                ok = warp_wait(&turn[4 * w + (warp & 3)], (uint32_t)((i + 1 - w) & 1), abort_flag, a.step.status, 13);
                if (!ok) continue;
            }
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                uint32_t p[16], rest[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float2 z = split(fma(pair(x[j][2 * e], x[j][2 * e + 1]), cc, mm));
                    const Pair y = pair(ex2(z.x), ex2(z.y));
                    sum[e & 1] = add(sum[e & 1], y);
                    p[e] = pack_bf16(y);
                    rest[e] = pack_bf16(fma(pair(p[e] << 16, p[e] & 0xFFFF0000u), minus, y));
                }
                tmem_st_32x16(s_addr + half * 32 + j * 16, p);
                tmem_st_32x16(s_addr + 64 + half * 32 + j * 16, rest);
            }
            if (active == 2 && lane == 0) mbar_arrive(&turn[4 * (w ^ 1) + (warp & 3)]);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&p_full[2 * w + half]);
            const float2 part = split(add(sum[0], sum[1]));
            l += part.x + part.y;
        }
        if (ok) ok = warp_wait(&o_full[w], 0, abort_flag, a.step.status, 10);
        const float other = exchange(l);
        l = half ? other + l : l + other;
        const int id = w * TILE + r;
        if (ok) {
            tc_fence_after();
            const int64_t all = (int64_t)cs.nseq * group, unit = (int64_t)at.part * kv_heads + hk, row = (int64_t)b0 * group + id;
            if (id < rows && half == 0) {
                a.part_most[unit * all + row] = m;
                a.part_sum[unit * all + row] = m == -INFINITY && l == 0.f ? (seen ? 1.f : 0.f) : l;
            }
            // quads of columns, rows next to one another: a warp writes 512 bytes at a time
            float4 *out = reinterpret_cast<float4 *>(a.part) + unit * (DP / 4) * all + row;
#pragma unroll 1
            for (int j = half * (DP / 32); j < (half + 1) * (DP / 32); ++j) {
                uint32_t o[16];
                tmem_ld_32x16(o_addr + j * 16, o);
                tmem_ld_wait();
                if (id < rows)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        out[(j * 4 + e) * all] = make_float4(__uint_as_float(o[4 * e]), __uint_as_float(o[4 * e + 1]), __uint_as_float(o[4 * e + 2]),
                                                             __uint_as_float(o[4 * e + 3]));
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (threadIdx.x == 0 && *met) atomicExch(a.step.status + kWsStatusWord, (unsigned)ST_ERR_DEV_BOUNDS);
    if (warp == S::ISSUE) {
        tc_fence_after();
        tmem_dealloc(tmem, S::TMEM);
    }
}

// What a call's workspace holds behind its header.
struct SharedPlan {
    int tiles_of, seqs, slots, most_parts;
    size_t counts, cuts, most, sum, part, bytes;           // where they begin
    StepPlan step;
};
static bool shared_plan(int64_t nseq, int64_t heads, int64_t kv_heads, int64_t groups, SharedPlan *p)
{
    if (nseq <= 0 || heads <= 0 || kv_heads <= 0 || heads % kv_heads != 0 || groups <= 0 || nseq > 65535 || heads > 65535 || groups > 65535 || heads / kv_heads > shared::MOST_ROWS)
        return false;
    const int64_t group = heads / kv_heads, sms = sm_count_or_default();
    p->tiles_of = nseq * group <= TILE ? 1 : 2;
    p->seqs = (int)(p->tiles_of * TILE / group);
    const int64_t least = (nseq + p->seqs - 1) / p->seqs * kv_heads, most = most_tiles(nseq, groups, p->seqs) * kv_heads;
    if (most > INT32_MAX) return false;
    p->slots = (int)(most > sms ? most : sms);
    // room for as many parts of one prefix as the SMs can take at a time, beside the other tiles of rows that there are at least
    const int64_t parts = (sms + least - 1) / least;
    p->most_parts = (int)(parts < 1 ? 1 : parts > MAX_PARTS ? MAX_PARTS : parts);
    const size_t rows = (size_t)nseq * heads * (p->most_parts + 1);        // and one for the own tokens
    p->counts = kWsHeaderBytes;
    p->cuts = round_up(p->counts + nseq * sizeof(int), 256);
    p->most = round_up(p->cuts + (groups + 1) * sizeof(int), 256);
    p->sum = round_up(p->most + rows * sizeof(float), 256);
    p->part = round_up(p->sum + rows * sizeof(float), 256);
    p->step = step_plan(nseq, p->part + rows * 128 * sizeof(float));
    p->bytes = p->step.bytes;
    return true;
}

size_t attn_shared_workspace(int64_t nseq, int64_t heads, int64_t kv_heads, int64_t groups)
{
    SharedPlan p;
    return shared_plan(nseq, heads, kv_heads, groups, &p) ? p.bytes : 0;
}

template <int DP, int TILES, bool BOXES>
static st_status launch_prefix(const SharedArgs &a, const CUtensorMap &km, const CUtensorMap &vm, cudaStream_t stream)
{
    using S = shared::Shape<DP, TILES, BOXES>;
    if (!ensure_dynamic_smem(shared_prefix_kernel<DP, TILES, BOXES>, S::SMEM)) return ST_ERR_CUDA;
    return launch(shared_prefix_kernel<DP, TILES, BOXES>, dim3((unsigned)a.slots), S::THREADS, S::SMEM, stream, km, vm, a);
}

// Pages that a tile is a whole number of, or that are a whole number of tiles, come as boxes: of 8 rows and more, as the swizzle of a tile repeats every 8.
template <int DP, int TILES>
static st_status run_prefix(const SharedArgs &a, cudaStream_t stream)
{
    const Cells &c = a.step.c;
    CUtensorMap km = {}, vm = {};
    const bool boxes = c.page >= 8 && (TILE % c.page == 0 || c.page % TILE == 0);
    if (!boxes) return launch_prefix<DP, TILES, false>(a, km, vm, stream);
    const uint32_t rows = c.page < TILE ? c.page : TILE;
    if (!make_tmap_pages(&km, c.k, c, rows) || !make_tmap_pages(&vm, c.v, c, rows)) return ST_ERR_CUDA;
    return launch_prefix<DP, TILES, true>(a, km, vm, stream);
}

}  // namespace attn
}  // namespace st

using namespace st;
using namespace st::attn;

extern "C" st_status st_attn_shared_step(const st_cells *c, const void *q, int64_t q_row, int64_t q_head, const void *k_pages, const void *v_pages,
                                         const int32_t *prefix_table, int64_t prefix_cols, const int32_t *prefix_lens, int64_t groups,
                                         const int32_t *group_offsets, const int32_t *table, const int32_t *lens, float scale, void *out, void *ws,
                                         size_t ws_bytes, void *stream)
{
    if (!c) return ST_ERR_NULL;
    if (c->dtype != ST_BF16) return ST_ERR_DTYPE;
    st_status rc = check_cells(c, k_pages, v_pages, nullptr, nullptr, table, lens);
    if (rc != ST_OK) return rc;
    if ((rc = check_step(c, q, q_row, q_head, scale, out)) != ST_OK) return rc;
    if (prefix_cols <= 0 || groups <= 0) return ST_ERR_SHAPE;
    if (groups > 65535 || prefix_cols > (1 << 30) || prefix_cols * c->page > (1 << 30) || c->heads / c->kv_heads > shared::MOST_ROWS) return ST_ERR_UNSUPPORTED;
    if (!prefix_table || !prefix_lens || (!group_offsets && groups != 1)) return ST_ERR_NULL;
    if (!aligned4(prefix_table) || !aligned4(prefix_lens) || !aligned4(group_offsets)) return ST_ERR_ALIGN;
    SharedPlan p;
    if (!shared_plan(c->nseq, c->heads, c->kv_heads, groups, &p)) return ST_ERR_UNSUPPORTED;
    if (!ws || ws_bytes < p.bytes) return ST_ERR_WORKSPACE;
    if (!aligned256(ws)) return ST_ERR_ALIGN;
    SharedArgs a = {};
    a.step = step_args(c, q, q_row, q_head, k_pages, v_pages, nullptr, nullptr, table, lens, scale, out, ws);
    // out is written when all queries have been read
    const int64_t bytes = c->nseq * c->heads * c->d * 2;
    const Operand Q = {q, c->nseq, c->heads, c->d, a.step.q_row, a.step.q_head};
    if (Q.under(out, bytes, true) || meets_cells(c, k_pages, nullptr, out, bytes) || meets_cells(c, v_pages, nullptr, out, bytes) ||
        arrays_meet(out, bytes, table, c->nseq * c->table_cols * 4) || arrays_meet(out, bytes, lens, c->nseq * 4) ||
        arrays_meet(out, bytes, prefix_table, groups * prefix_cols * 4) || arrays_meet(out, bytes, prefix_lens, groups * 4) ||
        arrays_meet(out, bytes, group_offsets, (groups + 1) * 4))
        return ST_ERR_UNSUPPORTED;
    a.prefix_table = prefix_table;
    a.prefix_lens = prefix_lens;
    a.groups = (int)groups;
    a.step.groups = (int)groups;
    a.step.group_offsets = group_offsets;
    a.step.group_cuts = group_offsets ? (int *)((char *)ws + p.cuts) : nullptr;
    a.prefix_cols = (int)prefix_cols;
    a.seqs = p.seqs;
    a.slots = p.slots;
    a.most_parts = p.most_parts;
    a.part_most = (float *)((char *)ws + p.most);
    a.part_sum = (float *)((char *)ws + p.sum);
    a.part = (float *)((char *)ws + p.part);
    place_step(a.step, p.step, ws);
    a.step.part_count = (int *)((char *)ws + p.counts);
    a.step.own_part = p.most_parts;
    a.step.part_most = a.part_most;
    a.step.part_sum = a.part_sum;
    a.step.part = a.part;
    if ((rc = plan_step(a.step, ST_BF16, (cudaStream_t)stream)) != ST_OK) return rc;
    if ((rc = run_cells_step(a.step, ST_BF16, STEP_UNITS, (cudaStream_t)stream)) != ST_OK) return rc;
    if (c->d <= 64) rc = p.tiles_of == 1 ? run_prefix<64, 1>(a, (cudaStream_t)stream) : run_prefix<64, 2>(a, (cudaStream_t)stream);
    else rc = p.tiles_of == 1 ? run_prefix<128, 1>(a, (cudaStream_t)stream) : run_prefix<128, 2>(a, (cudaStream_t)stream);
    if (rc != ST_OK) return rc;
    return run_cells_step(a.step, ST_BF16, STEP_JOIN, (cudaStream_t)stream);
}
