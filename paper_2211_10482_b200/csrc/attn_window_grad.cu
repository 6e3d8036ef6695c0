// st_attn_window_grad on the tensor cores, without atomics: one kernel for dq, one for dk and dv, both from the saved log-sum-exp.
//
//   window_dq_kernel   a block owns 128 queries of one head and passes over the tiles of keys that they see:
//                      S = Q K^T, dP = dO V^T, dS = exp(scale S - lse) (dP - delta), dQ += dS K
//                      delta = dO.O is taken on the way in and kept for the second kernel.
//   window_dkv_kernel  a block owns 128 keys of one key head and passes over the heads that share it and the tiles of queries that see it,
//                      everything transposed:  S^T = K Q^T, dP^T = V dO^T, dV += P^T dO, dK += dS^T Q
//
// Seven products instead of the five of one pass over both, in exchange for sums in a fixed order: no atomics on dq, and the sum over the
// heads that share keys stays in the accumulator.  P and dS go to tensor memory as bf16, each in the place of the fp32
// scores it was made from, and are A operands there; a thread holds one row and half of a tile's columns, and writes where it has read.
// Products and exponentials overlap: while a tile's dS is made the tensor cores work on the next tile's S.
//
// The first columns (sinks) are seen by every later query, so that their tiles of keys would take as long as the whole sequence:
// queries beyond the window are cut into parts of 256 or 1024 for blocks of their own, which leave fp32 sums of the sinks' rows in the
// workspace; window_sinks_kernel adds them in the order of the parts.
//
// Rows behind a sequence may hold anything: where they would be multiplied by weights of 0 they are cleared in shared memory.
#include "attn_window.cuh"

namespace st {
namespace attn {

namespace wgrad {
constexpr int THREADS = 320;
// Tiles of queries of a part beyond the window: short ones where their sums are few, so that these blocks take no longer than the others (4
// sequences of up to 4096 tokens, window 1024, forward and backward: parts of 256 take 18 us less than parts of 1024, of some 510).
constexpr int part_log(int64_t sinks) { return sinks <= 32 ? 1 : 3; }
constexpr int part_rows(int64_t sinks) { return TILE << part_log(sinks); }
constexpr int MAX_SPLIT_SINKS = 2 * TILE;                    // with more first columns they are no small share of the work any more
template <int DP> struct Shape {
    static constexpr int TILE_BYTES = DP / 64 * SLAB;
    static constexpr size_t DQ_SMEM = 1024 + (size_t)TILE_BYTES * 7 + TILE * sizeof(float) + 256;
    static constexpr size_t DKV_SMEM = 1024 + (size_t)TILE_BYTES * 6 + 4 * TILE * sizeof(float) + 256;
};
}  // namespace wgrad

struct WindowGradArgs {
    WindowArgs w;
    const bf16 *o, *dout;
    const float *lse;
    bf16 *dq, *dk, *dv;
    float *delta;                  // [nq, heads]
    float *parts;                  // sums of the sinks' rows: [2: near, far][tile of keys][slot][key head][2: dk, dv][rows][d]
    int nslots, sink_tiles, sink_rows;   // 0 sink_tiles: nothing is split
    int part_log;                        // a part has 2^part_log tiles of queries
};

__device__ __forceinline__ float *part_of(const WindowGradArgs &g, int far, int kt, int slot, int hk)
{
    const int kv_heads = g.w.heads / g.w.group;
    return g.parts + ((((int64_t)far * g.sink_tiles + kt) * g.nslots + slot) * kv_heads + hk) * 2 * g.sink_rows * g.w.d;
}

// The tiles of queries that see the keys s0.. of a tile: [a, near) through the window, [near, all) through the first columns only.
struct QueryTiles {
    int a, near, all;
};
__device__ __forceinline__ QueryTiles query_tiles(const Mask &m, const Rows &rq, const Rows &rk, int s0)
{
    const int64_t off = rk.len - rq.len, last = min(s0 + TILE, rk.len) - 1;
    const int n = (rq.len + TILE - 1) / TILE;
    QueryTiles q;
    q.a = (int)(max((int64_t)0, s0 - off) / TILE);
    const int64_t end = last + m.window - 1 - off;         // the last query that sees the last key through the window
    q.near = end < 0 ? 0 : (int)min((int64_t)n, end / TILE + 1);
    q.near = max(q.near, min(q.a, n));
    q.a = min(q.a, n);
    q.all = s0 < m.sinks ? n : q.near;
    return q;
}
// First query tile that is left to the parts, where a tile of keys is split.
__device__ __forceinline__ int first_part(const WindowGradArgs &g, const QueryTiles &q) { return q.near + (1 << g.part_log); }

// The sequence one of whose parts begins in rows [slot P, slot P + P) for P rows a part, and that part; by a whole warp.  Parts begin P rows
// apart and the first of a sequence more than P rows behind its beginning, so that there is one at most.
struct PartOf {
    int seq, part;
};
__device__ __forceinline__ PartOf part_at(const WindowGradArgs &g, const Mask &m, int kt, int slot, int lane)
{
    const WindowArgs &a = g.w;
    const int shift = TILE_LOG + g.part_log, rows = 1 << shift;
    for (int b0 = 0; b0 < a.nseq; b0 += 32) {
        const int b = b0 + lane;
        int part = -1;
        if (b < a.nseq) {
            const Rows rq = rows_of(a.q_offsets, b, a.nq), rk = rows_of(a.k_offsets, b, a.nk);
            if (kt * TILE < rk.len) {
                const QueryTiles q = query_tiles(m, rq, rk, kt * TILE);
                const int begin = rq.first + first_part(g, q) * TILE, p = max(0, (slot * rows - begin + rows - 1) >> shift);
                const int row = begin + p * rows;
                if (first_part(g, q) + (p << g.part_log) < q.all && row >> shift == slot) part = p;
            }
        }
        const unsigned found = __ballot_sync(~0u, part >= 0);
        if (found) {
            const int l = __ffs(found) - 1;
            return {b0 + l, __shfl_sync(~0u, part, l)};
        }
    }
    return {-1, 0};
}

// 8 values of a row, products of which are summed in fp32
__device__ __forceinline__ float dot8(uint4 x, uint4 y)
{
    const __nv_bfloat162 *a = reinterpret_cast<const __nv_bfloat162 *>(&x), *b = reinterpret_cast<const __nv_bfloat162 *>(&y);
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 u = __bfloat1622float2(a[i]), v = __bfloat1622float2(b[i]);
        s = fmaf(u.x, v.x, fmaf(u.y, v.y, s));
    }
    return s;
}

template <int DP>
__global__ void __launch_bounds__(wgrad::THREADS, 1)
window_dq_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                 const __grid_constant__ CUtensorMap domap, const __grid_constant__ CUtensorMap dqmap, const WindowGradArgs g)
{
    using namespace wgrad;
    using namespace tc;
    constexpr int BYTES = Shape<DP>::TILE_BYTES, KS = 3, VS = 2;
    const WindowArgs &a = g.w;
    extern __shared__ unsigned char raw[];
    unsigned char *smem = align_smem(raw);
    unsigned char *Q = smem, *DO = Q + BYTES, *K = DO + BYTES, *V = K + KS * BYTES;
    float *deltas = (float *)(V + VS * BYTES);
    uint64_t *bars = (uint64_t *)(deltas + TILE);
    uint64_t *q_full = bars, *do_full = bars + 1, *k_full = bars + 2, *k_copied = k_full + KS, *k_empty = k_copied + KS, *v_full = k_empty + KS,
             *v_empty = v_full + VS, *s_full = v_empty + VS, *dp_full = s_full + 2, *ds_full = dp_full + 1, *done = ds_full + 1,
             *k_first = done + 1;
    uint32_t *tmem_slot = (uint32_t *)(k_first + 1);
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);
    const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, h = blockIdx.y;

    pdl_wait();
    if (blockIdx.x == 0 && blockIdx.y == 0) {
        const bool fine = offsets_fine(a.q_offsets, a.nseq, a.nq, threadIdx.x, THREADS) && offsets_fine(a.k_offsets, a.nseq, a.nk, threadIdx.x, THREADS);
        const int all = __syncthreads_and(fine);
        if (threadIdx.x == 0) {
            a.status[kWsStatusWord] = all ? 0u : (unsigned)ST_ERR_DEV_BOUNDS;
            a.status[kWsDetailWord] = 0u;
        }
    }
    const TileOf at = tile_of(a.q_offsets, a.nseq, a.nq, TILE, blockIdx.x, lane);
    if (at.seq < 0) return;
    const Rows rq = rows_of(a.q_offsets, at.seq, a.nq), rk = rows_of(a.k_offsets, at.seq, a.nk);
    const int i0 = at.tile * TILE, left = min(rq.len - i0, TILE), t0 = i0 + rk.len - rq.len;
    const Mask mask{a.window, a.sinks};
    const KeyTiles tiles = key_tiles(mask, t0, t0 + left - 1);
    const int n = tiles.count();

    if (threadIdx.x == 0) {
        mbar_init(q_full, 1);
        mbar_init(do_full, 1);
        for (int s = 0; s < KS; ++s) {
            mbar_init(&k_full[s], 1);
            mbar_init(&k_copied[s], 1);
            mbar_init(&k_empty[s], 1);
        }
        for (int s = 0; s < VS; ++s) {
            mbar_init(&v_full[s], 1);
            mbar_init(&v_empty[s], 1);
        }
        mbar_init(&s_full[0], 1);
        mbar_init(&s_full[1], 1);
        mbar_init(dp_full, 1);
        mbar_init(ds_full, 8);
        mbar_init(done, 1);
        mbar_init(k_first, 1);
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 9) {
        tmem_alloc(tmem_slot, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(~0u, *tmem_slot, 0), dp_col = tmem + 2 * TILE, dq_col = tmem + 3 * TILE;
    pdl_trigger();

    if (warp == 8) {
        const int hk = h / a.group;
        if (lane == 0 && n > 0) {
            mbar_expect_tx(q_full, BYTES);
            load_tile<DP>(Q, &qmap, q_full, h, rq.first + i0);
            mbar_expect_tx(do_full, BYTES);
            load_tile<DP>(DO, &domap, do_full, h, rq.first + i0);
        }
        bool ok = true;
        uint32_t copied = 0;
        // the last tile of first columns, where its keys are cleared behind them: when they have come, and the next tile has been asked for
        const int cleared = tiles.cleared();
        bool clear = false;
        auto clear_first = [&] {
            clear = false;
            const int s = cleared % KS;
            ok = warp_wait(k_first, 0, abort_flag, a.status, 12);
            if (!ok) return;
            clear_rows<DP>(K + s * BYTES, tiles.unseen(), tiles.used(), lane);
            if (lane == 0) mbar_arrive(&k_full[s]);
        };
        for (int i = 0; i < n && ok; ++i) {
            const int s0 = tiles.key(i), row = rk.first + s0, s = i % KS, sv = i % VS;
            const bool edge = s0 + TILE > rk.len && i != cleared;
            if (lane == 0) {
                ok = mbar_wait(&k_empty[s], (uint32_t)((i / KS + 1) & 1), abort_flag, a.status, 1);
                if (ok) {
                    uint64_t *bar = i == cleared ? k_first : edge ? &k_copied[s] : &k_full[s];
                    mbar_expect_tx(bar, BYTES);
                    load_tile<DP>(K + s * BYTES, &kmap, bar, hk, row);
                    ok = mbar_wait(&v_empty[sv], (uint32_t)((i / VS + 1) & 1), abort_flag, a.status, 2);
                }
                if (ok) {
                    mbar_expect_tx(&v_full[sv], BYTES);
                    load_tile<DP>(V + sv * BYTES, &vmap, &v_full[sv], hk, row);
                }
            }
            ok = __shfl_sync(~0u, ok, 0);
            if (clear && ok) clear_first();
            clear = i == cleared;
            if (edge && ok) {
                ok = __all_sync(~0u, mbar_wait(&k_copied[s], (copied >> s) & 1u, abort_flag, a.status, 3));
                copied ^= 1u << s;
                if (ok) {
                    clear_rows<DP>(K + s * BYTES, rk.len - s0, TILE, lane);
                    if (lane == 0) mbar_arrive(&k_full[s]);
                }
            }
        }
        if (clear && ok) clear_first();
    } else if (warp == 9) {
        if (n > 0) {
            const bool lead = elect_one();
            const uint32_t s_idesc = make_idesc(1, 0, 0, TILE, TILE), o_idesc = make_idesc(1, 0, 1, TILE, DP), piece_idesc = make_idesc(1, 0, 0, TILE, KeyTiles::PIECE);
            bool ok = true;
            auto score = [&](int j) {
                if (!ok || j >= n) return;
                ok = warp_wait(&k_full[j % KS], (uint32_t)((j / KS) & 1), abort_flag, a.status, 4);
                if (!ok) return;
                tc_fence_after();
                mma_rows<DP>(lead, tmem + (j & 1) * TILE, Q, K + (j % KS) * BYTES, tiles.piece(j) ? piece_idesc : s_idesc);
                commit(lead, &s_full[j & 1]);
            };
            auto dprob = [&](int j) {
                if (!ok || j >= n) return;
                ok = warp_wait(&v_full[j % VS], (uint32_t)((j / VS) & 1), abort_flag, a.status, 5);
                if (!ok) return;
                tc_fence_after();
                mma_rows<DP>(lead, dp_col, DO, V + (j % VS) * BYTES, tiles.piece(j) ? piece_idesc : s_idesc);
                commit(lead, dp_full);
                commit(lead, &v_empty[j % VS]);
            };
            ok = warp_wait(q_full, 0, abort_flag, a.status, 6);
            score(0);
            if (ok) ok = warp_wait(do_full, 0, abort_flag, a.status, 7);
            dprob(0);
            score(1);
            for (int j = 0; j < n && ok; ++j) {
                ok = warp_wait(ds_full, (uint32_t)(j & 1), abort_flag, a.status, 8);
                if (!ok) break;
                tc_fence_after();
                dprob(j + 1);
                if (!ok) break;
                if (tiles.piece(j)) mma_tokens<64, 0, KeyTiles::PIECE / 16>(lead, dq_col, tmem + (j & 1) * TILE, K + (j % KS) * BYTES, o_idesc, false);
                else mma_tokens<64>(lead, dq_col, tmem + (j & 1) * TILE, K + (j % KS) * BYTES, o_idesc, j > 0);
                commit(lead, &k_empty[j % KS]);
                score(j + 2);
            }
            if (ok) commit(lead, done);
        }
        __syncwarp();
    } else {
        // thread: row r, columns 64 half .. 64 half + 63
        const int half = warp >> 2, r = (warp & 3) * 32 + lane, t = t0 + r;
        const int64_t row = rq.first + i0 + r;
        const bool mine = r < left;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
        float lse2 = 0.f;
        if (mine) {
            const float lse = g.lse[row * a.heads + h];
            lse2 = lse == -INFINITY ? 0.f : lse * LOG2E;
        }
        // delta: a warp takes 16 rows, as many lanes to a row as it has pieces of 16 bytes, all loads at once
        {
            constexpr int LANES = DP / 8, AT_ONCE = 32 / LANES, N = 16 / AT_ONCE;
            const int piece = lane % LANES, first = warp * 16 + lane / LANES;
            uint4 x[N], y[N];
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int i = first + k * AT_ONCE;
                const bool in = i < left && piece * 8 < a.d;
                const int64_t at = ((int64_t)(rq.first + i0 + i) * a.heads + h) * a.d + piece * 8;
                x[k] = in ? *reinterpret_cast<const uint4 *>(g.o + at) : make_uint4(0u, 0u, 0u, 0u);
                y[k] = in ? *reinterpret_cast<const uint4 *>(g.dout + at) : make_uint4(0u, 0u, 0u, 0u);
            }
#pragma unroll
            for (int k = 0; k < N; ++k) {
                const int i = first + k * AT_ONCE;
                float sum = dot8(x[k], y[k]);
#pragma unroll
                for (int o = LANES / 2; o; o >>= 1) sum += __shfl_xor_sync(~0u, sum, o);
                if (piece == 0) {
                    deltas[i] = sum;
                    if (i < left) g.delta[(int64_t)(rq.first + i0 + i) * a.heads + h] = sum;
                }
            }
        }
        asm volatile("bar.sync 1, 256;" ::: "memory");
        const float delta = deltas[r];
        const float c = a.scale * LOG2E;
        bool ok = true;
        for (int j = 0; j < n; ++j) {
            const uint32_t s_addr = tmem + lanes + (j & 1) * TILE + half * 64, dp_addr = dp_col + lanes + half * 64;
            const bool cut = !tiles.all(mask, t0, t0 + TILE - 1, j), piece = tiles.piece(j);
            ok = __all_sync(~0u, mbar_wait(&s_full[j & 1], (uint32_t)((j >> 1) & 1), abort_flag, a.status, 9));
            if (!ok) break;
            tc_fence_after();
            const RowMask seen = tiles.row_mask(mask, t, j);
            Pair p[2][16];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                if (piece && half + b > 0) continue;
                uint32_t x[32];
                tmem_ld_32x32(s_addr + b * 32, x);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float2 z = split(fma(pair(x[2 * e], x[2 * e + 1]), pair(c, c), pair(-lse2, -lse2)));
                    p[b][e] = pair(ex2(z.x), ex2(z.y));
                }
                if (cut) keep(p[b], seen.of(half * 64 + b * 32));
            }
            ok = __all_sync(~0u, mbar_wait(dp_full, (uint32_t)(j & 1), abort_flag, a.status, 10));
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                if (piece && half + b > 0) continue;
                uint32_t dp[32], ds[16];
                tmem_ld_32x32(dp_addr + b * 32, dp);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; ++e) p[b][e] = mul(p[b][e], add(pair(dp[2 * e], dp[2 * e + 1]), pair(-delta, -delta)));
                if (cut) keep(p[b], seen.of(half * 64 + b * 32));        // a masked weight is 0 whatever its dP is
#pragma unroll
                for (int e = 0; e < 16; ++e) ds[e] = pack_bf16(p[b][e]);
                tmem_st_32x16(s_addr + b * 16, ds);
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(ds_full);
        }
        if (ok && n > 0) ok = __all_sync(~0u, mbar_wait(done, 0, abort_flag, a.status, 11));
        if (ok) {
            tc_fence_after();
            if (half == 0) {
                store_rows<DP>(dq_col + lanes, Q, &dqmap, g.dq, (int64_t)a.heads * a.d, a.d, rq.first + i0 + (warp & 3) * 32, h, r, left - (warp & 3) * 32, 0, a.scale,
                               n == 0);
                if (lane == 0) tma_store_wait();
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

template <int DP>
__global__ void __launch_bounds__(wgrad::THREADS, 1)
window_dkv_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
                  const __grid_constant__ CUtensorMap domap, const __grid_constant__ CUtensorMap dkmap, const __grid_constant__ CUtensorMap dvmap,
                  const WindowGradArgs g)
{
    using namespace wgrad;
    using namespace tc;
    constexpr int BYTES = Shape<DP>::TILE_BYTES, ST = 2;
    const WindowArgs &a = g.w;
    extern __shared__ unsigned char raw[];
    unsigned char *smem = align_smem(raw);
    unsigned char *K = smem, *V = K + BYTES, *Q = V + BYTES, *DO = Q + ST * BYTES;
    float *stats = (float *)(DO + ST * BYTES);             // [stage][2: lse log2 e, delta][128]
    uint64_t *bars = (uint64_t *)(stats + ST * 2 * TILE);
    uint64_t *k_full = bars, *v_full = bars + 1, *q_full = bars + 2, *q_copied = q_full + ST, *q_empty = q_copied + ST, *do_full = q_empty + ST,
             *do_copied = do_full + ST, *do_empty = do_copied + ST, *s_full = do_empty + ST, *dp_full = s_full + 1, *p_full = dp_full + 1,
             *ds_full = p_full + 1, *done = ds_full + 1;
    uint32_t *tmem_slot = (uint32_t *)(done + 1);
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);
    const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, hk = blockIdx.y;

    pdl_wait();
    const Mask mask{a.window, a.sinks};
    const int far_blocks = g.sink_tiles * g.nslots;
    const bool far = (int)blockIdx.x < far_blocks;
    int seq, kt, slot = 0;
    QueryTiles qt;
    Rows rq, rk;
    if (far) {
        kt = blockIdx.x / g.nslots;
        slot = blockIdx.x % g.nslots;
        const PartOf p = part_at(g, mask, kt, slot, lane);
        if (p.seq < 0) return;
        seq = p.seq;
        rq = rows_of(a.q_offsets, seq, a.nq);
        rk = rows_of(a.k_offsets, seq, a.nk);
        qt = query_tiles(mask, rq, rk, kt * TILE);
        qt.a = first_part(g, qt) + (p.part << g.part_log);
        qt.all = min(qt.all, qt.a + (1 << g.part_log));
    } else {
        const TileOf at = tile_of(a.k_offsets, a.nseq, a.nk, TILE, blockIdx.x - far_blocks, lane);
        if (at.seq < 0) return;
        seq = at.seq;
        kt = at.tile;
        rq = rows_of(a.q_offsets, seq, a.nq);
        rk = rows_of(a.k_offsets, seq, a.nk);
        qt = query_tiles(mask, rq, rk, kt * TILE);
    }
    // rows whose sums are finished elsewhere: the sinks', where parts of the queries are left to other blocks
    int partial_rows = 0;
    if (far) {
        partial_rows = min(a.sinks - kt * TILE, TILE);
    } else if (kt < g.sink_tiles && first_part(g, qt) < qt.all) {
        partial_rows = min(a.sinks - kt * TILE, TILE);
        slot = (rq.first + first_part(g, qt) * TILE) >> (TILE_LOG + g.part_log);
        qt.all = first_part(g, qt);
    }
    const int s0 = kt * TILE, per_head = max(0, qt.all - qt.a), n = per_head * a.group, off = rk.len - rq.len;

    if (threadIdx.x == 0) {
        mbar_init(k_full, 1);
        mbar_init(v_full, 1);
        for (int s = 0; s < ST; ++s) {
            mbar_init(&q_full[s], 1);
            mbar_init(&q_copied[s], 1);
            mbar_init(&q_empty[s], 1);
            mbar_init(&do_full[s], 1);
            mbar_init(&do_copied[s], 1);
            mbar_init(&do_empty[s], 1);
        }
        mbar_init(s_full, 1);
        mbar_init(dp_full, 1);
        mbar_init(p_full, 8);
        mbar_init(ds_full, 8);
        mbar_init(done, 1);
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 9) {
        tmem_alloc(tmem_slot, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(~0u, *tmem_slot, 0), dp_col = tmem + TILE, dv_col = tmem + 2 * TILE, dk_col = tmem + 2 * TILE + DP;
    pdl_trigger();

    if (warp == 8) {
        if (lane == 0 && n > 0) {
            mbar_expect_tx(k_full, BYTES);
            load_tile<DP>(K, &kmap, k_full, hk, rk.first + s0);
            mbar_expect_tx(v_full, BYTES);
            load_tile<DP>(V, &vmap, v_full, hk, rk.first + s0);
        }
        bool ok = true;
        uint32_t copied = 0;
        int h = hk * a.group, tile = qt.a;
        for (int i = 0; i < n && ok; ++i) {
            const int s = i % ST, i0 = tile * TILE;
            const uint32_t parity = (uint32_t)((i / ST + 1) & 1);
            const int unseen = -off - i0;              // rows before the first key, which may hold anything
            const bool edge = i0 + TILE > rq.len || unseen > 0;
            float lse[4], delta[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const int j = i0 + k * 32 + lane;
                const bool in = j < rq.len && k * 32 + lane >= unseen;
                const int64_t at = (int64_t)(rq.first + j) * a.heads + h;
                lse[k] = in ? g.lse[at] : -INFINITY;
                delta[k] = in ? g.delta[at] : 0.f;
            }
            ok = __all_sync(~0u, mbar_wait(&q_empty[s], parity, abort_flag, a.status, 1));
            if (!ok) break;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                // negative, as they are added; a row that sees nothing, or is none, has weights exp2(x - inf) = 0
                stats[s * 2 * TILE + k * 32 + lane] = lse[k] == -INFINITY ? -INFINITY : -lse[k] * LOG2E;
                stats[s * 2 * TILE + TILE + k * 32 + lane] = -delta[k];
            }
            __syncwarp();
            if (lane == 0) {
                uint64_t *bar = edge ? &q_copied[s] : &q_full[s];
                mbar_expect_tx(bar, BYTES);
                load_tile<DP>(Q + s * BYTES, &qmap, bar, h, rq.first + i0);
                ok = mbar_wait(&do_empty[s], parity, abort_flag, a.status, 2);
                if (ok) {
                    bar = edge ? &do_copied[s] : &do_full[s];
                    mbar_expect_tx(bar, BYTES);
                    load_tile<DP>(DO + s * BYTES, &domap, bar, h, rq.first + i0);
                }
            }
            ok = __shfl_sync(~0u, ok, 0);
            if (edge && ok) {
                ok = __all_sync(~0u, mbar_wait(&q_copied[s], (copied >> s) & 1u, abort_flag, a.status, 3));
                if (ok) {
                    clear_rows<DP>(Q + s * BYTES, rq.len - i0, TILE, lane);
                    clear_rows<DP>(Q + s * BYTES, 0, unseen, lane);
                    if (lane == 0) mbar_arrive(&q_full[s]);
                    ok = __all_sync(~0u, mbar_wait(&do_copied[s], (copied >> s) & 1u, abort_flag, a.status, 4));
                }
                if (ok) {
                    clear_rows<DP>(DO + s * BYTES, rq.len - i0, TILE, lane);
                    clear_rows<DP>(DO + s * BYTES, 0, unseen, lane);
                    if (lane == 0) mbar_arrive(&do_full[s]);
                }
                copied ^= 1u << s;
            }
            if (++tile == qt.all) {
                tile = qt.a;
                ++h;
            }
        }
    } else if (warp == 9) {
        if (n > 0) {
            const bool lead = elect_one();
            const uint32_t s_idesc = make_idesc(1, 0, 0, TILE, TILE), o_idesc = make_idesc(1, 0, 1, TILE, DP);
            bool ok = true;
            auto score = [&](int i) {
                if (!ok || i >= n) return;
                ok = warp_wait(&q_full[i % ST], (uint32_t)((i / ST) & 1), abort_flag, a.status, 5);
                if (!ok) return;
                tc_fence_after();
                mma_rows<DP>(lead, tmem, K, Q + (i % ST) * BYTES, s_idesc);
                commit(lead, s_full);
            };
            auto dprob = [&](int i) {
                if (!ok || i >= n) return;
                ok = warp_wait(&do_full[i % ST], (uint32_t)((i / ST) & 1), abort_flag, a.status, 6);
                if (!ok) return;
                tc_fence_after();
                mma_rows<DP>(lead, dp_col, V, DO + (i % ST) * BYTES, s_idesc);
                commit(lead, dp_full);
            };
            ok = warp_wait(k_full, 0, abort_flag, a.status, 7);
            score(0);
            if (ok) ok = warp_wait(v_full, 0, abort_flag, a.status, 8);
            dprob(0);
            for (int i = 0; i < n && ok; ++i) {
                ok = warp_wait(p_full, (uint32_t)(i & 1), abort_flag, a.status, 9);
                if (!ok) break;
                tc_fence_after();
                mma_tokens<64>(lead, dv_col, tmem, DO + (i % ST) * BYTES, o_idesc, i > 0);
                commit(lead, &do_empty[i % ST]);
                score(i + 1);
                if (ok) ok = warp_wait(ds_full, (uint32_t)(i & 1), abort_flag, a.status, 10);
                if (!ok) break;
                tc_fence_after();
                mma_tokens<64>(lead, dk_col, dp_col, Q + (i % ST) * BYTES, o_idesc, i > 0);
                commit(lead, &q_empty[i % ST]);
                dprob(i + 1);
            }
            if (ok) commit(lead, done);
        }
        __syncwarp();
    } else {
        // thread: key r, queries 64 half .. 64 half + 63 of a tile
        const int half = warp >> 2, r = (warp & 3) * 32 + lane, s = s0 + r;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, s_addr = tmem + lanes + half * 64, dp_addr = dp_col + lanes + half * 64;
        const float c = a.scale * LOG2E;
        bool ok = true;
        int tile = qt.a;
        for (int i = 0; i < n; ++i) {
            const int st = i % ST, t0 = tile * TILE + off;
            const float *lse2 = stats + st * 2 * TILE + half * 64, *delta = lse2 + TILE;
            const bool cut = !mask.all(t0, t0 + TILE - 1, s0, s0 + TILE - 1);
            ok = __all_sync(~0u, mbar_wait(&q_full[st], (uint32_t)((i / ST) & 1), abort_flag, a.status, 11));
            if (ok) ok = __all_sync(~0u, mbar_wait(s_full, (uint32_t)(i & 1), abort_flag, a.status, 12));
            if (!ok) break;
            tc_fence_after();
            const ColumnMask seen(mask, s, t0);
            Pair y[2][16];
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                uint32_t x[32], p[16];
                tmem_ld_32x32(s_addr + b * 32, x);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const float4 l = *reinterpret_cast<const float4 *>(lse2 + b * 32 + 2 * e);
                    const float2 z0 = split(fma(pair(x[2 * e], x[2 * e + 1]), pair(c, c), pair(l.x, l.y))),
                                 z1 = split(fma(pair(x[2 * e + 2], x[2 * e + 3]), pair(c, c), pair(l.z, l.w)));
                    y[b][e] = pair(ex2(z0.x), ex2(z0.y));
                    y[b][e + 1] = pair(ex2(z1.x), ex2(z1.y));
                }
                if (cut) keep(y[b], seen.of(half * 64 + b * 32));
#pragma unroll
                for (int e = 0; e < 16; ++e) p[e] = pack_bf16(y[b][e]);
                tmem_st_32x16(s_addr + b * 16, p);
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(p_full);
            ok = __all_sync(~0u, mbar_wait(dp_full, (uint32_t)(i & 1), abort_flag, a.status, 13));
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                uint32_t dp[32], ds[16];
                tmem_ld_32x32(dp_addr + b * 32, dp);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 16; e += 2) {
                    const float4 d = *reinterpret_cast<const float4 *>(delta + b * 32 + 2 * e);
                    ds[e] = pack_bf16(mul(y[b][e], add(pair(dp[2 * e], dp[2 * e + 1]), pair(d.x, d.y))));
                    ds[e + 1] = pack_bf16(mul(y[b][e + 1], add(pair(dp[2 * e + 2], dp[2 * e + 3]), pair(d.z, d.w))));
                }
                tmem_st_32x16(dp_addr + b * 16, ds);
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(ds_full);
            if (++tile == qt.all) tile = qt.a;
        }
        if (ok && n > 0) ok = __all_sync(~0u, mbar_wait(done, 0, abort_flag, a.status, 14));
        if (ok) {
            tc_fence_after();
            // the first half of the threads has dk, the second dv
            const uint32_t acc = (half ? dv_col : dk_col) + lanes;
            const float scale = half ? 1.f : a.scale;
            const int kv_heads = a.heads / a.group, wr = (warp & 3) * 32;
            const bool inside = s < rk.len, partial = r < partial_rows;
            if (!far) {
                // K and V have been read for the last time
                // a key that no query sees, the first one at `off` neither: its value may hold anything, and 0 times dP - delta be NaN
                const bool unseen = s >= a.sinks && s <= off - a.window;
                store_rows<DP>(acc, half ? V : K, half ? &dvmap : &dkmap, half ? g.dv : g.dk, (int64_t)kv_heads * a.d, a.d, rk.first + s0 + wr, hk, r, rk.len - s0 - wr,
                               partial_rows - wr, scale, n == 0 || unseen);
                if (lane == 0) tma_store_wait();
            }
            if (partial_rows > (warp & 3) * 32) {
                float *part = part_of(g, far, kt, slot, hk) + ((int64_t)half * g.sink_rows + r) * a.d;
#pragma unroll
                for (int j = 0; j < DP / 32; ++j) {
                    uint32_t o[32];
                    tmem_ld_32x32(acc + j * 32, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int e = 0; e < 32; e += 4)
                        if (partial && inside && j * 32 + e < a.d)
                            *reinterpret_cast<float4 *>(part + j * 32 + e) =
                                n == 0 ? make_float4(0.f, 0.f, 0.f, 0.f)
                                       : make_float4(__uint_as_float(o[e]) * scale, __uint_as_float(o[e + 1]) * scale, __uint_as_float(o[e + 2]) * scale,
                                                     __uint_as_float(o[e + 3]) * scale);
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 9) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// dk and dv of the sinks' rows of the sequences whose queries were split: the sum of the block near them and of the parts.
__global__ void __launch_bounds__(256) window_sinks_kernel(const WindowGradArgs g)
{
    const WindowArgs &a = g.w;
    pdl_wait();
    pdl_trigger();
    const int kt = blockIdx.z, hk = blockIdx.y, kv_heads = a.heads / a.group;
    const Mask mask{a.window, a.sinks};
    const PartOf p = part_at(g, mask, kt, blockIdx.x, threadIdx.x & 31);
    if (p.seq < 0 || p.part != 0) return;
    const Rows rq = rows_of(a.q_offsets, p.seq, a.nq), rk = rows_of(a.k_offsets, p.seq, a.nk);
    const QueryTiles qt = query_tiles(mask, rq, rk, kt * TILE);
    const int first = first_part(g, qt), parts = (qt.all - first + (1 << g.part_log) - 1) >> g.part_log;
    const int rows = min(min(a.sinks - kt * TILE, TILE), rk.len - kt * TILE), quads = a.d / 4;
    for (int i = threadIdx.x; i < 2 * rows * quads; i += blockDim.x) {
        const int which = i / (rows * quads), r = i / quads % rows, c = i % quads * 4;
        const int64_t at = ((int64_t)which * g.sink_rows + r) * a.d + c;
        float4 sum = *reinterpret_cast<const float4 *>(part_of(g, 0, kt, blockIdx.x, hk) + at);
        constexpr int AT_ONCE = 8;
        for (int k0 = 0; k0 < parts; k0 += AT_ONCE) {
            float4 x[AT_ONCE];
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k) {
                const int tile = rq.first / TILE + first + (min(k0 + k, parts - 1) << g.part_log);
                x[k] = *reinterpret_cast<const float4 *>(part_of(g, 1, kt, tile >> g.part_log, hk) + at);
            }
#pragma unroll
            for (int k = 0; k < AT_ONCE; ++k)
                if (k0 + k < parts) sum = make_float4(sum.x + x[k].x, sum.y + x[k].y, sum.z + x[k].z, sum.w + x[k].w);
        }
        bf16 *dst = (which ? g.dv : g.dk) + ((int64_t)(rk.first + kt * TILE + r) * kv_heads + hk) * a.d + c;
        *reinterpret_cast<uint2 *>(dst) = make_uint2(pack_bf16(sum.x, sum.y), pack_bf16(sum.z, sum.w));
    }
}

// Sums of parts: for up to two tiles of first columns, one slot per part's queries.
static size_t parts_floats(int64_t nq, int64_t kv_heads, int64_t sinks, int64_t d)
{
    if (sinks <= 0 || sinks > wgrad::MAX_SPLIT_SINKS) return 0;
    const int64_t tiles = (sinks + TILE - 1) / TILE, rows = sinks < TILE ? sinks : TILE;
    return (size_t)(2 * tiles * (nq / wgrad::part_rows(sinks) + 1) * kv_heads * 2 * rows * d);
}

template <int DP>
static st_status run_grad(WindowGradArgs &g, const st_tokens *t, cudaStream_t stream)
{
    const WindowArgs &a = g.w;
    CUtensorMap qm, km, vm, dom, dqm, dkm, dvm;
    const Table dq{g.dq, (int64_t)t->heads * t->d, t->d}, dk{g.dk, (int64_t)t->kv_heads * t->d, t->d}, dv{g.dv, (int64_t)t->kv_heads * t->d, t->d};
    if (!make_tmap_table(&dqm, dq, t->nq, t->heads, t->d, 32) || !make_tmap_table(&dkm, dk, t->nk, t->kv_heads, t->d, 32) ||
        !make_tmap_table(&dvm, dv, t->nk, t->kv_heads, t->d, 32))
        return ST_ERR_CUDA;
    const Table dout{g.dout, (int64_t)t->heads * t->d, t->d};
    if (!make_tmap_table(&qm, a.q, t->nq, t->heads, t->d) || !make_tmap_table(&km, a.k, t->nk, t->kv_heads, t->d) ||
        !make_tmap_table(&vm, a.v, t->nk, t->kv_heads, t->d) || !make_tmap_table(&dom, dout, t->nq, t->heads, t->d))
        return ST_ERR_CUDA;
    using S = wgrad::Shape<DP>;
    if (!ensure_dynamic_smem(window_dq_kernel<DP>, S::DQ_SMEM) || !ensure_dynamic_smem(window_dkv_kernel<DP>, S::DKV_SMEM)) return ST_ERR_CUDA;
    st_status rc = launch(window_dq_kernel<DP>, dim3((unsigned)most_tiles(t->nq, t->nseq, TILE), (unsigned)t->heads), wgrad::THREADS, S::DQ_SMEM, stream,
                          qm, km, vm, dom, dqm, g);
    if (rc != ST_OK) return rc;
    const dim3 grid((unsigned)(g.sink_tiles * g.nslots + most_tiles(t->nk, t->nseq, TILE)), (unsigned)t->kv_heads);
    rc = launch(window_dkv_kernel<DP>, grid, wgrad::THREADS, S::DKV_SMEM, stream, qm, km, vm, dom, dkm, dvm, g);
    if (rc != ST_OK || g.sink_tiles == 0) return rc;
    return launch(window_sinks_kernel, dim3((unsigned)g.nslots, (unsigned)t->kv_heads, (unsigned)g.sink_tiles), 256, 0, stream, g);
}

}  // namespace attn

size_t attn_window_grad_workspace(int64_t nq, int64_t heads, int64_t kv_heads, int64_t sinks)
{
    if (nq <= 0 || heads <= 0 || kv_heads <= 0 || kv_heads > heads || sinks < 0 || nq > (1 << 29) || heads > 65535) return 0;
    return kWsHeaderBytes + round_up((size_t)nq * heads * sizeof(float), 256) + attn::parts_floats(nq, kv_heads, sinks, 128) * sizeof(float);
}

}  // namespace st

using namespace st;
using namespace st::attn;

extern "C" st_status st_attn_window_grad(const st_tokens *tokens, const void *q, const void *k, const void *v, const void *out,
                                         const float *lse, const void *dout, const int32_t *q_offsets, const int32_t *k_offsets,
                                         int64_t window, int64_t sinks, float scale, void *dq, void *dk, void *dv, void *ws,
                                         size_t ws_bytes, void *stream)
{
    const st_status rc = check_window(tokens, q_offsets, k_offsets, window, sinks, scale);
    if (rc != ST_OK) return rc;
    if (!q || !k || !v || !out || !lse || !dout || !dq || !dk || !dv) return ST_ERR_NULL;
    for (const void *p : {q, k, v, out, (const void *)lse, dout, (const void *)dq, (const void *)dk, (const void *)dv, (const void *)q_offsets, (const void *)k_offsets})
        if (!aligned16(p)) return ST_ERR_ALIGN;
    if (!ws || ws_bytes < attn_window_grad_workspace(tokens->nq, tokens->heads, tokens->kv_heads, sinks)) return ST_ERR_WORKSPACE;
    if (!aligned256(ws)) return ST_ERR_ALIGN;
    // the second kernel reads q, dout and lse again; a block of it reads its own keys and values alone
    {
        const int64_t rows = tokens->nq * tokens->heads, q_bytes = rows * tokens->d * 2, k_bytes = tokens->nk * tokens->kv_heads * tokens->d * 2;
        const Operand Q = q_of(tokens, q), K = k_of(tokens, k), V = v_of(tokens, v), O = dense_of(out, tokens->nq, tokens->heads, tokens->d),
                      D = dense_of(dout, tokens->nq, tokens->heads, tokens->d);
        bool wrong = Q.under(dq, q_bytes) || K.under(dq, q_bytes) || V.under(dq, q_bytes) || D.under(dq, q_bytes) || O.under(dq, q_bytes, true) ||
                     arrays_meet(dq, q_bytes, lse, rows * 4) || arrays_meet(dq, q_bytes, dk, k_bytes) || arrays_meet(dq, q_bytes, dv, k_bytes) ||
                     arrays_meet(dk, k_bytes, dv, k_bytes);
        for (const void *to : {dk, dv})
            wrong = wrong || Q.under(to, k_bytes) || D.under(to, k_bytes) || arrays_meet(to, k_bytes, lse, rows * 4) || K.under(to, k_bytes, true) ||
                    V.under(to, k_bytes, true);
        if (wrong) return ST_ERR_UNSUPPORTED;
    }
    WindowGradArgs g = {};
    g.w = window_args(tokens, q, k, v, q_offsets, k_offsets, window, sinks, scale, ws);
    g.o = (const bf16 *)out;
    g.dout = (const bf16 *)dout;
    g.lse = lse;
    g.dq = (bf16 *)dq;
    g.dk = (bf16 *)dk;
    g.dv = (bf16 *)dv;
    g.delta = (float *)((unsigned char *)ws + kWsHeaderBytes);
    g.parts = (float *)((unsigned char *)ws + kWsHeaderBytes + round_up((size_t)tokens->nq * tokens->heads * sizeof(float), 256));
    // Queries beyond the window and a part: with as many keys as queries only a table that is longer has them.  Behind cached keys shorter ones have
    // them too; their sinks' rows are summed by one block.
    if (sinks > 0 && sinks <= wgrad::MAX_SPLIT_SINKS && tokens->nq - wgrad::part_rows(sinks) > window) {
        g.sink_tiles = (int)((sinks + TILE - 1) / TILE);
        g.sink_rows = (int)(sinks < TILE ? sinks : TILE);
        g.part_log = wgrad::part_log(sinks);
        g.nslots = (int)(tokens->nq / wgrad::part_rows(sinks) + 1);
    }
    return g.w.d <= 64 ? run_grad<64>(g, tokens, (cudaStream_t)stream) : run_grad<128>(g, tokens, (cudaStream_t)stream);
}
