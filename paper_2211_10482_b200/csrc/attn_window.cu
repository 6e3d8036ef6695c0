// st_attn_window: softmax attention over a causal band and the first columns, on the tensor cores.
//
// A block owns 256 queries of one head as two tiles of 128.  For every tile of 128 keys that a tile of queries sees
//     S = Q K^T  (tcgen05, fp32 in tensor memory);   P = exp2(c S - c m)  (one thread per query row);   O += P V
// with c = scale log2 e and m a running row maximum.  P goes back to tensor memory as bf16, over S, and is the A operand of the
// second product; O stays in tensor memory.  While one tile's rows are in the exponential, the tensor cores work for the
// other.  m moves only when a row's maximum has grown by more than 8 / c: any m gives the same quotient O / l, and P up to 2^8
// loses nothing in bf16 or fp32, so that O is read and rescaled for the first tiles only.  P is rounded to bf16 once,
// for the tensor cores; the row sum l is taken from the fp32 values.
//
// Only tiles with a visible pair are loaded and multiplied (the sinks' tiles, then the band's), and only tiles that the mask
// cuts are masked.  Values behind a sequence's last key may be anything: their weight is 0, and their rows of V are
// cleared in shared memory, as 0 times NaN would be NaN.
//
// Bound by power where many tiles of keys are seen: 32768 tokens, 16 heads of 128, window 4096 run at 960 to 990 TFLOP/s whether the exponentials and the
// products alternate (3100 cycles for both tiles, at 1.4 GHz) or not (3960, at 1.8), and slower with part of the exponentials as
// polynomials on the FMA units (1050 us, so 1185 with an eighth of them).  Few tiles of keys: by a block's beginning and end.
//
// Warps: 0..3 and 4..7 one row per thread of the first and second tile of queries, 8 copies (TMA), 9 and 10 issue the products of one tile
// each: by one warp for both the issue itself took longer than the products.
#include "attn_window.cuh"

namespace st {
namespace attn {

namespace wfwd {
constexpr int THREADS = 352;
constexpr int STAGES = 2;
template <int DP> struct Shape {
    static constexpr int TILE_BYTES = DP / 64 * SLAB;
    static constexpr size_t SMEM = 1024 + (size_t)TILE_BYTES * (2 + 2 * STAGES) + 256;
};
}  // namespace wfwd

template <int DP>
__global__ void __launch_bounds__(wfwd::THREADS, 1)
window_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap,
              const __grid_constant__ CUtensorMap outmap, const WindowArgs a)
{
    using namespace wfwd;
    using namespace tc;
    using S = Shape<DP>;
    extern __shared__ unsigned char raw[];
    unsigned char *smem = align_smem(raw);
    unsigned char *Q = smem, *K = Q + 2 * S::TILE_BYTES, *V = K + STAGES * S::TILE_BYTES;
    uint64_t *bars = (uint64_t *)(V + STAGES * S::TILE_BYTES);
    uint64_t *q_full = bars, *k_full = bars + 2, *k_empty = k_full + STAGES, *v_full = k_empty + STAGES, *v_empty = v_full + STAGES,
             *v_copied = v_empty + STAGES, *s_full = v_copied + STAGES, *p_full = s_full + 2, *o_full = p_full + 4, *v_first = o_full + 2;
    uint32_t *tmem_slot = (uint32_t *)(v_first + 1);
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);
    const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, h = blockIdx.y;

    if (warp == 8 && lane < 4) prefetch_tmap(lane == 0 ? &qmap : lane == 1 ? &kmap : lane == 2 ? &vmap : &outmap);
    pdl_wait();
    if (blockIdx.x == 0 && blockIdx.y == 0) {
        const bool fine = offsets_fine(a.q_offsets, a.nseq, a.nq, threadIdx.x, THREADS) && offsets_fine(a.k_offsets, a.nseq, a.nk, threadIdx.x, THREADS);
        const int all = __syncthreads_and(fine);
        if (threadIdx.x == 0) {
            a.status[kWsStatusWord] = all ? 0u : (unsigned)ST_ERR_DEV_BOUNDS;
            a.status[kWsDetailWord] = 0u;
        }
    }
    const TileOf at = tile_of(a.q_offsets, a.nseq, a.nq, 2 * TILE, blockIdx.x, lane);
    if (at.seq < 0) return;
    const Rows rq = rows_of(a.q_offsets, at.seq, a.nq), rk = rows_of(a.k_offsets, at.seq, a.nk);
    const int i0 = at.tile * 2 * TILE, left = min(rq.len - i0, 2 * TILE), t0 = i0 + rk.len - rq.len;
    const Mask mask{a.window, a.sinks};
    const KeyTiles tiles = key_tiles(mask, t0, t0 + left - 1);
    const int n = tiles.count();
    // positions of the rows of a tile of queries (none: t1 < t0), and whether it sees a tile of keys
    auto sees = [&](int w, int i) {
        const int first = t0 + w * TILE, s0 = tiles.key(i);
        return mask.any(first, min(first + TILE, t0 + left) - 1, s0, s0 + TILE - 1);
    };

    if (threadIdx.x == 0) {
        for (int w = 0; w < 2; ++w) {
            mbar_init(&q_full[w], 1);
            mbar_init(&s_full[w], 1);
            mbar_init(&p_full[2 * w], 4);
            mbar_init(&p_full[2 * w + 1], 4);
            mbar_init(&o_full[w], 1);
        }
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(&k_full[s], 1);
            mbar_init(&k_empty[s], 2);
            mbar_init(&v_full[s], 1);
            mbar_init(&v_empty[s], 2);
            mbar_init(&v_copied[s], 1);
        }
        mbar_init(v_first, 1);
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
    const uint32_t tmem = __shfl_sync(~0u, *tmem_slot, 0);
    pdl_trigger();

    if (warp == 8) {
        const int hk = h / a.group;
        bool q_asked[2] = {false, false};       // queries that see nothing are not copied: their place is used for the output at once
        int use = 0;
        uint32_t copied = 0;                    // parity of v_copied, by stage
        bool ok = true;
        // the last tile of first columns, where its values are cleared behind them: when they have come, and the next tile has been asked for
        const int cleared = tiles.cleared();
        bool clear = false;
        auto clear_first = [&] {
            clear = false;
            const int s = cleared % STAGES;
            ok = warp_wait(v_first, 0, abort_flag, a.status, 10);
            if (!ok) return;
            clear_rows<DP>(V + s * S::TILE_BYTES, tiles.unseen(), tiles.used(), lane);
            if (lane == 0) mbar_arrive(&v_full[s]);
        };
        for (int i = 0; i < n && ok; ++i) {
            const bool a0 = sees(0, i), a1 = sees(1, i);
            if (!a0 && !a1) continue;
            for (int w = 0; w < 2; ++w)
                if ((w ? a1 : a0) && !q_asked[w]) {
                    q_asked[w] = true;
                    if (lane == 0) {
                        mbar_expect_tx(&q_full[w], S::TILE_BYTES);
                        load_tile<DP>(Q + w * S::TILE_BYTES, &qmap, &q_full[w], h, rq.first + i0 + w * TILE);
                    }
                }
            const int s = use % STAGES, s0 = tiles.key(i), row = rk.first + s0;
            const uint32_t parity = (uint32_t)((use / STAGES + 1) & 1);
            const bool edge = s0 + TILE > rk.len && i != cleared;
            if (lane == 0) {
                ok = mbar_wait(&k_empty[s], parity, abort_flag, a.status, 1);
                if (ok) {
                    mbar_expect_tx(&k_full[s], S::TILE_BYTES);
                    load_tile<DP>(K + s * S::TILE_BYTES, &kmap, &k_full[s], hk, row);
                    ok = mbar_wait(&v_empty[s], parity, abort_flag, a.status, 2);
                }
                if (ok) {
                    uint64_t *bar = i == cleared ? v_first : edge ? &v_copied[s] : &v_full[s];
                    mbar_expect_tx(bar, S::TILE_BYTES);
                    load_tile<DP>(V + s * S::TILE_BYTES, &vmap, bar, hk, row);
                }
            }
            ok = __shfl_sync(~0u, ok, 0);
            if (clear && ok) clear_first();
            clear = i == cleared;
            if (edge && ok) {
                ok = __all_sync(~0u, mbar_wait(&v_copied[s], (copied >> s) & 1u, abort_flag, a.status, 3));
                copied ^= 1u << s;
                if (ok) {
                    clear_rows<DP>(V + s * S::TILE_BYTES, rk.len - s0, TILE, lane);
                    if (lane == 0) mbar_arrive(&v_full[s]);
                }
            }
            ++use;
        }
        if (clear && ok) clear_first();
    } else if (warp >= 9) {
        // One warp for each tile of queries: its scores S of a tile of keys follow its product with V of the tile before, whose weights they
        // overwrite (products are carried out in the order of their issue), and the other tile's products fill the time between.
        const int w = warp - 9;
        const bool lead = elect_one();
        const uint32_t s_idesc = make_idesc(1, 0, 0, TILE, TILE), o_idesc = make_idesc(1, 0, 1, TILE, DP), piece_idesc = make_idesc(1, 0, 0, TILE, KeyTiles::PIECE);
        const uint32_t s_col = tmem + w * TILE, o_col = tmem + 2 * TILE + w * DP;
        const unsigned char *mine = Q + w * S::TILE_BYTES;
        bool ok = true, started = false;
        int i = 0, use = 0, done = 0;                            // tiles looked at, copied, used by this tile of queries
        int at_stage = -1;                                       // the stage whose scores are in the exponential
        uint32_t at_parity = 0;
        bool at_piece = false;
        while (ok) {
            // the next tile that was copied
            bool a0 = false, a1 = false;
            for (; i < n && !(a0 || a1); ++i) {
                a0 = sees(0, i);
                a1 = sees(1, i);
            }
            const bool more = a0 || a1, score = w ? a1 : a0, piece = more && tiles.piece(i - 1);
            const int s = use % STAGES;
            const uint32_t parity = (uint32_t)((use / STAGES) & 1);
            if (at_stage >= 0 && (score || !more)) {
                ok = warp_wait(&v_full[at_stage], at_parity, abort_flag, a.status, 6);
                if (ok) ok = warp_wait(&p_full[2 * w], (uint32_t)(done & 1), abort_flag, a.status, 7);
                if (!ok) break;
                tc_fence_after();
                if (at_piece) mma_tokens<32, 0, KeyTiles::PIECE / 16>(lead, o_col, s_col, V + at_stage * S::TILE_BYTES, o_idesc, started);
                else mma_tokens<32, 0, 4>(lead, o_col, s_col, V + at_stage * S::TILE_BYTES, o_idesc, started);
                ok = warp_wait(&p_full[2 * w + 1], (uint32_t)(done & 1), abort_flag, a.status, 7);
                if (!ok) break;
                tc_fence_after();
                if (!at_piece) mma_tokens<32, 4, 8>(lead, o_col, s_col, V + at_stage * S::TILE_BYTES, o_idesc, true);
                commit(lead, &v_empty[at_stage]);
                at_stage = -1;
                started = true;
                ++done;
            }
            if (!more) break;
            ok = warp_wait(&k_full[s], parity, abort_flag, a.status, 5);
            if (ok && score && !started && done == 0 && at_stage < 0) ok = warp_wait(&q_full[w], 0, abort_flag, a.status, 4);
            if (!ok) break;
            if (score) {
                tc_fence_after();
                mma_rows<DP>(lead, s_col, mine, K + s * S::TILE_BYTES, piece ? piece_idesc : s_idesc);
                commit(lead, &s_full[w]);
                at_stage = s;
                at_piece = piece;
                at_parity = parity;
            } else {
                // a tile that the other queries alone see: given back once it is there, so that the stages' turns stay in order
                ok = warp_wait(&v_full[s], parity, abort_flag, a.status, 8);
                if (!ok) break;
                if (lead) mbar_arrive(&v_empty[s]);
            }
            commit(lead, &k_empty[s]);
            ++use;
        }
        if (ok && started) commit(lead, &o_full[w]);
        __syncwarp();
    } else {
        const int w = warp >> 2, r = (warp & 3) * 32 + lane, t = t0 + w * TILE + r;      // this thread's row and its position
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, s_addr = tmem + lanes + w * TILE, o_addr = tmem + lanes + 2 * TILE + w * DP;
        const float c = a.scale * LOG2E;
        float m = -INFINITY, l = 0.f;
        uint32_t parity = 0;
        bool ok = true, started = false;
        for (int i = 0; i < n; ++i) {
            if (!sees(w, i)) continue;
            ok = __all_sync(~0u, mbar_wait(&s_full[w], parity, abort_flag, a.status, 8));
            if (!ok) break;
            parity ^= 1u;
            tc_fence_after();
            if (tiles.piece(i)) {                         // comes first, and every query sees the same columns
                uint32_t x[32], p[16];
                tmem_ld_32x32(s_addr, x);
                tmem_ld_wait();
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    if (e >= tiles.sinks) x[e] = __float_as_uint(-INFINITY);
                    m = fmaxf(m, __uint_as_float(x[e]));
                }
                const float mc = m == -INFINITY ? 0.f : -m * c;
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float2 y = {ex2(fmaf(__uint_as_float(x[2 * e]), c, mc)), ex2(fmaf(__uint_as_float(x[2 * e + 1]), c, mc))};
                    l += y.x + y.y;
                    p[e] = pack_bf16(y.x, y.y);
                }
                tmem_st_32x16(s_addr, p);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane < 2) mbar_arrive(&p_full[2 * w + lane]);
                started = true;
                continue;
            }
            const bool cut = !tiles.all(mask, t0 + w * TILE, t0 + w * TILE + TILE - 1, i);
            uint32_t x[4][32];
#pragma unroll
            for (int j = 0; j < 4; ++j) tmem_ld_32x32(s_addr + j * 32, x[j]);
            tmem_ld_wait();
            if (cut) {
                const RowMask seen = tiles.row_mask(mask, t, i);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const unsigned bits = seen.of(j * 32);
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (!(bits >> e & 1u)) x[j][e] = __float_as_uint(-INFINITY);
                }
            }
            float most[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int e = 0; e < 32; e += 2) most[e / 2 & 3] = max3(most[e / 2 & 3], __uint_as_float(x[j][e]), __uint_as_float(x[j][e + 1]));
            const float top = fmaxf(fmaxf(most[0], most[1]), fmaxf(most[2], most[3]));
            // the reference moves: 8 is the factor 2^8 that P may exceed 1 by
            if (__any_sync(~0u, c * (top - m) > 8.f)) {
                const float now = fmaxf(top, m), f = now == -INFINITY ? 1.f : ex2(c * (m - now));
                m = now;
                l *= f;
                if (started) {
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
            started = true;
            const float mc = m == -INFINITY ? 0.f : -m * c;
            const Pair cc = pair(c, c), mm = pair(mc, mc);
            Pair sum[2] = {pair(0.f, 0.f), pair(0.f, 0.f)};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t p[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    const float2 z = split(fma(pair(x[j][2 * e], x[j][2 * e + 1]), cc, mm));
                    const Pair y = pair(ex2(z.x), ex2(z.y));
                    sum[e & 1] = add(sum[e & 1], y);
                    p[e] = pack_bf16(y);
                }
                tmem_st_32x16(s_addr + j * 16, p);
                if (j & 1) {                              // the product with V begins when half of the keys' weights are there
                    tmem_st_wait();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&p_full[2 * w + j / 2]);
                }
            }
            const float2 part = split(add(sum[0], sum[1]));
            l += part.x + part.y;
        }
        if (ok && started) ok = __all_sync(~0u, mbar_wait(&o_full[w], 0, abort_flag, a.status, 9));
        if (ok) {
            tc_fence_after();
            const int wr = (warp & 3) * 32, first = w * TILE + wr, row = rq.first + i0 + first;      // this warp's rows
            // a query from position 0 on sees itself at least: where its sum is NaN (a score is, or is +inf) or 0 (all scores are -inf), so is the row NaN
            const bool seen = t >= 0, all = first + 32 <= left;
            const Pair inv = pair(seen ? 1.f / l : 0.f, seen ? 1.f / l : 0.f);
            if (first + lane < left) a.lse[(int64_t)(row + lane) * a.heads + h] = seen ? (m * c + log2f(l)) * LN2 : -INFINITY;
            // Rows go out through the shared memory of the queries, which no product reads any more: a warp's 32 rows in one copy for each
            // 64 columns, or at a sequence's end one by one.
            unsigned char *rows = Q + w * S::TILE_BYTES;
            const int r8 = r & 7;
#pragma unroll 1
            for (int j = 0; j < DP / 16; ++j) {
                uint32_t o[16];
                if (started) {
                    tmem_ld_32x16(o_addr + j * 16, o);
                    tmem_ld_wait();
                }
                uint4 v[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    uint32_t u[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) u[k] = seen ? pack_bf16(mul(pair(o[e * 8 + 2 * k], o[e * 8 + 2 * k + 1]), inv)) : 0u;
                    v[e] = make_uint4(u[0], u[1], u[2], u[3]);
                }
                unsigned char *at = rows + (j / 4) * SLAB + r * 128;
                *reinterpret_cast<uint4 *>(at + (((j % 4) * 2) ^ r8) * 16) = v[0];
                *reinterpret_cast<uint4 *>(at + (((j % 4) * 2 + 1) ^ r8) * 16) = v[1];
                if (all && j % 4 == 3) {
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) tma_store_3d(&outmap, rows + (j / 4) * SLAB + wr * 128, j / 4 * 64, h, row);
                }
            }
            __syncwarp();
            if (!all) {
                for (int k = 0; k < 32 && first + k < left; ++k)
                    if (lane * 8 < a.d && lane < DP / 8)
                        *reinterpret_cast<uint4 *>(a.out + ((int64_t)(row + k) * a.heads + h) * a.d + lane * 8) =
                            *reinterpret_cast<const uint4 *>(rows + (lane / 8) * SLAB + (wr + k) * 128 + (((lane & 7) ^ (k & 7)) << 4));
            }
            if (lane == 0) tma_store_wait();
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
static st_status run_window(const WindowArgs &a, const st_tokens *t, cudaStream_t stream)
{
    CUtensorMap qm, km, vm, om;
    const Table out{a.out, (int64_t)t->heads * t->d, t->d};
    if (!make_tmap_table(&om, out, t->nq, t->heads, t->d, 32)) return ST_ERR_CUDA;
    if (!make_tmap_table(&qm, a.q, t->nq, t->heads, t->d) || !make_tmap_table(&km, a.k, t->nk, t->kv_heads, t->d) ||
        !make_tmap_table(&vm, a.v, t->nk, t->kv_heads, t->d))
        return ST_ERR_CUDA;
    if (!ensure_dynamic_smem(window_kernel<DP>, wfwd::Shape<DP>::SMEM)) return ST_ERR_CUDA;
    const dim3 grid((unsigned)most_tiles(t->nq, t->nseq, 2 * TILE), (unsigned)t->heads);
    return launch(window_kernel<DP>, grid, wfwd::THREADS, wfwd::Shape<DP>::SMEM, stream, qm, km, vm, om, a);
}

}  // namespace attn
}  // namespace st

using namespace st;
using namespace st::attn;

extern "C" st_status st_attn_window(const st_tokens *tokens, const void *q, const void *k, const void *v, const int32_t *q_offsets,
                                    const int32_t *k_offsets, int64_t window, int64_t sinks, float scale, void *out, float *lse,
                                    void *ws, size_t ws_bytes, void *stream)
{
    const st_status rc = check_window(tokens, q_offsets, k_offsets, window, sinks, scale);
    if (rc != ST_OK) return rc;
    if (!q || !k || !v || !out || !lse) return ST_ERR_NULL;
    for (const void *p : {q, k, v, (const void *)out, (const void *)lse, (const void *)q_offsets, (const void *)k_offsets})
        if (!aligned16(p)) return ST_ERR_ALIGN;
    if (!ws || ws_bytes < kWsHeaderBytes) return ST_ERR_WORKSPACE;
    if (!aligned256(ws)) return ST_ERR_ALIGN;
    // a block reads its own queries alone, and every key and value of its band
    const Operand Q = q_of(tokens, q), K = k_of(tokens, k), V = v_of(tokens, v);
    const int64_t rows = tokens->nq * tokens->heads, out_bytes = rows * tokens->d * 2, lse_bytes = rows * 4;
    if (Q.under(out, out_bytes, true) || K.under(out, out_bytes) || V.under(out, out_bytes) || Q.under(lse, lse_bytes) || K.under(lse, lse_bytes) ||
        V.under(lse, lse_bytes) || arrays_meet(out, out_bytes, lse, lse_bytes))
        return ST_ERR_UNSUPPORTED;
    WindowArgs a = window_args(tokens, q, k, v, q_offsets, k_offsets, window, sinks, scale, ws);
    a.out = (bf16 *)out;
    a.lse = lse;
    return a.d <= 64 ? run_window<64>(a, tokens, (cudaStream_t)stream) : run_window<128>(a, tokens, (cudaStream_t)stream);
}
