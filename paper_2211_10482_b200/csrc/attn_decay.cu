// st_attn_decay and its gradient on the tensor cores: four runs of one operator, a causal sum of outer products that fades,
//     S = e^a S + in_scale y[t] (x) z[t],   out[t] = out_scale x[t].S
// forwards in time for out (x, y, z = q, k, v) and dq (dout, v, k), backwards for dk (v, dout, q) and dv (k, q, dout).
//
// Tokens are taken in chunks of 128.  With w = e^a, L the tokens of a chunk, and S the state that enters it, forwards
//     out = P Z + diag(w^(t+1)) X S,   P[t,s] = w^(t-s) x[t].y[s] for s <= t;     S <- w^L S + Y^T diag(w^(L-1-s)) Z
// and backwards (S holds its factor w already)
//     out = P Z + diag(w^(L-1-t)) X S, P[t,s] = w^(s-t) x[t].y[s] for s >= t;     S <- w^L S + Y^T diag(w^(s+1)) Z.
// No power is of a positive exponent, whatever the decay.  Four products a chunk on the tensor cores, all accumulators in tensor memory:
//     scores X Y^T;  P Z with P as bf16 in the place of the scores;  X S;  Y^T (weights Z).
// S itself stays in fp32 registers, one row to a thread, and the chunk's sum is added to it there, so that no long chain of additions
// runs through the tensor cores' accumulators (which do not round to nearest).  For a state that the caller gets, which is fp32, the weighted Z is
// the sum of three bf16 numbers (2e-7 off in the root mean square); for one that only meets bf16 tables of two (5e-6), in 15 % less time.
// P, and S where it meets X, are rounded to bf16 once: out is bf16 itself.
//
// A block owns 64 columns of z, out and S for a run of chunks: with 128 columns two stages of X, Y and Z, S and the weighted Z
// would not fit in shared memory.  The two blocks of a head read X and Y at about the same time, the second time from L2.
// Where heads and sequences are few, sequences are cut into segments: one kernel sums each segment's own state, one carries the states
// over the segments and behind the last, then all segments run at once.
//
// Bound by what a chunk does in turn: P Z and X S have one place each in tensor memory and are issued in a fixed order, so that X S of a chunk and the
// scores behind it wait until P of the chunk before has been made, multiplied and read.  One head of 128 alone takes 1.4 us a chunk (1.8 with the third
// part), 148 blocks at once 1.9 (2.4).  Some 370 KB go through shared memory for it (80 of copies, 190 of operands, 100 of Z, S and out; 64 more with
// a third part), and about a third of its wavefronts are bank conflicts.  65536 tokens of 16 heads run at 1000 W and 1.4 to 1.5 GHz.
// Two warps that issue products, or four more that write out, changed nothing or lost 5 %: they leave the wait where it is.
//
// Warps: 0..3 make P (a thread = a token), 4..7 weigh Z (a thread = a token), 8..11 keep S (a thread = a row of it) and write out (a thread = a
// token), 12 copies, 13 issues the products.
#include "attn_tc.cuh"
#include <algorithm>
#include <utility>

namespace st {
namespace attn {

struct FadeArgs {
    CUtensorMap xmap, ymap, zmap, outmap;
    Table x, y, z;
    int dx, dz;                       // extent of x and y, extent of z and out
    const float *log_decay;
    const int *offsets;
    int nseq, n, heads;
    const float *init;                // the state before the first (after the last) token: [nseq, heads, dx, dz] or null
    float *last;                      // [nseq, heads, dx, dz] or null
    int transposed, backwards;        // transposed: init and states are [.., dz, dx]
    float in_scale, out_scale;
    bf16 *out;
    unsigned *status;
    int check;                        // look the offsets over and set the status: the call's first kernel
    int chunks;                       // of a segment
    int tiles;                        // segments that the grid and the states have room for
    float *states;                    // [segment][heads][dx][dz], or null: no sequence has more than one segment
};

namespace fade {
constexpr int THREADS = 448, ZC = 64;               // ZC: columns of z of a block
template <int DX, bool STATE> struct Shape {
    static constexpr int STAGES = DX == 64 ? 3 : 2;
    static constexpr int BUFS = STATE ? 2 : 1;                                      // of the weighted Z and of U
    static constexpr int X_BYTES = DX / 64 * SLAB, Z_BYTES = SLAB, S_BYTES = STATE ? 0 : DX * 128;
    static constexpr int STAGE = (STATE ? 1 : 2) * X_BYTES + Z_BYTES;               // Y, Z, X
    static constexpr size_t SMEM = 1024 + (size_t)STAGES * STAGE + S_BYTES + 3 * BUFS * Z_BYTES + 2 * TILE * sizeof(float) + 320;
};
}  // namespace fade

// w^m for w = e^a, a2 = a log2 e <= 0: 1 for m = 0 whatever the decay
__device__ __forceinline__ float power(float a2, int m) { return m == 0 ? 1.f : exp2f(a2 * (float)m); }
// the factor of a state over `m` tokens: it enters as many times as there are chunks, so that its error counts
__device__ __forceinline__ float carry(float a, int m) { return m == 0 ? 1.f : (float)exp((double)a * m); }

// b z for two values z at a time as a sum of bf16 numbers.  Two, b = b_hi + b_lo: hi the rounded product, its remainder exact (two
// significands of 8 bits have a product of 16), lo the remainder and b_lo z rounded: 2^-17 of b z is lost.
__device__ __forceinline__ void times(__nv_bfloat162 b_hi, __nv_bfloat162 b_lo, uint32_t z, uint32_t &hi, uint32_t &lo)
{
    const __nv_bfloat162 x = *reinterpret_cast<const __nv_bfloat162 *>(&z), h = __hmul2(b_hi, x), l = __hfma2(b_lo, x, __hfma2(b_hi, x, __hneg2(h)));
    hi = *reinterpret_cast<const uint32_t *>(&h);
    lo = *reinterpret_cast<const uint32_t *>(&l);
}
// Three: each the rounded remainder of the fp32 product, which fp32 holds exactly.
__device__ __forceinline__ void times(float b, uint32_t z, uint32_t &hi, uint32_t &mid, uint32_t &lo)
{
    auto wide = [](uint32_t x) { return pair(x << 16, x & 0xffff0000u); };
    const Pair minus = pair(-1.f, -1.f), x = mul(pair(b, b), wide(z));
    hi = pack_bf16(x);
    const Pair y = fma(minus, wide(hi), x);
    mid = pack_bf16(y);
    lo = pack_bf16(fma(minus, wide(mid), y));
}

// The segment that a block works on.
struct Segment {
    int seq, first, len, index, count;     // rows of the table; number among its sequence's segments
};
__device__ __forceinline__ Segment segment_of(const FadeArgs &a, int tile, int lane)
{
    const int rows = a.chunks * TILE;
    const TileOf at = tile_of(a.offsets, a.nseq, a.n, rows, tile, lane, 1);
    if (at.seq < 0) return {-1, 0, 0, 0, 0};
    const Rows r = rows_of(a.offsets, at.seq, a.n);
    return {at.seq, r.first + at.tile * rows, min(r.len - at.tile * rows, rows), at.tile, max((r.len + rows - 1) / rows, 1)};
}

// The runs of one launch, one to a plane of the grid: those of the gradient are independent, and together fill the SMs where one alone has as
// many blocks as heads and columns (6 sequences of up to 4096 tokens, 16 heads: one after another 274 us, together 231; with two parts of Z everywhere).
constexpr int MAX_RUNS = 3;
struct FadeRuns {
    FadeArgs run[MAX_RUNS];
};

// STATE: only the segment's own sum of outer products, to `states`.
template <int DX, bool STATE>
__global__ void __launch_bounds__(fade::THREADS, 1)
fade_kernel(const __grid_constant__ FadeRuns runs)
{
    const FadeArgs &a = runs.run[blockIdx.z];
    using namespace fade;
    using namespace tc;
    using Sh = Shape<DX, STATE>;
    constexpr int STAGES = Sh::STAGES, BUFS = Sh::BUFS, U_COLS = 256;
    extern __shared__ unsigned char raw[];
    unsigned char *smem = align_smem(raw);
    unsigned char *stages = smem, *S_op = stages + STAGES * Sh::STAGE, *Z_parts = S_op + Sh::S_BYTES,      // Z_parts: [buffer][3]
                  *out_rows = Z_parts + (3 * BUFS - 1) * Sh::Z_BYTES;                   // in the place of the third part
    float *table = (float *)(out_rows + Sh::Z_BYTES);              // in_scale w^m on one side of the middle, zeros on the other
    uint64_t *bars = (uint64_t *)(table + 2 * TILE);
    uint64_t *xy_full = bars, *z_full = xy_full + STAGES, *xy_empty = z_full + STAGES, *z_empty = xy_empty + STAGES, *sc_full = z_empty + STAGES, *p_full = sc_full + 2, *o_full = p_full + 2, *o_free = o_full + 1,
             *z_ready = o_free + 1, *s_ready = z_ready + BUFS, *u_full = s_ready + 1, *u_free = u_full + BUFS, *xs_done = u_free + BUFS;
    uint32_t *tmem_slot = (uint32_t *)(xs_done + 1);
    volatile int *abort_flag = (volatile int *)(tmem_slot + 1);
    const int warp = __shfl_sync(~0u, threadIdx.x >> 5, 0), lane = threadIdx.x & 31, h = blockIdx.y;
    // the state that the caller gets takes every weighted value as three bf16 numbers, one that only meets bf16 tables as two
    const bool back = a.backwards, third = STATE ? a.last != nullptr : a.last && !a.states;
    const SlabOf place = slab_of(blockIdx.x, (a.dz + ZC - 1) / ZC, a.tiles);
    const int slab = place.slab, tile = place.tile;

    pdl_wait();
    if (a.check && blockIdx.x == 0 && blockIdx.y == 0) {
        const int all = __syncthreads_and(offsets_fine(a.offsets, a.nseq, a.n, threadIdx.x, THREADS));
        if (threadIdx.x == 0) {
            a.status[kWsStatusWord] = all ? 0u : (unsigned)ST_ERR_DEV_BOUNDS;
            a.status[kWsDetailWord] = 0u;
        }
    }
    if (tile < 0) return;
    const Segment seg = segment_of(a, tile, lane);
    if (seg.seq < 0) return;
    // the sum of the segment that comes last only goes to the caller
    if (STATE && !a.last && seg.index == (back ? 0 : seg.count - 1)) return;
    const int n = (seg.len + TILE - 1) / TILE;
    const float decay = a.log_decay[h], a2 = decay * LOG2E;
    auto chunk_of = [&](int i) { return back ? n - 1 - i : i; };
    auto tokens_of = [&](int i) { return min(seg.len - chunk_of(i) * TILE, TILE); };

    // the weight of column s for token t is table[128 + t - s], 0 on the side of the diagonal that is not summed
    if (threadIdx.x < 2 * TILE) {
        const int gap = back ? TILE - (int)threadIdx.x : (int)threadIdx.x - TILE;
        table[threadIdx.x] = gap < 0 ? 0.f : a.in_scale * power(a2, gap);
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(&xy_full[s], 1);
            mbar_init(&z_full[s], 1);
            mbar_init(&xy_empty[s], 1);
            mbar_init(&z_empty[s], STATE ? 4 : 1);
        }
        mbar_init(&sc_full[0], 1);
        mbar_init(&sc_full[1], 1);
        // one for each buffer of scores: P of a chunk may be made before that of the chunk before it has been used
        mbar_init(&p_full[0], 4);
        mbar_init(&p_full[1], 4);
        mbar_init(o_full, 1);
        mbar_init(o_free, 4);
        for (int b = 0; b < BUFS; ++b) {
            mbar_init(&z_ready[b], 4);
            mbar_init(&u_full[b], 1);
            mbar_init(&u_free[b], 4);
        }
        mbar_init(s_ready, 4);
        mbar_init(xs_done, 1);
        *abort_flag = 0;
        fence_barrier_init();
    }
    if (warp == 13) {
        tmem_alloc(tmem_slot, 512);
        tmem_relinquish();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(~0u, *tmem_slot, 0), pz_col = tmem + 2 * TILE, xs_col = pz_col + ZC, u_col = STATE ? tmem : xs_col + ZC;
    pdl_trigger();

    if (warp == 12) {
        if (elect_one()) {
            // a stage's tiles come back from the products one after another; what comes next is on its way to L2 before there is room for it
            auto ahead = [&](int i) {
                if (i >= n) return;
                const int row = seg.first + chunk_of(i) * TILE;
                prefetch_3d(&a.zmap, slab * ZC, h, row);
                if (slab != 0) return;
                prefetch_tile<DX>(&a.ymap, h, row);
                if (!STATE) prefetch_tile<DX>(&a.xmap, h, row);
            };
            for (int i = 0; i < n; ++i) {
                const int s = i % STAGES, row = seg.first + chunk_of(i) * TILE;
                const uint32_t parity = (uint32_t)((i / STAGES + 1) & 1);
                unsigned char *st = stages + s * Sh::STAGE;
                auto load_z = [&] {
                    if (!mbar_wait(&z_empty[s], parity, abort_flag, a.status, 15)) return false;
                    mbar_expect_tx(&z_full[s], Sh::Z_BYTES);
                    tma_load_3d(st + Sh::X_BYTES, &a.zmap, &z_full[s], slab * ZC, h, row);
                    return true;
                };
                // without scores Z is given back as soon as it is weighted, before Y
                if (STATE && !load_z()) break;
                if (!mbar_wait(&xy_empty[s], parity, abort_flag, a.status, 1)) break;
                mbar_expect_tx(&xy_full[s], Sh::STAGE - Sh::Z_BYTES);
                load_tile<DX>(st, &a.ymap, &xy_full[s], h, row);
                if (!STATE) load_tile<DX>(st + Sh::X_BYTES + Sh::Z_BYTES, &a.xmap, &xy_full[s], h, row);
                if (!STATE && !load_z()) break;
                ahead(i + STAGES);
            }
        }
        __syncwarp();
    } else if (warp == 13) {
        {
            const bool lead = elect_one();
            const uint32_t sc_idesc = make_idesc(1, 0, 0, TILE, TILE), pz_idesc = make_idesc(1, 0, 1, TILE, ZC), third_idesc = make_idesc(1, 1, 1, TILE, ZC);
            bool ok = true;
            // U and XS of a chunk, scores of the next, PZ of the chunk: each product has one place in the code, for the instruction cache
            for (int i = -1; i < n && ok; ++i) {
                const unsigned char *Y = stages + ((i + STAGES) % STAGES) * Sh::STAGE, *Z = Y + Sh::X_BYTES, *X = Z + Sh::Z_BYTES;
                if (i >= 0) {
                    if (STATE) ok = warp_wait(&xy_full[i % STAGES], (uint32_t)((i / STAGES) & 1), abort_flag, a.status, 12);
                    if (ok) ok = warp_wait(&z_ready[i % BUFS], (uint32_t)((i / BUFS) & 1), abort_flag, a.status, 3);
                    if (ok && i >= BUFS) ok = warp_wait(&u_free[i % BUFS], (uint32_t)((i / BUFS - 1) & 1), abort_flag, a.status, 13);
                    if (!ok) break;
                    tc_fence_after();
                    // Y^T times all parts side by side: the tile of Y is read once.  Beside scores there is tensor memory for two, and the third is added
                    // to the second.
                    const uint32_t u_idesc = make_idesc(1, 1, 1, TILE, STATE && third ? 3 * ZC : 2 * ZC);
                    const uint64_t y = make_smem_desc(smem_u32(Y), SLAB, 1024), z = make_smem_desc(smem_u32(Z_parts + (i % BUFS) * 3 * Sh::Z_BYTES), SLAB, 1024);
#pragma unroll
                    for (int k = 0; k < TILE / 16; ++k)
                        mma_ss(lead, u_col + (i % BUFS) * U_COLS, y + (uint64_t)(k * 2048 >> 4), z + (uint64_t)(k * 2048 >> 4), u_idesc, k > 0);
                    if (!STATE && third) {
#pragma unroll
                        for (int k = 0; k < TILE / 16; ++k)
                            mma_ss(lead, u_col + ZC, y + (uint64_t)(k * 2048 >> 4), z + (uint64_t)((2 * SLAB + k * 2048) >> 4), third_idesc, true);
                    }
                    commit(lead, &u_full[i % BUFS]);
                    if (STATE) {
                        commit(lead, &xy_empty[i % STAGES]);
                        continue;
                    }
                    if (i > 0) ok = warp_wait(o_free, (uint32_t)((i - 1) & 1), abort_flag, a.status, 4);
                    if (ok) ok = warp_wait(s_ready, (uint32_t)(i & 1), abort_flag, a.status, 5);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t x = make_smem_desc(smem_u32(X), 16, 1024), st = make_smem_desc(smem_u32(S_op), SLAB, 1024);
#pragma unroll
                    for (int k = 0; k < DX / 16; ++k)
                        mma_ss(lead, xs_col, x + (uint64_t)(((k >> 2) * SLAB + (k & 3) * 32) >> 4), st + (uint64_t)(k * 2048 >> 4), pz_idesc, k > 0);
                    commit(lead, xs_done);
                    commit(lead, &xy_empty[i % STAGES]);
                }
                if (!STATE && i + 1 < n) {
                    const int e = i + 1;
                    ok = warp_wait(&xy_full[e % STAGES], (uint32_t)((e / STAGES) & 1), abort_flag, a.status, 2);
                    // rows behind the sequence are cleared first
                    if (ok && tokens_of(e) < TILE) ok = warp_wait(&z_ready[e % BUFS], (uint32_t)((e / BUFS) & 1), abort_flag, a.status, 16);
                    if (!ok) break;
                    tc_fence_after();
                    const unsigned char *st = stages + (e % STAGES) * Sh::STAGE;
                    mma_rows<DX>(lead, tmem + (e & 1) * TILE, st + Sh::X_BYTES + Sh::Z_BYTES, st, sc_idesc);
                    commit(lead, &sc_full[e & 1]);
                }
                if (!STATE && i >= 0) {
                    ok = warp_wait(&p_full[i & 1], (uint32_t)((i >> 1) & 1), abort_flag, a.status, 6);
                    if (!ok) break;
                    tc_fence_after();
                    mma_tokens(lead, pz_col, tmem + (i & 1) * TILE, Z, pz_idesc, false);
                    commit(lead, o_full);
                    commit(lead, &z_empty[i % STAGES]);
                }
            }
        }
        __syncwarp();
    } else if (warp < 4 && !STATE) {
        // thread: token t of a chunk.  Scores to weights.
        {
            const uint32_t lanes = (uint32_t)(warp * 32) << 16;
            bool ok = true;
            const float *w = table + TILE + threadIdx.x;
            for (int i = 0; i < n; ++i) {
                ok = __all_sync(~0u, mbar_wait(&sc_full[i & 1], (uint32_t)((i >> 1) & 1), abort_flag, a.status, 8));
                if (!ok) break;
                tc_fence_after();
                const uint32_t addr = tmem + lanes + (i & 1) * TILE;
                // Weights go over scores that have been read: 16 columns for 32.  The loops of this kernel are no more unrolled than they have to
                // be: one warp of each kind runs on every quarter of an SM, and with all loops unrolled the instruction cache missed
                // in every chunk (65536 tokens of 16 heads 1070 us, 530 with loops like this one).
#pragma unroll 1
                for (int j = 0; j < 4; ++j) {
                    uint32_t p[16];
                    if (back ? j < warp : j > warp) {                     // all zeros
#pragma unroll
                        for (int e = 0; e < 16; ++e) p[e] = 0u;
                    } else {
                        uint32_t x[32];
                        tmem_ld_32x32(addr + j * 32, x);
                        const float *wj = w - j * 32;
                        tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const int c = 2 * e;
                            p[e] = pack_bf16(wj[-c] * __uint_as_float(x[c]), wj[-c - 1] * __uint_as_float(x[c + 1]));
                        }
                    }
                    tmem_st_32x16(addr + j * 16, p);
                }
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&p_full[i & 1]);
            }
        }
    } else if (warp < 8) {
        // thread: token t of a chunk.  Z times its weights, in three parts; where there are no scores warps 0..3 take every other chunk.
        const int t = threadIdx.x & 127, swz = t & 7;
        bool ok = true;
        for (int i = STATE ? warp >> 2 : 0; i < n; i += STATE ? 2 : 1) {
            const int L = tokens_of(i);
            const float beta = t < L ? a.in_scale * power(a2, back ? t + 1 : L - 1 - t) : 0.f;
            ok = __all_sync(~0u, mbar_wait(&z_full[i % STAGES], (uint32_t)((i / STAGES) & 1), abort_flag, a.status, 10));
            if (ok && L < TILE) ok = __all_sync(~0u, mbar_wait(&xy_full[i % STAGES], (uint32_t)((i / STAGES) & 1), abort_flag, a.status, 17));
            if (ok && i >= BUFS) ok = __all_sync(~0u, mbar_wait(&u_full[i % BUFS], (uint32_t)((i / BUFS - 1) & 1), abort_flag, a.status, 9));
            if (!ok) break;
            unsigned char *Y = stages + (i % STAGES) * Sh::STAGE, *Z = Y + Sh::X_BYTES, *Z_hi = Z_parts + (i % BUFS) * 3 * Sh::Z_BYTES;
            if (t >= L) {                              // rows behind the sequence: they meet weights of 0
#pragma unroll 1
                for (int j = 0; j < 8; ++j) {
                    *reinterpret_cast<uint4 *>(Z + t * 128 + j * 16) = make_uint4(0u, 0u, 0u, 0u);
                    for (int c = 0; c < DX / 64; ++c) *reinterpret_cast<uint4 *>(Y + c * SLAB + t * 128 + j * 16) = make_uint4(0u, 0u, 0u, 0u);
                }
            }
            // a row is one thread's, in any order: this one meets every bank once in eight lanes
            const __nv_bfloat162 b_hi = __float2bfloat162_rn(beta), b_lo = __float2bfloat162_rn(beta - __low2float(b_hi));
#pragma unroll 1
            for (int b = 0; b < 2; ++b) {
                uint4 v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = *reinterpret_cast<const uint4 *>(Z + t * 128 + (((b * 4 + j) ^ swz) << 4));
                if (third) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int o = t * 128 + (((b * 4 + j) ^ swz) << 4);
                        uint4 hi, mid, lo;
                        times(beta, v[j].x, hi.x, mid.x, lo.x);
                        times(beta, v[j].y, hi.y, mid.y, lo.y);
                        times(beta, v[j].z, hi.z, mid.z, lo.z);
                        times(beta, v[j].w, hi.w, mid.w, lo.w);
                        *reinterpret_cast<uint4 *>(Z_hi + o) = hi;
                        *reinterpret_cast<uint4 *>(Z_hi + Sh::Z_BYTES + o) = mid;
                        *reinterpret_cast<uint4 *>(Z_hi + 2 * Sh::Z_BYTES + o) = lo;
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const int o = t * 128 + (((b * 4 + j) ^ swz) << 4);
                        uint4 hi, lo;
                        times(b_hi, b_lo, v[j].x, hi.x, lo.x);
                        times(b_hi, b_lo, v[j].y, hi.y, lo.y);
                        times(b_hi, b_lo, v[j].z, hi.z, lo.z);
                        times(b_hi, b_lo, v[j].w, hi.w, lo.w);
                        *reinterpret_cast<uint4 *>(Z_hi + o) = hi;
                        *reinterpret_cast<uint4 *>(Z_hi + Sh::Z_BYTES + o) = lo;
                    }
                }
            }
            fence_proxy_async();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(&z_ready[i % BUFS]);
                if (STATE) mbar_arrive(&z_empty[i % STAGES]);
            }
        }
    } else {
        // thread: row r of S, and token r of a chunk's out
        const int r = threadIdx.x - 256, swz = r & 7, w = warp & 3;
        const uint32_t lanes = (uint32_t)(w * 32) << 16;
        const bool row = r < a.dx;
        const int64_t plane = (int64_t)a.dx * a.dz, at = (int64_t)r * a.dz + slab * ZC;
        Pair S[32];
        {
            const float *from = nullptr;
            if (!STATE) from = a.states ? a.states + ((int64_t)tile * a.heads + h) * plane : a.init ? a.init + ((int64_t)seg.seq * a.heads + h) * plane : nullptr;
            const int64_t step = a.transposed ? a.dx : 1;
            if (from) from += a.transposed ? (int64_t)slab * ZC * a.dx + r : at;
#pragma unroll
            for (int c = 0; c < 32; ++c) {
                const bool in = from && row && slab * ZC + 2 * c < a.dz;
                S[c] = pair(in ? from[2 * c * step] : 0.f, in ? from[(2 * c + 1) * step] : 0.f);
            }
        }
        bool ok = true;
        const float keep_full = carry(decay, TILE);
        const float full_alpha = a.out_scale * power(a2, back ? TILE - 1 - r : r + 1);
        auto write = [&](int i) {
            const int first = chunk_of(i) * TILE, L = tokens_of(i);
            const float alpha = !back || L == TILE ? full_alpha : a.out_scale * power(a2, max(L - 1 - r, 0));
            ok = __all_sync(~0u, mbar_wait(o_full, (uint32_t)(i & 1), abort_flag, a.status, 7));
            if (!ok) return;
            tc_fence_after();
            if (!third) {
                // a warp's 32 rows go through shared memory and out in one copy; rows at a sequence's end are written one by one
                if (lane == 0) tma_store_wait_read();
                __syncwarp();
#pragma unroll 1
                for (int b = 0; b < 4; ++b) {
                    uint32_t pz[16], xs[16];
                    tmem_ld_32x16(pz_col + lanes + b * 16, pz);
                    tmem_ld_32x16(xs_col + lanes + b * 16, xs);
                    tmem_ld_wait();
                    if (b == 3) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(o_free);
                    }
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        uint32_t u[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const int c = j * 8 + 2 * k;
                            u[k] = pack_bf16(fma(pair(alpha, alpha), pair(xs[c], xs[c + 1]), mul(pair(a.out_scale, a.out_scale), pair(pz[c], pz[c + 1]))));
                        }
                        *reinterpret_cast<uint4 *>(out_rows + r * 128 + (((b * 2 + j) ^ swz) << 4)) = make_uint4(u[0], u[1], u[2], u[3]);
                    }
                }
                const int row = seg.first + first + w * 32;
                if (w * 32 + 32 <= L) {
                    fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) tma_store_3d(&a.outmap, out_rows + w * 4096, slab * ZC, h, row);
                } else {
                    __syncwarp();
                    const int c = lane & 7;
                    for (int k = lane / 8; w * 32 + k < L; k += 4)
                        if (slab * ZC + c * 8 < a.dz)
                            *reinterpret_cast<uint4 *>(a.out + ((int64_t)(row + k) * a.heads + h) * a.dz + slab * ZC + c * 8) =
                                *reinterpret_cast<const uint4 *>(out_rows + (w * 32 + k) * 128 + ((c ^ (k & 7)) << 4));
                }
            } else {
                // Four lanes exchange their rows' pieces, so that they write 64 bytes of a row side by side; one by one every piece of 16 bytes
                // took a cycle of the store (65536 tokens of 16 heads 300 us in this kernel, so 271).
                bf16 *to = a.out + ((int64_t)(seg.first + first + w * 32 + (lane & ~3)) * a.heads + h) * a.dz + slab * ZC + (lane & 3) * 8;
                const int64_t stride = (int64_t)a.heads * a.dz;
                const int rows = L - (w * 32 + (lane & ~3)), cols = a.dz - slab * ZC - (lane & 3) * 8;
#pragma unroll 1
                for (int b = 0; b < 2; ++b) {
                    uint32_t v[4][4];
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        uint32_t pz[16], xs[16];
                        tmem_ld_32x16(pz_col + lanes + b * 32 + j * 16, pz);
                        tmem_ld_32x16(xs_col + lanes + b * 32 + j * 16, xs);
                        tmem_ld_wait();
#pragma unroll
                        for (int k = 0; k < 8; ++k)
                            v[j * 2 + k / 4][k % 4] = pack_bf16(fma(pair(alpha, alpha), pair(xs[2 * k], xs[2 * k + 1]),
                                                                    mul(pair(a.out_scale, a.out_scale), pair(pz[2 * k], pz[2 * k + 1]))));
                    }
                    if (b == 1) {
                        tc_fence_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(o_free);
                    }
#pragma unroll
                    for (int s = 1; s < 4; s *= 2)
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (!(k & s))
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    const bool odd = lane & s;
                                    const uint32_t got = __shfl_xor_sync(~0u, odd ? v[k][e] : v[k | s][e], s);
                                    if (odd) v[k][e] = got;
                                    else v[k | s][e] = got;
                                }
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k < rows && b * 32 < cols) *reinterpret_cast<uint4 *>(to + k * stride + b * 32) = make_uint4(v[k][0], v[k][1], v[k][2], v[k][3]);
                }
            }
        };
        for (int i = 0; i < n; ++i) {
            const int L = tokens_of(i);
            const float keep = L == TILE ? keep_full : carry(decay, L);
            if (!STATE) {
                if (i > 0) ok = __all_sync(~0u, mbar_wait(xs_done, (uint32_t)((i - 1) & 1), abort_flag, a.status, 11));
                if (!ok) break;
                if (r < DX) {
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        *reinterpret_cast<uint4 *>(S_op + r * 128 + ((j ^ swz) << 4)) =
                            make_uint4(pack_bf16(S[j * 4]), pack_bf16(S[j * 4 + 1]), pack_bf16(S[j * 4 + 2]), pack_bf16(S[j * 4 + 3]));
                }
                fence_proxy_async();
                __syncwarp();
                if (lane == 0) mbar_arrive(s_ready);
                if (i > 0) write(i - 1);
                if (!ok) break;
            }
            ok = __all_sync(~0u, mbar_wait(&u_full[i % BUFS], (uint32_t)((i / BUFS) & 1), abort_flag, a.status, 14));
            if (!ok) break;
            tc_fence_after();
            const uint32_t u_addr = u_col + lanes + (i % BUFS) * U_COLS;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t hi[16], lo[16];
                tmem_ld_32x16(u_addr + j * 16, hi);
                tmem_ld_32x16(u_addr + ZC + j * 16, lo);
                tmem_ld_wait();
                if (STATE && third) {
                    uint32_t more[16];
                    tmem_ld_32x16(u_addr + 2 * ZC + j * 16, more);
                    tmem_ld_wait();
#pragma unroll
                    for (int c = 0; c < 16; ++c) lo[c] = __float_as_uint(__uint_as_float(lo[c]) + __uint_as_float(more[c]));
                }
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    S[j * 8 + c] = fma(pair(keep, keep), S[j * 8 + c], add(pair(hi[2 * c], hi[2 * c + 1]), pair(lo[2 * c], lo[2 * c + 1])));
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&u_free[i % BUFS]);
        }
        if (!STATE && ok && n > 0) write(n - 1);
        if (!STATE && lane == 0) tma_store_wait();
        const bool end = seg.index == (back ? 0 : seg.count - 1);
        float *to = STATE ? a.states + ((int64_t)tile * a.heads + h) * plane : end && third ? a.last + ((int64_t)seg.seq * a.heads + h) * plane : nullptr;
        if (ok && to && row) {
#pragma unroll
            for (int c = 0; c < 64; c += 4)
                if (slab * ZC + c < a.dz) {
                    const float2 u = split(S[c / 2]), v = split(S[c / 2 + 1]);
                    *reinterpret_cast<float4 *>(to + at + c) = make_float4(u.x, u.y, v.x, v.y);
                }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 13) {
        tc_fence_after();
        tmem_dealloc(tmem, 512);
    }
}

// The segments' own sums become the states that enter the segments and the one behind the last; a thread owns four elements of a head's state.
__global__ void __launch_bounds__(256) fade_carry_kernel(const __grid_constant__ FadeRuns runs, int parts)
{
    const FadeArgs &a = runs.run[blockIdx.z / parts];
    pdl_wait();
    pdl_trigger();
    const Segment seg = segment_of(a, blockIdx.x, threadIdx.x & 31);
    // offsets that decrease can make more segments than there is room for: those have no states
    if (seg.seq < 0 || seg.index != 0 || blockIdx.x + seg.count > gridDim.x) return;
    const int h = blockIdx.y, plane = a.dx * a.dz, e = (blockIdx.z % parts * 256 + threadIdx.x) * 4;
    if (e >= plane) return;
    const Rows r = rows_of(a.offsets, seg.seq, a.n);
    const int rows = a.chunks * TILE;
    const int64_t step = (int64_t)a.heads * plane;
    float *states = a.states + ((int64_t)blockIdx.x * a.heads + h) * plane + e;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (a.init) s = *reinterpret_cast<const float4 *>(a.init + ((int64_t)seg.seq * a.heads + h) * plane + e);
    const float decay = a.log_decay[h], whole = carry(decay, rows);
    constexpr int AT_ONCE = 8;
    for (int i0 = 0; i0 < seg.count; i0 += AT_ONCE) {
        float4 own[AT_ONCE];
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const int i = i0 + j, k = a.backwards ? seg.count - 1 - i : i;
            own[j] = i < seg.count && (a.last || i + 1 < seg.count) ? *reinterpret_cast<const float4 *>(states + k * step) : make_float4(0.f, 0.f, 0.f, 0.f);
        }
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const int i = i0 + j, k = a.backwards ? seg.count - 1 - i : i;
            if (i >= seg.count) break;
            const float f = (k + 1) * rows <= r.len ? whole : carry(decay, r.len - k * rows);
            *reinterpret_cast<float4 *>(states + k * step) = s;
            s = make_float4(fmaf(f, s.x, own[j].x), fmaf(f, s.y, own[j].y), fmaf(f, s.z, own[j].z), fmaf(f, s.w, own[j].w));
        }
    }
    if (a.last) *reinterpret_cast<float4 *>(a.last + ((int64_t)seg.seq * a.heads + h) * plane + e) = s;
}

// Chunks of a segment, 0: whole sequences.  Whole, a call takes the longest sequence's chunks one after another, here estimated as twice the mean
// (the lengths are on the device); in segments 1.6 times its share of all chunks, as the states are summed first, and the time of some 12
// chunks for two launches more.  Segments are so long that two come to every SM.
// us, in segments / whole: 6 sequences of up to 4096 tokens, 16 heads, with gradient 355 / 256; 9 of up to 1333, 8 heads of 64 28 / 27; 2 of up to 4000 28 / 64.
static int segment_chunks(int64_t n, int64_t nseq, int64_t heads, int64_t d)
{
    const int64_t sms = sm_count_or_default(), blocks = heads * ((d + fade::ZC - 1) / fade::ZC), wanted = 2 * sms / blocks;
    const int64_t chunks = (n + TILE - 1) / TILE, mean = (chunks + nseq - 1) / nseq, longest = 2 * mean < chunks ? 2 * mean : chunks;
    if (wanted <= 1 || longest <= chunks * blocks * 8 / (5 * sms) + 12) return 0;
    const int64_t each = (chunks + wanted - 1) / wanted, some = each < 4 ? 4 : each;
    return some >= chunks ? 0 : (int)some;
}

template <int DX, bool STATE>
static st_status launch_fade(const FadeRuns &r, int count, cudaStream_t stream)
{
    const size_t smem = fade::Shape<DX, STATE>::SMEM;
    if (!ensure_dynamic_smem(fade_kernel<DX, STATE>, smem)) return ST_ERR_CUDA;
    const FadeArgs &a = r.run[0];
    int slabs = 1;
    for (int i = 0; i < count; ++i) slabs = std::max(slabs, (r.run[i].dz + fade::ZC - 1) / fade::ZC);
    return launch(fade_kernel<DX, STATE>, dim3((unsigned)((int64_t)a.tiles * slabs), (unsigned)a.heads, (unsigned)count), fade::THREADS, smem, stream, r);
}

// `count` runs over the same tokens at once: their states that enter the segments (of y (x) z as it is kept: not transposed), or all of them.
template <bool STATE>
static st_status run_fades(FadeRuns &r, int count, cudaStream_t stream)
{
    bool wide = false;
    for (int i = 0; i < count; ++i) {
        FadeArgs &a = r.run[i];
        const Table out{a.out, (int64_t)a.heads * a.dz, a.dz};
        if (!make_tmap_table(&a.ymap, a.y, a.n, a.heads, a.dx) || !make_tmap_table(&a.zmap, a.z, a.n, a.heads, a.dz)) return ST_ERR_CUDA;
        if (!STATE && (!make_tmap_table(&a.xmap, a.x, a.n, a.heads, a.dx) || !make_tmap_table(&a.outmap, out, a.n, a.heads, a.dz, 32))) return ST_ERR_CUDA;
        wide = wide || a.dx > 64;
    }
    const st_status rc = wide ? launch_fade<128, STATE>(r, count, stream) : launch_fade<64, STATE>(r, count, stream);
    if (!STATE || rc != ST_OK) return rc;
    const FadeArgs &a = r.run[0];
    const int parts = (a.dx * a.dz + 1023) / 1024;
    return launch(fade_carry_kernel, dim3((unsigned)a.tiles, (unsigned)a.heads, (unsigned)(parts * count)), 256, 0, stream, r, parts);
}

// The states of the segments of one run.
static size_t states_floats(int64_t n, int64_t nseq, int64_t heads, int64_t d)
{
    const int chunks = segment_chunks(n, nseq, heads, d);
    return chunks ? (size_t)most_tiles(n, nseq, (int64_t)chunks * TILE) * heads * d * d : 0;
}

static st_status check_decay(const st_tokens *t, const int32_t *offsets)
{
    const st_status rc = check_tokens(t);
    if (rc != ST_OK) return rc;
    if (t->nq != t->nk || t->heads != t->kv_heads) return ST_ERR_SHAPE;
    return !offsets && t->nseq != 1 ? ST_ERR_NULL : ST_OK;
}

static FadeArgs fade_args(const st_tokens *t, const float *log_decay, const int32_t *offsets, void *ws)
{
    FadeArgs a = {};
    a.status = (unsigned *)ws;
    a.check = 1;
    a.chunks = segment_chunks(t->nq, t->nseq, t->heads, t->d > t->dv ? t->d : t->dv);
    a.states = a.chunks ? (float *)((unsigned char *)ws + kWsHeaderBytes) : nullptr;
    if (!a.chunks) a.chunks = 1 << 22;                                 // 2^29 tokens, as many as a sequence can have
    a.dx = (int)t->d;
    a.dz = (int)t->dv;
    a.log_decay = log_decay;
    a.offsets = offsets;
    a.nseq = (int)t->nseq;
    a.n = (int)t->nq;
    a.tiles = (int)most_tiles(a.n, a.nseq, (int64_t)a.chunks * TILE);
    a.heads = (int)t->heads;
    a.in_scale = a.out_scale = 1.f;
    return a;
}

static Table table_of(const void *p, int64_t rows, int64_t heads, int64_t row, int64_t head)
{
    return {(const bf16 *)p, stride_of(rows, row), stride_of(heads, head)};
}

}  // namespace attn

size_t attn_decay_workspace(int64_t n, int64_t nseq, int64_t heads, int64_t d, bool gradient)
{
    if (n <= 0 || nseq <= 0 || heads <= 0 || d <= 0 || d > 128 || n > (1 << 29) || heads > 65535 || nseq > (1 << 20)) return 0;
    return kWsHeaderBytes + round_up((gradient ? 2 : 1) * attn::states_floats(n, nseq, heads, d) * sizeof(float), 256);
}

}  // namespace st

using namespace st;
using namespace st::attn;

extern "C" {

st_status st_attn_decay(const st_tokens *t, const void *q, const void *k, const void *v, const float *log_decay,
                        const int32_t *offsets, const float *state_in, float scale, void *out, float *state_out,
                        void *ws, size_t ws_bytes, void *stream)
{
    st_status rc = check_decay(t, offsets);
    if (rc != ST_OK) return rc;
    if (!q || !k || !v || !log_decay || !out) return ST_ERR_NULL;
    for (const void *p : {q, k, v, (const void *)log_decay, (const void *)offsets, (const void *)state_in, (const void *)out, (const void *)state_out})
        if (!aligned16(p)) return ST_ERR_ALIGN;
    if (!ws || ws_bytes < attn_decay_workspace(t->nq, t->nseq, t->heads, t->d > t->dv ? t->d : t->dv, false)) return ST_ERR_WORKSPACE;
    if (!aligned256(ws)) return ST_ERR_ALIGN;
    // the blocks of a head share its x and y; what one reads of z and of the first state it alone writes
    const int64_t out_bytes = t->nq * t->heads * t->dv * 2, state_bytes = t->nseq * t->heads * t->d * t->dv * 4;
    const Operand Q = q_of(t, q), K = k_of(t, k), V = v_of(t, v);
    const bool alone = t->dv <= fade::ZC;
    if (Q.under(out, out_bytes, alone) || K.under(out, out_bytes, alone) || V.under(out, out_bytes, true) || arrays_meet(out, out_bytes, state_in, state_bytes) ||
        arrays_meet(out, out_bytes, state_out, state_bytes))
        return ST_ERR_UNSUPPORTED;
    if (state_out && (Q.under(state_out, state_bytes) || K.under(state_out, state_bytes) || V.under(state_out, state_bytes) ||
                      (state_out != state_in && arrays_meet(state_out, state_bytes, state_in, state_bytes))))
        return ST_ERR_UNSUPPORTED;
    FadeArgs a = fade_args(t, log_decay, offsets, ws);
    a.x = table_of(q, t->nq, t->heads, t->q_row, t->q_head);
    a.y = table_of(k, t->nk, t->heads, t->k_row, t->k_head);
    a.z = table_of(v, t->nk, t->heads, t->v_row, t->v_head);
    a.init = state_in;
    a.last = state_out;
    a.out_scale = scale;
    a.out = (bf16 *)out;
    FadeRuns r = {};
    r.run[0] = a;
    if (a.states) {
        if ((rc = run_fades<true>(r, 1, (cudaStream_t)stream)) != ST_OK) return rc;
        r.run[0].check = 0;
    }
    return run_fades<false>(r, 1, (cudaStream_t)stream);
}

st_status st_attn_decay_grad(const st_tokens *t, const void *q, const void *k, const void *v, const float *log_decay,
                             const void *dout, const int32_t *offsets, const float *state_in, const float *dstate_out,
                             float scale, void *dq, void *dk, void *dv, float *dstate_in, void *ws, size_t ws_bytes,
                             void *stream)
{
    st_status rc = check_decay(t, offsets);
    if (rc != ST_OK) return rc;
    if (!q || !k || !v || !log_decay || !dout || !dq || !dk || !dv) return ST_ERR_NULL;
    // the runs go at once: one reads what another would write
    if (dstate_in && (dstate_in == dstate_out || dstate_in == state_in)) return ST_ERR_UNSUPPORTED;
    for (const void *p : {q, k, v, (const void *)log_decay, dout, (const void *)offsets, (const void *)state_in, (const void *)dstate_out,
                          (const void *)dq, (const void *)dk, (const void *)dv, (const void *)dstate_in})
        if (!aligned16(p)) return ST_ERR_ALIGN;
    if (!ws || ws_bytes < attn_decay_workspace(t->nq, t->nseq, t->heads, t->d > t->dv ? t->d : t->dv, true)) return ST_ERR_WORKSPACE;
    if (!aligned256(ws)) return ST_ERR_ALIGN;
    {
        // nor may any other result take the place of an operand or of a result
        struct Result {
            const void *p;
            int64_t bytes;
        };
        const int64_t rows = t->nq * t->heads, state_bytes = t->nseq * t->heads * t->d * t->dv * 4;
        const Operand tables[] = {q_of(t, q), k_of(t, k), v_of(t, v), dense_of(dout, t->nq, t->heads, t->dv)};
        const Result results[] = {{dq, rows * t->d * 2}, {dk, rows * t->d * 2}, {dv, rows * t->dv * 2}, {dstate_in, dstate_in ? state_bytes : 0}};
        for (int i = 0; i < 4; ++i) {
            const Result &r = results[i];
            if (!r.p) continue;
            bool wrong = arrays_meet(r.p, r.bytes, state_in, state_bytes) || arrays_meet(r.p, r.bytes, dstate_out, state_bytes);
            for (const Operand &o : tables) wrong = wrong || o.under(r.p, r.bytes);
            for (int j = 0; j < i; ++j) wrong = wrong || arrays_meet(r.p, r.bytes, results[j].p, results[j].bytes);
            if (wrong) return ST_ERR_UNSUPPORTED;
        }
    }
    const Table Q = table_of(q, t->nq, t->heads, t->q_row, t->q_head), K = table_of(k, t->nk, t->heads, t->k_row, t->k_head),
                V = table_of(v, t->nk, t->heads, t->v_row, t->v_head), O = table_of(dout, t->nq, t->heads, t->heads * t->dv, t->dv);
    cudaStream_t s = (cudaStream_t)stream;
    FadeArgs a = fade_args(t, log_decay, offsets, ws);
    FadeRuns r = {};
    FadeArgs &dq_run = r.run[0], &dv_run = r.run[1], &dk_run = r.run[2];
    // dq[t] = scale sum e^{a(t-s)} (dout[t].v[s]) k[s], with the states of k (x) v
    a.y = K;
    a.z = V;
    a.init = state_in;
    dq_run = a;
    // dv[s] = sum e^{a(t-s)} (k[s].q[t]) scale dout[t], backwards, with the states of q (x) dout
    a.x = K;
    a.y = Q;
    a.z = O;
    a.backwards = 1;
    a.check = 0;
    a.init = dstate_out;
    a.in_scale = scale;
    a.out = (bf16 *)dv;
    if (a.states) a.states += states_floats(t->nq, t->nseq, t->heads, t->d > t->dv ? t->d : t->dv);
    dv_run = a;
    dv_run.last = dstate_in;
    if (a.states) {
        if ((rc = run_fades<true>(r, 2, s)) != ST_OK) return rc;
        dq_run.check = 0;
    }
    dq_run.x = O;
    dq_run.y = V;
    dq_run.z = K;
    std::swap(dq_run.dx, dq_run.dz);
    dq_run.transposed = 1;
    dq_run.out_scale = scale;
    dq_run.out = (bf16 *)dq;
    // dk[s] = sum e^{a(t-s)} (v[s].dout[t]) scale q[t], backwards, with the same states
    a.x = V;
    a.y = O;
    a.z = Q;
    std::swap(a.dx, a.dz);
    a.transposed = 1;
    a.out = (bf16 *)dk;
    dk_run = a;
    return run_fades<false>(r, 3, s);
}

}  // extern "C"
