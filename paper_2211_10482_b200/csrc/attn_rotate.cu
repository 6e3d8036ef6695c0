// st_attn_rotate and its gradient: an RMS norm of every head and a rotation of pairs of its columns, in one pass.
//
// Bound by memory as long as a row (one head of one token) takes few instructions.  8 lanes (4 up to 64 columns) own a row, each 16 of its columns as two
// pieces of 16 bytes which hold both columns of eight pairs, whichever way they are paired: a lane turns its pairs by itself, two at a time in packed fp32.  A
// warp takes a token, or some of its heads.  Its lanes make the sines and cosines of two of its angles each, all others take them by shuffles, once for all
// heads.  An angle is position freq / 2 pi turns, of which only the fraction counts: with freq / 2 pi in units of 2^-64, cut off by less than two of them, the
// product's low 64 bits are that fraction of a turn.  Its first 32 are kept: off by at most 2^-32 + |position| 2^-63 turns, 2^-31 at any position.  The nearest quarter of a
// turn is its top two bits, and the rest, at most pi / 4, goes into the Taylor series of sine and cosine (their next terms are below 2^-25).  Rows come by asynchronous copies to a ring of the warp's own, over the ends of tokens and of q.
//
// The gradient's warps keep the weights' sums in registers; a second kernel adds the blocks' sums in a fixed order.
//
// 32768 tokens of 16 + 4 heads of 128 with norms, inputs not in L2: forward and gradient together 161.6 us (149 where a part of them is), of which the gradient
// 93 (5.4 TB/s) and the sums 4; 12289 tokens of 24 heads without norms 29.5 us (5.1 TB/s).  (With 16 lanes to a row and rows loaded when they are needed
// forward and gradient took 504 us together.)
//
// Where `rot` is no multiple of 16, pieces of a half begin off their 16 bytes, and pairs and pieces do not fit together: columns are then taken one by one,
// from shared memory and with stores of 2 bytes, at a fifth of the speed.  32768 tokens of 24 heads of 80 with norms: 20 turning columns 337 us, 32 of them 68;
// with the gradient 752 and 169.
#include "attn_common.cuh"
#include "tc_common.cuh"

namespace st {
namespace attn {

struct RotateArgs {
    const bf16 *q, *k;
    int64_t q_row, q_head, k_row, k_head;
    const bf16 *dq_out, *dk_out;           // gradient only
    bf16 *q_out, *k_out;                   // gradient: dq, dk
    const int *positions;
    const float *freq;
    const void *q_weight, *k_weight;
    bool weight_f32;
    int n, heads, width, d, rot;           // width: heads of q and k
    float eps, factor;
    int cols, chunks, items;               // heads of an item, items of a token, items
    float *part;                           // [block][q, k][128] sums of the weights' gradient, or NULL
};

namespace rot {
constexpr int MAX_D = 128, WEIGHTS = 2 * 4 * 16;      // pieces of the weights in shared memory
ST_HD constexpr int warps(bool grad) { return grad ? 6 : 8; }                            // of a block
ST_HD constexpr int min_blocks(bool odd, bool grad) { return odd || grad ? 2 : 3; }       // on an SM
constexpr int AHEAD = 4;                                                                 // rows of a lane on their way
}  // namespace rot

// The fraction of freq / 2 pi, in units of 2^-64: the frequency's 24 bits times the first 128 bits of 1 / 2 pi, in whole numbers.  |freq| below 2^24.  (One
// product in 64-bit floating point takes as long, within 0.4 us of a call, and keeps too few bits of the fraction where a frequency is many turns.)
__device__ __forceinline__ uint64_t turns_of(float freq)
{
    const uint32_t bits = __float_as_uint(freq), exponent = bits >> 23 & 255;
    const uint64_t m = (bits & 0x7FFFFF) | (exponent ? 0x800000 : 0);
    const int shift = 150 - (int)max(exponent, 1u);        // m 2^-shift
    const uint64_t low = m * 0x28be60db9391054aull, p = low + __umul64hi(m, 0x7f09d5f47d4d3770ull), q = __umul64hi(m, 0x28be60db9391054aull) + (p < low);
    const uint64_t t = shift <= 0 ? p : shift < 64 ? p >> shift | q << (64 - shift) : shift < 128 ? q >> (shift - 64) : 0;
    return bits >> 31 ? 0 - t : t;
}

// Sum over the lanes of a row, the same in all of them.
template <int LANES>
__device__ __forceinline__ float row_sum(float x)
{
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
    return x;
}
__device__ __forceinline__ void copy_piece(uint32_t dst, const void *src, bool there)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %2, 0;\n\t@p cp.async.cg.shared.global [%0], [%1], 16;\n\t}" ::"r"(dst), "l"(src), "r"((int)there) : "memory");
}
// Cosines and sines of two angles, given as fractions of 2^32 turns.
__device__ __forceinline__ void cos_sin(uint32_t t0, uint32_t t1, float (&c)[2], float (&s)[2])
{
    const uint32_t q0 = t0 + 0x20000000u, q1 = t1 + 0x20000000u;          // top two bits: the nearest quarter
    constexpr float unit = 1.4629180792671596e-9f;                         // 2 pi / 2^32
    const Pair x = pair((float)(int)(t0 - (q0 & 0xC0000000u)) * unit, (float)(int)(t1 - (q1 & 0xC0000000u)) * unit), y = mul(x, x);
    auto all = [](float v) { return pair(v, v); };
    const Pair si = fma(mul(x, y), fma(y, fma(y, fma(y, all(1.f / 362880), all(-1.f / 5040)), all(1.f / 120)), all(-1.f / 6)), x);
    const Pair co = fma(y, fma(y, fma(y, fma(y, all(1.f / 40320), all(-1.f / 720)), all(1.f / 24)), all(-0.5f)), all(1.f));
    const float2 ss = split(si), cc = split(co);
    const uint32_t q[2] = {q0, q1};
    const float sv[2] = {ss.x, ss.y}, cv[2] = {cc.x, cc.y};
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        // quarters 0..3: (c, s), (-s, c), (-c, -s), (s, -c)
        const bool odd = q[i] & 0x40000000u;
        const float a = odd ? sv[i] : cv[i], b = odd ? cv[i] : sv[i];
        c[i] = __uint_as_float(__float_as_uint(a) ^ ((q[i] ^ (q[i] << 1)) & 0x80000000u));
        s[i] = __uint_as_float(__float_as_uint(b) ^ (q[i] & 0x80000000u));
    }
}
// Eight pairs from two pieces of a row: first columns in a, second ones in b.
template <bool INTER>
__device__ __forceinline__ void pairs_of(const uint4 &p, const uint4 &q, Pair (&a)[4], Pair (&b)[4])
{
    if (!INTER) {
        unpack8(p, a);
        unpack8(q, b);
    } else {
        const uint32_t w[8] = {p.x, p.y, p.z, p.w, q.x, q.y, q.z, q.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = pair(w[2 * i] << 16, w[2 * i + 1] << 16);
            b[i] = pair(w[2 * i] & 0xFFFF0000u, w[2 * i + 1] & 0xFFFF0000u);
        }
    }
}
template <bool INTER>
__device__ __forceinline__ void pieces_of(const Pair (&a)[4], const Pair (&b)[4], uint4 &p, uint4 &q)
{
    if (!INTER) {
        p = pack8(a);
        q = pack8(b);
    } else {
        Pair x[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = split(a[i]), g = split(b[i]);
            (i < 2 ? x[2 * i] : y[2 * i - 4]) = pair(f.x, g.x);
            (i < 2 ? x[2 * i + 1] : y[2 * i - 3]) = pair(f.y, g.y);
        }
        p = pack8(x);
        q = pack8(y);
    }
}

// MIXED: all rows of a token, of q and of k, fit a warp's groups of lanes and are taken at once; a group's row is of one table for good.
// LANES to a row; ODD: `rot` is no multiple of 16, so that pieces and pairs do not fit together and columns are taken one by one.
template <int LANES, bool NORM, bool INTER, bool ODD, bool GRAD, bool MIXED>
__global__ void __launch_bounds__(rot::warps(GRAD) * 32, rot::min_blocks(ODD, GRAD)) rotate_kernel(const RotateArgs a)
{
    using namespace rot;
    constexpr int ROWS = 32 / LANES, WARPS = rot::warps(GRAD);
    constexpr bool TWO = GRAD && NORM;                     // tables that are read: x and dy, or one of them
    constexpr int TABLE = ODD ? 32 : 64, STAGE = TABLE * (TWO ? 2 : 1);       // pieces of a step
    extern __shared__ __align__(16) uint4 smem[];
    float4(*weights)[4][LANES] = reinterpret_cast<float4(*)[4][LANES]>(smem);      // [q, k][a's pairs 0..3, 4..7, b's][lane of a row]
    uint4 *ring = smem + (NORM ? WEIGHTS : 0);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, sub = lane / LANES, l = lane % LANES, half = a.rot / 2;
    uint4 *mine = ring + warp * AHEAD * STAGE;
    // A lane's pieces begin at columns a0 and b0, both of which are next to its neighbours': pairs in halves 8 l .. 8 l + 7, then the lanes whose columns do
    // not turn; neighbours 8 columns each of the row's halves.  p0 and p1: the first pairs of a0..7 and b0..7.
    const int turning = (half + 7) / 8, resting = (a.d - a.rot + 15) / 16;
    const bool turns = l < turning;                        // halves
    const int a0 = INTER || turns ? 8 * l : a.rot + 8 * (l - turning) + (ODD ? 8 * (l - turning) : 0);
    const int b0 = INTER ? 8 * (l + LANES) : turns ? half + 8 * l : a0 + (ODD ? 8 : l - turning < resting ? 8 * resting : MAX_D);
    const bool turn_a = ODD || (INTER ? a0 < a.rot : turns), turn_b = ODD || (INTER ? b0 < a.rot : turns);
    const bool in_a = a0 < a.d && (INTER || turns || l - turning < resting), in_b = b0 < a.d;
    // columns of pair e
    auto col_a = [&](int e) { return INTER ? (ODD ? 16 * l + 2 * e : (e < 4 ? a0 : b0 - 8) + 2 * e) : a0 + e; };
    auto col_b = [&](int e) { return INTER ? col_a(e) + 1 : b0 + e; };
    auto has_a = [&](int e) { return ODD ? col_a(e) < (!INTER && turns ? half : a.d) : INTER && e >= 4 ? in_b : in_a; };
    auto has_b = [&](int e) { return ODD ? col_b(e) < (!INTER && turns ? a.rot : a.d) : INTER && e < 4 ? in_a : in_b; };
    // this lane's angles, of pairs 2 lane and 2 lane + 1, as fractions of 2^64 turns a position
    uint64_t turn[2] = {0, 0};
    const float inv_d = 1.f / a.d;
    Pair dwa[2][4], dwb[2][4];
    if (TWO)
#pragma unroll
        for (int e = 0; e < 4; ++e) dwa[0][e] = dwa[1][e] = dwb[0][e] = dwb[1][e] = pair(0.f, 0.f);

#pragma unroll
    for (int i = 0; i < AHEAD * STAGE / 32; ++i) mine[i * 32 + lane] = make_uint4(0u, 0u, 0u, 0u);      // what no copy reaches
    pdl_wait();
    pdl_trigger();
    float freq[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) freq[i] = 2 * lane + i < half ? a.freq[2 * lane + i] : 0.f;
    // whether one of the row's is no number, or more than the product is exact for
    auto no_turn = [](float f) { return !(fabsf(f) < 16777216.f); };
    const bool some_none = __any_sync(~0u, no_turn(freq[0]) || no_turn(freq[1]));
    const int kv_heads = a.width - a.heads;
    // Heads q0.. of nq of q and k0.. of nk of k of a token: an item.
    struct Item {
        int t, q0, nq, k0, nk;
    };
    auto item_of = [&](int i) {
        if (a.chunks == 1) return Item{i, 0, a.heads, 0, kv_heads};
        const int t = i / a.chunks, c0 = (i - t * a.chunks) * a.cols, c1 = min(c0 + a.cols, a.width);
        const int q0 = min(c0, a.heads), k0 = max(c0, a.heads);
        return Item{t, q0, min(c1, a.heads) - q0, k0 - a.heads, max(c1 - k0, 0)};
    };
    const int hop = gridDim.x * WARPS, begin = blockIdx.x * WARPS + warp;
    // What is fetched next: rows `f_left` and on of a table's heads (q's, then k's) of item f_item.
    int f_item = begin, f_left = 0, f_stage = 0;
    bool f_k = false, f_begun = false;                     // k's heads are what is fetched; there was a fetch before
    const bf16 *f_x = nullptr, *f_dy = nullptr;
    int64_t f_hop = 0;
    auto fetch = [&] {
        if (f_left <= 0) {                                 // the next table with rows, if there is one
            if (f_begun) {                                 // (f_x may be NULL where the gradient needs no x)
                if (MIXED || f_k) f_item += hop;
                f_k = !MIXED && !f_k;
            }
            f_begun = true;
            while (f_item < a.items) {
                const Item f = item_of(f_item);
                f_left = MIXED ? a.width : f_k ? f.nk : f.nq;
                if (f_left > 0) {
                    const bool of_k = MIXED ? sub >= a.heads : f_k;
                    const int h = MIXED ? sub - (of_k ? a.heads : 0) : (of_k ? f.k0 : f.q0) + sub;
                    const int64_t head = of_k ? a.k_head : a.q_head;
                    f_x = (of_k ? a.k + f.t * a.k_row : a.q + f.t * a.q_row) + h * head;
                    f_hop = ROWS * head;
                    if (GRAD) f_dy = (of_k ? a.dk_out + (int64_t)f.t * kv_heads * a.d : a.dq_out + (int64_t)f.t * a.heads * a.d) + h * a.d;
                    break;
                }
                if (f_k) f_item += hop;
                f_k = !f_k;
            }
        }
        if (f_item < a.items) {
            // a row that is not there leaves an older one in its place, of which nothing is kept
            const bool in = sub < f_left, there = in && (ODD ? 8 * l < a.d : in_a), more = in && in_b;
            const uint32_t to = tc::smem_u32(mine + f_stage * STAGE + lane);
            if (!GRAD || TWO) {
                copy_piece(to, f_x + (ODD ? 8 * l : a0), there);
                if (!ODD) copy_piece(to + 512, f_x + b0, more);
            }
            if (GRAD) {
                copy_piece(to + (TWO ? TABLE * 16 : 0), f_dy + (ODD ? 8 * l : a0), there);
                if (!ODD) copy_piece(to + (TWO ? TABLE * 16 : 0) + 512, f_dy + b0, more);
            }
            f_left -= ROWS;
            f_x += f_hop;
            if (GRAD) f_dy += ROWS * a.d;
        }
        if (++f_stage == AHEAD) f_stage = 0;
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll 1
    for (int i = 0; i < AHEAD; ++i) fetch();
    if (NORM) {
        // a warp each for the weights of q and k; ones where there are none
        if (warp < 2 && sub == 0)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const void *w = warp ? a.k_weight : a.q_weight;
                auto weight = [&](int col, bool has) { return !w || !has ? 1.f : a.weight_f32 ? ((const float *)w)[col] : __bfloat162float(((const bf16 *)w)[col]); };
                reinterpret_cast<float *>(&weights[warp][e / 4][l])[e % 4] = weight(col_a(e), has_a(e));
                reinterpret_cast<float *>(&weights[warp][2 + e / 4][l])[e % 4] = weight(col_b(e), has_b(e));
            }
        __syncthreads();
    }
    int stage = 0, next_position = begin < a.items ? a.positions[item_of(begin).t] : 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) turn[i] = turns_of(freq[i]);
    for (int i = begin; i < a.items; i += hop) {
        const Item it = item_of(i);
        // cosine and sine of every pair: y'[a] = c y[a] - s y[b], y'[b] = c y[b] + s y[a]
        Pair c[4], s[4], minus_s[4];
        {
            const int64_t position = next_position;
            if (i + hop < a.items) next_position = a.positions[item_of(i + hop).t];
            float mine_c[2], mine_s[2];
            cos_sin((uint32_t)((uint64_t)position * turn[0] >> 32), (uint32_t)((uint64_t)position * turn[1] >> 32), mine_c, mine_s);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                mine_c[i] *= a.factor;
                mine_s[i] *= GRAD ? -a.factor : a.factor;
            }
            if (some_none)                                 // read again: kept, a factor for each would take registers in every call (training 152 us, so 150)
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    if (2 * lane + i < half && no_turn(a.freq[2 * lane + i])) mine_c[i] = mine_s[i] = NAN;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                // pairs 8 l + 2 e and the next; neighbours, where the row is in two halves: 4 l + 2 e, and from e = 2 on the second half's
                const int from = (INTER && !ODD ? 2 * (e < 2 ? l : l + LANES) + (e & 1) : 4 * l + e) & 31;
                float x[2], y[2];
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    x[i] = __shfl_sync(~0u, mine_c[i], from);
                    y[i] = __shfl_sync(~0u, mine_s[i], from);
                }
                c[e] = pair(x[0], x[1]);
                s[e] = pair(y[0], y[1]);
                minus_s[e] = pair(-y[0], -y[1]);
            }
        }
#pragma unroll
        for (int m = 0; m < (MIXED ? 1 : 2); ++m) {        // heads of q, then of k
            const bool of_k = MIXED ? sub >= a.heads : m;
            const int first = MIXED ? (of_k ? -a.heads : 0) : m ? it.k0 : it.q0, n = MIXED ? a.width : m ? it.nk : it.nq;
            if (n == 0) continue;
            Pair wa[4], wb[4];
            if (NORM)
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float4 x = weights[of_k][e][l], y = weights[of_k][2 + e][l];
                    wa[2 * e] = pair(x.x, x.y);
                    wa[2 * e + 1] = pair(x.z, x.w);
                    wb[2 * e] = pair(y.x, y.y);
                    wb[2 * e + 1] = pair(y.z, y.w);
                }
            bf16 *dst = (of_k ? a.k_out : a.q_out) + ((int64_t)it.t * (of_k ? kv_heads : a.heads) + first + sub) * a.d;
            for (int h = 0; h < n; h += ROWS, dst += ROWS * a.d) {
                const bool in = h + sub < n;
                asm volatile("cp.async.wait_group %0;" ::"n"(AHEAD - 1) : "memory");
                __syncwarp();
                const uint4 *x_at = mine + stage * STAGE, *u_at = x_at + (TWO ? TABLE : 0);       // u: what is turned, x or dy
                Pair xa[4], xb[4], ua[4], ub[4];
                if (ODD) {
                    auto column = [&](const uint4 *at, int col, bool has) { return has ? __bfloat162float(reinterpret_cast<const bf16 *>(at + sub * LANES)[col]) : 0.f; };
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        ua[e] = pair(column(u_at, col_a(2 * e), has_a(2 * e)), column(u_at, col_a(2 * e + 1), has_a(2 * e + 1)));
                        ub[e] = pair(column(u_at, col_b(2 * e), has_b(2 * e)), column(u_at, col_b(2 * e + 1), has_b(2 * e + 1)));
                        if (TWO) {
                            xa[e] = pair(column(x_at, col_a(2 * e), has_a(2 * e)), column(x_at, col_a(2 * e + 1), has_a(2 * e + 1)));
                            xb[e] = pair(column(x_at, col_b(2 * e), has_b(2 * e)), column(x_at, col_b(2 * e + 1), has_b(2 * e + 1)));
                        }
                    }
                    __syncwarp();                          // rows of several lanes: read by all of them before the next copy
                } else {
                    pairs_of<INTER>(u_at[lane], u_at[lane + 32], ua, ub);
                    if (TWO) pairs_of<INTER>(x_at[lane], x_at[lane + 32], xa, xb);
                }
                fetch();                                   // into the place that has been read
                if (++stage == AHEAD) stage = 0;
                float r = 1.f;
                if (NORM) {
                    const Pair *y = TWO ? xa : ua, *z = TWO ? xb : ub;
                    Pair sum = mul(y[0], y[0]), sum1 = mul(z[0], z[0]);
#pragma unroll
                    for (int e = 1; e < 4; ++e) {
                        sum = fma(y[e], y[e], sum);
                        sum1 = fma(z[e], z[e], sum1);
                    }
                    const float2 two = split(add(sum, sum1));
                    r = rsqrtf(fmaf(row_sum<LANES>(two.x + two.y), inv_d, a.eps));
                }
                if (TWO && !in) {                          // a row that is not there adds nothing to the weights' sums
                    r = 0.f;
#pragma unroll
                    for (int e = 0; e < 4; ++e) xa[e] = xb[e] = ua[e] = ub[e] = pair(0.f, 0.f);
                }
                const Pair rr = pair(r, r);
                if (NORM && !GRAD)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        ua[e] = mul(mul(ua[e], wa[e]), rr);
                        ub[e] = mul(mul(ub[e], wb[e]), rr);
                    }
                // columns that do not turn stay as they are, whatever lies beside them
#pragma unroll
                for (int g = 0; g < 2; ++g) {
                    if (!(g ? turn_b : turn_a)) continue;
#pragma unroll
                    for (int e = 2 * g; e < 2 * g + 2; ++e) {
                        const Pair x = fma(minus_s[e], ub[e], mul(c[e], ua[e])), y = fma(s[e], ua[e], mul(c[e], ub[e]));
                        if (ODD) {
                            const bool t0 = 8 * l + 2 * e < half, t1 = 8 * l + 2 * e + 1 < half;
                            const float2 x2 = split(x), y2 = split(y), a2 = split(ua[e]), b2 = split(ub[e]);
                            ua[e] = pair(t0 ? x2.x : a2.x, t1 ? x2.y : a2.y);
                            ub[e] = pair(t0 ? y2.x : b2.x, t1 ? y2.y : b2.y);
                        } else {
                            ua[e] = x;
                            ub[e] = y;
                        }
                    }
                }
                if (TWO) {
                    Pair sum = pair(0.f, 0.f), sum1 = pair(0.f, 0.f);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        xa[e] = mul(xa[e], rr);
                        xb[e] = mul(xb[e], rr);
                        dwa[m][e] = fma(ua[e], xa[e], dwa[m][e]);
                        dwb[m][e] = fma(ub[e], xb[e], dwb[m][e]);
                        ua[e] = mul(ua[e], wa[e]);
                        ub[e] = mul(ub[e], wb[e]);
                        sum = fma(ua[e], xa[e], sum);
                        sum1 = fma(ub[e], xb[e], sum1);
                    }
                    const float2 two = split(add(sum, sum1));
                    const float mean = -row_sum<LANES>(two.x + two.y) * inv_d;
                    const Pair mm = pair(mean, mean);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        ua[e] = mul(rr, fma(mm, xa[e], ua[e]));
                        ub[e] = mul(rr, fma(mm, xb[e], ub[e]));
                    }
                }
                if (ODD) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const float2 x = split(ua[e / 2]), y = split(ub[e / 2]);
                        if (in && has_a(e)) dst[col_a(e)] = __float2bfloat16(e % 2 ? x.y : x.x);
                        if (in && has_b(e)) dst[col_b(e)] = __float2bfloat16(e % 2 ? y.y : y.x);
                    }
                } else {
                    uint4 p, q;
                    pieces_of<INTER>(ua, ub, p, q);
                    if (in && in_a) *reinterpret_cast<uint4 *>(dst + a0) = p;
                    if (in && in_b) *reinterpret_cast<uint4 *>(dst + b0) = q;
                }
            }
        }
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (TWO && a.part) {
        float *sums = reinterpret_cast<float *>(ring);     // [warp][column]
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float2 x = split(dwa[MIXED ? 0 : m][e / 2]), y = split(dwb[MIXED ? 0 : m][e / 2]);
                float va = e % 2 ? x.y : x.x, vb = e % 2 ? y.y : y.x;
                if (MIXED && (sub >= a.heads) != (m == 1)) va = vb = 0.f;
#pragma unroll
                for (int o = 16; o >= LANES; o >>= 1) {
                    va += __shfl_xor_sync(~0u, va, o);
                    vb += __shfl_xor_sync(~0u, vb, o);
                }
                if (sub == 0 && has_a(e)) sums[warp * MAX_D + col_a(e)] = va;
                if (sub == 0 && has_b(e)) sums[warp * MAX_D + col_b(e)] = vb;
            }
            __syncthreads();
            if (threadIdx.x < a.d) {
                float sum = 0.f;
#pragma unroll
                for (int g = 0; g < WARPS; ++g) sum += sums[g * MAX_D + threadIdx.x];
                a.part[((int64_t)blockIdx.x * 2 + m) * MAX_D + threadIdx.x] = sum;
            }
        }
    }
}

// The blocks' sums, 32 columns of one weight to a block, in a fixed order.
__global__ void __launch_bounds__(1024) rotate_weight_kernel(const float *part, int blocks, int d, float *dq_weight, float *dk_weight)
{
    __shared__ float sums[32][33];
    pdl_wait();
    pdl_trigger();
    const int col = blockIdx.x * 32 + (threadIdx.x & 31), first = threadIdx.x >> 5;
    float *out = blockIdx.y ? dk_weight : dq_weight;
    if (!out) return;
    float sum = 0.f;
    if (col < d) {
#pragma unroll 8
        for (int b = first; b < blocks; b += 32) sum += part[((int64_t)b * 2 + blockIdx.y) * rot::MAX_D + col];
    }
    sums[first][threadIdx.x & 31] = sum;
    __syncthreads();
    if (threadIdx.x < 32) {
        sum = 0.f;
#pragma unroll
        for (int r = 0; r < 32; ++r) sum += sums[r][threadIdx.x];
        if (col < d) out[col] = sum;
    }
}

size_t rotate_partials(bool wanted) { return wanted ? (size_t)sm_count_or_default() * rot::min_blocks(false, true) * 2 * rot::MAX_D * sizeof(float) : 0; }

template <int LANES, bool ODD, bool GRAD, bool MIXED>
static st_status launch_rotate(const RotateArgs &a, bool norm, bool inter, int grid, cudaStream_t stream)
{
    using namespace rot;
    void (*kernel)(RotateArgs) = norm ? (inter ? rotate_kernel<LANES, true, true, ODD, GRAD, MIXED> : rotate_kernel<LANES, true, false, ODD, GRAD, MIXED>)
                                      : (inter ? rotate_kernel<LANES, false, true, ODD, GRAD, MIXED> : rotate_kernel<LANES, false, false, ODD, GRAD, MIXED>);
    const size_t smem = (size_t)warps(GRAD) * 32 * AHEAD * 16 * (ODD ? 1 : 2) * (GRAD && norm ? 2 : 1) + (norm ? WEIGHTS * 16 : 0);
    if (!ensure_dynamic_smem(kernel, smem)) return ST_ERR_CUDA;
    return launch(kernel, dim3((unsigned)grid), warps(GRAD) * 32, smem, stream, a);
}

// An item is a token where half of the warps have one; where not, its heads are divided, down to one row of each group of lanes.
template <bool GRAD>
static st_status run_rotate(RotateArgs &a, bool norm, bool inter, cudaStream_t stream, int *blocks)
{
    using namespace rot;
    constexpr int WARPS = warps(GRAD);
    const bool odd = a.rot % 16 != 0;
    const int rows = odd ? 2 : a.d <= 64 ? 8 : 4;          // of a warp at a time
    const int64_t sms = sm_count_or_default(), most = sms * min_blocks(odd, GRAD);
    a.cols = a.width;
    while ((int64_t)a.n * ((a.width + a.cols - 1) / a.cols) < most * WARPS / 2 && a.cols > rows) a.cols = ((a.cols + 1) / 2 + rows - 1) / rows * rows;
    a.chunks = (a.width + a.cols - 1) / a.cols;
    a.items = a.n * a.chunks;
    int64_t grid = ((int64_t)a.items + WARPS - 1) / WARPS;
    if (grid > most) grid = most;
    *blocks = (int)grid;
    if (odd) return launch_rotate<16, true, GRAD, false>(a, norm, inter, (int)grid, stream);
    if (a.chunks == 1 && a.width > a.heads && a.width <= rows)
        return a.d <= 64 ? launch_rotate<4, false, GRAD, true>(a, norm, inter, (int)grid, stream) : launch_rotate<8, false, GRAD, true>(a, norm, inter, (int)grid, stream);
    return a.d <= 64 ? launch_rotate<4, false, GRAD, false>(a, norm, inter, (int)grid, stream) : launch_rotate<8, false, GRAD, false>(a, norm, inter, (int)grid, stream);
}

static st_status check_rotation(const st_rotation *r, const void *positions, const void *freq)
{
    if (!r) return ST_ERR_NULL;
    if (r->dtype != ST_BF16 || (r->weight_dtype != ST_BF16 && r->weight_dtype != ST_F32)) return ST_ERR_DTYPE;
    if ((r->norm | 1) != 1 || (r->interleaved | 1) != 1 || r->n <= 0 || r->heads <= 0 || r->kv_heads < 0 || r->d <= 0 || r->rot < 0 || r->rot > r->d || r->rot % 2 != 0)
        return ST_ERR_SHAPE;
    if (r->n > (1 << 29) || r->heads > 65535 || r->kv_heads > 65535 || r->d % 8 != 0 || r->d > rot::MAX_D) return ST_ERR_UNSUPPORTED;
    if (!(r->eps >= 0.f && r->eps < INFINITY) || !(r->factor > -INFINITY && r->factor < INFINITY)) return ST_ERR_UNSUPPORTED;
    if (!positions || (r->rot > 0 && !freq)) return ST_ERR_NULL;
    return aligned4(positions) && aligned16(freq) ? ST_OK : ST_ERR_ALIGN;
}

// A table of the call; its heads may be 0.
static st_status check_rows(const st_rotation *r, const void *p, int64_t heads, int64_t row, int64_t head)
{
    if (heads == 0) return ST_OK;
    if (!p) return ST_ERR_NULL;
    if (!stride_ok(r->n, row, r->d) || !stride_ok(heads, head, r->d)) return ST_ERR_SHAPE;
    if (row > ((int64_t)1 << 38) || head > ((int64_t)1 << 38)) return ST_ERR_UNSUPPORTED;
    if ((r->n > 1 && row % 8 != 0) || (heads > 1 && head % 8 != 0) || !aligned16(p)) return ST_ERR_ALIGN;
    return ST_OK;
}

static RotateArgs rotate_args(const st_rotation *r, const void *q, const void *k, const int32_t *positions, const float *freq, const void *qw, const void *kw)
{
    RotateArgs a = {};
    a.q = (const bf16 *)q;
    a.k = (const bf16 *)k;
    a.q_row = stride_of(r->n, r->q_row);
    a.q_head = stride_of(r->heads, r->q_head);
    a.k_row = stride_of(r->n, r->k_row);
    a.k_head = stride_of(r->kv_heads, r->k_head);
    a.positions = positions;
    a.freq = freq;
    a.q_weight = qw;
    a.k_weight = kw;
    a.weight_f32 = r->weight_dtype == ST_F32;
    a.n = (int)r->n;
    a.heads = (int)r->heads;
    a.width = (int)(r->heads + r->kv_heads);
    a.d = (int)r->d;
    a.rot = (int)r->rot;
    a.eps = r->eps;
    a.factor = r->factor;
    return a;
}

}  // namespace attn
}  // namespace st

using namespace st;
using namespace st::attn;

extern "C" st_status st_attn_rotate(const st_rotation *r, const void *q, const void *k, const int32_t *positions, const float *freq, const void *q_weight,
                                    const void *k_weight, void *q_out, void *k_out, void *stream)
{
    st_status rc = check_rotation(r, positions, freq);
    if (rc == ST_OK) rc = check_rows(r, q, r->heads, r->q_row, r->q_head);
    if (rc == ST_OK) rc = check_rows(r, k, r->kv_heads, r->k_row, r->k_head);
    if (rc != ST_OK) return rc;
    if (!q_out || (r->kv_heads > 0 && !k_out)) return ST_ERR_NULL;
    for (const void *p : {q_weight, k_weight, (const void *)q_out, (const void *)k_out})
        if (!aligned16(p)) return ST_ERR_ALIGN;
    RotateArgs a = rotate_args(r, q, k, positions, freq, q_weight, k_weight);
    a.q_out = (bf16 *)q_out;
    a.k_out = (bf16 *)k_out;
    // a row is read by the lanes that write it; everything else is read by all blocks
    const int64_t q_bytes = r->n * r->heads * r->d * 2, k_bytes = r->n * r->kv_heads * r->d * 2, w_bytes = r->d * (a.weight_f32 ? 4 : 2);
    const Operand Q = {q, r->n, r->heads, r->d, a.q_row, a.q_head}, K = {k, r->n, r->kv_heads, r->d, a.k_row, a.k_head};
    if (Q.under(q_out, q_bytes, true)) return ST_ERR_UNSUPPORTED;
    if (r->kv_heads > 0 && (Q.under(k_out, k_bytes) || K.under(q_out, q_bytes) || K.under(k_out, k_bytes, true) || arrays_meet(q_out, q_bytes, k_out, k_bytes)))
        return ST_ERR_UNSUPPORTED;
    for (const auto &o : {std::make_pair((const void *)q_out, q_bytes), std::make_pair((const void *)k_out, k_bytes)})
        if (arrays_meet(o.first, o.second, positions, r->n * 4) || arrays_meet(o.first, o.second, freq, r->rot * 2) ||
            arrays_meet(o.first, o.second, q_weight, w_bytes) || arrays_meet(o.first, o.second, k_weight, w_bytes))
            return ST_ERR_UNSUPPORTED;
    int blocks;
    return run_rotate<false>(a, r->norm, r->interleaved, (cudaStream_t)stream, &blocks);
}

extern "C" st_status st_attn_rotate_grad(const st_rotation *r, const void *q, const void *k, const void *dq_out, const void *dk_out, const int32_t *positions,
                                         const float *freq, const void *q_weight, const void *k_weight, void *dq, void *dk, float *dq_weight,
                                         float *dk_weight, void *ws, size_t ws_bytes, void *stream)
{
    st_status rc = check_rotation(r, positions, freq);
    if (rc == ST_OK && r->norm) rc = check_rows(r, q, r->heads, r->q_row, r->q_head);
    if (rc == ST_OK && r->norm) rc = check_rows(r, k, r->kv_heads, r->k_row, r->k_head);
    if (rc != ST_OK) return rc;
    if (!dq_out || !dq || (r->kv_heads > 0 && (!dk_out || !dk))) return ST_ERR_NULL;
    if ((!r->norm && (dq_weight || dk_weight)) || (r->kv_heads == 0 && dk_weight)) return ST_ERR_SHAPE;
    for (const void *p : {q_weight, k_weight, dq_out, dk_out, (const void *)dq, (const void *)dk, (const void *)dq_weight, (const void *)dk_weight})
        if (!aligned16(p)) return ST_ERR_ALIGN;
    const bool weights = dq_weight || dk_weight;
    if (!ws || ws_bytes < kWsHeaderBytes + rotate_partials(weights)) return ST_ERR_WORKSPACE;
    if (!aligned256(ws)) return ST_ERR_ALIGN;
    RotateArgs a = rotate_args(r, q, k, positions, freq, q_weight, k_weight);
    a.dq_out = (const bf16 *)dq_out;
    a.dk_out = (const bf16 *)dk_out;
    a.q_out = (bf16 *)dq;
    a.k_out = (bf16 *)dk;
    a.part = weights ? (float *)((char *)ws + kWsHeaderBytes) : nullptr;
    const int64_t q_bytes = r->n * r->heads * r->d * 2, k_bytes = r->n * r->kv_heads * r->d * 2, w_bytes = r->d * (a.weight_f32 ? 4 : 2), dw_bytes = r->d * 4;
    const Operand Q = {q, r->n, r->heads, r->d, a.q_row, a.q_head}, K = {k, r->n, r->kv_heads, r->d, a.k_row, a.k_head};
    const std::pair<const void *, int64_t> outs[4] = {{dq, q_bytes}, {dk, k_bytes}, {dq_weight, dw_bytes}, {dk_weight, dw_bytes}};
    for (int i = 0; i < 4; ++i) {
        const void *p = outs[i].first;
        const int64_t bytes = outs[i].second;
        if (!p || bytes == 0) continue;
        if ((r->norm && (Q.under(p, bytes) || (r->kv_heads > 0 && K.under(p, bytes)))) || arrays_meet(p, bytes, positions, r->n * 4) || arrays_meet(p, bytes, freq, r->rot * 2) ||
            arrays_meet(p, bytes, q_weight, w_bytes) || arrays_meet(p, bytes, k_weight, w_bytes) || (!(i == 0 && p == dq_out) && arrays_meet(p, bytes, dq_out, q_bytes)) ||
            (!(i == 1 && p == dk_out) && arrays_meet(p, bytes, dk_out, k_bytes)))
            return ST_ERR_UNSUPPORTED;
        for (int j = 0; j < i; ++j)
            if (arrays_meet(p, bytes, outs[j].first, outs[j].second)) return ST_ERR_UNSUPPORTED;
    }
    int blocks = 0;
    rc = run_rotate<true>(a, r->norm, r->interleaved, (cudaStream_t)stream, &blocks);
    if (rc != ST_OK || !weights) return rc;
    return launch(rotate_weight_kernel, dim3((unsigned)((r->d + 31) / 32), 2), 1024, 0, (cudaStream_t)stream, (const float *)a.part, blocks, (int)r->d, dq_weight, dk_weight);
}
