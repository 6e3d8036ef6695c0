// st_attn_rotate and its gradient: an RMS norm of every head and a rotation of pairs of its columns, in one pass.
//
// Bound by memory: a result is 8 multiplications and additions for each 4 bytes (8 for each 8 in the gradient).  16 lanes own a row (one head of
// one token), each 8 of its columns: 16 bytes.  A block has T tokens and C of their heads of q and k; the angles of its T tokens, which all heads
// share, are turned into sines and cosines once, while the block's first rows are on their way: in fp64 up to the fraction of a turn
// (position freq / 2 pi reaches 2^17 turns and more, where fp32 has no digits left for the fraction), then in fp32.
//
// The gradient's blocks take several tiles in turn and keep the weights' sums in registers; a second kernel adds the blocks' sums in a
// fixed order.
#include "attn_common.cuh"

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
    int tokens, cols, col_tiles;           // of a tile
    int64_t tiles;
    float *part;                           // [block][q, k][128] sums of the weights' gradient, or NULL
};

namespace rot {
constexpr int THREADS = 256, LANES = 16, ROWS = THREADS / LANES;      // rows that a block has in hand at a time
enum Pairs { HALF = 0, INTERLEAVED = 1, HALF_ODD = 2 };               // HALF_ODD: a half that is no whole number of lanes
constexpr int MAX_D = 128;
}  // namespace rot

// Sum over the 16 lanes of a row, the same in all of them.
__device__ __forceinline__ float row_sum(float x)
{
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) x += __shfl_xor_sync(~0u, x, o);
    return x;
}

// R rows of each group of 16 lanes: rows g R .. g R + R - 1 of the tile, so that a group's rows share their token's angles.
template <int R, bool NORM, int PAIRS, bool GRAD>
__global__ void __launch_bounds__(rot::THREADS) rotate_kernel(const RotateArgs a)
{
    using namespace rot;
    extern __shared__ __align__(16) float smem[];
    float *weights = smem;                                 // [q, k][128]
    float *turns = smem + (NORM ? 2 * MAX_D : 0);          // [token][cosines, sines][rot / 2]
    const int lane = threadIdx.x & 31, group = threadIdx.x / LANES, e0 = (threadIdx.x % LANES) * 8, half = a.rot / 2;
    const bool inside = e0 < a.d;
    // the other half's columns are in another lane; a lane without any meets itself
    const int there = PAIRS == HALF && e0 < a.rot ? (e0 < half ? lane + half / 8 : lane - half / 8) : lane;
    const int p0 = PAIRS == INTERLEAVED ? e0 / 2 : e0 < half ? e0 : e0 - half;       // first pair of this lane
    const int stride = (half + 3) / 4 * 4;                 // of a token's cosines: whole 16-byte pieces
    float dw[2][8];
    if (GRAD && NORM)
#pragma unroll
        for (int e = 0; e < 8; ++e) dw[0][e] = dw[1][e] = 0.f;

    pdl_wait();
    pdl_trigger();
    if (NORM)
        for (int i = threadIdx.x; i < 2 * MAX_D; i += THREADS) {
            const void *w = i < MAX_D ? a.q_weight : a.k_weight;
            const int e = i % MAX_D;
            weights[i] = e >= a.d ? 0.f : !w ? 1.f : a.weight_f32 ? ((const float *)w)[e] : __bfloat162float(((const bf16 *)w)[e]);
        }
    for (int64_t tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
        const int t0 = (int)(tile / a.col_tiles) * a.tokens, c0 = (int)(tile % a.col_tiles) * a.cols;
        const int nt = min(a.tokens, a.n - t0), nc = min(a.cols, a.width - c0);
        // the rows on their way
        uint4 x[R], y[R];
        float other[PAIRS == HALF_ODD ? R : 1][8];
        int token[R], col[R];
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int row = group * R + j;
            token[j] = row / a.cols;
            col[j] = row - token[j] * a.cols;
            const bool in = token[j] < nt && col[j] < nc;
            if (!in) token[j] = -1;
            const int h = c0 + col[j], t = t0 + token[j];
            const bool is_q = h < a.heads;
            const bf16 *src = is_q ? a.q + t * a.q_row + h * a.q_head : a.k + t * a.k_row + (h - a.heads) * a.k_head;
            const bf16 *dy = is_q ? a.dq_out + ((int64_t)t * a.heads + h) * a.d : a.dk_out + ((int64_t)t * (a.width - a.heads) + h - a.heads) * a.d;
            x[j] = (NORM || !GRAD) && in && inside ? *reinterpret_cast<const uint4 *>(src + e0) : make_uint4(0u, 0u, 0u, 0u);
            if (GRAD) y[j] = in && inside ? *reinterpret_cast<const uint4 *>(dy + e0) : make_uint4(0u, 0u, 0u, 0u);
            if (PAIRS == HALF_ODD)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int i = e0 + e;
                    other[j][e] = in && i < a.rot ? __bfloat162float((GRAD ? dy : src)[i < half ? i + half : i - half]) : 0.f;
                }
        }
        for (int i = threadIdx.x; i < nt * half; i += THREADS) {
            const int t = i / half, p = i - t * half;
            // the fraction of a turn, -1/2 to 1/2
            const double turn = (double)a.positions[t0 + t] * ((double)a.freq[p] * 0.15915494309189533577);
            float s, c;
            sincospif(2.f * (float)(turn - rint(turn)), &s, &c);
            turns[(2 * t) * stride + p] = a.factor * c;
            turns[(2 * t + 1) * stride + p] = a.factor * (GRAD ? -s : s);
        }
        __syncthreads();
        float c[8], s[8];
        int held = -1;
#pragma unroll
        for (int j = 0; j < R; ++j) {
            const int h = c0 + col[j];
            const bool is_q = h < a.heads;
            // cosine and sine of every column, the sine with the sign that its product has: y'[i] = c[i] y[i] + s[i] y[other column of the pair]
            if (token[j] != held && token[j] >= 0) {
                held = token[j];
                const float *at = turns + 2 * held * stride;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool turned = e0 + e < a.rot;
                    const int p = PAIRS == INTERLEAVED ? p0 + e / 2 : PAIRS == HALF ? p0 + e : e0 + e < half ? e0 + e : e0 + e - half;
                    const bool first = PAIRS == INTERLEAVED ? e % 2 == 0 : e0 + e < half;
                    c[e] = turned ? at[p] : 1.f;
                    s[e] = turned ? (first ? -at[stride + p] : at[stride + p]) : 0.f;
                }
            }
            const float *w = weights + (is_q ? 0 : MAX_D);
            float v[8], o[8], r = 1.f, z[8];
            unpack8(x[j], v);
            if (NORM) {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) sum = fmaf(v[e], v[e], sum);
                r = rsqrtf(row_sum(sum) / a.d + a.eps);
            }
            // what is turned, and the other columns of its pairs
            const uint4 mine = GRAD ? y[j] : x[j];
            float u[8];
            unpack8(mine, u);
            if (PAIRS == HALF) {
                const uint4 theirs = make_uint4(__shfl_sync(~0u, mine.x, there), __shfl_sync(~0u, mine.y, there), __shfl_sync(~0u, mine.z, there),
                                                __shfl_sync(~0u, mine.w, there));
                unpack8(theirs, o);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const int i = e0 + e, pair = PAIRS == INTERLEAVED ? (i ^ 1) : i < half ? i + half : i - half;
                if (PAIRS == INTERLEAVED) o[e] = u[e ^ 1];
                if (PAIRS == HALF_ODD) o[e] = other[j][e];
                if (NORM && !GRAD) {
                    z[e] = r * fmaf(c[e], u[e] * w[i], s[e] * (i < a.rot ? o[e] * w[pair] : 0.f));
                } else {
                    z[e] = i < a.rot ? fmaf(c[e], u[e], s[e] * o[e]) : u[e];
                }
            }
            if (GRAD && NORM) {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    v[e] *= r;
                    if (token[j] >= 0) {
                        // one of the two is added 0 of what is finite: which head a row is, lanes of a warp may differ in
                        dw[0][e] += is_q ? z[e] * v[e] : 0.f;
                        dw[1][e] += is_q ? 0.f : z[e] * v[e];
                    }
                    z[e] *= w[e0 + e];
                    sum = fmaf(z[e], v[e], sum);
                }
                sum = row_sum(sum) / a.d;
#pragma unroll
                for (int e = 0; e < 8; ++e) z[e] = r * fmaf(-sum, v[e], z[e]);
            }
            if (token[j] >= 0 && inside) {
                const int64_t t = t0 + token[j];
                bf16 *dst = is_q ? a.q_out + (t * a.heads + h) * a.d : a.k_out + (t * (a.width - a.heads) + h - a.heads) * a.d;
                *reinterpret_cast<uint4 *>(dst + e0) = pack8(z);
            }
        }
        if (GRAD) __syncthreads();                         // the next tile's angles take this one's place
    }
    if (GRAD && NORM && a.part) {
        __shared__ float sums[ROWS][MAX_D];
#pragma unroll
        for (int m = 0; m < 2; ++m) {
            __syncthreads();
#pragma unroll
            for (int e = 0; e < 8; ++e) sums[group][e0 + e] = dw[m][e];
            __syncthreads();
            if (threadIdx.x < MAX_D) {
                float sum = 0.f;
#pragma unroll
                for (int g = 0; g < ROWS; ++g) sum += sums[g][threadIdx.x];
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
    for (int b = first; b < blocks; b += 32) sum += part[((int64_t)b * 2 + blockIdx.y) * rot::MAX_D + col];
    sums[first][threadIdx.x & 31] = sum;
    __syncthreads();
    if (threadIdx.x < 32) {
        sum = 0.f;
#pragma unroll
        for (int r = 0; r < 32; ++r) sum += sums[r][threadIdx.x];
        if (col < d) out[col] = sum;
    }
}

namespace rot {
constexpr int GRAD_BLOCKS = 4;             // blocks of the gradient to an SM
}

size_t rotate_partials(bool wanted) { return wanted ? (size_t)sm_count_or_default() * rot::GRAD_BLOCKS * 2 * rot::MAX_D * sizeof(float) : 0; }

template <int R, bool GRAD>
static st_status run_rotate(RotateArgs a, bool norm, int pairs, cudaStream_t stream, int *blocks)
{
    using namespace rot;
    a.cols = a.width < ROWS * R ? a.width : ROWS * R;
    a.tokens = ROWS * R / a.cols;
    a.col_tiles = (a.width + a.cols - 1) / a.cols;
    a.tiles = ((int64_t)a.n + a.tokens - 1) / a.tokens * a.col_tiles;
    const size_t smem = ((norm ? 2 * MAX_D : 0) + (size_t)a.tokens * 2 * ((a.rot / 2 + 3) / 4 * 4)) * sizeof(float);
    int64_t grid = a.tiles;
    if (GRAD && grid > (int64_t)sm_count_or_default() * GRAD_BLOCKS) grid = (int64_t)sm_count_or_default() * GRAD_BLOCKS;
    if (grid > INT32_MAX) return ST_ERR_UNSUPPORTED;
    *blocks = (int)grid;
    void (*kernel)(RotateArgs) = nullptr;
    if (norm) kernel = pairs == HALF ? rotate_kernel<R, true, HALF, GRAD> : pairs == INTERLEAVED ? rotate_kernel<R, true, INTERLEAVED, GRAD> : rotate_kernel<R, true, HALF_ODD, GRAD>;
    else kernel = pairs == HALF ? rotate_kernel<R, false, HALF, GRAD> : pairs == INTERLEAVED ? rotate_kernel<R, false, INTERLEAVED, GRAD> : rotate_kernel<R, false, HALF_ODD, GRAD>;
    if (!ensure_dynamic_smem(kernel, smem)) return ST_ERR_CUDA;
    return launch(kernel, dim3((unsigned)grid), THREADS, smem, stream, a);
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

static int pairs_of(const st_rotation *r) { return r->interleaved ? rot::INTERLEAVED : r->rot % 16 == 0 ? rot::HALF : rot::HALF_ODD; }

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
    // rows for four blocks on every SM: four rows to a group of lanes, so that a token's angles serve more of its heads
    if ((int64_t)a.n * a.width >= (int64_t)sm_count_or_default() * 4 * rot::ROWS * 4) return run_rotate<4, false>(a, r->norm, pairs_of(r), (cudaStream_t)stream, &blocks);
    return run_rotate<1, false>(a, r->norm, pairs_of(r), (cudaStream_t)stream, &blocks);
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
    if ((int64_t)a.n * a.width >= (int64_t)sm_count_or_default() * rot::GRAD_BLOCKS * rot::ROWS * 2) rc = run_rotate<2, true>(a, r->norm, pairs_of(r), (cudaStream_t)stream, &blocks);
    else rc = run_rotate<1, true>(a, r->norm, pairs_of(r), (cudaStream_t)stream, &blocks);
    if (rc != ST_OK || !weights) return rc;
    return launch(rotate_weight_kernel, dim3((unsigned)((r->d + 31) / 32), 2), 1024, 0, (cudaStream_t)stream, (const float *)a.part, blocks, (int)r->d, dq_weight, dk_weight);
}
