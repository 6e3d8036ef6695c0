// st_attn_decay_step: S <- e^a S + k (x) v, out = scale S^T q, for one token of every sequence.
//
// The states are read and written once, 8 bytes an element; everything else is small.  A block owns 64 columns of one head's state,
// a thread four of them (16 bytes) and every 16th row: all its loads are in flight before the first is needed.  The rows' sums are
// joined in shared memory.
#include "attn_common.cuh"

namespace st {
namespace attn {

namespace dstep {
constexpr int COLS = 64, ROWS = 16, THREADS = COLS / 4 * ROWS;
}

// NR: rows of a thread
template <int NR>
__global__ void __launch_bounds__(dstep::THREADS) decay_step_kernel(const bf16 *q, const bf16 *k, const bf16 *v, const float *log_decay, float *state,
                                                                    float scale, bf16 *out, int heads, int d, int dv)
{
    using namespace dstep;
    __shared__ float4 part[ROWS][COLS / 4];
    pdl_wait();
    pdl_trigger();
    const int slabs = (dv + COLS - 1) / COLS, h = blockIdx.x / slabs, col = blockIdx.x % slabs * COLS + (threadIdx.x % (COLS / 4)) * 4, r0 = threadIdx.x / (COLS / 4);
    const int64_t bh = (int64_t)blockIdx.y * heads + h;
    const bool in = col < dv;
    float4 s[NR];
    float kk[NR], qq[NR];
    float *at = state + (bh * d + r0) * dv + col;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const bool row = in && r0 + i * ROWS < d;
        s[i] = row ? *reinterpret_cast<const float4 *>(at + (int64_t)i * ROWS * dv) : make_float4(0.f, 0.f, 0.f, 0.f);
        kk[i] = row ? __bfloat162float(k[bh * d + r0 + i * ROWS]) : 0.f;
        qq[i] = row ? __bfloat162float(q[bh * d + r0 + i * ROWS]) : 0.f;
    }
    float z[4] = {0.f, 0.f, 0.f, 0.f};
    if (in)
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = __bfloat162float(v[bh * dv + col + e]);
    const float w = expf(log_decay[h]);
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        s[i] = make_float4(fmaf(w, s[i].x, kk[i] * z[0]), fmaf(w, s[i].y, kk[i] * z[1]), fmaf(w, s[i].z, kk[i] * z[2]), fmaf(w, s[i].w, kk[i] * z[3]));
        if (in && r0 + i * ROWS < d) *reinterpret_cast<float4 *>(at + (int64_t)i * ROWS * dv) = s[i];
        o = make_float4(fmaf(qq[i], s[i].x, o.x), fmaf(qq[i], s[i].y, o.y), fmaf(qq[i], s[i].z, o.z), fmaf(qq[i], s[i].w, o.w));
    }
    part[r0][threadIdx.x % (COLS / 4)] = o;
    __syncthreads();
    if (threadIdx.x < COLS) {
        const int c = blockIdx.x % slabs * COLS + threadIdx.x;
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < ROWS; ++r) sum += reinterpret_cast<const float *>(&part[r][0])[threadIdx.x];
        if (c < dv) out[bh * dv + c] = __float2bfloat16(scale * sum);
    }
}

}  // namespace attn
}  // namespace st

using namespace st;
using namespace st::attn;

extern "C" st_status st_attn_decay_step(const st_tokens *t, const void *q, const void *k, const void *v, const float *log_decay,
                                        float *state, float scale, void *out, void *stream)
{
    const st_status rc = check_tokens(t);
    if (rc != ST_OK) return rc;
    if (t->nq != t->nk || t->heads != t->kv_heads || t->nseq != t->nq) return ST_ERR_SHAPE;
    // the kernel takes the tables as contiguous ones
    auto contiguous = [t](int64_t cols, int64_t row, int64_t head) { return (t->heads == 1 || head == cols) && (t->nq == 1 || row == t->heads * cols); };
    if (!contiguous(t->d, t->q_row, t->q_head) || !contiguous(t->d, t->k_row, t->k_head) || !contiguous(t->dv, t->v_row, t->v_head)) return ST_ERR_SHAPE;
    if (!q || !k || !v || !log_decay || !state || !out) return ST_ERR_NULL;
    if (t->nq > 65535) return ST_ERR_UNSUPPORTED;
    for (const void *p : {q, k, v, (const void *)log_decay, (const void *)state, (const void *)out})
        if (!aligned16(p)) return ST_ERR_ALIGN;
    // a block reads all of its head's q and k, and of v the columns that it writes
    const int64_t rows = t->nq * t->heads, out_bytes = rows * t->dv * 2, state_bytes = rows * t->d * t->dv * 4;
    const Operand Q = q_of(t, q), K = k_of(t, k), V = v_of(t, v);
    const bool alone = t->dv <= dstep::COLS;
    if (Q.under(out, out_bytes, alone) || K.under(out, out_bytes, alone) || V.under(out, out_bytes, true) || Q.under(state, state_bytes) ||
        K.under(state, state_bytes) || V.under(state, state_bytes) || arrays_meet(out, out_bytes, state, state_bytes))
        return ST_ERR_UNSUPPORTED;
    const dim3 grid((unsigned)(t->heads * ((t->dv + dstep::COLS - 1) / dstep::COLS)), (unsigned)t->nq);
    return launch(t->d <= 64 ? decay_step_kernel<4> : decay_step_kernel<8>, grid, dstep::THREADS, 0, (cudaStream_t)stream, (const bf16 *)q, (const bf16 *)k,
                  (const bf16 *)v, log_decay, state, scale, (bf16 *)out, (int)t->heads, (int)t->d, (int)t->dv);
}
