// st_attn_window_step: one new token of every sequence against a cache in pages.
//
// Bound by the cache's bytes: every visible row of K and V is read once for all query heads that share it.  A cluster of blocks owns
// one key head of one sequence (and 16 of its query heads); its warps take tiles of 16 visible keys in turn.  Each warp copies its own
// tiles to its own ring in shared memory (cp.async, a tile ahead; page numbers one tile further), so that no barrier lies in the loop,
// and multiplies with mma.sync: the 16 rows of the fragments are query heads, of which a group of 1 to 16 is filled.  The tensor
// cores of tcgen05 would need 128 rows, and 2 to 32 flops a byte need no more than a tenth of mma.sync's rate.
// Rows that are not visible are never read: their place in shared memory is zeroed by the copy.
//
// Warps, then blocks of the cluster, join their maxima, sums and outputs in shared memory, the blocks over distributed shared
// memory: one kernel, behind a small one that clears the status, and no workspace however the keys are split.
#include "attn_common.cuh"
#include "tc_common.cuh"

namespace st {
namespace attn {

struct StepArgs {
    const bf16 *q, *k, *v;
    bf16 *k_pages, *v_pages;
    const int *table, *lens;
    int nseq, heads, group, d, pages, page, cols, window, sinks;
    unsigned page_magic;               // floor((2^32 - 1) / page): __umulhi with it is s / page or one less, s below 2^31
    int64_t page_stride, token_stride, head_stride;
    float scale;
    bf16 *out;
    unsigned *status;
};

namespace wstep {
constexpr int KEYS = 16, HEADS = 16, MAX_SPLITS = 16;
constexpr int FEWEST = 2;                  // tiles of a warp, where keys are split further
template <int DP, int WARPS, int STAGES> struct Shape {
    static constexpr int TILE_BYTES = KEYS * DP * 2, STAGE = 2 * TILE_BYTES, RING = STAGES * STAGE;
    static constexpr size_t SMEM = (size_t)WARPS * RING + (2 * WARPS + 2 + MAX_SPLITS) * HEADS * sizeof(float) + WARPS * KEYS * sizeof(int64_t) + 16;
    static_assert(HEADS * DP * 4 <= RING, "a warp's output takes the place of its ring");
};
}  // namespace wstep

__device__ __forceinline__ void copy16(uint32_t dst, const void *src, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldmatrix4_trans(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ld_cluster(uint32_t addr)
{
    float x;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(x) : "r"(addr) : "memory");
    return x;
}

__device__ __forceinline__ float fast_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <int DP, int WARPS, int STAGES>
__global__ void __launch_bounds__(WARPS * 32) window_step_kernel(const StepArgs a)
{
    using namespace wstep;
    using S = Shape<DP, WARPS, STAGES>;
    constexpr int CHUNKS = DP / 8;                        // 16-byte pieces of a row
    extern __shared__ __align__(128) unsigned char smem[];
    float *most_w = (float *)(smem + WARPS * S::RING), *sum_w = most_w + WARPS * HEADS, *most_b = sum_w + WARPS * HEADS, *sum_b = most_b + HEADS;
    float *share = sum_b + HEADS;                          // weight of every block's part, over the sum: [block][head]
    int64_t *offsets = (int64_t *)(share + MAX_SPLITS * HEADS);
    int *bad = (int *)(offsets + WARPS * KEYS);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int splits = gridDim.x, split = blockIdx.x, chunks = (a.group + HEADS - 1) / HEADS, b = blockIdx.z;
    const int hk = blockIdx.y / chunks, g0 = blockIdx.y % chunks * HEADS, g = min(a.group - g0, HEADS), kv_heads = a.heads / a.group;

    if (threadIdx.x == 0) *bad = 0;
    pdl_wait();
    pdl_trigger();
    __syncthreads();
    const int told = a.lens[b], len = (int)min((int64_t)max(told, 0), (int64_t)a.cols * a.page), t = len - 1;
    if (told != len && threadIdx.x == 0) *bad = 1;
    // visible keys: [0, first) and [lo, t), which are cached, and t, the new one
    const int lo = max(0, t - a.window + 1), first = min(a.sinks, lo), cached = first + max(t, 0) - lo, tiles = (cached + KEYS - 1) / KEYS;
    const bf16 *kn = a.k + ((int64_t)b * kv_heads + hk) * a.d, *vn = a.v + ((int64_t)b * kv_heads + hk) * a.d;
    const bf16 *kc = a.k_pages + hk * a.head_stride, *vc = a.v_pages + hk * a.head_stride;
    const uint32_t ring = tc::smem_u32(smem + warp * S::RING);
    const int step = splits * WARPS, tile0 = split * WARPS + warp;

    // the queries as fragments: row = head
    uint32_t q[DP / 16][4];
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = lane / 4 + (i & 1) * 8, col = k * 16 + (lane & 3) * 2 + (i >> 1) * 8;
            q[k][i] = row < g && col < a.d ? *reinterpret_cast<const uint32_t *>(a.q + ((int64_t)b * a.heads + hk * a.group + g0 + row) * a.d + col) : 0u;
        }

    // The new token's row of the cache; nobody reads it there in this call: it is taken from k and v, behind the cached keys.
    if (split == 0 && warp == 0 && g0 == 0 && len > 0) {
        const int p = a.table[(int64_t)b * a.cols + t / a.page], col = lane * 8 % DP;
        if ((unsigned)p >= (unsigned)a.pages) *bad = 1;
        else if (lane * 8 < 2 * DP && col < a.d)
            *reinterpret_cast<uint4 *>((lane * 8 < DP ? a.k_pages : a.v_pages) + (int64_t)p * a.page_stride + (t % a.page) * a.token_stride + hk * a.head_stride + col) =
                *reinterpret_cast<const uint4 *>((lane * 8 < DP ? kn : vn) + col);
    }

    // Lane r (of 16) finds row r of a tile: its page (-1: none, or outside the cache), then its offset in the pages, which goes where all lanes
    // that copy a piece of the row see it.
    auto page_of = [&](int tile, int &slot) -> int {
        const int u = tile * KEYS + (lane & 15), s = u < first ? u : lo + u - first;
        slot = 0;
        if (u >= cached) return -1;
        const int p = (int)__umulhi((unsigned)s, a.page_magic), q = s - p * a.page >= a.page ? p + 1 : p;
        slot = s - q * a.page;
        const int page = a.table[(int64_t)b * a.cols + q];
        if ((unsigned)page < (unsigned)a.pages) return page;
        *bad = 1;
        return -1;
    };
    int64_t *at = offsets + warp * KEYS;
    const int piece = lane % CHUNKS, row0 = lane / CHUNKS;
    const bool inside = piece * 8 < a.d;
    constexpr int ROWS = 32 / CHUNKS;                      // rows that a warp copies at a time
    // bit r: row r of the tile is there.  What is not there is zeros.
    auto fetch = [&](int tile, int stage, int page, int slot) -> unsigned {
        const unsigned there = __ballot_sync(~0u, page >= 0) & 0xFFFFu;
        if (tile < tiles) {
            __syncwarp();
            if (lane < KEYS) at[lane] = page >= 0 ? (int64_t)page * a.page_stride + slot * a.token_stride : 0;
            __syncwarp();
            const uint32_t dst = ring + stage * S::STAGE;
#pragma unroll
            for (int i = 0; i < KEYS / ROWS; ++i) {
                const int row = row0 + i * ROWS;
                const int64_t from = at[row] + piece * 8;
                const bool in = inside && (there >> row & 1);
                const uint32_t o = dst + row * (DP * 2) + ((piece ^ (row & 7)) << 4);
                copy16(o, kc + from, in);
                copy16(o + S::TILE_BYTES, vc + from, in);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        return there;
    };

    const float c = a.scale * 1.4426950408889634f;
    float o[DP / 8][4], most[2] = {-INFINITY, -INFINITY}, sum[2] = {0.f, 0.f};
#pragma unroll
    for (int n = 0; n < DP / 8; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[n][i] = 0.f;
    // 16 keys in a stage
    auto attend = [&](int stage, unsigned there) {
        const uint32_t K = ring + stage * S::STAGE, V = K + S::TILE_BYTES;
        float x[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int k = 0; k < DP / 32; ++k)
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                uint32_t f[4];                             // 8 keys, 32 columns
                ldmatrix4(f, K + (n * 8 + (lane & 7)) * (DP * 2) + (((k * 4 + lane / 8) ^ (lane & 7)) << 4));
                mma16816(x[n], q[2 * k], f[0], f[1]);
                mma16816(x[n], q[2 * k + 1], f[2], f[3]);
            }
        if (there != 0xFFFFu)
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (!(there >> (n * 8 + (lane & 3) * 2 + (i & 1)) & 1)) x[n][i] = -INFINITY;
        float top[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            top[i] = fmaxf(fmaxf(x[0][2 * i], x[0][2 * i + 1]), fmaxf(x[1][2 * i], x[1][2 * i + 1]));
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
            }
#pragma unroll
            for (int n = 0; n < DP / 8; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) o[n][i] *= f[i >> 1];
        }
        const float ref[2] = {most[0] == -INFINITY ? 0.f : c * most[0], most[1] == -INFINITY ? 0.f : c * most[1]};
        uint32_t p[4];
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float y0 = fast_exp2(fmaf(c, x[n][2 * i], -ref[i])), y1 = fast_exp2(fmaf(c, x[n][2 * i + 1], -ref[i]));
                sum[i] += y0 + y1;
                const __nv_bfloat162 w = __floats2bfloat162_rn(y0, y1);          // rounded once, for the product with V
                p[n * 2 + i] = *reinterpret_cast<const uint32_t *>(&w);
            }
#pragma unroll
        for (int n = 0; n < DP / 16; ++n) {
            uint32_t f[4];                                 // 16 keys, 16 columns
            ldmatrix4_trans(f, V + (lane & 15) * (DP * 2) + (((n * 2 + lane / 16) ^ (lane & 7)) << 4));
            mma16816(o[2 * n], p, f[0], f[1]);
            mma16816(o[2 * n + 1], p, f[2], f[3]);
        }
    };
    unsigned there[STAGES];
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
        attend(stage, there[0]);
#pragma unroll
        for (int s = 0; s + 1 < STAGES; ++s) there[s] = there[s + 1];
        if (++stage == STAGES) stage = 0;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    __syncwarp();
    if (split == 0 && warp == 0 && len > 0) {              // the new token, as a tile of one key
        for (int i = lane; i < 2 * KEYS * CHUNKS; i += 32) {
            const int v = i / (KEYS * CHUNKS), row = i / CHUNKS % KEYS, ch = i % CHUNKS;
            const bool in = row == 0 && ch * 8 < a.d;
            *reinterpret_cast<uint4 *>(smem + v * S::TILE_BYTES + row * (DP * 2) + ((ch ^ (row & 7)) << 4)) =
                in ? *reinterpret_cast<const uint4 *>((v ? vn : kn) + ch * 8) : make_uint4(0u, 0u, 0u, 0u);
        }
        __syncwarp();
        attend(0, 1u);
        __syncwarp();
    }

    // join the warps: each leaves its output where its ring was
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        sum[i] += __shfl_xor_sync(~0u, sum[i], 1);
        sum[i] += __shfl_xor_sync(~0u, sum[i], 2);
        if ((lane & 3) == 0) {
            most_w[warp * HEADS + i * 8 + lane / 4] = most[i];
            sum_w[warp * HEADS + i * 8 + lane / 4] = sum[i];
        }
    }
    float *mine = (float *)(smem + warp * S::RING);
#pragma unroll
    for (int n = 0; n < DP / 8; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i)
            *reinterpret_cast<float2 *>(mine + (lane / 4 + i * 8) * DP + n * 8 + (lane & 3) * 2) = make_float2(o[n][2 * i], o[n][2 * i + 1]);
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
        sum_b[threadIdx.x] = s;
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
    // then the blocks: their shares first, each read once, then every block its piece of the output
    if (threadIdx.x < HEADS) {
        float m[MAX_SPLITS], l[MAX_SPLITS], all = -INFINITY, s = 0.f;
#pragma unroll
        for (int r = 0; r < MAX_SPLITS; ++r) {
            m[r] = -INFINITY;
            l[r] = 0.f;
            if (r < splits) {
                m[r] = splits > 1 ? ld_cluster(tc::map_to_cta(tc::smem_u32(most_b + threadIdx.x), r)) : most_b[threadIdx.x];
                l[r] = splits > 1 ? ld_cluster(tc::map_to_cta(tc::smem_u32(sum_b + threadIdx.x), r)) : sum_b[threadIdx.x];
            }
            all = fmaxf(all, m[r]);
        }
#pragma unroll
        for (int r = 0; r < MAX_SPLITS; ++r) {
            m[r] = weight(m[r], all);
            s = fmaf(m[r], l[r], s);
        }
        const float inv = len > 0 ? 1.f / s : 0.f;         // a sum of 0 (all scores are -inf) or NaN gives NaN
#pragma unroll
        for (int r = 0; r < MAX_SPLITS; ++r) share[r * HEADS + threadIdx.x] = m[r] * inv;
    }
    __syncthreads();
    for (int e = 2 * (split * WARPS * 32 + threadIdx.x); e < g * DP; e += 2 * splits * WARPS * 32) {
        const int row = e / DP, col = e % DP;
        float y0 = 0.f, y1 = 0.f;
        if (splits == 1) {
            y0 = share[row] * block[e];
            y1 = share[row] * block[e + 1];
        } else {
#pragma unroll 8
            for (int r = 0; r < splits; ++r) {
                const uint32_t at = tc::map_to_cta(tc::smem_u32(block + e), r);
                float x0, x1;
                asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(x0), "=f"(x1) : "r"(at) : "memory");
                y0 = fmaf(share[r * HEADS + row], x0, y0);
                y1 = fmaf(share[r * HEADS + row], x1, y1);
            }
        }
        if (col < a.d) *reinterpret_cast<__nv_bfloat162 *>(a.out + ((int64_t)b * a.heads + hk * a.group + g0 + row) * a.d + col) = __floats2bfloat162_rn(y0, y1);
    }
    if (splits > 1) tc::cluster_sync_all();                // no block ends while another reads its shared memory
    if (*bad && threadIdx.x == 0) atomicExch(a.status + kWsStatusWord, (unsigned)ST_ERR_DEV_BOUNDS);
}

// The status is cleared ahead of the blocks that may report: within one kernel no block is known to run before another.  A kernel, which the
// next one's blocks may be placed beside, takes 1.0 us of 8 heads with 8192 keys (16.3 to 17.3), a memset 2.4.
__global__ void step_status_kernel(unsigned *status)
{
    pdl_trigger();
    pdl_wait();
    status[kWsStatusWord] = 0u;
    status[kWsDetailWord] = 0u;
}

template <int DP, int WARPS, int STAGES>
static st_status launch_step(const StepArgs &a, int splits, cudaStream_t stream)
{
    const auto kernel = window_step_kernel<DP, WARPS, STAGES>;
    const size_t smem = wstep::Shape<DP, WARPS, STAGES>::SMEM;
    if (!ensure_dynamic_smem(kernel, smem) || !allow_large_clusters(kernel)) return ST_ERR_CUDA;
    const int chunks = (a.group + wstep::HEADS - 1) / wstep::HEADS;
    const st_status rc = launch(step_status_kernel, dim3(1), 1, 0, stream, a.status);
    if (rc != ST_OK) return rc;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)splits, (unsigned)(a.heads / a.group * chunks), (unsigned)a.nseq);
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

// Where heads and sequences are few the keys are split over a cluster of up to 16 blocks.  Blocks of four warps with one tile ahead leave room
// for three on an SM; where even 16 blocks a head do not fill the SMs once, six warps, of which two blocks still fit: clusters of 16 need 16
// blocks' room in one group of SMs, and with one block to an SM not all of them start (8 heads, 8192 keys: eight warps with two tiles ahead
// 25 us, four warps 17.5, six 15.8; 64 sequences of 8 heads: four warps with one tile ahead 65 us, with two 85).
template <int DP>
static st_status run_step(const StepArgs &a, cudaStream_t stream)
{
    const int64_t most = (int64_t)a.cols * a.page, visible = most < (int64_t)a.window + a.sinks ? most : (int64_t)a.window + a.sinks;
    const int64_t blocks = (int64_t)a.nseq * (a.heads / a.group) * ((a.group + wstep::HEADS - 1) / wstep::HEADS);
    const int64_t sms = sm_count_or_default(), tiles = (visible + wstep::KEYS - 1) / wstep::KEYS;
    int n = 1;
    while (n < wstep::MAX_SPLITS && blocks * n < 3 * sms && tiles > (int64_t)2 * n * 4 * wstep::FEWEST) n *= 2;
    if (blocks * n <= sms && tiles > (int64_t)n * 6) return launch_step<DP, 6, 2>(a, n, stream);
    return launch_step<DP, 4, 2>(a, n, stream);
}

}  // namespace attn
}  // namespace st

using namespace st;
using namespace st::attn;

extern "C" st_status st_attn_window_step(const st_cache *c, const void *q, const void *k, const void *v, void *k_pages,
                              void *v_pages, const int32_t *table, const int32_t *lens, int64_t window, int64_t sinks,
                              float scale, void *out, void *ws, size_t ws_bytes, void *stream)
{
    if (!c) return ST_ERR_NULL;
    if (c->dtype != ST_BF16) return ST_ERR_DTYPE;
    if (c->reserved != 0 || c->nseq <= 0 || c->heads <= 0 || c->kv_heads <= 0 || c->d <= 0 || c->pages <= 0 || c->page <= 0 || c->table_cols <= 0 ||
        c->heads % c->kv_heads != 0 || window < 1 || sinks < 0)
        return ST_ERR_SHAPE;
    if (c->nseq > 65535 || c->heads > 65535 || c->d % 8 != 0 || c->d > 128 || c->pages > (1 << 30) || c->page > (1 << 30) || c->table_cols > (1 << 30) ||
        c->page * c->table_cols > (1 << 30))               // tokens of a sequence
        return ST_ERR_UNSUPPORTED;
    if (!stride_ok(c->pages, c->page_stride, c->d) || !stride_ok(c->page, c->token_stride, c->d) || !stride_ok(c->kv_heads, c->head_stride, c->d))
        return ST_ERR_SHAPE;
    if ((c->pages > 1 && c->page_stride % 8 != 0) || (c->page > 1 && c->token_stride % 8 != 0) || (c->kv_heads > 1 && c->head_stride % 8 != 0))
        return ST_ERR_ALIGN;
    if (!(scale > 0.f && scale < INFINITY)) return ST_ERR_UNSUPPORTED;
    if (!q || !k || !v || !k_pages || !v_pages || !table || !lens || !out) return ST_ERR_NULL;
    for (const void *p : {q, k, v, (const void *)k_pages, (const void *)v_pages, (const void *)table, (const void *)lens, (const void *)out})
        if (!aligned16(p)) return ST_ERR_ALIGN;
    if (!ws || ws_bytes < kWsHeaderBytes) return ST_ERR_WORKSPACE;
    if (!aligned256(ws)) return ST_ERR_ALIGN;
    const int64_t out_bytes = c->nseq * c->heads * c->d * 2, new_bytes = c->nseq * c->kv_heads * c->d * 2;
    if (dense_of(q, c->nseq, c->heads, c->d).under(out, out_bytes, true) || arrays_meet(out, out_bytes, k, new_bytes) || arrays_meet(out, out_bytes, v, new_bytes))
        return ST_ERR_UNSUPPORTED;
    StepArgs a = {};
    a.q = (const bf16 *)q;
    a.k = (const bf16 *)k;
    a.v = (const bf16 *)v;
    a.k_pages = (bf16 *)k_pages;
    a.v_pages = (bf16 *)v_pages;
    a.table = table;
    a.lens = lens;
    a.nseq = (int)c->nseq;
    a.heads = (int)c->heads;
    a.group = (int)(c->heads / c->kv_heads);
    a.d = (int)c->d;
    a.pages = (int)c->pages;
    a.page = (int)c->page;
    a.page_magic = 0xFFFFFFFFu / (unsigned)c->page;
    a.cols = (int)c->table_cols;
    a.window = clamp_int(window, 1 << 30);
    a.sinks = clamp_int(sinks, 1 << 30);
    a.page_stride = stride_of(c->pages, c->page_stride);
    a.token_stride = stride_of(c->page, c->token_stride);
    a.head_stride = stride_of(c->kv_heads, c->head_stride);
    a.scale = scale;
    a.out = (bf16 *)out;
    a.status = (unsigned *)ws;
    return a.d <= 64 ? run_step<64>(a, (cudaStream_t)stream) : run_step<128>(a, (cudaStream_t)stream);
}
