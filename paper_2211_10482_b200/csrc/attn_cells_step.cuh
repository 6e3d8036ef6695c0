// Arguments of the single-token attention over a cache in cells, and the parts of a shared prefix that it may be joined with.
#pragma once
#include "attn_cells.cuh"

namespace st {
namespace attn {

struct CellsStepArgs {
    Cells c;
    const bf16 *q;
    int64_t q_row, q_head;
    int heads, group, window, sinks;
    float scale;
    bf16 *out;
    unsigned *status;
    // Parts of a prefix, [part][key head][sequence, head of the key head's group]: largest score (-inf: no visible key, or none above -inf), sum of the weights
    // (0: no visible key; 1 where the largest is -inf), sum of the weighted values, [part][key head][16 or 32 column quads][sequence, head][4].
    // part_count [sequence]: how many there are of each; NULL: none.
    const int *part_count;
    const float *part_most, *part_sum, *part;
};

constexpr int MAX_PARTS = 32;

st_status run_cells_step(const CellsStepArgs &a, int dtype, cudaStream_t stream);
st_status check_step(const st_cells *c, const void *q, int64_t q_row, int64_t q_head, float scale, const void *out);
CellsStepArgs step_args(const st_cells *c, const void *q, int64_t q_row, int64_t q_head, const void *k_pages, const void *v_pages, const void *k_scales,
                        const void *v_scales, const int32_t *table, const int32_t *lens, float scale, void *out, void *ws);

}  // namespace attn
}  // namespace st
