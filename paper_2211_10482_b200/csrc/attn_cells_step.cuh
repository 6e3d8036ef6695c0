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
    // Work: a line of units (one key head of one sequence with 16 or fewer query heads), each as long as its key tiles and what a unit costs beside them;
    // starts[b] is where sequence b's begin, starts[nseq] the whole length.
    int64_t *starts;
    int units, team;                       // of a sequence; neighbouring units that as many warps of a block take together, as one on the line
    // Partial results of warps, [warp][2][heads of a unit]: largest score, sum of the weights, sum of the weighted values (64 or 128 columns); 0: of the
    // unit that the warp goes on with, 1: of one that it begins and does not end.
    float *slot_most, *slot_sum, *slot;
    int slots;                             // warps
    // Parts of a prefix, [part][key head][sequence, head of the key head's group]: largest score (-inf: no visible key, or none above -inf), sum of the weights
    // (0: no visible key; 1 where the largest is -inf), sum of the weighted values, [part][key head][16 or 32 column quads][sequence, head][4].
    // part_count [sequence]: how many there are of each; NULL: none.  Part own_part holds the own tokens of units that one warp has the whole of.
    int *part_count;
    int own_part;
    // Where the groups of sequences that share a prefix begin, as they were told and, `group_cuts`, as no sequence is in two of them; NULL: one group of all.
    const int *group_offsets;
    int *group_cuts;
    int groups;
    float *part_most, *part_sum, *part;
};

constexpr int MAX_PARTS = 32;

// What a call's workspace holds behind its header: the starts of the work, the warps' partial results.
struct StepPlan {
    size_t starts, most, sum, values, bytes;
};
StepPlan step_plan(int64_t nseq, size_t from);
void place_step(CellsStepArgs &a, const StepPlan &p, void *ws);
// Clears the status and part_count, lays out the work and cuts the groups.
st_status plan_step(CellsStepArgs &a, int dtype, cudaStream_t stream);
// The units' kernel, the joins' or both.
constexpr unsigned STEP_UNITS = 1, STEP_JOIN = 2;
st_status run_cells_step(const CellsStepArgs &a, int dtype, unsigned what, cudaStream_t stream);
st_status check_step(const st_cells *c, const void *q, int64_t q_row, int64_t q_head, float scale, const void *out);
CellsStepArgs step_args(const st_cells *c, const void *q, int64_t q_row, int64_t q_head, const void *k_pages, const void *v_pages, const void *k_scales,
                        const void *v_scales, const int32_t *table, const int32_t *lens, float scale, void *out, void *ws);

}  // namespace attn
}  // namespace st
