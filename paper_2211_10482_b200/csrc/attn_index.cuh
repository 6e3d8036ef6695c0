// Index arithmetic of the attention calls (host + device).
#pragma once
#include <cstdint>
#include "st_index.cuh"

namespace st {
namespace attn {

// A table of n rows in nseq sequences has at most this many tiles of `rows` rows.
ST_HD int64_t most_tiles(int64_t n, int64_t nseq, int64_t rows) { return n / rows + nseq; }

// What block x of a run does whose results have `slabs` slabs of columns: slab `slab` of tile `tile`; tile -1: nothing.  Runs of one launch
// share a grid that is as wide as the one with the most slabs needs, and tiles from `tiles` on have no place in the workspace.
struct SlabOf {
    int tile, slab;
};
ST_HD SlabOf slab_of(int x, int slabs, int tiles)
{
    const int tile = x / slabs;
    return {tile < tiles ? tile : -1, x % slabs};
}

}  // namespace attn
}  // namespace st
