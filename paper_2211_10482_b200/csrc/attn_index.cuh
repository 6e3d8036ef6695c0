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

// Whether any of `bytes` bytes from address p on belongs to a table of rows x heads pieces of `piece` bytes, `row` and `head` bytes apart.
inline bool overlap(uint64_t table, uint64_t rows, uint64_t heads, uint64_t piece, uint64_t row, uint64_t head, uint64_t p, uint64_t bytes)
{
    const uint64_t end = p + bytes;
    if (p >= table + (rows - 1) * row + (heads - 1) * head + piece || end <= table) return false;
    for (uint64_t h = 0; h < heads; ++h) {
        const uint64_t at = table + h * head, r = p < at + piece ? 0 : (p - at - piece) / row + 1;     // the first row that ends behind p
        if (r < rows && at + r * row < end) return true;
    }
    return false;
}

}  // namespace attn
}  // namespace st
