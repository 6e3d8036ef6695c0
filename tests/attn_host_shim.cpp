// Host-side C shim over the attention calls' index arithmetic.  Built by tests/test_attn_index.py.
#include "attn_index.cuh"
extern "C" {
long long shim_most_tiles(long long n, long long nseq, long long rows) { return st::attn::most_tiles(n, nseq, rows); }
void shim_slab_of(int x, int slabs, int tiles, int *tile, int *slab)
{
    const st::attn::SlabOf s = st::attn::slab_of(x, slabs, tiles);
    *tile = s.tile;
    *slab = s.slab;
}
int shim_overlap(long long table, long long rows, long long heads, long long piece, long long row, long long head, long long p, long long bytes)
{
    return st::attn::overlap(table, rows, heads, piece, row, head, p, bytes);
}
}
