"""Index arithmetic of the attention calls, on the CPU: which places of a workspace the blocks of a launch reach."""
import ctypes
import os
import subprocess
import tempfile

import pytest

pytest.importorskip("torch")

import paper_2211_10482_b200 as st

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2211_10482_b200", "csrc")
CHUNK, SLAB = 128, 64


@pytest.fixture(scope="module")
def shim():
    out = os.path.join(tempfile.mkdtemp(prefix="st_attn_shim_"), "shim.so")
    subprocess.check_call(["g++", "-O2", "-shared", "-fPIC", "-std=c++17", "-x", "c++", "-I", CSRC,
                           os.path.join(ROOT, "tests", "attn_host_shim.cpp"), "-o", out])
    L = ctypes.CDLL(out)
    ll, ip = ctypes.c_longlong, ctypes.POINTER(ctypes.c_int)
    L.shim_most_tiles.argtypes, L.shim_most_tiles.restype = [ll] * 3, ll
    L.shim_slab_of.argtypes, L.shim_slab_of.restype = [ctypes.c_int] * 3 + [ip, ip], None
    L.shim_overlap.argtypes, L.shim_overlap.restype = [ll] * 8, ctypes.c_int
    return L


def place(shim, x, slabs, tiles):
    tile, slab = ctypes.c_int(), ctypes.c_int()
    shim.shim_slab_of(x, slabs, tiles, ctypes.byref(tile), ctypes.byref(slab))
    return tile.value, slab.value


@pytest.mark.parametrize("d,dv", [(64, 64), (72, 64), (64, 72), (64, 96), (96, 64), (8, 128), (128, 128)])
def test_runs_of_a_gradient_stay_within_their_states(shim, d, dv):
    """The runs of a gradient share a grid, as wide as the one with the most columns needs.  Offsets may name every row again, so that
    the sequences have more segments than there is room for: no block takes a tile behind the last one."""
    n, nseq, heads, wide = 300 * CHUNK, 4, 1, max(d, dv)
    states = (st.st_workspace_bytes(st.ST_OP_ATTN_DECAY_GRAD, n, nseq, heads, wide) - 256) // 4 // 2       # floats of one run
    tiles = states // (heads * wide * wide)
    # the room is that for segments of whole chunks, of which sequences that name all rows nseq times have more
    chunks = next(c for c in range(1, 301) if shim.shim_most_tiles(n, nseq, c * CHUNK) == tiles)
    assert 0 < tiles < nseq * -(-300 // chunks)
    slabs = [-(-z // SLAB) for z in (d, dv, d)]                                                            # dq, dv, dk
    for own, x_cols, z_cols in zip(slabs, (dv, d, dv), (d, dv, d)):
        seen = set()
        for x in range(tiles * max(slabs)):
            tile, slab = place(shim, x, own, tiles)
            assert 0 <= slab < own and tile < tiles
            if tile >= 0:
                assert (tile + 1) * heads * x_cols * z_cols <= states
                assert (tile, slab) not in seen
                seen.add((tile, slab))
        assert len(seen) == tiles * own                    # and none is left out


def test_every_sequence_has_its_tiles(shim):
    for n, lens, rows in ((1000, [1000], 128), (1000, [0, 1, 999], 256), (257, [128, 129], 128), (40, [1] * 40, 128), (5000, [4999, 1], 1 << 29)):
        assert sum(max(1, -(-x // rows)) for x in lens) <= shim.shim_most_tiles(n, len(lens), rows)


@pytest.mark.parametrize("rows,heads,piece,row,head", [(1, 1, 4, 4, 4), (3, 2, 4, 8, 4), (3, 2, 4, 4, 12), (4, 3, 2, 16, 4), (5, 2, 3, 3, 40), (1, 3, 2, 128, 5), (4, 1, 2, 7, 128)])
def test_overlap_is_that_of_the_bytes(shim, rows, heads, piece, row, head):
    table = 200
    bytes_of = {table + r * row + h * head + i for r in range(rows) for h in range(heads) for i in range(piece)}
    for p in range(table - 12, max(bytes_of) + 12):
        for n in (1, 2, 5, 30):
            assert bool(shim.shim_overlap(table, rows, heads, piece, row, head, p, n)) == bool(bytes_of & set(range(p, p + n)))
