"""Calls of the rotations, the caches and the steps at the edges of what they take."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import attn_more_reference as ref
import paper_2211_10482_b200 as st
from test_gpu_attn import near, normal, ok, spans
from test_gpu_attn_more import Cache, check_step, shared_inputs
from test_gpu_parity import GuardAllocator


@pytest.fixture(autouse=True)
def guard_bands_and_device_status():
    """Nothing writes outside its buffers."""
    guard = GuardAllocator()
    st.set_allocator(guard)
    yield
    st.set_allocator(None)
    guard.check()


# ---------------------------------------------------------------------------- scores of nothing


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("scale", [1.0, 1e-8, 1e-30, 1e-44])
@pytest.mark.parametrize("d", [64, 128])
def test_queries_of_nothing_take_the_mean_whatever_the_scale(d, scale, bits):
    """Heads of zeros, of the smallest numbers and of usual ones; keys that fill their tiles and that do not, and so many that warps share them."""
    for lens in ([32, 33, 64, 1, 0, 500], [9001]):
        c = Cache(401, lens, 2, d, 16, bits)
        q = normal(402, len(lens), 6, d)
        q[:, 0], q[:, 4] = 0, 0
        q[:, 1] = 2.0 ** -133
        q[:, 2] = q[:, 2] * 2.0 ** -122
        got = st.st_attn_cache_step(q, *c.pages(), 1 << 30, 0, scale=scale, **c.how())
        ok()
        assert bool(torch.isfinite(got).all())
        check_step(got, c, q, 1 << 30, 0, scale)


@pytest.mark.parametrize("scale", [1.0, 1e-8, 1e-44])
def test_queries_of_nothing_behind_a_prefix(scale):
    c, q, args, lens = shared_inputs(411, [3, 2], [300, 128], [7, 0, 40], 4, 2, 64, 16)
    q[:, 0] = 0
    q[:, 3] = 2.0 ** -133
    got = st.st_attn_shared_step(q, *c.cells, *args, scale=scale)
    ok()
    G = 2
    for g, (a, b) in enumerate(spans([3, 2])):
        for n in range(a, b):
            (k0, k1), (v0, v1) = (tuple(torch.cat(x) for x in zip(c.parts(i, g), c.parts(i, G + n))) for i in range(2))
            near(got[n], *ref.attend(q[n], (k0, k1), (v0, v1), scale), "out of sequence %d" % n)
