"""How near the steps come to 64 bits: their errors in the root mean square, beside what the roundings that they state leave (attn_precision_reference.py)."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import attn_precision_reference as precision
import paper_2211_10482_b200 as st
from test_gpu_attn import normal, ok, spans
from test_gpu_attn_more import Cache, shared_inputs

# Some columns of the keys are six times as large as the others, and scores of more than 1 in the root mean square leave a result to few weights, of which the
# largest is exact; with half the usual scale they are about 0.9.
FLAT = 0.5
WEIGHT = {16: precision.TWO_BF16, 8: precision.ONE_FP16, 4: precision.TWO_BF16}


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("lens,H,Hk,d", [([300, 700, 500, 640, 333, 900, 411, 512], 16, 4, 128), ([800] * 6, 32, 2, 64), ([9000], 64, 2, 128)])
def test_errors_of_the_step_in_the_root_mean_square(lens, H, Hk, d, bits):
    c = Cache(421, lens, Hk, d, 16, bits)
    q = normal(422, len(lens), H, d)
    got = st.st_attn_cache_step(q, *c.pages(), 1 << 30, 0, scale=FLAT * d ** -0.5, **c.how())
    ok()
    out, squares = (torch.stack(x) for x in zip(*(precision.attend(q[b], c.parts(0, b), c.parts(1, b), FLAT * d ** -0.5) for b in range(len(lens)))))
    error, most = precision.error(got, out), precision.bound(out, squares, WEIGHT[bits])
    assert error <= most, "%.3g of the bound" % (error / most)


@pytest.mark.parametrize("groups,prefix,own,H,Hk,d,page", [([8], [1500], [40], 8, 2, 128, 16), ([20, 20], [2000, 700], [3, 200], 16, 4, 128, 64), ([70], [900], [0], 8, 4, 64, 100)])
def test_errors_of_the_shared_step_in_the_root_mean_square(groups, prefix, own, H, Hk, d, page):
    c, q, args, lens = shared_inputs(431, groups, prefix, own, H, Hk, d, page)
    got = st.st_attn_shared_step(q, *c.cells, *args, scale=FLAT * d ** -0.5)
    ok()
    G, rows = len(groups), []
    for g, (a, b) in enumerate(spans(groups)):
        for n in range(a, b):
            (k0, k1), (v0, v1) = (tuple(torch.cat(x) for x in zip(c.parts(i, g), c.parts(i, G + n))) for i in range(2))
            rows.append(precision.attend(q[n], (k0, k1), (v0, v1), FLAT * d ** -0.5))
    out, squares = (torch.stack(x) for x in zip(*rows))
    error, most = precision.error(got, out), precision.bound(out, squares, precision.TWO_BF16)
    assert error <= most, "%.3g of the bound" % (error / most)
