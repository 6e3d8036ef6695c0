"""Calls of the rotations, the caches and the steps at the edges of what they take."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import attn_more_reference as ref
import paper_2211_10482_b200 as st
from test_gpu_attn import near, normal, ok, spans
from test_gpu_attn_more import Cache, check_shared, check_step, ints, shared_inputs
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


# --------------------------------------------------------------------------------------- groups


@pytest.mark.parametrize("told,cut", [
    ([0, 4, 2, 6], [0, 4, 4, 6]),
    ([0, 6, 0, 6], [0, 6, 6, 6]),                        # two groups of the same sequences
    ([3, 0, 5, 8], [3, 3, 5, 8]),
    ([-3, 2, 100, 5, 8], [0, 2, 8, 8, 8]),
    ([8, 0, 8, 0, 8], [8, 8, 8, 8, 8]),                  # nobody is left
    ([0, 2, 2, -1, 1, 7], [0, 2, 2, 2, 2, 7]),
    ([-(2**31), 2**31 - 1], [0, 8]),
])
@pytest.mark.parametrize("H,Hk", [(4, 2), (40, 1)])       # with 40 heads to a key head a tile of rows holds six sequences
def test_a_sequence_is_in_one_group_whatever_the_offsets(told, cut, H, Hk):
    G = len(told) - 1
    groups = [b - a for a, b in zip(cut, cut[1:])]
    c, q, args, lens = shared_inputs(501, [8] + [0] * (G - 1), [500, 130, 64, 900, 33][:G], [20, 0, 3], H, Hk, 64, 16)
    want = st.st_attn_shared_step(q, *c.cells, *args[:4], ints(*cut))
    ok()
    for _ in range(3):
        got = st.st_attn_shared_step(q, *c.cells, *args[:4], ints(*told))
        assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS
        assert torch.equal(got, want)
    alone = st.st_attn_cache_step(q, *c.cells, args[2], args[3], 1 << 30)
    assert torch.equal(got[: cut[0]], alone[: cut[0]]) and torch.equal(got[cut[-1] :], alone[cut[-1] :])
    prefix = [500, 130, 64, 900, 33]
    for g, (a, b) in enumerate(zip(cut, cut[1:])):
        for n in range(a, b):
            (k0, k1), (v0, v1) = (tuple(torch.cat(x) for x in zip(c.parts(i, g), c.parts(i, G + n))) for i in range(2))
            near(got[n], *ref.attend(q[n], (k0, k1), (v0, v1)), "out of sequence %d" % n)


def test_offsets_of_thousands_of_groups():
    """More groups than the block that cuts them has threads; some of them fall back, at the ends of warps and blocks too."""
    n, G = 300, 2500
    told = torch.tensor([i * n // G for i in range(G + 1)], dtype=torch.int32)
    for fine in (True, False):
        if not fine:
            told[[31, 32, 255, 256, 257, 1023, 1024, 1025, 2047, 2048, 2400]] = torch.tensor([0, 0, -1, 0, 3, 5, 0, 1, 0, 9, n], dtype=torch.int32)
        cut = told.clamp(0, n).cummax(0).values
        sizes = (cut[1:] - cut[:-1]).tolist()
        prefix = [17 if s else 0 for s in sizes]
        c, q, args, lens = shared_inputs(511, sizes, prefix, [2, 0], 2, 1, 32, 16)
        got = st.st_attn_shared_step(q, *c.cells, *args[:4], told.cuda())
        assert st.st_check_status() == (st.ST_OK if fine else st.ST_ERR_DEV_BOUNDS)
        check_shared(got, c, q, sizes, prefix, lens)


# ---------------------------------------------------------------------------------- frequencies


@pytest.mark.parametrize("rot,inter", [(64, False), (64, True), (20, False), (20, True)])
@pytest.mark.parametrize("norm", [False, True])
def test_frequencies_that_are_no_numbers_or_too_large_give_none(rot, inter, norm):
    """Their pairs are NaN, and the others what they are without them."""
    n, H, Hk, d = 70, 3, 2, 64
    q, k = normal(521, n, H, d), normal(522, n, Hk, d)
    positions = torch.arange(-3, n - 3, dtype=torch.int32, device="cuda")
    freq = st.st_rotary_frequencies(rot).cuda()
    bad = {0: float("inf"), 3: float("nan"), 5: 2.0 ** 24, 6: -(2.0 ** 40), rot // 2 - 1: -float("inf")}
    wrong, clean = freq.clone(), freq.clone()
    for i, f in bad.items():
        wrong[i], clean[i] = f, 0.0
    clean[1], wrong[1] = 16777215.0, 16777215.0          # the largest that there is an exact product for
    a, b = ref.pairs_of(rot, inter, q.device)
    hit = torch.zeros(d, dtype=torch.bool, device="cuda")
    hit[a[list(bad)]] = hit[b[list(bad)]] = True
    eps = 1e-6 if norm else None
    for got, want in zip(st.st_attn_rotate(q, k, positions, wrong, inter, eps=eps), st.st_attn_rotate(q, k, positions, clean, inter, eps=eps)):
        assert bool(got[..., hit].isnan().all()) and torch.equal(got[..., ~hit], want[..., ~hit])
    near(st.st_attn_rotate(q, k, positions, clean, inter, eps=eps)[0], *ref.rotate(q, None, positions, clean, inter, eps, 1.0), "clean")
    dq, dk = normal(523, n, H, d), normal(524, n, Hk, d)
    for got, want in zip(st.st_attn_rotate_grad(q, k, dq, dk, positions, wrong, inter, eps=eps)[:2], st.st_attn_rotate_grad(q, k, dq, dk, positions, clean, inter, eps=eps)[:2]):
        if norm:
            assert bool(got.isnan().all())                 # a row's mean is over all of its columns
        else:
            assert bool(got[..., hit].isnan().all()) and torch.equal(got[..., ~hit], want[..., ~hit])


# -------------------------------------------------------------------------------------- extents


@pytest.mark.parametrize("groups,prefix,own,H,Hk,d,page", [
    ([3], [200], [9, 0], 2, 1, 8, 16),                   # a box of 64 columns of which the table has 8
    ([2, 2], [90, 300], [5], 4, 2, 8, 8),
    ([5], [700], [1, 300], 6, 2, 72, 128),               # the second box of a row has 8 columns
    ([40], [515], [2], 8, 2, 104, 512),
    ([4], [260], [30], 4, 4, 64, 1024),                  # one page holds all
])
def test_shared_step_of_narrow_heads_and_long_pages(groups, prefix, own, H, Hk, d, page):
    c, q, args, lens = shared_inputs(531, groups, prefix, own, H, Hk, d, page)
    got = st.st_attn_shared_step(q, *c.cells, *args)
    ok()
    check_shared(got, c, q, groups, prefix, lens)


def repeated(c, n, page, pages):
    """What the first n tokens behind a table that goes through `pages` pages again and again count for: places and how often each is there."""
    place = torch.arange(pages * page, device="cuda")
    turns, rest = divmod(n, pages * page)
    return (c.table[0].long()[place // page], place % page), (turns + (place < rest)).double()


def weighted(q, k, v, times, scale):
    """ref.attend over keys that are there several times."""
    group = q.shape[0] // k[0].shape[1]
    Q = q.double()[:, None]
    (k0, k1), (v0, v1) = (tuple(z.repeat_interleave(group, 1).transpose(0, 1) for z in x) for x in (k, v))
    x = (Q @ (k0 + k1).transpose(1, 2)) * scale + times.log()
    p = torch.softmax(x, -1)
    off = ref.E * scale * (Q.abs() @ (k0.abs() + k1.abs()).transpose(1, 2)).amax(-1)
    out, size = p @ (v0 + v1), p @ (v0.abs() + v1.abs())
    return out.squeeze(1), (ref.B * (p @ v1.abs()) + ref.B * out.abs() + (ref.F + 2 * off[..., None]) * size).squeeze(1)


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_steps_over_sixteen_million_tokens(bits):
    """Pages that a table names again and again, so that positions, tiles and pieces are many and the cache is small."""
    page, pages, n, H, Hk, d = 256, 8, (1 << 24) + 77, 4, 1, 64
    c = Cache(541, [page * pages], Hk, d, page, bits)
    q = normal(542, 1, H, d)
    table = c.table[:, torch.arange((1 << 16) + 1, device="cuda") % pages].contiguous()
    at, times = repeated(c, n, page, pages)
    want = weighted(q[0], c.parts(0, 0, at), c.parts(1, 0, at), times, d ** -0.5)
    got = st.st_attn_cache_step(q, *c.cells, table, ints(n), 1 << 30, 0, **c.how())
    ok()
    near(got[0], *want, "step")
    if bits == 16:
        got = st.st_attn_shared_step(q, *c.cells, table, ints(n - page * pages), c.table, ints(page * pages))
        ok()
        near(got[0], *want, "behind a prefix")
