"""Attention over structured pairs on the GPU: every call against its definition in 64 bits (attn_reference.py, which derives the
tolerances), sequence by sequence, at the sizes and masks where tiles, chunks and pages end."""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import attn_reference as ref
import paper_2211_10482_b200 as st
from test_gpu_parity import GuardAllocator

BF16 = torch.bfloat16


@pytest.fixture(autouse=True)
def guard_bands_and_device_status():
    """Nothing writes outside its buffers, and the last call left no error in its workspace."""
    guard = GuardAllocator()
    st.set_allocator(guard)
    yield
    st.set_allocator(None)
    guard.check()


def ok():
    assert st.st_check_status() == st.ST_OK


def normal(seed, *shape):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda").to(BF16)


def floats(seed, *shape):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(shape, generator=g, device="cuda")


def offsets(lens, at=0):
    return torch.tensor([at] + [at + sum(lens[: i + 1]) for i in range(len(lens))], dtype=torch.int32, device="cuda")


def spans(lens, at=0):
    return [(at + sum(lens[:i]), at + sum(lens[: i + 1])) for i in range(len(lens))]


def near(got, want, tol, what):
    assert got.shape == want.shape, (what, got.shape, want.shape)
    got, finite = got.double(), torch.isfinite(want)
    assert bool((torch.isfinite(got) == finite).all()), "%s: not finite in other places" % what
    assert bool((got[~finite] == want[~finite]).all()), what
    over = ((got - want).abs() / (tol + 1e-30))[finite]
    assert not over.numel() or float(over.max()) <= 1.0, "%s: %.3g of the tolerance" % (what, float(over.max()))


# ------------------------------------------------------------------------------------- window

WINDOWS = [
    # query lengths, key lengths, heads, key heads, d, window, sinks
    ([1], [1], 1, 1, 8, 1, 0),
    ([197], [197], 8, 8, 64, 64, 4),
    ([1, 2, 127, 128, 129, 0, 255, 257], None, 4, 2, 64, 100, 4),
    ([300, 0, 31], None, 3, 3, 128, 1, 0),
    ([513], None, 8, 1, 128, 128, 130),
    ([640, 5], None, 4, 4, 128, 129, 1),
    ([384], None, 2, 2, 128, 1 << 40, 0),
    ([700, 33], None, 6, 2, 80, 65, 16),
    ([260, 130], None, 2, 1, 32, 1000, 2),
    ([400], None, 2, 2, 96, 37, 300),
    ([333], None, 2, 1, 128, 127, 1 << 35),
    ([5, 1, 200, 70], [45, 778, 240, 70], 4, 2, 64, 50, 4),
    ([1, 100, 129], [1000, 515, 1300], 4, 1, 128, 300, 130),
    ([50, 300, 8, 260], [20, 150, 0, 260], 2, 2, 64, 40, 3),       # fewer keys than queries: the first rows see nothing
    ([1500], [1500], 2, 2, 64, 600, 10),
    ([17] * 40, None, 2, 2, 64, 8, 1),
    # first columns that end just before, at and behind the band, and at the width that is multiplied alone
    ([300], None, 2, 1, 64, 200, 32),
    ([300], None, 2, 1, 64, 200, 33),
    ([259, 258], [290, 600], 2, 2, 128, 257, 31),
    ([130, 129, 200], [640, 257, 513], 2, 1, 64, 100, 128),
    ([40], [200], 1, 1, 64, 129, 64),
]


def window_inputs(seed, lq, lk, H, Hk, d):
    lk = lq if lk is None else lk
    return lk, normal(seed, sum(lq), H, d), normal(seed + 1, sum(lk), Hk, d), normal(seed + 2, sum(lk), Hk, d), offsets(lq), offsets(lk)


@pytest.mark.parametrize("lq,lk,H,Hk,d,window,sinks", WINDOWS)
def test_window_against_the_definition(lq, lk, H, Hk, d, window, sinks):
    lk, q, k, v, qo, ko = window_inputs(1, lq, lk, H, Hk, d)
    out, lse = st.st_attn_window(q, k, v, window, sinks, qo, ko)
    ok()
    for (a, b), (c, e) in zip(spans(lq), spans(lk)):
        o, l, ot, lt = ref.window(q[a:b], k[c:e], v[c:e], window, sinks)
        near(out[a:b], o, ot, "out")
        near(lse[a:b], l, lt, "lse")


@pytest.mark.parametrize("lq,lk,H,Hk,d,window,sinks", WINDOWS)
def test_window_gradient_against_the_definition(lq, lk, H, Hk, d, window, sinks):
    lk, q, k, v, qo, ko = window_inputs(11, lq, lk, H, Hk, d)
    dout = normal(14, *q.shape)
    out, lse = st.st_attn_window(q, k, v, window, sinks, qo, ko)
    got = st.st_attn_window_grad(q, k, v, out, lse, dout, window, sinks, qo, ko)
    ok()
    for (a, b), (c, e) in zip(spans(lq), spans(lk)):
        want = ref.window_grad(q[a:b], k[c:e], v[c:e], out[a:b], dout[a:b], window, sinks)
        for g, rows, (w, tol), name in zip(got, ((a, b), (c, e), (c, e)), want, ("dq", "dk", "dv")):
            near(g[rows[0] : rows[1]], w, tol, name)


@pytest.mark.parametrize("lq,lk,H,Hk,d,window,sinks", [
    ([3000, 200, 1, 2500], None, 4, 2, 64, 50, 4),
    ([2300], [2500], 2, 2, 128, 130, 130),
    ([1500, 4000], [7000, 4001], 2, 1, 80, 700, 256),
    ([1024, 1025, 1152, 1153, 1280], None, 2, 2, 64, 1, 1),
    ([3500], [3000], 2, 1, 64, 300, 200),
    ([257, 513, 769, 255, 900], [300, 513, 770, 400, 900], 2, 1, 64, 1, 32),
    ([2100, 700], None, 2, 2, 80, 129, 33),
])
def test_window_gradient_of_first_columns_that_many_later_queries_see(lq, lk, H, Hk, d, window, sinks):
    """Queries beyond the window are summed in parts for the sinks' rows."""
    test_window_gradient_against_the_definition(lq, lk, H, Hk, d, window, sinks)


def test_window_gradient_against_differences():
    H, Hk, d, n, window, sinks = 2, 1, 16, 40, 9, 3
    lk, q, k, v, qo, ko = window_inputs(21, [n], None, H, Hk, d)
    dout = normal(24, n, H, d)
    out, lse = st.st_attn_window(q, k, v, window, sinks)
    grads = st.st_attn_window_grad(q, k, v, out, lse, dout, window, sinks)
    tols = [t for _, t in ref.window_grad(q, k, v, out, dout, window, sinks)]
    loss = lambda *x: float((ref.window(*x, window, sinks)[0] * dout.double()).sum())
    base = [x.double() for x in (q, k, v)]
    # delta comes from the rounded out: off by half a step of every value of out
    delta_off = (dout.double().abs() * out.double().abs()).sum(-1).max() * ref.B
    for i, (g, tol) in enumerate(zip(grads, tols)):
        direction = floats(30 + i, *g.shape).double()
        h = 1e-5
        x0, x1 = list(base), list(base)
        x0[i], x1[i] = base[i] - h * direction, base[i] + h * direction
        slope = (loss(*x1) - loss(*x0)) / (2 * h)
        # a row's ds moves by p delta_off scale in all: against |k| or |q| of the largest
        slack = float((tol * direction.abs()).sum()) + float(delta_off) * d ** -0.5 * H * n * float(direction.abs().max()) * float(max(base[0].abs().max(), base[1].abs().max())) * d
        assert abs(float((g.double() * direction).sum()) - slope) <= slack


def test_window_takes_strided_slices_and_head_major_tables():
    n, H, Hk, d = 300, 6, 2, 80
    qkv = normal(41, n, H + 2 * Hk, d)
    q, k, v = qkv.split([H, Hk, Hk], 1)
    want = st.st_attn_window(q.contiguous(), k.contiguous(), v.contiguous(), 77, 5)
    got = st.st_attn_window(q, k, v, 77, 5)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    hq, hk, hv = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v))
    got = st.st_attn_window(hq, hk, hv, 77, 5)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    dout = normal(42, n, H, d)
    a = st.st_attn_window_grad(q, k, v, *want, dout, 77, 5)
    b = st.st_attn_window_grad(hq, hk, hv, *want, dout, 77, 5)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    out, lse = torch.empty_like(want[0]), torch.empty_like(want[1])
    r = st.st_attn_window(q, k, v, 77, 5, out=out, lse=lse, scale=d ** -0.5)
    assert r[0] is out and r[1] is lse and torch.equal(out, want[0])
    ok()


def test_window_other_scale():
    q, k, v = (normal(50 + i, 200, 2, 64) for i in range(3))
    scale = 0.5
    out, lse = st.st_attn_window(q, k, v, 90, 2, scale=scale)
    o, l, ot, lt = ref.window(q, k, v, 90, 2, scale)
    # scores are scale sqrt(d) times larger than at the usual scale, and so are their errors
    wide = scale * 8
    near(out, o, ot * wide, "out")
    near(lse, l, lt * wide, "lse")
    dout = normal(54, 200, 2, 64)
    for g, (w, tol) in zip(st.st_attn_window_grad(q, k, v, out, lse, dout, 90, 2, scale=scale), ref.window_grad(q, k, v, out, dout, 90, 2, scale)):
        near(g, w, tol * wide, "gradient")
    for scale in (0.0, -0.2, math.nan, math.inf):
        with pytest.raises(st.StError) as e:
            st.st_attn_window(q, k, v, 90, 2, scale=scale)
        assert e.value.status == st.ST_ERR_UNSUPPORTED


def test_large_scores_do_not_overflow():
    q, k, v = normal(55, 300, 2, 64) * 30, normal(56, 300, 2, 64) * 30, normal(57, 300, 2, 64)
    out, lse = st.st_attn_window(q, k, v, 100, 4)
    o, l, ot, lt = ref.window(q, k, v, 100, 4)
    # the scores reach some 5000: their fp32 errors, 64 products of up to 10^4 at 2^-24 each times scale, are up to 64*1e4*6e-8/8 = 5e-3
    near(lse, l, lt + 5e-3, "lse")
    assert bool(torch.isfinite(out).all())
    see = ref.visible(300, 300, 100, 4, "cuda")
    V = ref.heads_first(v)
    p = torch.exp((ref.heads_first(q) @ ref.heads_first(k).transpose(1, 2) / 8).masked_fill(~see, -math.inf) - l.transpose(0, 1)[..., None])
    near(out, o, ot + 1.1e-2 * (p @ V.abs()).transpose(0, 1), "out")


@pytest.mark.parametrize("what", ["q nan", "k nan", "k inf", "all -inf", "overflow"])
@pytest.mark.parametrize("window,sinks", [(50, 3), (300, 0), (20, 140)])
def test_scores_that_are_not_finite_are_not_taken_for_none(what, window, sinks):
    """A query whose visible scores hold NaN or +inf, or are all -inf, gets NaN as by the definition, and every other one its row;
    the gradient of such a query is NaN.  The same for a single token.  (The other rows are held against the definition and not bit for bit
    against a call without: the reference that weights are relative to moves for the 32 rows of a warp together, and a weight is
    rounded relative to it, by half a step at most wherever it lies.)"""
    n, H, d, bad = 300, 2, 64, 140
    q, k, v, do = (normal(170 + i, n, H, d) for i in range(4))
    t = torch.arange(n, device="cuda")
    sees_bad = ref.visible(n, n, window, sinks, "cuda")[:, bad]
    if what == "q nan":
        put, at, value, rows = q, (bad, 0, 5), math.nan, t == bad
    elif what == "k nan":
        put, at, value, rows = k, (bad, 0, 7), math.nan, sees_bad
    elif what == "k inf":
        q[:, 0, 9] = q[:, 0, 9].abs() + 1
        put, at, value, rows = k, (bad, 0, 9), math.inf, sees_bad
    elif what == "all -inf":
        q[bad, 0], k[:, 0, 0] = 0.0, k[:, 0, 0].abs() + 1
        put, at, value, rows = q, (bad, 0, 0), -math.inf, t == bad
    else:                                                  # finite values whose products leave fp32
        q[:, 0, 9], k[:, 0, 9] = 2.0 ** 100, 0.0
        put, at, value, rows = k, (bad, 0, 9), 2.0 ** 100, sees_bad
    want, wl, tol, lt = ref.window(q, k, v, window, sinks)
    put[at] = value
    out, lse = st.st_attn_window(q, k, v, window, sinks)
    ok()
    assert bool(out[rows, 0].isnan().all())
    assert bool((lse[rows, 0] == -math.inf).all() if what == "all -inf" else lse[rows, 0].isnan().all())
    for h, others in ((0, ~rows), (1, torch.ones_like(rows))):
        near(out[others, h], want[others, h], tol[others, h], "out")
        near(lse[others, h], wl[others, h], lt[others, h], "lse")
    dq = st.st_attn_window_grad(q, k, v, out, lse, do, window, sinks)[0]
    assert bool(dq[rows, 0].isnan().all()) and bool(torch.isfinite(dq[:, 1].float()).all())
    for i in (bad, bad + 1, bad + 30, n - 1):
        kp, vp = torch.zeros(1, 320, H, d, dtype=BF16, device="cuda"), torch.zeros(1, 320, H, d, dtype=BF16, device="cuda")
        kp[0, :i], vp[0, :i] = k[:i], v[:i]
        o = st.st_attn_window_step(q[i : i + 1], k[i : i + 1], v[i : i + 1], kp, vp, torch.zeros(1, 1, dtype=torch.int32, device="cuda"),
                                   torch.tensor([i + 1], dtype=torch.int32, device="cuda"), window, sinks)
        assert bool(o[0, 0].isnan().all()) == bool(rows[i]) and bool(torch.isfinite(o[0, 1].float()).all())
    ok()


def test_rows_of_no_sequence_are_neither_read_nor_written():
    """Rows before, between and behind the sequences hold NaN; so do the other sequences, one at a time."""
    lq, H, Hk, d = [70, 130, 200], 4, 2, 64
    total = 30 + sum(lq) + 100
    base = [normal(60 + i, total, h, d) for i, h in enumerate((H, Hk, Hk))]
    dout = normal(64, total, H, d)
    at = offsets(lq, 30)
    sp = spans(lq, 30)
    clean = st.st_attn_window(*base, 60, 3, at)
    cleang = st.st_attn_window_grad(*base, *clean, dout, 60, 3, at)
    for keep in range(3):
        a, b = sp[keep]
        live = torch.zeros(total, dtype=torch.bool, device="cuda")
        live[a:b] = True
        q, k, v, do = (torch.where(live[:, None, None], x, torch.full_like(x, math.nan)) for x in (*base, dout))
        out, lse = torch.full_like(base[0], 7.0), torch.full((total, H), 7.0, device="cuda")
        st.st_attn_window(q, k, v, 60, 3, at, out=out, lse=lse)
        assert torch.equal(out[a:b], clean[0][a:b]) and torch.equal(lse[a:b], clean[1][a:b])
        inside = torch.zeros_like(live)
        inside[sp[0][0] : sp[-1][1]] = True
        assert bool((out[~inside] == 7.0).all()) and bool((lse[~inside] == 7.0).all())
        grads = [torch.full_like(x, 7.0) for x in base]
        st.st_attn_window_grad(q, k, v, out, lse, do, 60, 3, at, dq=grads[0], dk=grads[1], dv=grads[2])
        for g, c in zip(grads, cleang):
            assert torch.equal(g[a:b], c[a:b])
            assert bool((g[~inside] == 7.0).all())
    ok()


@pytest.mark.parametrize("lq,lk,window,sinks", [
    ([300, 40], [900, 1000], 100, 4), ([300], [900], 100, 40), ([513, 3], [900, 700], 100, 130), ([300], [900], 128, 128), ([300, 200], [1400, 700], 33, 32),
    ([300, 1], [900, 500], 100, 0), ([2100], [2600], 70, 7), ([2100], [2600], 70, 200),
    ([300, 260, 140], [100, 0, 20], 50, 3), ([400, 300], [130, 171], 1000, 0)])
@pytest.mark.parametrize("d", [64, 128, 80])
def test_rows_of_a_sequence_that_no_pair_meets_may_hold_anything(lq, lk, window, sinks, d):
    """Keys and values between the first columns and the window of the first query, as a cache leaves them that keeps no more, and queries that
    stand before the first key: NaN there changes no bit, and their own gradients are 0."""
    H, Hk = 4, 2
    lk, q, k, v, qo, ko = window_inputs(63, lq, lk, H, Hk, d)
    do = normal(66, *q.shape)
    seen_k, seen_q = [], []
    for x, y in zip(lq, lk):
        see = ref.visible(x, y, window, sinks, "cuda")
        seen_k.append(see.any(0))
        seen_q.append(see.any(1))
    none_k, none_q = ~torch.cat(seen_k), ~torch.cat(seen_q)
    assert bool(none_k.any() | none_q.any())

    def run(q, k, v, do):
        out, lse = st.st_attn_window(q, k, v, window, sinks, qo, ko)
        grads = st.st_attn_window_grad(q, k, v, out, lse, do, window, sinks, qo, ko)
        ok()
        return out, lse, *grads

    want = run(q, k, v, do)
    for value in (math.nan, math.inf, -math.inf):
        for which in ((0,), (1,), (2,), (3,), (0, 1, 2, 3)):
            tables = [x.clone() for x in (q, k, v, do)]
            for i in which:
                tables[i][none_k if i in (1, 2) else none_q] = value
            got = run(*tables)
            assert all(torch.equal(x, y) for x, y in zip(got, want)), (value, which)
    for g, rows in ((want[0], none_q), (want[2], none_q), (want[3], none_k), (want[4], none_k)):
        assert bool((g[rows] == 0).all())


@pytest.mark.parametrize("bad", [[0, 50, 40, 100], [0, 50, 60, 101], [-1, 50, 60, 100], [0, 1 << 30, 5, 100]])
def test_bad_offsets_are_reported_and_touch_nothing_outside(bad):
    q, k, v = (normal(70 + i, 100, 2, 64) for i in range(3))
    at = torch.tensor(bad, dtype=torch.int32, device="cuda")
    good = offsets([50, 10, 40])
    out, lse = st.st_attn_window(q, k, v, 20, 2, at)
    assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS
    st.st_attn_window(q, k, v, 20, 2, good, at)
    assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS
    st.st_attn_window_grad(q, k, v, q, torch.zeros(100, 2, device="cuda"), q, 20, 2, at)
    assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS
    a = -torch.ones(2, device="cuda")
    st.st_attn_decay(q, k, v, a, at)
    assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS
    st.st_attn_decay_grad(q, k, v, a, q, at)
    assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS
    st.st_attn_window(q, k, v, 20, 2, good)
    ok()


def test_offsets_that_name_the_same_rows_again_stay_within_the_workspace():
    """More segments than the lengths can have: reported, and no state outside of its place (the guard bands see to that)."""
    n = 128 * 300
    q, k, v = (normal(75 + i, n, 1, 64) for i in range(3))
    at = torch.tensor([0, n, 0, n, 0, n, 0, n], dtype=torch.int32, device="cuda")
    a = -torch.ones(1, device="cuda")
    assert st.st_workspace_bytes(st.ST_OP_ATTN_DECAY, n, 1, 1, 64) > 256                 # one sequence of that length is cut
    st.st_attn_decay(q, k, v, a, at)
    assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS
    st.st_attn_decay_grad(q, k, v, a, q, at)
    assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS
    out, lse = st.st_attn_window(q, k, v, 20, 2, at)
    assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS
    st.st_attn_window_grad(q, k, v, out, lse, q, 20, 2, at)
    assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS


@pytest.mark.parametrize("d,dv", [(64, 96), (96, 64), (72, 64), (64, 72)])
def test_offsets_that_name_the_same_rows_again_with_states_of_two_widths(d, dv):
    """Rows of queries and of values in different numbers of 64 columns: the runs of the gradient have grids of different widths.  (What each
    block may reach is tested on the CPU.)"""
    n = 128 * 300
    q, k, v, do = normal(76, n, 1, d), normal(77, n, 1, d), normal(78, n, 1, dv), normal(79, n, 1, dv)
    at = torch.tensor([0, n, 0, n, 0, n, 0, n], dtype=torch.int32, device="cuda")
    a = -torch.ones(1, device="cuda")
    assert st.st_workspace_bytes(st.ST_OP_ATTN_DECAY_GRAD, n, 4, 1, max(d, dv)) > 256
    st.st_attn_decay(q, k, v, a, at)
    assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS
    st.st_attn_decay_grad(q, k, v, a, do, at)
    assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS
    # the same rows as one sequence, in segments as well
    one_at = offsets([n])
    got, want = st.st_attn_decay_grad(q, k, v, a, do, one_at), st.st_attn_decay_grad(q, k, v, a, do)
    ok()
    assert all(torch.equal(x, y) for x, y in zip(got[:3], want[:3]))


# --------------------------------------------------------------------------------- window: step

STEPS = [
    # lengths with the new token, heads, key heads, d, page, window, sinks
    ([1], 1, 1, 8, 1, 1, 0),
    ([1, 2, 16, 17, 33, 0], 4, 2, 64, 16, 10, 0),
    ([300, 1, 77], 8, 8, 128, 64, 1 << 33, 0),
    ([1000, 999, 31, 128], 8, 2, 128, 100, 250, 4),
    ([4000], 8, 1, 128, 7, 3000, 130),
    ([2500, 65], 32, 2, 80, 256, 700, 16),
    ([513] * 5, 6, 3, 96, 64, 64, 1000),
    ([20000], 4, 4, 32, 1000, 16000, 1),
    ([129, 5], 20, 1, 64, 32, 128, 2),
]


def cache_of(seed, lens, Hk, d, page, spare=2):
    used = [-(-n // page) for n in lens]
    pages = sum(used) + spare
    g = torch.Generator().manual_seed(seed)
    order = torch.randperm(pages, generator=g).to(torch.int32)
    table = torch.full((len(lens), max(1, max(used))), -1, dtype=torch.int32)
    for b, u in enumerate(used):
        table[b, :u] = order[sum(used[:b]) : sum(used[:b]) + u]
    return normal(seed, pages, page, Hk, d), normal(seed + 1, pages, page, Hk, d), table.cuda()


def gathered(pages, table, b, n):
    page = pages.shape[1]
    i = torch.arange(n, device="cuda")
    return pages[table[b, i // page].long(), i % page]


@pytest.mark.parametrize("lens,H,Hk,d,page,window,sinks", STEPS)
def test_window_step_against_the_definition(lens, H, Hk, d, page, window, sinks):
    kp, vp, table = cache_of(80, lens, Hk, d, page)
    q, k, v = normal(82, len(lens), H, d), normal(83, len(lens), Hk, d), normal(84, len(lens), Hk, d)
    # what lies behind a sequence's length, and pages of nobody, may hold anything
    live = torch.zeros(kp.shape[:2], dtype=torch.bool, device="cuda")
    for b, n in enumerate(lens):
        i = torch.arange(max(0, n - 1), device="cuda")
        live[table[b, i // page].long(), i % page] = True
    kp, vp = (torch.where(live[..., None, None], x, torch.full_like(x, math.nan)) for x in (kp, vp))
    before = kp.clone(), vp.clone()
    out = st.st_attn_window_step(q, k, v, kp, vp, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), window, sinks)
    ok()
    for b, n in enumerate(lens):
        if n == 0:
            assert bool((out[b] == 0).all())
            continue
        K, V = gathered(kp, table, b, n), gathered(vp, table, b, n)
        assert torch.equal(K[-1], k[b]) and torch.equal(V[-1], v[b])
        o, _, ot, _ = ref.window(q[b : b + 1], K, V, window, sinks)
        near(out[b : b + 1], o, ot, "out")
        last = table[b, (n - 1) // page].long(), (n - 1) % page
        before[0][last], before[1][last] = k[b], v[b]
    # nothing else in the cache moved
    for x, y in zip((kp, vp), before):
        assert torch.equal(x.view(torch.int16), y.view(torch.int16))


def test_step_takes_interleaved_and_head_major_caches():
    lens, H, Hk, d, page = [200, 90], 4, 2, 64, 32
    kp, vp, table = cache_of(90, lens, Hk, d, page)
    q, k, v = normal(92, 2, H, d), normal(93, 2, Hk, d), normal(94, 2, Hk, d)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    want = st.st_attn_window_step(q, k, v, kp.clone(), vp.clone(), table, n, 100, 4)
    both = torch.stack([kp, vp], 1)                                    # [pages, 2, page, Hk, d]
    assert torch.equal(st.st_attn_window_step(q, k, v, both[:, 0], both[:, 1], table, n, 100, 4), want)
    major = torch.stack([kp.transpose(1, 2), vp.transpose(1, 2)], 1)   # [pages, 2, Hk, page, d]
    assert torch.equal(st.st_attn_window_step(q, k, v, major[:, 0].transpose(1, 2), major[:, 1].transpose(1, 2), table, n, 100, 4), want)
    assert torch.equal(gathered(major[:, 1].transpose(1, 2), table, 0, 200)[-1], v[0])
    ok()


def test_step_leaves_out_bad_pages_and_reports_them():
    lens, H, Hk, d, page = [100, 64], 4, 2, 64, 16
    kp, vp, table = cache_of(95, lens, Hk, d, page)
    q, k, v = normal(97, 2, H, d), normal(98, 2, Hk, d), normal(99, 2, Hk, d)
    n = torch.tensor(lens, dtype=torch.int32, device="cuda")
    want = st.st_attn_window_step(q, k, v, kp, vp, table, n, 1000, 0)
    ok()
    for wrong in (-1, kp.shape[0], 1 << 30):
        bad = table.clone()
        bad[0, 2] = wrong
        out = st.st_attn_window_step(q, k, v, kp, vp, bad, n, 1000, 0)
        assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS
        assert torch.equal(out[1], want[1])
        keep = torch.cat([torch.arange(32), torch.arange(48, 100)]).cuda()
        o, _, ot, _ = ref.window(q[:1], gathered(kp, table, 0, 100)[keep], gathered(vp, table, 0, 100)[keep], 1000, 0)
        near(out[:1], o, ot, "out")
    long = torch.tensor([100, 7 * 16 + 1], dtype=torch.int32, device="cuda")
    st.st_attn_window_step(q, k, v, kp, vp, table.clamp(min=0), long, 1000, 0)
    assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS
    st.st_attn_window_step(q, k, v, kp, vp, table, torch.tensor([100, -5], dtype=torch.int32, device="cuda"), 1000, 0)
    assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS
    st.st_attn_window_step(q, k, v, kp, vp, table, n, 1000, 0)
    ok()


def test_step_reports_are_ordered_by_the_stream_and_not_by_time():
    """The status is cleared ahead of all blocks that may report, so that a report is neither lost nor has to wait: 3000 sequences with
    bad pages, seven turns of blocks, take no longer than with good ones, and one bad sequence is seen wherever it stands."""
    n, d, page = 3000, 64, 16
    q, k, v = normal(105, n, 1, d), normal(106, n, 1, d), normal(107, n, 1, d)
    kp, vp = normal(108, 3 * n, page, 1, d), normal(109, 3 * n, page, 1, d)
    lens = torch.full((n,), 40, dtype=torch.int32, device="cuda")
    good = torch.arange(3 * n, dtype=torch.int32, device="cuda").view(n, 3)
    bad = torch.full_like(good, -1)
    out, ws = torch.empty_like(q), torch.empty(256, dtype=torch.uint8, device="cuda")

    def timed(table):
        begin, end = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        begin.record()
        for _ in range(5):
            st.st_attn_window_step(q, k, v, kp, vp, table, lens, 100, 4, out=out, ws=ws)
        end.record()
        end.synchronize()
        return begin.elapsed_time(end)

    for _ in range(3):
        fine = timed(good)
        assert st.st_check_status(ws) == st.ST_OK
        wrong = timed(bad)
        assert st.st_check_status(ws) == st.ST_ERR_DEV_BOUNDS
    assert wrong < 5 * fine, (wrong, fine)
    for b in (0, 1, n // 2, n - 1):
        table = good.clone()
        table[b, 1] = -1
        for _ in range(5):
            st.st_attn_window_step(q, k, v, kp, vp, table, lens, 100, 4, out=out, ws=ws)
            assert st.st_check_status(ws) == st.ST_ERR_DEV_BOUNDS
        st.st_attn_window_step(q, k, v, kp, vp, good, lens, 100, 4, out=out, ws=ws)
        assert st.st_check_status(ws) == st.ST_OK


def test_step_on_a_cache_whose_offsets_pass_32_bits():
    page, Hk, d = 64, 8, 128
    pages = (1 << 31) // (page * Hk * d) + 40                          # elements: beyond 2^31
    kp, vp = torch.zeros(pages, page, Hk, d, dtype=BF16, device="cuda"), torch.zeros(pages, page, Hk, d, dtype=BF16, device="cuda")
    last = torch.arange(pages - 3, pages, device="cuda")
    kp[last], vp[last] = normal(100, 3, page, Hk, d), normal(101, 3, page, Hk, d)
    table = last.to(torch.int32)[None]
    q, k, v = normal(102, 1, 8, d), normal(103, 1, Hk, d), normal(104, 1, Hk, d)
    out = st.st_attn_window_step(q, k, v, kp, vp, table, torch.tensor([190], dtype=torch.int32, device="cuda"), 150, 4)
    o, _, ot, _ = ref.window(q, gathered(kp, table, 0, 190), gathered(vp, table, 0, 190), 150, 4)
    near(out, o, ot, "out")
    ok()


# -------------------------------------------------------------------------------------- decay

DECAYS = [
    # lengths, heads, d, dv, log decays, state
    ([1], 1, 8, 8, [-0.1], True),
    ([1, 2, 127, 128, 129, 0, 255, 257], 2, 64, 64, [-0.5, -0.004], True),
    ([700], 3, 128, 128, [-0.02, 0.0, -3.0], False),
    ([700, 0, 31], 2, 128, 128, [-0.02, -0.3], True),
    ([300, 77], 2, 80, 32, [-0.1, -0.001], True),
    ([130], 2, 32, 96, [-math.inf, -20.0], True),
    ([1100], 1, 64, 128, [-0.003], True),
    ([1100], 1, 128, 40, [-0.003], False),
    ([16] * 30, 2, 64, 64, [-0.05, -0.7], True),
    ([6000], 1, 128, 128, [-0.0005], True),
    ([5000, 0, 1, 900], 1, 64, 72, [-0.01], True),                 # in segments, one sequence without any token
]


def decay_inputs(seed, lens, H, d, dv, a, state):
    n = sum(lens)
    s = floats(seed + 3, len(lens), H, d, dv) if state else None
    return normal(seed, n, H, d), normal(seed + 1, n, H, d), normal(seed + 2, n, H, dv), torch.tensor(a, device="cuda"), s, offsets(lens)


def one(x, b):
    return None if x is None else x[b]


@pytest.mark.parametrize("lens,H,d,dv,a,state", DECAYS)
def test_decay_against_the_definition(lens, H, d, dv, a, state):
    q, k, v, a, s, at = decay_inputs(110, lens, H, d, dv, a, state)
    out, last = st.st_attn_decay(q, k, v, a, at, s)
    ok()
    for b, (x, y) in enumerate(spans(lens)):
        o, l, ot, lt = ref.decay(q[x:y], k[x:y], v[x:y], a, one(s, b))
        near(out[x:y], o, ot, "out")
        near(last[b], l, lt, "state")


@pytest.mark.parametrize("lens,H,d,dv,a,state", DECAYS)
def test_decay_gradient_against_the_definition(lens, H, d, dv, a, state):
    q, k, v, a, s, at = decay_inputs(120, lens, H, d, dv, a, state)
    dout = normal(124, *v.shape)
    dlast = floats(125, len(lens), H, d, dv) if state else None
    got = st.st_attn_decay_grad(q, k, v, a, dout, at, s, dlast)
    ok()
    assert (got[3] is None) == (not state)
    for b, (x, y) in enumerate(spans(lens)):
        want = ref.decay_grad(q[x:y], k[x:y], v[x:y], a, dout[x:y], one(s, b), one(dlast, b))
        for g, (w, tol), name in zip(got, want, ("dq", "dk", "dv")):
            near(g[x:y], w, tol, name)
        if state:
            near(got[3][b], *want[3], "dstate")


@pytest.mark.parametrize("d", [64, 128])
def test_decay_states_have_the_precision_of_fp32(d):
    """Sequences of two tokens: a state is the sum of two products, nothing cancels in the sum of their absolute values.  Off by at most
    2^-22 of a term (exp2f: two units) and 2^-23 (its rounded argument, |a2| < 1, and the product), 2^-25 (what three parts leave) and
    2^-23 for each of up to six summands on the tensor cores: below 2^-19."""
    H, n = 2, 40
    q, k, v, do = (normal(170 + i, 2 * n, H, d) for i in range(4))
    a = torch.tensor([-0.3, -0.6], device="cuda")
    at = offsets([2] * n)
    w = torch.exp(a.double())[None, :, None, None]
    zero = torch.zeros(n, H, d, d, device="cuda")
    _, last = st.st_attn_decay(q, k, v, a, at)
    dstate = st.st_attn_decay_grad(q, k, v, a, do, at, zero, None, scale=1.0)[3]
    ok()
    for got, x, y, first, second in ((last, k, v, w, 1.0), (dstate, q, do, w, w * w)):
        t = torch.einsum("nthd,nthe->nthde", x.double().view(n, 2, H, d), y.double().view(n, 2, H, d))
        want, size = first * t[:, 0] + second * t[:, 1], first * t[:, 0].abs() + second * t[:, 1].abs()
        assert bool(((got.double() - want).abs() <= size * 2.0 ** -19).all())


@pytest.mark.parametrize("lens,H", [([300, 0, 77], 2), ([5000, 0, 900], 1)])
def test_decay_state_in_place(lens, H):
    q, k, v, a, s, at = decay_inputs(180, lens, H, 64, 64, [-0.02] * H, True)
    want = st.st_attn_decay(q, k, v, a, at, s)
    same = s.clone()
    got = st.st_attn_decay(q, k, v, a, at, same, state_out=same)
    ok()
    assert got[1] is same and torch.equal(got[0], want[0]) and torch.equal(same, want[1])


def test_decay_gradient_against_differences():
    q, k, v, a, s, at = decay_inputs(130, [50], 2, 16, 24, [-0.2, -0.01], True)
    dout, dlast = normal(134, *v.shape), floats(135, 1, 2, 16, 24)
    got = st.st_attn_decay_grad(q, k, v, a, dout, None, s, dlast)
    want = ref.decay_grad(q, k, v, a, dout, s[0], dlast[0])

    def loss(q, k, v, s):
        out, last, _, _ = ref.decay(q, k, v, a, s[0])
        return float((out * dout.double()).sum() + (last * dlast[0].double()).sum())

    base = [x.double() for x in (q, k, v, s)]
    for i, g in enumerate(got):
        direction = floats(140 + i, *g.shape).double()
        x0, x1 = list(base), list(base)
        x0[i], x1[i] = base[i] - 1e-4 * direction, base[i] + 1e-4 * direction
        slope = (loss(*x1) - loss(*x0)) / 2e-4
        tol = want[i][1] if i < 3 else want[i][1][None]
        # the differences themselves: sums of some 10^5 terms of a few units in 64 bits over 2e-4
        assert abs(float((g.double() * direction).sum()) - slope) <= float((tol * direction.abs()).sum()) + 1e-5


def test_decay_takes_strided_tables_and_results_that_the_caller_has():
    n, H, d = 300, 2, 64
    qkv = normal(150, n, 3 * H, d)
    q, k, v = qkv.split(H, 1)
    a = torch.tensor([-0.1, -0.01], device="cuda")
    want = st.st_attn_decay(q.contiguous(), k.contiguous(), v.contiguous(), a)
    out, last = torch.empty_like(want[0]), torch.empty_like(want[1])
    got = st.st_attn_decay(q, k, v, a, out=out, state_out=last, scale=d ** -0.5)
    assert got[0] is out and got[1] is last and torch.equal(out, want[0]) and torch.equal(last, want[1])
    hq, hk, hv = (x.transpose(0, 1).contiguous().transpose(0, 1) for x in (q, k, v))
    assert torch.equal(st.st_attn_decay(hq, hk, hv, a)[0], out)
    dout = normal(151, n, H, d)
    x, y = st.st_attn_decay_grad(q, k, v, a, dout), st.st_attn_decay_grad(hq, hk, hv, a, dout)
    assert all(torch.equal(i, j) for i, j in zip(x[:3], y[:3]))
    # the last state may replace the first
    s = floats(152, 1, H, d, d)
    w = st.st_attn_decay(q, k, v, a, None, s.clone())
    got = st.st_attn_decay(q, k, v, a, None, s, state_out=s)
    assert got[1] is s and torch.equal(s, w[1]) and torch.equal(got[0], w[0])
    ok()


def test_decay_rows_of_no_sequence_are_neither_read_nor_written():
    lens, H, d = [70, 130, 200], 2, 64
    total = 30 + sum(lens) + 100
    base = [normal(160 + i, total, H, d) for i in range(4)]
    a, at, sp = torch.tensor([-0.1, -0.01], device="cuda"), offsets(lens, 30), spans(lens, 30)
    clean, last = st.st_attn_decay(*base[:3], a, at)
    cleang = st.st_attn_decay_grad(*base[:3], a, base[3], at)
    for keep in range(3):
        x, y = sp[keep]
        live = torch.zeros(total, dtype=torch.bool, device="cuda")
        live[x:y] = True
        q, k, v, do = (torch.where(live[:, None, None], t, torch.full_like(t, math.nan)) for t in base)
        out = torch.full_like(base[0], 7.0)
        _, l = st.st_attn_decay(q, k, v, a, at, out=out)
        inside = torch.zeros_like(live)
        inside[sp[0][0] : sp[-1][1]] = True
        assert torch.equal(out[x:y], clean[x:y]) and torch.equal(l[keep], last[keep]) and bool((out[~inside] == 7.0).all())
        grads = [torch.full_like(base[0], 7.0) for _ in range(3)]
        st.st_attn_decay_grad(q, k, v, a, do, at, dq=grads[0], dk=grads[1], dv=grads[2])
        for g, c in zip(grads, cleang):
            assert torch.equal(g[x:y], c[x:y]) and bool((g[~inside] == 7.0).all())
    ok()


@pytest.mark.parametrize("n,H,d,dv", [(1, 1, 8, 8), (3, 2, 64, 64), (70, 4, 128, 128), (5, 3, 80, 40), (300, 2, 32, 128)])
def test_decay_step_against_the_definition(n, H, d, dv):
    q, k, v, s = normal(170, n, H, d), normal(171, n, H, d), normal(172, n, H, dv), floats(173, n, H, d, dv)
    a = torch.linspace(-2.0, -0.001, H, device="cuda")
    state = s.clone()
    out = st.st_attn_decay_step(q, k, v, a, state)
    kept = s.double() * torch.exp(a.double()).view(-1, 1, 1)
    want = kept + k.double()[..., None] * v.double()[:, :, None]
    # two products and a sum in fp32, the decay's exponential within a few steps of it
    near(state, want, 2.0 ** -20 * (kept.abs() + (k.double()[..., None] * v.double()[:, :, None]).abs()), "state")
    o = torch.einsum("nhd,nhde->nhe", q.double(), want) * d ** -0.5
    near(out, o, ref.B * o.abs() + ref.F * torch.einsum("nhd,nhde->nhe", q.double().abs(), want.abs()) * d ** -0.5, "out")


# --------------------------------------------------------------------------- used together, and otherwise

def test_tables_whose_offsets_pass_32_bits():
    st.set_allocator(None)
    H, d, last = 64, 128, 300
    n = (1 << 31) // (H * d) + 500
    q = torch.zeros(n, H, d, dtype=BF16, device="cuda")
    k, v, do = (torch.zeros_like(q) for _ in range(3))
    for i, x in enumerate((q, k, v, do)):
        x[-last:] = normal(190 + i, last, H, d)
    at = torch.tensor([0, n - last, n], dtype=torch.int32, device="cuda")
    a = -torch.linspace(0.01, 1.0, H, device="cuda")
    tail = [x[-last:].clone() for x in (q, k, v, do)]
    out, lse = st.st_attn_window(q, k, v, 70, 3, at)
    want = st.st_attn_window(*tail[:3], 70, 3)
    assert torch.equal(out[-last:], want[0]) and torch.equal(lse[-last:], want[1])
    for g, w in zip(st.st_attn_window_grad(q, k, v, out, lse, do, 70, 3, at), st.st_attn_window_grad(*tail[:3], *want, tail[3], 70, 3)):
        assert torch.equal(g[-last:], w)
    out, s = st.st_attn_decay(q, k, v, a, at)
    want = st.st_attn_decay(*tail[:3], a)
    assert torch.equal(out[-last:], want[0]) and torch.equal(s[1:], want[1])
    for g, w in zip(st.st_attn_decay_grad(q, k, v, a, do, at)[:3], st.st_attn_decay_grad(*tail[:3], a, tail[3])[:3]):
        assert torch.equal(g[-last:], w)
    ok()


def test_a_prompt_and_its_steps_are_the_whole_sequence():
    """Two layers, one of each kind: a prompt of 150 tokens, then 20 single steps, against one pass over all 170."""
    n, p, H, Hk, d, window, sinks, page = 170, 150, 4, 2, 64, 48, 3, 16
    q, k, v = normal(180, n, H, d), normal(181, n, Hk, d), normal(182, n, Hk, d)
    whole, _ = st.st_attn_window(q, k, v, window, sinks)
    kp, vp = torch.full((12, page, Hk, d), math.nan, dtype=BF16, device="cuda"), torch.full((12, page, Hk, d), math.nan, dtype=BF16, device="cuda")
    table = torch.tensor([[7, 2, 9, 0, 4, 11, 1, 3, 10, 5, 8]], dtype=torch.int32, device="cuda")
    i = torch.arange(p, device="cuda")
    kp[table[0, i // page].long(), i % page], vp[table[0, i // page].long(), i % page] = k[:p], v[:p]
    rows = [st.st_attn_window(q[:p], k[:p], v[:p], window, sinks)[0]]
    for t in range(p, n):
        rows.append(st.st_attn_window_step(q[t : t + 1], k[t : t + 1], v[t : t + 1], kp, vp, table, torch.tensor([t + 1], dtype=torch.int32, device="cuda"), window, sinks))
    want, _, tol, _ = ref.window(q, k, v, window, sinks)
    near(torch.cat(rows), want, tol, "window")
    near(whole, want, tol, "window")
    a = torch.tensor([-0.3, -0.05, -0.01, 0.0], device="cuda")
    k4, v4 = whole, q
    whole2, last = st.st_attn_decay(q, k4, v4, a)
    out, state = st.st_attn_decay(q[:p], k4[:p], v4[:p], a)
    rows = [out]
    for t in range(p, n):
        rows.append(st.st_attn_decay_step(q[t : t + 1], k4[t : t + 1], v4[t : t + 1], a, state))
    want, wl, tol, lt = ref.decay(q, k4, v4, a, None)
    near(torch.cat(rows), want, tol, "decay")
    near(whole2, want, tol, "decay")
    near(state[0], wl, 2 * lt, "state")
    near(last[0], wl, lt, "state")
    ok()


@pytest.mark.parametrize("d,sinks", [(64, 3), (128, 40)])
def test_results_in_the_place_of_operands_that_are_not_read_again(d, sinks):
    """out over q or v, dq over out, dk and dv over k and v: the same bits as with results of their own."""
    st.set_allocator(None)
    lens, H = [700, 33, 0, 1300], 2
    q, k, v, do = (normal(300 + i, sum(lens), H, d) for i in range(4))
    at, a = offsets(lens), torch.tensor([-0.1, -0.01], device="cuda")
    out, lse = st.st_attn_window(q, k, v, 60, sinks, at)
    x = q.clone()
    assert st.st_attn_window(x, k, v, 60, sinks, at, out=x)[0] is x and torch.equal(x, out)
    want = st.st_attn_window_grad(q, k, v, out, lse, do, 60, sinks, at)
    for swap in (False, True):
        o, x, y = out.clone(), k.clone(), v.clone()
        dk, dv = (y, x) if swap else (x, y)
        got = st.st_attn_window_grad(q, x, y, o, lse, do, 60, sinks, at, dq=o, dk=dk, dv=dv)
        assert all(torch.equal(g, w) for g, w in zip(got, want))
    s = floats(305, len(lens), H, d, d)
    out, last = st.st_attn_decay(q, k, v, a, at, s)
    x, y = v.clone(), s.clone()
    st.st_attn_decay(q, k, x, a, at, y, out=x, state_out=y)
    assert torch.equal(x, out) and torch.equal(y, last)
    n = 4
    q1, k1, v1, s1 = q[:n].clone(), k[:n].clone(), v[:n].clone(), s.clone()
    out = st.st_attn_decay_step(q1, k1, v1, a, s1)
    x = v1.clone()
    assert torch.equal(st.st_attn_decay_step(q1, k1, x, a, s.clone(), out=x), out)
    kp, vp, table = cache_of(306, [200] * n, H, d, 16)
    ns = torch.tensor([200, 17, 1, 0], dtype=torch.int32, device="cuda")
    out = st.st_attn_window_step(q1, k1, v1, kp, vp, table, ns, 100, sinks)
    assert torch.equal(st.st_attn_window_step(q1, k1, v1, kp, vp, table, ns, 100, sinks, out=q1), out)
    with pytest.raises(st.StError) as e:
        st.st_attn_window(q, k, v, 60, sinks, at, out=k)
    assert e.value.status == st.ST_ERR_UNSUPPORTED
    with pytest.raises(st.StError) as e:
        st.st_attn_decay_grad(q, k, v, a, do, at, dv=v)
    assert e.value.status == st.ST_ERR_UNSUPPORTED
    ok()


def everything(seed, H=2, d=64, lens=(150, 40, 300)):
    """One call of each kind, as a list of (inputs to overwrite, function)."""
    lens = list(lens)
    n = sum(lens)
    q, k, v, do = (normal(seed + i, n, H, d) for i in range(4))
    a, at = -torch.rand(H, device="cuda"), offsets(lens)
    kp, vp, table = cache_of(seed + 5, lens, H, d, 16)
    ns = torch.tensor(lens, dtype=torch.int32, device="cuda")
    q1, k1, v1 = (normal(seed + 7 + i, len(lens), H, d) for i in range(3))
    s = floats(seed + 11, len(lens), H, d, d)

    def run():
        out, lse = st.st_attn_window(q, k, v, 60, 4, at)
        g = st.st_attn_window_grad(q, k, v, out, lse, do, 60, 4, at)
        o1 = st.st_attn_window_step(q1, k1, v1, kp, vp, table, ns, 100, 4)
        o2, last = st.st_attn_decay(q, k, v, a, at, s)
        g2 = st.st_attn_decay_grad(q, k, v, a, do, at, s, last)
        s1 = s.clone()
        o3 = st.st_attn_decay_step(q1, k1, v1, a, s1)
        return [out, lse, *g, o1, o2, last, *g2, o3, s1]
    return (q, k, v, do, a, q1, k1, v1, s), at, run


def test_the_same_bits_twenty_times():
    _, _, run = everything(200)
    first = [x.clone() for x in run()]
    for _ in range(20):
        assert all(torch.equal(x, y) for x, y in zip(run(), first))
    ok()


def test_captured_graphs_replay_with_new_inputs_and_offsets():
    """Two graphs, each with its own workspaces, replayed in turn; an eager call between them."""
    st.set_allocator(None)
    made = []
    side = torch.cuda.Stream()
    for seed in (210, 230):
        inputs, at, run = everything(seed)
        with torch.cuda.stream(side):
            run()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            results = run()
        made.append((inputs, at, run, graph, results))
    for step, lens in enumerate(([150, 40, 300], [1, 488, 1], [200, 0, 290])):
        for inputs, at, run, graph, results in made:
            for x in inputs:
                x.mul_(0.75 if step == 1 else 1.0)
            at.copy_(offsets(lens))
            want = [x.clone() for x in run()]
            for r in results:
                r.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(results, want))


def test_calls_on_two_streams_at_once():
    st.set_allocator(None)
    runs = [everything(seed, lens=(700, 20, 900))[2] for seed in (250, 270)]
    want = [[x.clone() for x in run()] for run in runs]
    streams = [torch.cuda.Stream() for _ in runs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(5):
        for i, (run, s) in enumerate(zip(runs, streams)):
            with torch.cuda.stream(s):
                got[i].append(run())
    torch.cuda.synchronize()
    for g, w in zip(got, want):
        for r in g:
            assert all(torch.equal(x, y) for x, y in zip(r, w))


def test_wrong_tensors_are_refused():
    q, k = normal(290, 10, 4, 64), normal(291, 10, 2, 64)
    a, at = torch.zeros(4, device="cuda"), offsets([4, 6])
    with pytest.raises(TypeError, match="k must be bfloat16"):
        st.st_attn_window(q, k.float(), k, 4)
    with pytest.raises(ValueError, match="shape mismatch"):
        st.st_attn_window(q, k, k[:9], 4)
    with pytest.raises(ValueError, match="last dimension of q"):
        st.st_attn_window(q.transpose(1, 2), k, k, 4)
    with pytest.raises(ValueError, match="k_offsets are needed"):
        st.st_attn_window(q, k[:9], k[:9], 4, 0, at)
    with pytest.raises(ValueError, match="same length"):
        st.st_attn_window(q, k, k, 4, 0, at, offsets([10]))
    with pytest.raises(TypeError, match="q_offsets must be int32"):
        st.st_attn_window(q, k, k, 4, 0, at.long())
    with pytest.raises(ValueError, match="out has the wrong shape"):
        st.st_attn_window(q, k, k, 4, out=q[:5].clone())
    with pytest.raises(st.StError) as e:
        st.st_attn_window(q, k, k, 0)
    assert e.value.status == st.ST_ERR_SHAPE
    with pytest.raises(st.StError) as e:
        st.st_attn_window(q[:0], k, k, 3)
    assert e.value.status == st.ST_ERR_SHAPE
    with pytest.raises(st.StError) as e:
        st.st_attn_decay(q, k, k, a)
    assert e.value.status == st.ST_ERR_SHAPE
    with pytest.raises(ValueError, match="state has the wrong shape"):
        st.st_attn_decay(q, q, q, a, at, torch.zeros(1, 4, 64, 64, device="cuda"))
    with pytest.raises(ValueError, match="dout has the wrong shape"):
        st.st_attn_decay_grad(q, q, q, a, q[:4], at)
    with pytest.raises(ValueError, match="k must be contiguous"):
        st.st_attn_decay_step(q, torch.cat([q, q], 2)[..., :64], q, a, torch.zeros(10, 4, 64, 64, device="cuda"))
    with pytest.raises(ValueError, match="same strides"):
        kp = normal(292, 3, 8, 2, 64)
        st.st_attn_window_step(q, k, k, kp, kp.transpose(1, 2).contiguous().transpose(1, 2), torch.zeros(10, 1, dtype=torch.int32, device="cuda"),
                               torch.ones(10, dtype=torch.int32, device="cuda"), 4)
