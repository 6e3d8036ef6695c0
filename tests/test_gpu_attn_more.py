"""Norms with rotation, a cache in cells and the steps over it on the GPU: every call against its definition in 64 bits
(attn_more_reference.py, which derives the tolerances), at the sizes, types and masks where tiles, pages and groups end."""
import ctypes

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

import attn_more_reference as ref
import paper_2211_10482_b200 as st
from test_gpu_attn import floats, near, normal, offsets, ok, spans
from test_gpu_parity import GuardAllocator

BF16 = torch.bfloat16
NAN = float("nan")


@pytest.fixture(autouse=True)
def guard_bands_and_device_status():
    """Nothing writes outside its buffers."""
    guard = GuardAllocator()
    st.set_allocator(guard)
    yield
    st.set_allocator(None)
    guard.check()


def ints(*values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------ rotation

ROTATIONS = [
    # tokens, heads, key heads, d, rot, interleaved, norm, weight type, factor
    (1, 1, 1, 8, 8, False, True, BF16, 1.0),
    (1, 1, 0, 8, 2, True, False, None, 1.0),
    (48, 32, 8, 128, 128, False, True, BF16, 1.0),
    (5, 3, 1, 64, 64, False, True, torch.float32, 1.3),
    (37, 4, 4, 64, 64, True, True, BF16, 0.7),
    (300, 2, 1, 80, 80, False, True, BF16, 1.0),
    (300, 2, 1, 80, 80, True, False, None, 1.0),
    (129, 6, 3, 80, 20, False, True, BF16, 1.0),         # a half of 10 columns
    (129, 6, 3, 80, 20, True, True, None, 1.0),
    (63, 3, 2, 96, 34, False, False, None, 1.1),
    (63, 3, 2, 96, 6, True, True, torch.float32, 1.0),
    (70, 5, 0, 128, 16, False, True, BF16, 1.0),
    (33, 130, 7, 32, 32, False, True, BF16, 1.0),        # more heads than a tile has rows
    (40, 1, 1, 128, 0, False, True, BF16, 1.0),          # norms alone
    (40, 1, 1, 128, 0, False, False, None, 1.0),         # neither: copies
    (6001, 16, 4, 128, 128, False, True, BF16, 1.0),     # four rows to a group of lanes
    (6001, 16, 4, 128, 64, True, False, None, 1.0),
    (4000, 7, 5, 72, 72, False, True, BF16, 1.0),
    (50000, 1, 0, 64, 64, False, True, None, 1.0),
]


def rotation_inputs(seed, n, H, Hk, d, rot, norm, wtype, far=1 << 20):
    q = normal(seed, n, H, d)
    k = normal(seed + 1, n, Hk, d) if Hk else None
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 2)
    positions = torch.randint(-far, far, (n,), generator=g, device="cuda", dtype=torch.int32)
    freq = st.st_rotary_frequencies(rot, 10000.0).cuda() if rot else None
    qw, kw = ((1 + 0.3 * floats(seed + 3 + i, d)).to(wtype) if norm and wtype is not None and (i == 0 or Hk) else None for i in range(2))
    return q, k, (positions, freq), (qw, kw, 1e-6 if norm else None)


@pytest.mark.parametrize("n,H,Hk,d,rot,inter,norm,wtype,factor", ROTATIONS)
def test_rotation_against_the_definition(n, H, Hk, d, rot, inter, norm, wtype, factor):
    q, k, at, (qw, kw, eps) = rotation_inputs(1, n, H, Hk, d, rot, norm, wtype)
    got = st.st_attn_rotate(q, k, *at, inter, qw, kw, eps, factor)
    assert (got[1] is None) == (Hk == 0)
    for g, x, w, name in zip(got, (q, k), (qw, kw), "qk"):
        if x is not None:
            want, tol = ref.rotate(x, w, *at, inter, eps, factor)
            near(g, want, tol, name)


@pytest.mark.parametrize("n,H,Hk,d,rot,inter,norm,wtype,factor", ROTATIONS)
def test_rotation_gradient_against_the_definition(n, H, Hk, d, rot, inter, norm, wtype, factor):
    q, k, at, (qw, kw, eps) = rotation_inputs(11, n, H, Hk, d, rot, norm, wtype)
    dq, dk = normal(17, *q.shape), normal(18, *k.shape) if Hk else None
    got = st.st_attn_rotate_grad(q, k, dq, dk, *at, inter, qw, kw, eps, factor)
    ok()
    for i, (x, w, dy) in enumerate(((q, qw, dq), (k, kw, dk))):
        if x is None:
            assert got[i] is None and got[2 + i] is None
            continue
        (dx, tol), weight = ref.rotate_grad(x, w, dy, *at, inter, eps, factor)
        near(got[i], dx, tol, "dx")
        if w is None:
            assert got[2 + i] is None
        else:
            assert got[2 + i].dtype == torch.float32
            near(got[2 + i], *weight, "dw")


@pytest.mark.parametrize("inter,rot", [(False, 16), (True, 16), (False, 12)])
def test_rotation_gradient_against_differences(inter, rot):
    n, H, Hk, d = 5, 2, 1, 16
    q, k, at, (qw, kw, eps) = rotation_inputs(21, n, H, Hk, d, rot, True, torch.float32, 50)
    dq, dk = normal(27, *q.shape), normal(28, *k.shape)
    grads = st.st_attn_rotate_grad(q, k, dq, dk, *at, inter, qw, kw, 0.01, 1.2)
    def loss(q, k, qw, kw):
        return sum(float((ref.rotate(x, w, *at, inter, 0.01, 1.2)[0] * dy.double()).sum()) for x, w, dy in ((q, qw, dq), (k, kw, dk)))
    base = [x.double() for x in (q, k, qw, kw)]
    tols = [ref.rotate_grad(x, w, dy, *at, inter, 0.01, 1.2) for x, w, dy in ((q, qw, dq), (k, kw, dk))]
    tols = [tols[0][0][1], tols[1][0][1], tols[0][1][1], tols[1][1][1]]
    h = 1e-5
    for i in range(4):
        flat = base[i].flatten()
        for e in range(0, flat.numel(), max(1, flat.numel() // 24)):
            ends = []
            for sign in (1, -1):
                moved = flat.clone()
                moved[e] += sign * h
                ends.append(loss(*[moved.view_as(base[i]) if j == i else b for j, b in enumerate(base)]))
            slope = (ends[0] - ends[1]) / (2 * h)
            # the difference's own error: h^2 times a third derivative of order 10^2, and 2^-52 of the loss over h
            assert abs(float(grads[i].flatten()[e]) - slope) <= float(tols[i].flatten()[e]) + 1e-6, (i, e)


def test_far_positions_keep_their_angles():
    """The angle is an exact product: positions up to the ends of 32 bits."""
    q, k, (_, freq), _ = rotation_inputs(31, 8, 2, 2, 64, 64, False, None)
    positions = ints(2**31 - 1, -(2**31), 1 << 24, (1 << 24) + 1, 999999937, -999999937, 0, 1)
    got = st.st_attn_rotate(q, k, positions, freq)
    for g, x in zip(got, (q, k)):
        near(g, *ref.rotate(x, None, positions, freq, False, None, 1.0), "far")


def test_rotation_takes_slices_of_a_projection_and_head_major_tables():
    n, H, Hk, d = 70, 4, 2, 64
    joined = normal(41, n, H + 2 * Hk, d)
    q, k, _ = joined.split([H, Hk, Hk], 1)
    _, _, at, (qw, kw, eps) = rotation_inputs(42, n, H, Hk, d, 64, True, BF16)
    want = st.st_attn_rotate(q.contiguous(), k.contiguous(), *at, False, qw, kw, eps)
    for a, b in ((q, k), (q.transpose(0, 1).contiguous().transpose(0, 1), k.transpose(0, 1).contiguous().transpose(0, 1))):
        got = st.st_attn_rotate(a, b, *at, False, qw, kw, eps)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    grads = [st.st_attn_rotate_grad(a, b, *want, *at, False, qw, kw, eps) for a, b in ((q, k), (q.contiguous(), k.contiguous()))]
    assert all(torch.equal(a, b) for a, b in zip(*grads))


@pytest.mark.parametrize("rot,inter", [(64, False), (64, True), (20, False)])
def test_rotation_in_place(rot, inter):
    q, k, at, (qw, kw, eps) = rotation_inputs(51, 200, 4, 2, 64, rot, True, BF16)
    want = st.st_attn_rotate(q, k, *at, inter, qw, kw, eps)
    dq, dk = normal(57, *q.shape), normal(58, *k.shape)
    grads = st.st_attn_rotate_grad(q, k, dq, dk, *at, inter, qw, kw, eps)
    a, b = dq.clone(), dk.clone()
    again = st.st_attn_rotate_grad(q, k, a, b, *at, inter, qw, kw, eps, dq=a, dk=b)
    assert again[0] is a and all(torch.equal(x, y) for x, y in zip(grads, again))
    a, b = q.clone(), k.clone()
    got = st.st_attn_rotate(a, b, *at, inter, qw, kw, eps, q_out=a, k_out=b)
    assert got[0] is a and torch.equal(a, want[0]) and torch.equal(b, want[1])


def test_norms_of_zero_and_of_large_rows():
    q, k, at, (qw, kw, eps) = rotation_inputs(61, 20, 2, 1, 64, 64, True, BF16)
    q[3] = 0
    q[4] *= 2.0 ** 50
    q[5] *= 2.0 ** -60
    got = st.st_attn_rotate(q, k, *at, False, qw, kw, eps)[0]
    near(got, *ref.rotate(q, qw, *at, False, eps, 1.0), "q")
    dq, dk = normal(67, *q.shape), normal(68, *k.shape)
    got = st.st_attn_rotate_grad(q, k, dq, dk, *at, False, qw, kw, eps)
    (dx, tol), (dw, wtol) = ref.rotate_grad(q, qw, dq, *at, False, eps, 1.0)
    near(got[0], dx, tol, "dx")
    near(got[2], dw, wtol, "dw")


def test_a_row_that_is_not_finite_stays_alone():
    q, k, at, (qw, kw, eps) = rotation_inputs(71, 40, 3, 2, 64, 64, True, BF16)
    clean = st.st_attn_rotate(q, k, *at, False, qw, kw, eps)
    q[7, 1, 5], k[9, 0, 2] = NAN, float("inf")
    got = st.st_attn_rotate(q, k, *at, False, qw, kw, eps)
    assert bool(torch.isnan(got[0][7, 1]).all())
    keep = torch.ones_like(q, dtype=torch.bool)
    keep[7, 1] = False
    assert torch.equal(got[0][keep], clean[0][keep])
    keep = torch.ones_like(k, dtype=torch.bool)
    keep[9, 0] = False
    assert torch.equal(got[1][keep], clean[1][keep])


def test_rotations_of_tables_whose_offsets_pass_32_bits():
    if torch.cuda.mem_get_info()[0] < 30 << 30:
        pytest.skip("needs 30 GB")
    st.set_allocator(None)
    n, H, d = 70000, 260, 128                            # 2.3 x 10^9 elements
    q = torch.empty((n, H, d), dtype=BF16, device="cuda")
    q[:50], q[-50:] = normal(81, 50, H, d), normal(82, 50, H, d)
    q[50:-50] = 1
    positions = torch.arange(n, dtype=torch.int32, device="cuda")
    freq = st.st_rotary_frequencies(128).cuda()
    got, _ = st.st_attn_rotate(q, None, positions, freq, False, None, None, 1e-6)
    for rows in (slice(0, 50), slice(n - 50, n)):
        near(got[rows], *ref.rotate(q[rows], None, positions[rows], freq, False, 1e-6, 1.0), "rows")
    dq = st.st_attn_rotate_grad(q, None, got, None, positions, freq, False, None, None, 1e-6)[0]
    for rows in (slice(0, 50), slice(n - 50, n)):
        near(dq[rows], *ref.rotate_grad(q[rows], None, got[rows], positions[rows], freq, False, 1e-6, 1.0)[0], "gradient")


# --------------------------------------------------------------------------------------- cells


class Cache:
    """Pages of keys and values in any order, of every type; `lens` tokens of each sequence get pages, the last `spare` pages nobody's."""

    def __init__(self, seed, lens, Hk, d, page, bits, spare=2, fill=True):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        self.bits, self.page, self.lens_host, self.d, self.Hk = bits, page, list(lens), d, Hk
        used = [-(-n // page) for n in lens]
        pages = sum(used) + spare
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        self.table = torch.full((len(lens), max(1, max(used))), -1, dtype=torch.int32, device="cuda")
        for b, (at, n) in enumerate(zip((sum(used[:b]) for b in range(len(lens))), used)):
            self.table[b, :n] = order[at : at + n]
        self.lens = ints(*lens)
        shape = (pages, page, Hk)
        if bits == 16:
            self.cells = [torch.full((*shape, d), NAN, dtype=BF16, device="cuda") for _ in range(2)]
            self.scales = [None, None]
        elif bits == 8:
            self.cells = [torch.full((*shape, d), 77, dtype=torch.int8, device="cuda") for _ in range(2)]
            self.scales = [torch.full(shape, NAN, device="cuda") for _ in range(2)]
        else:
            self.cells = [torch.full((*shape, d // 2), 0xA5, dtype=torch.uint8, device="cuda") for _ in range(2)]
            self.scales = [torch.full((*shape, -(-d // 32), 2), NAN, dtype=BF16, device="cuda") for _ in range(2)]
        if fill:
            for b, n in enumerate(lens):
                for i in range(2):
                    self.put(i, b, 0, (floats(seed + 10 * b + i, n, Hk, d) * (1 + 5 * (floats(seed + 5, d) > 1.5))).to(BF16))

    def where(self, b, first, n):
        s = torch.arange(first, first + n, device="cuda")
        return self.table[b].long()[s // self.page], s % self.page

    def put(self, i, b, first, x):
        at = self.where(b, first, x.shape[0])
        if self.bits == 16:
            self.cells[i][at] = x
        else:
            self.cells[i][at], self.scales[i][at] = ref.quantise(x, self.bits)

    def parts(self, i, b, at=None, n=None):
        at = self.where(b, 0, self.lens_host[b] if n is None else n) if at is None else at
        return ref.parts_of(self.cells[i][at], None if self.bits == 16 else self.scales[i][at], self.bits)

    def values(self, i, b, first, n):
        at = self.where(b, first, n)
        return ref.values(self.cells[i][at], None if self.bits == 16 else self.scales[i][at], self.bits)

    def pages(self):
        return self.cells[0], self.cells[1], self.table, self.lens

    def how(self):
        return dict(k_scales=self.scales[0], v_scales=self.scales[1])

    def copies(self):
        return [x.clone() for x in (*self.cells, *self.scales) if x is not None]

    def held(self):
        return [x for x in (*self.cells, *self.scales) if x is not None]


def same(a, b):
    return torch.equal(a, b) if not a.is_floating_point() else torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a.nan_to_num(), b.nan_to_num())


STORES = [
    # new tokens, tokens cached before, key heads, d, page
    ([1], [0], 1, 16, 1),
    ([57, 3, 0, 20], [300, 0, 7, 1], 8, 128, 16),
    ([1] * 37, [3] * 37, 2, 64, 16),
    ([130, 1, 64], [5, 200, 0], 3, 80, 100),
    ([33], [2], 40, 32, 7),                              # more rows of a token than a tile has
    ([5, 0, 0, 0, 9], [1, 0, 5, 0, 2], 1, 96, 256),
    ([1, 2] * 150, [0, 4] * 150, 1, 48, 4),
    ([700, 1], [0, 65], 4, 112, 64),
]


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("new,old,Hk,d,page", STORES)
def test_cache_written_and_read_back(new, old, Hk, d, page, bits):
    lens = [a + b for a, b in zip(new, old)]
    want, got = (Cache(1, lens, Hk, d, page, bits, fill=True) for _ in range(2))
    n = sum(new)
    k, v = normal(3, n + 2, Hk, d), normal(4, n + 2, Hk, d)[:, :, :]
    at = offsets(new, 1)                                 # the first and the last row are no sequence's
    for b, (lo, hi) in enumerate(spans(new, 1)):
        want.put(0, b, old[b], k[lo:hi])
        want.put(1, b, old[b], v[lo:hi])
    st.st_attn_cache_write(k, v, *got.pages(), at, **got.how())
    ok()
    for a, b in zip(got.held(), want.held()):
        assert same(a, b)
    # all of it, and the last tokens of every sequence
    for counts in (lens, [min(x, 3) for x in lens]):
        rows = sum(counts) + 2
        ko, vo = (torch.full((rows, Hk, d), 5.0, dtype=BF16, device="cuda") for _ in range(2))
        out = st.st_attn_cache_read(*got.pages(), offsets(counts, 1), rows, k=ko, v=vo, **got.how())
        ok()
        assert out[0] is ko
        for b, (lo, hi) in enumerate(spans(counts, 1)):
            for i in range(2):
                assert same(out[i][lo:hi], want.values(i, b, lens[b] - counts[b], counts[b]))
        for x in out:
            assert bool((x[0] == 5).all()) and bool((x[-1] == 5).all())


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_cache_rows_without_offsets(bits):
    """A row for every sequence, or one sequence of all rows."""
    for lens, rows in (([5, 1, 17, 200], 4), ([90], 31)):
        c, want = (Cache(11, lens, 2, 64, 16, bits) for _ in range(2))
        k, v = normal(12, rows, 2, 64), normal(13, rows, 2, 64)
        counts = [1] * 4 if rows == 4 else [31]
        for b, (lo, hi) in enumerate(spans(counts)):
            want.put(0, b, lens[b] - counts[b], k[lo:hi])
            want.put(1, b, lens[b] - counts[b], v[lo:hi])
        st.st_attn_cache_write(k, v, *c.pages(), **c.how())
        ok()
        assert all(same(a, b) for a, b in zip(c.held(), want.held()))
        got = st.st_attn_cache_read(*c.pages(), None, rows, **c.how())
        ok()
        for b, (lo, hi) in enumerate(spans(counts)):
            assert same(got[0][lo:hi], want.values(0, b, lens[b] - counts[b], counts[b]))


@pytest.mark.parametrize("bits", [8, 4])
def test_cells_of_rows_at_the_ends_of_the_numbers(bits):
    d = 64
    rows = normal(21, 16, 1, d)
    rows[0] = 0
    rows[1] = -3.0
    rows[2, 0, 5] = NAN
    rows[3, 0, 40] = float("inf")
    rows[4, 0, 0] = -float("inf")
    rows[5] *= 2.0 ** -120
    rows[6] *= 2.0 ** 120
    rows[7] = torch.finfo(BF16).max
    rows[8, 0, ::2], rows[8, 0, 1::2] = torch.finfo(BF16).max, -torch.finfo(BF16).max
    rows[9] = 2.0 ** -133                                # below the normal numbers
    rows[10, 0, :32] = 2.0 ** -100 * 15
    rows[11] = torch.arange(d, device="cuda") - 32.0     # borders between cells
    rows[12] = torch.arange(d, device="cuda") % 2 + 100.0
    c, want = (Cache(22, [16], 1, d, 8, bits, fill=False) for _ in range(2))
    for i in range(2):
        want.put(i, 0, 0, rows)
    st.st_attn_cache_write(rows, rows, *c.pages(), **c.how())
    ok()
    assert all(same(a, b) for a, b in zip(c.held(), want.held()))
    got = st.st_attn_cache_read(*c.pages(), None, 16, **c.how())[0]
    assert same(got, want.values(0, 0, 0, 16))
    assert bool(torch.isnan(got[2, 0, :32]).all()) and bool((got[0] == 0).all())
    assert bool(torch.isnan(got[2]).all()) == (bits == 8)


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_cache_takes_strided_rows_and_interleaved_pages(bits):
    lens, Hk, d, page = [30, 9], 2, 64, 16
    c = Cache(31, lens, Hk, d, page, bits)
    joined = normal(32, sum(lens), 3 * Hk, d)
    k, v = joined[:, Hk : 2 * Hk], joined[:, 2 * Hk :]
    st.st_attn_cache_write(k.contiguous(), v.contiguous(), *c.pages(), offsets(lens), **c.how())
    want = c.copies()
    # keys and values of a page side by side, heads before tokens
    cells = torch.zeros((c.cells[0].shape[0], 2, Hk, page, c.cells[0].shape[3]), dtype=c.cells[0].dtype, device="cuda")
    pages = [cells[:, i].transpose(1, 2) for i in range(2)]
    scales = [None, None]
    if bits != 16:
        s = torch.zeros((cells.shape[0], 2, Hk, page, *c.scales[0].shape[3:]), dtype=c.scales[0].dtype, device="cuda")
        scales = [s[:, i].transpose(1, 2) for i in range(2)]
    st.st_attn_cache_write(k, v, *pages, c.table, c.lens, offsets(lens), *scales)
    ok()
    for b, n in enumerate(lens):
        at = c.where(b, 0, n)
        for i, x in enumerate((*pages, *scales)):
            if x is not None:
                assert same(x[at], want[i][at])
    got = st.st_attn_cache_read(*pages, c.table, c.lens, offsets(lens), sum(lens), *scales)
    for i in range(2):
        for b, (lo, hi) in enumerate(spans(lens)):
            assert same(got[i][lo:hi], c.values(i, b, 0, lens[b]))
    q = normal(33, 2, 4, d)
    a = st.st_attn_cache_step(q, *pages, c.table, c.lens, 100, 0, *scales)
    ok()
    assert torch.equal(a, st.st_attn_cache_step(q, *c.pages(), 100, 0, **c.how()))


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_cache_leaves_out_tokens_without_a_place_and_reports_them(bits):
    lens, Hk, d, page = [40, 20], 1, 32, 8
    for what in ("page behind", "page negative", "length beyond", "more rows than tokens", "length negative"):
        c, want = (Cache(41, lens, Hk, d, page, bits) for _ in range(2))
        k, v = normal(42, 24, Hk, d), normal(43, 24, Hk, d)
        out = set()                                      # rows without a place
        if what.startswith("page"):
            c.table[0, 4] = c.cells[0].shape[0] if what == "page behind" else -5
            out = {8 + e for e in range(8)}              # tokens 32..39 of 24..39
        elif what == "length beyond":
            c.lens[0] = 48                               # five pages of eight in a row
            out = {8 + e for e in range(8)}
        elif what == "more rows than tokens":
            c.lens[0] = 10
            out = set(range(6))
        else:
            c.lens[0] = -3
            out = set(range(16))
        told = int(c.lens[0])
        for r in range(16):
            if r not in out:
                want.put(0, 0, told - 16 + r, k[r : r + 1])
                want.put(1, 0, told - 16 + r, v[r : r + 1])
        want.put(0, 1, 12, k[16:])
        want.put(1, 1, 12, v[16:])
        st.st_attn_cache_write(k, v, *c.pages(), offsets([16, 8]), **c.how())
        assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS, what
        assert all(same(a, b) for a, b in zip(c.held(), want.held())), what
        got = st.st_attn_cache_read(*c.pages(), offsets([16, 8]), 24, **c.how())
        assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS, what
        for r in range(16):
            if r in out:
                assert bool((got[0][r] == 0).all()) and bool((got[1][r] == 0).all()), what
            else:
                assert same(got[0][r : r + 1], want.values(0, 0, told - 16 + r, 1)), what
        assert same(got[1][16:], want.values(1, 1, 12, 8)), what
    c = Cache(41, lens, Hk, d, page, bits)
    for bad in ([0, 30, 24], [0, 5, 25], [-1, 5, 24]):
        st.st_attn_cache_write(normal(44, 24, Hk, d), normal(45, 24, Hk, d), *c.pages(), ints(*bad), **c.how())
        assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_cache_whose_offsets_pass_32_bits(bits):
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    st.set_allocator(None)
    page, Hk, d = 128, 8, 128
    pages = (1 << 31) // (page * Hk * (d if bits != 4 else d // 2)) + 40          # more than 2^31 bytes or elements
    c = Cache(51, [page * 2 + 3], Hk, d, page, bits, spare=1)
    cells = [torch.empty((pages, page, Hk, c.cells[0].shape[3]), dtype=c.cells[0].dtype, device="cuda") for _ in range(2)]
    scales = [None if s is None else torch.empty((pages, *s.shape[1:]), dtype=s.dtype, device="cuda") for s in c.scales]
    table = ints(pages - 1, 3, pages - 7).view(1, 3)
    k, v = normal(52, 259, Hk, d), normal(53, 259, Hk, d)
    st.st_attn_cache_write(k, v, *cells, table, c.lens, None, *scales)
    st.st_attn_cache_write(k, v, *c.pages(), None, **c.how())
    ok()
    for a, b in zip(st.st_attn_cache_read(*cells, table, c.lens, None, 259, *scales), st.st_attn_cache_read(*c.pages(), None, 259, **c.how())):
        assert same(a, b)
    q = normal(54, 1, 16, d)
    assert torch.equal(st.st_attn_cache_step(q, *cells, table, c.lens, 1 << 30, 0, *scales), st.st_attn_cache_step(q, *c.pages(), 1 << 30, 0, **c.how()))
    if bits == 16:
        prefix, own = ints(pages - 1, 3).view(1, 2), ints(pages - 7).view(1, 1)
        got = st.st_attn_shared_step(q, *cells, prefix, ints(256), own, ints(3))
        o, tol = ref.attend(q[0], c.parts(0, 0), c.parts(1, 0))
        near(got[0], o, tol, "shared")
    ok()


# --------------------------------------------------------------------------------------- steps

STEPS = [
    # lengths, heads, key heads, d, page, window, sinks
    ([1], 1, 1, 16, 1, 1, 0),
    ([1, 2, 15, 16, 17, 31, 32, 33, 0, 64, 65], 4, 2, 64, 16, 1 << 30, 0),
    ([500, 3, 129], 8, 2, 128, 16, 100, 4),
    ([777], 17, 1, 128, 100, 300, 130),
    ([300, 41], 34, 2, 64, 7, 1 << 40, 0),
    ([90, 1000, 10], 6, 3, 80, 64, 65, 1),
    ([256, 257, 4], 3, 3, 96, 256, 256, 300),
    ([400], 5, 1, 32, 3, 1, 5),
    ([3001], 32, 8, 128, 16, 2000, 16),
    ([9000], 2, 1, 64, 64, 1 << 30, 0),
    ([40] * 30 + [0, 700], 8, 8, 48, 16, 200, 3),
]


def check_step(got, c, q, window, sinks, scale=None):
    for b, n in enumerate(c.lens_host):
        lo = max(0, n - window)
        first = min(sinks, lo)
        s = torch.cat([torch.arange(first, device="cuda"), torch.arange(lo, n, device="cuda")])
        at = (c.table[b].long()[s // c.page], s % c.page)
        o, tol = ref.attend(q[b], c.parts(0, b, at), c.parts(1, b, at), scale)
        near(got[b], o, tol, "out of sequence %d" % b)


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("lens,H,Hk,d,page,window,sinks", STEPS)
def test_cache_step_against_the_definition(lens, H, Hk, d, page, window, sinks, bits):
    """Everything that is not visible is NaN, and so are pages of nobody."""
    c = Cache(61, lens, Hk, d, page, bits)
    for b, n in enumerate(lens):
        for s in range(min(sinks, n), max(0, n - window))[:50]:
            at = c.where(b, s, 1)
            for x in c.held():
                if x.is_floating_point():
                    x[at] = NAN
    q = normal(62, len(lens), H, d)
    got = st.st_attn_cache_step(q, *c.pages(), window, sinks, **c.how())
    ok()
    check_step(got, c, q, window, sinks)


def test_cache_step_of_plain_pages_is_the_window_step():
    lens, H, Hk, d = [300, 1, 77], 8, 2, 128
    c = Cache(71, lens, Hk, d, 16, 16)
    q = normal(72, 3, H, d)
    k, v = (torch.stack([c.cells[i][c.where(b, n - 1, 1)][0] for b, n in enumerate(lens)]) for i in range(2))
    a = st.st_attn_cache_step(q, *c.pages(), 64, 4)
    b = st.st_attn_window_step(q, k, v, *c.pages(), 64, 4)
    # both are rounded twice
    assert float((a.double() - b.double()).abs().max()) <= 4 * ref.B * float(c.cells[1][c.cells[1].isfinite()].abs().max())


@pytest.mark.parametrize("bits", [8, 4])
def test_cache_step_with_strided_queries_other_scale_and_in_place(bits):
    c = Cache(81, [100, 260, 31], 2, 64, 16, bits)
    joined = normal(82, 3, 12, 64)
    q = joined[:, :8]
    got = st.st_attn_cache_step(q, *c.pages(), 200, 2, scale=0.3, **c.how())
    ok()
    check_step(got, c, q, 200, 2, 0.3)
    own = q.contiguous()
    assert st.st_attn_cache_step(own, *c.pages(), 200, 2, scale=0.3, out=own, **c.how()) is own
    assert torch.equal(own, got)


@pytest.mark.parametrize("bits", [8, 4])
def test_cache_step_pages_that_are_not_whole_pieces_of_16_bytes(bits):
    """Rows 8 bytes off 16-byte boundaries."""
    lens, H, Hk, d = [70, 200, 3], 4, 2, 128
    c = Cache(91, lens, Hk, d, 16, bits)
    wide = [torch.zeros((*x.shape[:3], x.shape[3] + 8), dtype=x.dtype, device="cuda") for x in c.cells]
    pages = [w[..., :-8] for w in wide]
    for a, b in zip(pages, c.cells):
        a.copy_(b)
    q = normal(92, 3, H, d)
    got = st.st_attn_cache_step(q, *pages, c.table, c.lens, 150, 3, **c.how())
    ok()
    check_step(got, c, q, 150, 3)


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_cache_step_large_values_do_not_overflow(bits):
    c = Cache(101, [200], 1, 64, 16, bits, fill=False)
    k, v = normal(102, 200, 1, 64), normal(103, 200, 1, 64)
    c.put(0, 0, 0, (k.float() * 300).to(BF16))
    c.put(1, 0, 0, (v.float() * 1e30).to(BF16))
    q = (normal(104, 1, 4, 64).float() * 20).to(BF16)
    got = st.st_attn_cache_step(q, *c.pages(), 1 << 30, **c.how())
    check_step(got, c, q, 1 << 30, 0)


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_cache_step_values_that_are_not_finite_are_seen(bits):
    for what in (0, 1):
        c = Cache(111, [50, 50], 1, 32, 16, bits)
        clean = st.st_attn_cache_step(normal(112, 2, 2, 32), *c.pages(), 20, 3, **c.how())
        x = normal(113, 1, 1, 32)
        x[..., 3] = NAN
        c.put(what, 0, 10, x)                            # hidden
        assert torch.equal(st.st_attn_cache_step(normal(112, 2, 2, 32), *c.pages(), 20, 3, **c.how()), clean)
        c.put(what, 0, 40, x)
        got = st.st_attn_cache_step(normal(112, 2, 2, 32), *c.pages(), 20, 3, **c.how())
        hit = got[0].isnan()
        assert bool(hit.all()) if what == 0 or bits != 16 else bool(hit[:, 3].all())
        assert torch.equal(got[1], clean[1])
    if bits == 16:
        c = Cache(114, [20, 20], 1, 32, 16, 16)
        q = torch.ones((2, 2, 32), dtype=BF16, device="cuda")
        c.put(0, 0, 0, torch.full((20, 1, 32), -float("inf"), dtype=BF16, device="cuda"))
        got = st.st_attn_cache_step(q, *c.pages(), 100)
        assert bool(got[0].isnan().all()) and bool(got[1].isfinite().all())       # all scores -inf


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_cache_step_leaves_out_bad_pages_and_reports_them(bits):
    lens, H, Hk, d, page = [100, 40, 16], 4, 2, 64, 16
    c = Cache(121, lens, Hk, d, page, bits)
    q = normal(122, 3, H, d)
    full = st.st_attn_cache_step(q, *c.pages(), 1 << 30, **c.how())
    ok()
    table = c.table.clone()
    table[0, 2], table[2, 0] = c.cells[0].shape[0], -9
    got = st.st_attn_cache_step(q, *c.cells, table, c.lens, 1 << 30, **c.how())
    assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS
    s = torch.cat([torch.arange(0, 32, device="cuda"), torch.arange(48, 100, device="cuda")])
    at = (c.table[0].long()[s // page], s % page)
    o, tol = ref.attend(q[0], c.parts(0, 0, at), c.parts(1, 0, at))
    near(got[0], o, tol, "what is left")
    assert torch.equal(got[1], full[1]) and bool((got[2] == 0).all())
    # a page that no visible token lies in is not looked at
    got = st.st_attn_cache_step(q[:1], *c.cells, table[:1].contiguous(), c.lens[:1], 30, **c.how())
    ok()
    # lengths that the table's rows do not hold are cut, negative ones are none
    c.lens[0], c.lens[1] = 10000, -4
    c.table[0, -1] = c.table[0, 0]
    got = st.st_attn_cache_step(q, *c.pages(), 1, **c.how())
    assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS
    at = (c.table[0].long()[-1:], torch.tensor([page - 1], device="cuda"))
    o, tol = ref.attend(q[0], c.parts(0, 0, at), c.parts(1, 0, at))
    if bits == 16 or bool(c.scales[0][at].isfinite().all()):
        near(got[0], o, tol, "cut")
    assert bool((got[1] == 0).all())


# -------------------------------------------------------------------------------------- shared

SHARED = [
    # sequences of every group, prefixes, own lengths (cycled), heads, key heads, d, page
    ([1], [1], [0], 1, 1, 8, 1),
    ([8], [4001], [120, 1, 0, 33], 8, 2, 128, 16),
    ([3, 5], [127, 129], [7, 40], 4, 2, 64, 16),
    ([2, 0, 1, 4], [300, 50, 0, 128], [0, 1, 17], 6, 3, 80, 100),
    ([40], [1000], [5, 200], 8, 1, 128, 64),             # 320 rows: two tiles, the second in part
    ([33], [700], [3], 8, 2, 96, 256),                   # 132 rows
    ([70], [257], [1, 2], 17, 1, 64, 7),                 # 15 sequences to a tile
    ([1, 1, 1, 1, 1], [2000, 3, 1500, 128, 999], [50], 4, 1, 128, 32),
    ([20, 30], [5000, 100], [10], 16, 4, 128, 16),
    ([1], [300], [20], 200, 1, 32, 16),                  # 200 heads to a key head
    ([150], [513], [0, 9], 2, 2, 32, 16),
]


def shared_inputs(seed, groups, prefix, own, H, Hk, d, page):
    n = sum(groups)
    lens = [own[i % len(own)] for i in range(n)]
    c = Cache(seed, prefix + lens, Hk, d, page, 16)
    G = len(groups)
    args = (c.table[:G].contiguous(), c.lens[:G].contiguous(), c.table[G:].contiguous(), c.lens[G:].contiguous(), offsets(groups))
    return c, normal(seed + 1, n, H, d), args, lens


def check_shared(got, c, q, groups, prefix, lens):
    G = len(groups)
    for g, (a, b) in enumerate(spans(groups)):
        for n in range(a, b):
            (k0, k1), (v0, v1) = (tuple(torch.cat(x) for x in zip(c.parts(i, g), c.parts(i, G + n))) for i in range(2))
            o, tol = ref.attend(q[n], (k0, k1), (v0, v1))
            near(got[n], o, tol, "out of sequence %d" % n)


@pytest.mark.parametrize("groups,prefix,own,H,Hk,d,page", SHARED)
def test_shared_step_against_the_definition(groups, prefix, own, H, Hk, d, page):
    c, q, args, lens = shared_inputs(1, groups, prefix, own, H, Hk, d, page)
    got = st.st_attn_shared_step(q, *c.cells, *args)
    ok()
    check_shared(got, c, q, groups, prefix, lens)


def test_shared_step_with_one_group_without_offsets_and_strided_queries():
    c, _, args, lens = shared_inputs(11, [6], [500], [3, 0], 8, 2, 64, 16)
    q = normal(12, 6, 12, 64)[:, 2:10]
    got = st.st_attn_shared_step(q, *c.cells, *args[:4])
    ok()
    check_shared(got, c, q, [6], [500], lens)
    own = q.contiguous()
    assert st.st_attn_shared_step(own, *c.cells, *args, out=own) is own and torch.equal(own, got)


def test_shared_step_of_sequences_in_no_group_is_the_cache_step():
    c, q, args, lens = shared_inputs(21, [2, 3], [200, 300], [30, 4, 100], 4, 2, 64, 16)
    alone = st.st_attn_cache_step(q, *c.cells, args[2], args[3], 1 << 30)
    got = st.st_attn_shared_step(q, *c.cells, *args[:4], ints(1, 1, 3))
    ok()
    assert torch.equal(got[0], alone[0]) and torch.equal(got[3:], alone[3:])
    (k0, k1), (v0, v1) = (tuple(torch.cat(x) for x in zip(c.parts(i, 1), c.parts(i, 3))) for i in range(2))
    o, tol = ref.attend(q[1], (k0, k1), (v0, v1))
    near(got[1], o, tol, "the second group's first")


def test_shared_step_large_scores_and_values_that_are_not_finite():
    c, q, args, lens = shared_inputs(31, [5], [600], [10], 4, 1, 64, 16)
    q = (q.float() * 50).to(BF16)
    got = st.st_attn_shared_step(q, *c.cells, *args)
    ok()
    check_shared(got, c, q, [5], [600], lens)
    x = normal(32, 1, 1, 64)
    x[..., 7] = NAN
    c.put(0, 0, 333, x)
    assert bool(st.st_attn_shared_step(q, *c.cells, *args).isnan().all())
    c, q, args, lens = shared_inputs(31, [5], [600], [10], 4, 1, 64, 16)
    c.put(0, 2, 4, x)                                    # a token of its own: the others do not see it
    got = st.st_attn_shared_step(q, *c.cells, *args)
    assert bool(got[1].isnan().all()) and bool(got[[0, 2, 3, 4]].isfinite().all())
    # scores of the prefix all -inf: the own tokens count alone; without any, NaN
    c, q, args, lens = shared_inputs(31, [5], [600], [10, 0], 4, 1, 64, 16)
    q = q.abs()
    c.put(0, 0, 0, torch.full((600, 1, 64), -float("inf"), dtype=BF16, device="cuda"))
    got = st.st_attn_shared_step(q, *c.cells, *args)
    for n, own in enumerate(lens):
        if own:
            o, tol = ref.attend(q[n], c.parts(0, 1 + n), c.parts(1, 1 + n))
            near(got[n], o, tol, "own tokens")
        else:
            assert bool(got[n].isnan().all())
    ok()


def test_shared_step_leaves_out_bad_pages_and_reports_them():
    groups, prefix = [4, 2], [400, 90]
    c, q, (pt, pl, t, l, go), lens = shared_inputs(41, groups, prefix, [20, 0], 4, 2, 64, 16)
    bad = pt.clone()
    bad[0, 3], bad[1] = 1 << 29, -1
    got = st.st_attn_shared_step(q, *c.cells, bad, pl, t, l, go)
    assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS
    s = torch.cat([torch.arange(48, device="cuda"), torch.arange(64, 400, device="cuda")])
    at = (c.table[0].long()[s // 16], s % 16)
    for n in range(4):
        (k0, k1), (v0, v1) = (tuple(torch.cat(x) for x in zip(c.parts(i, 0, at), c.parts(i, 2 + n))) for i in range(2))
        near(got[n], *ref.attend(q[n], (k0, k1), (v0, v1)), "what is left")
    near(got[4], *ref.attend(q[4], c.parts(0, 6), c.parts(1, 6)), "own tokens alone")
    assert bool((got[5] == 0).all())
    for bad_offsets, bad_lens in (([0, 5, 4], pl), ([0, 4, 7], pl), ([-1, 4, 6], pl), ([0, 4, 6], ints(-2, 90)), ([0, 4, 6], ints(400, 1 << 30))):
        st.st_attn_shared_step(q, *c.cells, pt, bad_lens, t, l, ints(*bad_offsets))
        assert st.st_check_status() == st.ST_ERR_DEV_BOUNDS


# ----------------------------------------------------------------------------------- together


def test_a_prompt_then_steps_over_the_cache_are_attention_over_the_whole():
    """Projections of a prompt are normed and turned, stored, read back for st_attn_window, and tokens follow one by one."""
    H, Hk, d, page, n, steps = 4, 2, 64, 16, 50, 3
    q, k, v = normal(1, n + steps, H, d), normal(2, n + steps, Hk, d), normal(3, n + steps, Hk, d)
    positions, freq = torch.arange(n + steps, dtype=torch.int32, device="cuda"), st.st_rotary_frequencies(d).cuda()
    w = (1 + 0.1 * floats(4, d)).to(BF16)
    how = (False, w, w, 1e-6)
    c = Cache(5, [n + steps], Hk, d, page, 16, fill=False)
    c.lens.fill_(n)
    qr, kr = st.st_attn_rotate(q[:n], k[:n], positions[:n], freq, *how)
    st.st_attn_cache_write(kr, v[:n], *c.pages())
    kc, vc = st.st_attn_cache_read(*c.pages(), None, n)
    assert torch.equal(kc, kr) and torch.equal(vc, v[:n])
    out = [st.st_attn_window(qr, kc, vc, 1 << 30)[0]]
    for i in range(n, n + steps):
        c.lens.fill_(i + 1)
        qr, kr = st.st_attn_rotate(q[i : i + 1], k[i : i + 1], positions[i : i + 1], freq, *how)
        st.st_attn_cache_write(kr, v[i : i + 1], *c.pages())
        a = st.st_attn_cache_step(qr, *c.pages(), 1 << 30)
        b = st.st_attn_shared_step(qr, *c.cells, c.table[:, :2].contiguous(), ints(32), c.table[:, 2:].contiguous(), c.lens - 32)
        assert float((a.double() - b.double()).abs().max()) <= 4 * ref.B * float(v.abs().max())
        out.append(a)
    ok()
    qa, ka = st.st_attn_rotate(q, k, positions, freq, *how)
    for i in range(n + steps):
        o, tol = ref.attend(qa[i], *((torch.zeros_like(x[: i + 1], dtype=torch.float64), x[: i + 1].double()) for x in (ka, v)))
        near(torch.cat(out)[i], o, tol, "token %d" % i)


def test_training_through_norm_rotation_and_attention_against_differences():
    H, Hk, d, n = 2, 1, 16, 12
    q, k, v, do = normal(11, n, H, d), normal(12, n, Hk, d), normal(13, n, Hk, d), normal(14, n, H, d)
    positions, freq = torch.arange(n, dtype=torch.int32, device="cuda"), st.st_rotary_frequencies(d).cuda()
    w = (1 + 0.1 * floats(15, d)).to(BF16)
    how = (positions, freq, False, w, w, 1e-6)
    qr, kr = st.st_attn_rotate(q, k, *how)
    out, lse = st.st_attn_window(qr, kr, v, 5, 1)
    dqr, dkr, _ = st.st_attn_window_grad(qr, kr, v, out, lse, do, 5, 1)
    grads = st.st_attn_rotate_grad(q, k, dqr, dkr, *how)
    import attn_reference as attn
    def loss(q, k, qw):
        a, b = ref.rotate(q, qw, positions, freq, False, 1e-6, 1.0)[0], ref.rotate(k, w, positions, freq, False, 1e-6, 1.0)[0]
        return float((attn.window(a, b, v, 5, 1)[0] * do.double()).sum())
    base = [x.double() for x in (q, k, w)]
    # rounded tables in between: bf16 queries, keys, outputs and their gradients, each B of sums of some 10 terms
    sizes = [float(grads[0].abs().max()), float(grads[1].abs().max()), float(grads[2].abs().max())]
    for i in range(3):
        flat = base[i].flatten()
        for e in range(0, flat.numel(), max(1, flat.numel() // 20)):
            ends = []
            for sign in (1, -1):
                moved = flat.clone()
                moved[e] += sign * 1e-5
                ends.append(loss(*[moved.view_as(base[i]) if j == i else b for j, b in enumerate(base)]))
            assert abs(float(grads[i].flatten()[e]) - (ends[0] - ends[1]) / 2e-5) <= 16 * ref.B * sizes[i]


def everything(seed):
    """All calls on their own inputs: a function that runs them, and what it reads."""
    q, k, at, (qw, kw, eps) = rotation_inputs(seed, 90, 4, 2, 64, 64, True, BF16)
    dq, dk = normal(seed + 20, *q.shape), normal(seed + 21, *k.shape)
    caches = [Cache(seed + 22, [30, 60], 2, 64, 16, bits) for bits in (16, 8, 4)]
    c, qs, args, _ = shared_inputs(seed + 23, [3, 4], [300, 200], [9, 0], 4, 2, 64, 16)
    new = offsets([30, 60])
    def run():
        out = [*st.st_attn_rotate(q, k, *at, False, qw, kw, eps), *st.st_attn_rotate_grad(q, k, dq, dk, *at, False, qw, kw, eps)]
        for x in caches:
            st.st_attn_cache_write(k, dk, *x.pages(), new, **x.how())
            out += st.st_attn_cache_read(*x.pages(), new, 90, **x.how())
            out.append(st.st_attn_cache_step(q[:2], *x.pages(), 40, 3, **x.how()))
        out.append(st.st_attn_shared_step(qs, *c.cells, *args))
        return out
    return run, (q, k, dq, dk, qs)


def test_the_same_bits_twenty_times():
    run, _ = everything(201)
    want = [x.clone() for x in run()]
    for _ in range(20):
        assert all(torch.equal(a, b) for a, b in zip(run(), want))


def test_captured_graphs_replay_with_new_inputs_and_lengths():
    st.set_allocator(None)
    run, reads = everything(211)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs = run()
        graphs.append((graph, outs))
    for i in range(3):
        for x in reads:
            x.copy_(normal(220 + i, *x.shape))
        for graph, outs in graphs:
            graph.replay()
        torch.cuda.synchronize()
        got = [[x.clone() for x in outs] for _, outs in graphs]
        want = run()
        for outs in got:
            assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_calls_on_two_streams_at_once():
    runs = [everything(231 + i)[0] for i in range(2)]
    want = [[x.clone() for x in r()] for r in runs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i] = runs[i]()
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_wrong_tensors_are_refused():
    q, k, at, (qw, kw, eps) = rotation_inputs(241, 6, 4, 2, 64, 64, True, BF16)
    rotate = st.st_attn_rotate
    for bad, error in (
        (lambda: rotate(q.float(), k, *at), TypeError), (lambda: rotate(q, k[:3], *at), ValueError), (lambda: rotate(q.cpu(), k, *at), ValueError),
        (lambda: rotate(q, k, at[0].long(), at[1]), TypeError), (lambda: rotate(q, k, at[0][:3], at[1]), ValueError),
        (lambda: rotate(q, k, at[0], at[1].double()), TypeError), (lambda: rotate(q, k, *at, False, qw), ValueError),
        (lambda: rotate(q, k, *at, False, qw, kw.float(), eps), TypeError), (lambda: rotate(q, k, *at, False, qw[:32], kw, eps), ValueError),
        (lambda: rotate(q, None, *at, False, qw, kw, eps), ValueError), (lambda: rotate(q, k, at[0], torch.ones(40, device="cuda")), st.StError),
        (lambda: rotate(q, k, *at, k_out=q[:, :2]), ValueError), (lambda: rotate(q, k, *at, q_out=k), ValueError),
        (lambda: rotate(q[:, :2], q[:, 2:], *at, q_out=q.view(-1)[: 6 * 2 * 64].view(6, 2, 64)), st.StError),
        (lambda: st.st_attn_rotate_grad(q, k, q, None, *at), ValueError), (lambda: st.st_attn_rotate_grad(q, k, q.float(), k, *at), TypeError)):
        with pytest.raises(error):
            bad()
    c, four = Cache(242, [20, 30], 2, 64, 16, 8), Cache(242, [20, 30], 2, 64, 16, 4)
    step = st.st_attn_cache_step
    x = normal(243, 2, 4, 64)
    for bad, error in (
        (lambda: step(x, *c.pages(), 10), TypeError), (lambda: step(x, *c.pages(), 10, 0, c.scales[0].double(), c.scales[1]), TypeError),
        (lambda: step(x, *c.pages(), 10, 0, c.scales[0][1:], c.scales[1][1:]), ValueError), (lambda: step(x, *four.pages(), 10, **c.how()), TypeError),
        (lambda: step(x[:1], *c.pages(), 10, **c.how()), ValueError), (lambda: step(x, *c.pages(), 0, **c.how()), st.StError),
        (lambda: step(x[:, :3], *c.pages(), 10, **c.how()), st.StError), (lambda: step(x, *c.pages(), 10, scale=0.0, **c.how()), st.StError),
        (lambda: step(x[..., :32], *c.pages(), 10, **c.how()), ValueError), (lambda: step(x, c.cells[0], c.cells[1][:1], c.table, c.lens, 10, **c.how()), ValueError),
        (lambda: st.st_attn_cache_write(x[:, :2], x[:, :2], *c.pages(), ints(0, 2), **c.how()), ValueError),
        (lambda: st.st_attn_cache_write(x[:, :1], x[:, :1], *c.pages(), **c.how()), ValueError),
        (lambda: st.st_attn_cache_read(*c.pages(), None, 5, **c.how()), ValueError), (lambda: st.st_attn_cache_read(*c.pages(), ints(0, 1, 2), 0, **c.how()), ValueError),
        (lambda: st.st_attn_shared_step(x, *c.pages()[:2], c.table[:1], c.lens[:1], c.table, c.lens), TypeError)):
        with pytest.raises(error):
            bad()
    plain = Cache(244, [20, 30], 2, 64, 16, 16)
    shared = st.st_attn_shared_step
    for bad, error in (
        (lambda: step(x, *plain.pages(), 10, **c.how()), ValueError),
        (lambda: shared(x, *plain.cells, plain.table, plain.lens, plain.table, plain.lens), ValueError),
        (lambda: shared(x, *plain.cells, plain.table, plain.lens[:1], plain.table, plain.lens), ValueError),
        (lambda: shared(x, *plain.cells, plain.table[:1], plain.lens[:1], plain.table, plain.lens, ints(0, 1, 2)), ValueError),
        (lambda: shared(x, *plain.cells, plain.table[:1], plain.lens[:1], plain.table, plain.lens, ws=torch.empty(512, dtype=torch.uint8, device="cuda")), st.StError)):
        with pytest.raises(error):
            bad()


# ------------------------------------------------------------------------- extents and layouts


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_caches_whose_heads_lie_apart(bits):
    """Heads before pages, and tokens before pages: the other strides are the largest."""
    lens, Hk, d, page = [40, 0, 133], 3, 64, 16
    c = Cache(251, lens, Hk, d, page, bits)
    q = normal(252, 3, 6, d)
    k, v = normal(253, 6, Hk, d), normal(254, 6, Hk, d)
    at = offsets([3, 0, 3])
    plain = [c.copies() for _ in range(2)]
    n = len(plain[0]) // 2
    for order in ((2, 0, 1), (1, 0, 2), (0, 2, 1)):
        def moved(x):
            if x is None:
                return None
            rest = tuple(range(3, x.dim()))
            y = torch.empty([x.shape[i] for i in order] + list(x.shape[3:]), dtype=x.dtype, device="cuda")
            view = y.permute(*[order.index(i) for i in range(3)], *rest)
            view.copy_(x)
            return view
        cells, scales = [moved(x) for x in c.cells], [moved(x) for x in c.scales]
        if bits == 4 and scales[0].stride(-2) != 2:
            continue
        how = dict(k_scales=scales[0], v_scales=scales[1])
        got = st.st_attn_cache_step(q, *cells, c.table, c.lens, 100, 3, **how)
        want = st.st_attn_cache_step(q, *c.pages(), 100, 3, **c.how())
        ok()
        assert torch.equal(got, want)
        for a, b in zip(st.st_attn_cache_read(*cells, c.table, c.lens, at, 6, **how), st.st_attn_cache_read(*c.pages(), at, 6, **c.how())):
            assert same(a, b)
        kept = Cache(251, lens, Hk, d, page, bits)
        st.st_attn_cache_write(k, v, *kept.pages(), at, **kept.how())
        st.st_attn_cache_write(k, v, *cells, c.table, c.lens, at, **how)
        ok()
        for a, b in zip((*cells, *scales), (*kept.cells, *kept.scales)):
            assert a is None or same(a.contiguous(), b)
        if bits == 16:
            args = c.table[2:].contiguous(), c.lens[2:].contiguous(), c.table, c.lens
            cells = [moved(x) for x in c.cells]
            assert torch.equal(st.st_attn_shared_step(q, *cells, *args), st.st_attn_shared_step(q, *c.cells, *args))
            ok()


@pytest.mark.parametrize("bits", [16, 8, 4])
@pytest.mark.parametrize("H,Hk,d", [(1, 1, 64), (16, 1, 128), (9, 3, 80)])
def test_one_long_sequence_is_every_warps(H, Hk, d, bits):
    n, page = 40003, 64
    c = Cache(261, [n], Hk, d, page, bits)
    q = normal(262, 1, H, d)
    got = st.st_attn_cache_step(q, *c.pages(), 1 << 62, 0, **c.how())
    ok()
    check_step(got, c, q, 1 << 62, 0)


@pytest.mark.parametrize("bits,H,Hk", [(16, 4, 4), (8, 4, 2), (4, 6, 6), (8, 10, 1)])
def test_more_sequences_than_a_block_has_threads(bits, H, Hk):
    lens = [(i * 7) % 45 if i % 11 else 0 for i in range(2100)] + [3000]
    c = Cache(271, lens, Hk, 32, 16, bits, fill=False)
    for i in range(2):                                   # one random fill of all pages instead of a sequence's each
        x = normal(272 + i, *c.cells[i].shape[:3], 32)
        if bits == 16:
            c.cells[i] = x
        else:
            c.cells[i], c.scales[i] = ref.quantise(x, bits)
    q = normal(274, len(lens), H, 32)
    got = st.st_attn_cache_step(q, *c.pages(), 30, 2, **c.how())
    ok()
    some = [0, 1, 2, 10, 11, 12, 255, 256, 257, 1022, 1023, 1024, 1025, 2047, 2048, 2098, 2099, 2100]
    for b in some:
        n = lens[b]
        lo = max(0, n - 30)
        s = torch.cat([torch.arange(min(2, lo), device="cuda"), torch.arange(lo, n, device="cuda")])
        at = (c.table[b].long()[s // 16], s % 16)
        near(got[b], *ref.attend(q[b], c.parts(0, b, at), c.parts(1, b, at)), "out of sequence %d" % b)
    # each alone gives the same up to the order of its sums, and what is empty is zeros
    empty = torch.tensor([n == 0 for n in lens], device="cuda")
    assert bool((got[empty] == 0).all()) and not bool(torch.isnan(got).any())


def test_more_groups_than_a_warp_has_lanes():
    groups = [(i * 5) % 4 for i in range(75)]
    prefix = [(i * 37) % 300 if i % 6 else 0 for i in range(75)]
    c, q, args, lens = shared_inputs(281, groups, prefix, [0, 3, 17], 4, 2, 64, 16)
    got = st.st_attn_shared_step(q, *c.cells, *args)
    ok()
    check_shared(got, c, q, groups, prefix, lens)


def test_a_batch_of_more_than_a_thousand_with_prefixes():
    groups = [700, 0, 500]
    prefix, own = [390, 5, 200], [2, 0, 33, 1]
    c, q, args, lens = shared_inputs(291, groups, prefix, own, 16, 1, 64, 32)      # 16 heads to a key head
    got = st.st_attn_shared_step(q, *c.cells, *args)
    ok()
    keep = [0, 1, 7, 8, 9, 15, 16, 17, 255, 256, 698, 699, 700, 701, 702, 703, 1023, 1024, 1198, 1199]
    for n in keep:
        g = 0 if n < 700 else 2
        (k0, k1), (v0, v1) = (tuple(torch.cat(x) for x in zip(c.parts(i, g), c.parts(i, 3 + n))) for i in range(2))
        near(got[n], *ref.attend(q[n], (k0, k1), (v0, v1)), "out of sequence %d" % n)


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_sequences_may_share_pages(bits):
    """The same row of the table for all, the same page more than once in a row."""
    c = Cache(301, [64], 2, 64, 16, bits)
    table = c.table[:, [0, 1, 0, 3, 3]].expand(5, 5).contiguous()
    lens = ints(80, 80, 33, 16, 71)
    q = normal(302, 1, 4, 64).expand(5, 4, 64).contiguous()
    got = st.st_attn_cache_step(q, c.cells[0], c.cells[1], table, lens, 1 << 30, 0, **c.how())
    ok()
    for b, n in enumerate(lens.tolist()):
        s = torch.arange(n, device="cuda")
        at = (table[b].long()[s // 16], s % 16)
        near(got[b], *ref.attend(q[b], c.parts(0, 0, at), c.parts(1, 0, at)), "out of sequence %d" % b)
    if bits == 16:
        got = st.st_attn_shared_step(q, *c.cells, table[:1].contiguous(), ints(80), table, lens)
        ok()
        for b, n in enumerate(lens.tolist()):
            s = torch.cat([torch.arange(80, device="cuda"), torch.arange(n, device="cuda")])
            at = (table[b].long()[s // 16], s % 16)
            near(got[b], *ref.attend(q[b], c.parts(0, 0, at), c.parts(1, 0, at)), "out of sequence %d" % b)


def test_the_ends_of_the_positions():
    q = normal(311, 4, 2, 64)
    positions = ints(2**31 - 1, -(2**31), 0, -1)
    freq = st.st_rotary_frequencies(64).cuda()
    freq[3], freq[4], freq[5] = 3.0e4, -0.75, 0.0
    for inter in (False, True):
        got, _ = st.st_attn_rotate(q, None, positions, freq, inter)
        near(got, *ref.rotate(q, None, positions, freq, inter, None, 1.0), "rotated")


def test_one_workspace_for_calls_one_after_the_other():
    """A workspace holds nothing from one call for the next: not after a larger call, a failed one or another kind."""
    big, small = Cache(321, [900, 44, 0, 7], 2, 64, 16, 16), Cache(322, [3, 50], 1, 128, 16, 8)
    n = max(st.st_workspace_bytes(st.ST_OP_ATTN_CACHE_STEP, 4, 0), st.st_workspace_bytes(st.ST_OP_ATTN_SHARED_STEP, 4, 8, 2, 1))
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda")
    q, r = normal(323, 4, 8, 64), normal(324, 2, 3, 128)
    args = big.table[:1].contiguous(), big.lens[:1].contiguous(), big.table, big.lens
    want = st.st_attn_cache_step(q, *big.pages(), 500, 1), st.st_attn_cache_step(r, *small.pages(), 40, **small.how()), st.st_attn_shared_step(q, *big.cells, *args)
    for _ in range(2):
        assert torch.equal(st.st_attn_cache_step(q, *big.pages(), 500, 1, ws=ws), want[0])
        assert torch.equal(st.st_attn_shared_step(q, *big.cells, *args, ws=ws), want[2])
        assert torch.equal(st.st_attn_cache_step(r, *small.pages(), 40, **small.how(), ws=ws), want[1])
        ok()
        bad = small.table.clone()
        bad[1, 0] = 1 << 20
        st.st_attn_cache_step(r, small.cells[0], small.cells[1], bad, small.lens, 100, **small.how(), ws=ws)
        assert st.st_check_status(ws) == st.ST_ERR_DEV_BOUNDS
    assert torch.equal(st.st_attn_cache_step(r, *small.pages(), 40, **small.how(), ws=ws), want[1])
    ok()


@pytest.mark.parametrize("n,H,Hk,d", [(7, 1, 1, 64), (5000, 1, 1, 128), (5000, 1, 0, 64), (9, 4, 2, 128), (3001, 6, 3, 64)])
def test_a_gradient_without_norms_needs_no_operands(n, H, Hk, d):
    """q and k may be NULL: they are not read."""
    dq, dk = normal(331, n, H, d), normal(332, n, Hk, d) if Hk else None
    at, freq = torch.arange(n, dtype=torch.int32, device="cuda"), st.st_rotary_frequencies(d).cuda()
    out = [torch.full_like(x, NAN) if x is not None else None for x in (dq, dk)]
    ws = torch.empty(256, dtype=torch.uint8, device="cuda")
    p = lambda x: None if x is None else x.data_ptr()
    r = st.StRotation(st.ST_BF16, st.ST_BF16, 0, 0, n, H, Hk, d, d, 0, 0, 0, 0, 0.0, 1.0)
    rc = st.lib().st_attn_rotate_grad(ctypes.byref(r), None, None, p(dq), p(dk), p(at), p(freq), None, None, p(out[0]), p(out[1]), None, None, p(ws), 256,
                                      torch.cuda.current_stream().cuda_stream)
    assert rc == st.ST_OK
    for x, g in ((dq, out[0]), (dk, out[1])):
        if x is not None:
            near(g, *ref.rotate_grad(x, None, x, at, freq, False, None, 1.0)[0], "gradient")


@pytest.mark.parametrize("n,H,Hk,d", [(1, 1, 1, 32), (20000, 2, 2, 32), (20000, 1, 1, 128), (9001, 2, 1, 96), (15000, 5, 3, 64), (15000, 4, 4, 48), (12000, 5, 4, 64)])
@pytest.mark.parametrize("inter", [False, True])
def test_rotations_of_tokens_of_few_heads(n, H, Hk, d, inter):
    """All heads of a token, or all but one, fit a warp at once."""
    both = normal(341, n, H + Hk + 1, d)
    q, k = both[:, :H], both[:, H : H + Hk]
    qw, kw = 1 + 0.3 * floats(342, d), 1 - 0.3 * floats(343, d)
    at = torch.arange(n, dtype=torch.int32, device="cuda") - n // 2
    rot = d - d % 16
    freq = st.st_rotary_frequencies(rot).cuda()
    out = st.st_attn_rotate(q, k, at, freq, inter, qw, kw, 1e-5)
    for got, x, w in zip(out, (q, k), (qw, kw)):
        near(got, *ref.rotate(x, w, at, freq, inter, 1e-5, 1.0), "rotated")
    dq, dk = normal(344, n, H, d), normal(345, n, Hk, d)
    gq, gk, gqw, gkw = st.st_attn_rotate_grad(q, k, dq, dk, at, freq, inter, qw, kw, 1e-5)
    for got, gotw, x, w, dy in ((gq, gqw, q, qw, dq), (gk, gkw, k, kw, dk)):
        (dx, tol), (dw, wtol) = ref.rotate_grad(x, w, dy, at, freq, inter, 1e-5, 1.0)
        near(got, dx, tol, "gradient")
        near(gotw, dw, wtol, "gradient of the weights")


@pytest.mark.parametrize("bits", [16, 8, 4])
def test_steps_where_nothing_is_to_be_seen(bits):
    c = Cache(351, [0, 0, 0], 2, 64, 16, bits)
    q = normal(352, 3, 4, 64)
    out = torch.full_like(q, NAN)
    st.st_attn_cache_step(q, *c.pages(), 7, 2, **c.how(), out=out)
    ok()
    assert bool((out == 0).all())
    if bits == 16:
        for at in (offsets([1, 2]), offsets([0, 0]), offsets([3, 0])):
            out.fill_(NAN)
            st.st_attn_shared_step(q, *c.cells, c.table[:2].contiguous(), c.lens[:2].contiguous(), c.table, c.lens, at, out=out)
            ok()
            assert bool((out == 0).all())


@pytest.mark.parametrize("H,Hk,d", [(4, 2, 64), (10, 1, 128)])
def test_scales_of_values_far_apart(H, Hk, d):
    """Cells that are not 0 beside scales over 80 powers of two, growing, falling, in any order, or 0: the weights times scales keep their places."""
    n = 300
    c = Cache(361, [n] * 4, Hk, d, 16, 8)
    g = torch.Generator(device="cuda")
    g.manual_seed(362)
    for b in range(4):
        at = c.where(b, 0, n)
        cells = torch.randint(1, 128, c.cells[1][at].shape, generator=g, device="cuda") * (2 * torch.randint(0, 2, c.cells[1][at].shape, generator=g, device="cuda") - 1)
        c.cells[1][at] = cells.to(torch.int8)
        power = torch.linspace(-40, 40, n, device="cuda")
        power = power if b == 0 else power.flip(0) if b == 1 else power[torch.randperm(n, generator=g, device="cuda")]
        scale = torch.exp2(power)[:, None].expand(n, Hk).clone()
        if b == 3:
            scale[::2] = 0
        c.scales[1][at] = scale
    q = normal(363, 4, H, d)
    for window, sinks in ((1 << 30, 0), (40, 3), (33, 0)):
        got = st.st_attn_cache_step(q, *c.pages(), window, sinks, **c.how())
        ok()
        check_step(got, c, q, window, sinks)
