"""Refusals of the rotations, the cache in cells and the steps over it: found on the host, before anything touches a device; and the frequencies."""
import ctypes
import math

import pytest

torch = pytest.importorskip("torch")

import attn_more_reference as ref
import paper_2211_10482_b200 as st

P = [(i + 1) << 32 for i in range(16)]           # addresses that are never read, and whose tables do not meet
BIG = 1 << 50
NAN, INF = float("nan"), float("inf")


def rotation(**change):
    r = dict(dtype=st.ST_BF16, weight_dtype=st.ST_BF16, norm=1, interleaved=0, n=100, heads=4, kv_heads=2, d=64, rot=32, q_row=512, q_head=64, k_row=512,
             k_head=64, eps=1e-6, factor=1.0)
    r.update(change)
    return ctypes.byref(st.StRotation(*(r[n] for n, _ in st.StRotation._fields_)))


def rotate(r=None, q=P[0], k=P[1], at=P[2], freq=P[3], qw=P[4], kw=P[5], qo=P[6], ko=P[7]):
    return st.lib().st_attn_rotate(r or rotation(), q, k, at, freq, qw, kw, qo, ko, None)


def rotate_grad(r=None, q=P[0], k=P[1], dqo=P[8], dko=P[9], at=P[2], freq=P[3], qw=P[4], kw=P[5], dq=P[6], dk=P[7], dqw=P[10], dkw=P[11], ws=P[12], n=BIG):
    return st.lib().st_attn_rotate_grad(r or rotation(), q, k, dqo, dko, at, freq, qw, kw, dq, dk, dqw, dkw, ws, n, None)


# three sequences, two key heads of 64 columns, pages of 16 tokens
ROW = {st.ST_BF16: 128, st.ST_I8: 64, st.ST_I4: 32}
SCALES = {st.ST_BF16: 0, st.ST_I8: 1, st.ST_I4: 2}
TYPES = list(ROW)


def cells(dtype=st.ST_I8, **change):
    row, scales = ROW.get(dtype, 128), SCALES.get(dtype, 0)
    c = dict(dtype=dtype, reserved=0, nseq=3, heads=4, kv_heads=2, d=64, pages=10, page=16, table_cols=5, page_stride=32 * row, token_stride=2 * row,
             head_stride=row, scale_page=32 * scales, scale_token=2 * scales, scale_head=scales)
    c.update(change)
    return ctypes.byref(st.StCells(*(c[n] for n, _ in st.StCells._fields_)))


def rows(**change):
    t = dict(dtype=st.ST_BF16, reserved=0, nseq=0, nq=0, nk=100, heads=0, kv_heads=2, d=64, dv=64, q_row=0, q_head=0, k_row=128, k_head=64, v_row=128, v_head=64)
    t.update(change)
    return ctypes.byref(st.StTokens(*(t[n] for n, _ in st.StTokens._fields_)))


def scales_of(c, ks, vs):
    plain = c is not None and c._obj.dtype == st.ST_BF16
    return (None if plain and ks == P[4] else ks), (None if plain and vs == P[5] else vs)


def write(c=None, t=None, k=P[0], v=P[1], table=P[6], lens=P[7], at=P[8], kp=P[2], vp=P[3], ks=P[4], vs=P[5], ws=P[9], n=256):
    c = c or cells()
    return st.lib().st_attn_cache_write(c, t or rows(), k, v, table, lens, at, kp, vp, *scales_of(c, ks, vs), ws, n, None)


def read(c=None, count=100, kp=P[2], vp=P[3], ks=P[4], vs=P[5], table=P[6], lens=P[7], at=P[8], k=P[0], v=P[1], ws=P[9], n=256):
    c = c or cells()
    return st.lib().st_attn_cache_read(c, count, kp, vp, *scales_of(c, ks, vs), table, lens, at, k, v, ws, n, None)


def step(c=None, q=P[0], row=256, head=64, kp=P[2], vp=P[3], ks=P[4], vs=P[5], table=P[6], lens=P[7], w=10, sinks=0, scale=1.0, out=P[1], ws=P[9], n=BIG):
    c = c or cells()
    return st.lib().st_attn_cache_step(c, q, row, head, kp, vp, *scales_of(c, ks, vs), table, lens, w, sinks, scale, out, ws, n, None)


def shared(c=None, q=P[0], row=256, head=64, kp=P[2], vp=P[3], prefix=P[10], cols=7, told=P[11], groups=2, at=P[8], table=P[6], lens=P[7], scale=1.0, out=P[1],
           ws=P[9], n=BIG):
    return st.lib().st_attn_shared_step(c or cells(st.ST_BF16), q, row, head, kp, vp, prefix, cols, told, groups, at, table, lens, scale, out, ws, n, None)


@pytest.mark.parametrize("change,status", [
    (dict(dtype=st.ST_F32), st.ST_ERR_DTYPE), (dict(weight_dtype=st.ST_F64), st.ST_ERR_DTYPE), (dict(weight_dtype=st.ST_I8), st.ST_ERR_DTYPE),
    (dict(norm=2), st.ST_ERR_SHAPE), (dict(norm=-1), st.ST_ERR_SHAPE), (dict(interleaved=3), st.ST_ERR_SHAPE), (dict(n=0), st.ST_ERR_SHAPE),
    (dict(heads=0), st.ST_ERR_SHAPE), (dict(kv_heads=-1), st.ST_ERR_SHAPE), (dict(d=0), st.ST_ERR_SHAPE), (dict(rot=-2), st.ST_ERR_SHAPE),
    (dict(rot=31), st.ST_ERR_SHAPE), (dict(rot=66), st.ST_ERR_SHAPE), (dict(n=(1 << 29) + 1), st.ST_ERR_UNSUPPORTED), (dict(heads=1 << 16), st.ST_ERR_UNSUPPORTED),
    (dict(kv_heads=1 << 40), st.ST_ERR_UNSUPPORTED), (dict(d=60, rot=8), st.ST_ERR_UNSUPPORTED), (dict(d=136), st.ST_ERR_UNSUPPORTED),
    (dict(eps=-1e-6), st.ST_ERR_UNSUPPORTED), (dict(eps=NAN), st.ST_ERR_UNSUPPORTED), (dict(eps=INF), st.ST_ERR_UNSUPPORTED), (dict(factor=INF), st.ST_ERR_UNSUPPORTED),
    (dict(factor=NAN), st.ST_ERR_UNSUPPORTED), (dict(q_row=56), st.ST_ERR_SHAPE), (dict(q_head=-64), st.ST_ERR_SHAPE), (dict(k_row=0), st.ST_ERR_SHAPE),
    (dict(q_row=516), st.ST_ERR_ALIGN), (dict(k_head=68), st.ST_ERR_ALIGN), (dict(k_row=1 << 50), st.ST_ERR_UNSUPPORTED)])
def test_rotations_are_checked(change, status):
    assert rotate(rotation(**change)) == status
    assert rotate_grad(rotation(**change)) == status


def test_rotation_refusals():
    null, align = st.ST_ERR_NULL, st.ST_ERR_ALIGN
    L = st.lib()
    assert L.st_attn_rotate(None, *P[:8], None) == L.st_attn_rotate_grad(None, *P[:13], BIG, None) == null
    assert rotate(q=None) == rotate(k=None) == rotate(at=None) == rotate(freq=None) == rotate(qo=None) == rotate(ko=None) == null
    assert rotate_grad(q=None) == rotate_grad(dqo=None) == rotate_grad(dko=None) == rotate_grad(dq=None) == rotate_grad(dk=None) == null
    for f in (rotate, rotate_grad):
        assert f(q=P[0] + 8) == f(at=P[2] + 2) == f(freq=P[3] + 4) == f(qw=P[4] + 2) == f(kw=P[5] + 8) == align
    assert rotate(qo=P[6] + 8) == rotate(ko=P[7] + 2) == rotate_grad(dqo=P[8] + 8) == rotate_grad(dk=P[7] + 8) == rotate_grad(dqw=P[10] + 4) == align
    assert rotate_grad(ws=None) == rotate_grad(n=255) == st.ST_ERR_WORKSPACE
    need = st.st_workspace_bytes(st.ST_OP_ATTN_ROTATE_GRAD, 64, 0)
    assert need > 256 and rotate_grad(n=need - 1) == st.ST_ERR_WORKSPACE and rotate_grad(ws=P[12] + 128) == align
    # where no weight has a gradient, the header is enough
    assert st.st_workspace_bytes(st.ST_OP_ATTN_ROTATE_GRAD, 0, 0) == 256
    assert rotate_grad(dqw=None, dkw=None, n=255) == st.ST_ERR_WORKSPACE and rotate_grad(dqw=None, dkw=None, n=256, ws=P[12] + 16) == align
    # gradients of weights that there are none of
    assert rotate_grad(rotation(norm=0)) == rotate_grad(rotation(kv_heads=0)) == st.ST_ERR_SHAPE


def test_rotations_over_operands_are_refused():
    bad, size = st.ST_ERR_UNSUPPORTED, 100 * 4 * 64 * 2
    flat = rotation(q_row=256, k_row=128)
    for d in (16, size - 16, 16 - size):
        assert rotate(flat, qo=P[0] + d) == bad
    for d in (0, 16, size // 2 - 16, 16 - size):
        assert rotate(flat, qo=P[6] + d, ko=P[6]) == rotate(flat, qo=P[1] + d) == bad      # half as many heads
    assert rotate(flat, qo=P[1]) == rotate(flat, ko=P[0]) == rotate(flat, qo=P[2]) == rotate(flat, ko=P[3]) == rotate(flat, qo=P[4]) == rotate(flat, ko=P[5]) == bad
    assert rotate(qo=P[0]) == rotate(ko=P[1]) == bad                # slices of a projection: rows of the result lie over other ones
    for name, own in (("dq", P[8]), ("dk", P[9])):
        for p in (P[0], P[1], P[2], P[3], P[4], P[5], own + 16):
            assert rotate_grad(flat, **{name: p}) == bad, (name, p)
    assert rotate_grad(flat, dk=P[8]) == rotate_grad(flat, dq=P[9]) == rotate_grad(flat, dk=P[6]) == rotate_grad(flat, dqw=P[6]) == bad
    assert rotate_grad(flat, dkw=P[10] + 16) == rotate_grad(flat, dkw=P[5]) == rotate_grad(flat, dqw=P[8] + 32) == bad


CALLS = [write, read, step, shared]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("change,status", [
    (dict(reserved=1), st.ST_ERR_SHAPE), (dict(nseq=0), st.ST_ERR_SHAPE), (dict(heads=0), st.ST_ERR_SHAPE), (dict(heads=3), st.ST_ERR_SHAPE),
    (dict(kv_heads=0), st.ST_ERR_SHAPE), (dict(d=0), st.ST_ERR_SHAPE), (dict(pages=0), st.ST_ERR_SHAPE), (dict(page=-1), st.ST_ERR_SHAPE),
    (dict(table_cols=0), st.ST_ERR_SHAPE), (dict(nseq=(1 << 20) + 1), st.ST_ERR_UNSUPPORTED), (dict(heads=1 << 16), st.ST_ERR_UNSUPPORTED),
    (dict(d=60), st.ST_ERR_UNSUPPORTED), (dict(d=144), st.ST_ERR_UNSUPPORTED), (dict(page=1 << 20, table_cols=1 << 11), st.ST_ERR_UNSUPPORTED),
    (dict(page=1 << 62, table_cols=4), st.ST_ERR_UNSUPPORTED), (dict(token_stride=16), st.ST_ERR_SHAPE), (dict(head_stride=-128), st.ST_ERR_SHAPE),
    (dict(page_stride=0), st.ST_ERR_SHAPE), (dict(page_stride=1 << 40), st.ST_ERR_UNSUPPORTED), (dict(page_stride=1 << 36, pages=1 << 30), st.ST_ERR_UNSUPPORTED),
    (dict(page_stride=32 * 128 + 4), st.ST_ERR_ALIGN), (dict(head_stride=132), st.ST_ERR_ALIGN)])
def test_caches_are_checked(change, status, dtype):
    for f in CALLS:
        if f is not shared or dtype == st.ST_BF16:
            assert f(cells(dtype, **change)) == status, f.__name__


@pytest.mark.parametrize("dtype", TYPES)
def test_cache_arguments(dtype):
    c = cells(dtype)
    for f in CALLS:
        if f is shared and dtype != st.ST_BF16:
            assert f(c) == st.ST_ERR_DTYPE
            continue
        assert f(cells(st.ST_F32)) == f(cells(7)) == st.ST_ERR_DTYPE
        assert f(c, kp=None) == f(c, vp=None) == f(c, table=None) == f(c, lens=None) == st.ST_ERR_NULL
        assert f(c, kp=P[2] + 8) == f(c, vp=P[3] + 4) == f(c, table=P[6] + 2) == f(c, lens=P[7] + 1) == f(c, ws=P[9] + 128) == st.ST_ERR_ALIGN
        if f is not step:
            assert f(c, at=P[8] + 2) == st.ST_ERR_ALIGN
        assert f(c, ws=None) == f(c, n=255) == st.ST_ERR_WORKSPACE
    for f in (write, read, step):
        if dtype == st.ST_BF16:
            assert f(c, ks=P[12]) == f(c, vs=P[12]) == st.ST_ERR_SHAPE                     # scales of what has none
        else:
            assert f(c, ks=None) == f(c, vs=None) == st.ST_ERR_NULL
            assert f(c, ks=P[4] + 4) == f(c, vs=P[5] + 8) == st.ST_ERR_ALIGN
            assert f(cells(dtype, scale_head=0)) == f(cells(dtype, scale_token=SCALES[dtype] - 1)) == f(cells(dtype, scale_page=-1)) == st.ST_ERR_SHAPE
            assert f(cells(dtype, scale_page=1 << 40)) == f(cells(dtype, scale_page=1 << 34, pages=1 << 30)) == st.ST_ERR_UNSUPPORTED
            # rows of 8-byte pieces are enough for them, where plain ones want 16
            assert f(cells(dtype, head_stride=ROW[dtype] + 8, token_stride=3 * ROW[dtype] + 8, page_stride=64 * ROW[dtype]), ws=None) == st.ST_ERR_WORKSPACE
    if dtype == st.ST_I4:
        assert write(cells(dtype, d=40)) == step(cells(dtype, d=8)) == st.ST_ERR_UNSUPPORTED


def test_cache_write_and_read_refusals():
    L = st.lib()
    assert L.st_attn_cache_write(None, rows(), *P[:9], P[9], P[10], 256, None) == L.st_attn_cache_read(None, 5, *P[:10], 256, None) == st.ST_ERR_NULL
    assert L.st_attn_cache_write(cells(), None, P[0], P[1], P[6], P[7], P[8], P[2], P[3], P[4], P[5], P[9], 256, None) == st.ST_ERR_NULL
    assert write(k=None) == write(v=None) == read(k=None) == read(v=None) == st.ST_ERR_NULL
    for change in (dict(kv_heads=1), dict(d=32), dict(dv=32), dict(nk=0), dict(k_row=64 - 8), dict(v_head=-8), dict(reserved=1)):
        assert write(t=rows(**change)) == st.ST_ERR_SHAPE, change
    assert write(t=rows(dtype=st.ST_F32)) == st.ST_ERR_DTYPE
    assert write(t=rows(k_row=132)) == write(t=rows(v_head=68)) == write(k=P[0] + 8) == write(v=P[1] + 2) == read(k=P[0] + 8) == read(v=P[1] + 4) == st.ST_ERR_ALIGN
    assert write(t=rows(nk=(1 << 29) + 1)) == read(count=(1 << 29) + 1) == st.ST_ERR_UNSUPPORTED
    # three sequences of which nothing says where their rows are; with as many rows they have one each
    assert write(at=None) == read(at=None) == read(count=0) == read(count=-1) == st.ST_ERR_SHAPE
    assert write(t=rows(nk=3), at=None, ws=None) == read(count=3, at=None, ws=None) == write(cells(nseq=1), at=None, ws=None) == st.ST_ERR_WORKSPACE
    # rows in pages and in scales
    assert write(k=P[2]) == write(v=P[2] + 1024) == write(k=P[3]) == write(v=P[5]) == write(k=P[4] - 128) == st.ST_ERR_UNSUPPORTED
    assert read(k=P[2]) == read(v=P[3] + 512) == read(k=P[4]) == read(v=P[5]) == read(k=P[1]) == read(v=P[0] + 256) == st.ST_ERR_UNSUPPORTED
    assert read(k=P[6]) == read(v=P[7]) == read(k=P[8]) == st.ST_ERR_UNSUPPORTED
    assert st.st_workspace_bytes(st.ST_OP_ATTN_CACHE, 0, 0) == 256


def test_cache_step_refusals():
    L = st.lib()
    assert L.st_attn_cache_step(None, P[0], 256, 64, *P[2:8], 10, 0, 1.0, P[1], P[9], BIG, None) == st.ST_ERR_NULL
    assert step(q=None) == step(out=None) == st.ST_ERR_NULL
    assert step(w=0) == step(w=-5) == step(sinks=-1) == step(row=56) == step(head=0) == st.ST_ERR_SHAPE
    assert step(row=260) == step(head=68) == step(q=P[0] + 8) == step(out=P[1] + 2) == st.ST_ERR_ALIGN
    assert step(scale=0.0) == step(scale=-1.0) == step(scale=NAN) == step(scale=INF) == step(row=1 << 40) == step(cells(nseq=1 << 16)) == st.ST_ERR_UNSUPPORTED
    # 65535 sequences of 65535 heads with 2^30 tokens each
    assert step(cells(nseq=65535, heads=65535, kv_heads=65535, page=1 << 30, table_cols=1, pages=1), row=65535 * 64) == st.ST_ERR_UNSUPPORTED
    need = st.st_workspace_bytes(st.ST_OP_ATTN_CACHE_STEP, 3, 0)
    assert need > 256 and step(n=need - 1) == st.ST_ERR_WORKSPACE
    assert st.st_workspace_bytes(st.ST_OP_ATTN_CACHE_STEP, 0, 0) == st.st_workspace_bytes(st.ST_OP_ATTN_CACHE_STEP, 1 << 16, 0) == 0
    size = 3 * 256 * 2
    for p in (P[0] + 16, P[0] + size - 16, P[0] - size + 16, P[2], P[2] + 32 * 64 * 10 - 16, P[3] - size + 16, P[4], P[5], P[6], P[7]):
        assert step(out=p) == st.ST_ERR_UNSUPPORTED, hex(p)
    assert step(row=512, out=P[0]) == st.ST_ERR_UNSUPPORTED          # strided queries


def test_shared_step_refusals():
    L = st.lib()
    assert L.st_attn_shared_step(None, P[0], 256, 64, P[2], P[3], P[10], 7, P[11], 2, P[8], P[6], P[7], 1.0, P[1], P[9], BIG, None) == st.ST_ERR_NULL
    assert shared(q=None) == shared(out=None) == shared(prefix=None) == shared(told=None) == shared(at=None) == st.ST_ERR_NULL
    assert shared(cols=0) == shared(groups=0) == shared(groups=-1) == shared(row=56) == st.ST_ERR_SHAPE
    assert shared(prefix=P[10] + 2) == shared(told=P[11] + 1) == shared(q=P[0] + 8) == shared(head=68) == st.ST_ERR_ALIGN
    assert shared(cols=1 << 31) == shared(cols=1 << 28) == shared(groups=1 << 16) == shared(scale=-1.0) == shared(cells(st.ST_BF16, nseq=1 << 16)) == st.ST_ERR_UNSUPPORTED
    assert shared(cells(st.ST_BF16, heads=514), row=514 * 64) == st.ST_ERR_UNSUPPORTED       # 257 heads to a key head
    args = st.ST_OP_ATTN_SHARED_STEP, 3, 4, 2, 2
    need = st.st_workspace_bytes(*args)
    assert need > st.st_workspace_bytes(st.ST_OP_ATTN_CACHE_STEP, 3, 0) and shared(n=need - 1) == st.ST_ERR_WORKSPACE
    for a in ((0, 4, 2, 2), (3, 4, 3, 2), (3, 4, 2, 0), (1 << 16, 4, 2, 2), (3, 514, 2, 2), (3, 0, 2, 2), (65535, 65535, 65535, 65535)):
        assert st.st_workspace_bytes(st.ST_OP_ATTN_SHARED_STEP, *a) == 0, a
    size = 3 * 256 * 2
    for p in (P[0] + 16, P[0] - size + 16, P[2], P[3] + 1024, P[6], P[7], P[8], P[10], P[11]):
        assert shared(out=p) == st.ST_ERR_UNSUPPORTED, hex(p)


def test_tensors_on_the_host_are_refused_by_name():
    x, i = torch.zeros(4, 2, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int32)
    p = torch.zeros(3, 16, 2, 64, dtype=torch.bfloat16)
    for name, f in (("q", lambda: st.st_attn_rotate(x, x, i, None)), ("q", lambda: st.st_attn_rotate_grad(x, x, x, x, i, None)),
                    ("q", lambda: st.st_attn_cache_step(x, p, p, i, i, 4)), ("q", lambda: st.st_attn_shared_step(x, p, p, i, i, i, i)),
                    ("k", lambda: st.st_attn_cache_write(x, x, p, p, i, i)), ("k_pages", lambda: st.st_attn_cache_read(p, p, i, i, None, 4))):
        with pytest.raises(ValueError, match="%s must be a CUDA tensor" % name):
            f()
    with pytest.raises(TypeError, match="q must be a tensor"):
        st.st_attn_rotate(None, x, i, None)


# ------------------------------------------------------------------------------------ frequencies

def test_frequencies_are_the_definition():
    f = st.st_rotary_frequencies(64, 500000.0)
    assert f.dtype == torch.float32 and f.shape == (32,) and f.device.type == "cpu"
    for i in range(32):
        assert abs(f[i].item() / 500000.0 ** (-2 * i / 64) - 1) <= 2 ** -23
    assert torch.equal(st.st_rotary_frequencies(64, 500000.0, stretch=8.0), f)


def test_stretched_frequencies():
    f = st.st_rotary_frequencies(128).double()
    assert torch.allclose(st.st_rotary_frequencies(128, kind="linear", stretch=4.0).double() * 4, f, rtol=2 ** -23, atol=0)
    g = st.st_rotary_frequencies(128, kind="base", stretch=4.0).double()
    assert g[0] == f[0] == 1 and abs(g[-1] * 4 / f[-1] - 1) < 2 ** -22 and bool((g[1:] < f[1:]).all())
    h = st.st_rotary_frequencies(128, kind="turns", stretch=4.0, trained=4096, turns=(1.0, 32.0)).double()
    turns = 4096 * f / (2 * math.pi)
    assert torch.equal(h[turns >= 33], f[turns >= 33]) and torch.allclose(h[turns <= 0.99] * 4, f[turns <= 0.99], rtol=2 ** -23, atol=0)
    between = (turns > 1.01) & (turns < 31.9)
    assert bool(between.any()) and bool(((h < f) & (h * 4 > f))[between].all())


@pytest.mark.parametrize("how", [dict(rot=0), dict(rot=7), dict(rot=-2), dict(rot=8, base=0.0), dict(rot=8, base=NAN), dict(rot=8, stretch=0.0), dict(rot=8, kind="other"),
                                 dict(rot=2, kind="base"), dict(rot=8, kind="turns"), dict(rot=8, kind="turns", trained=10, turns=(2.0, 1.0))])
def test_frequencies_that_are_refused(how):
    with pytest.raises(ValueError):
        st.st_rotary_frequencies(**how)


# ------------------------------------------------------------------------------------ the oracle

@pytest.mark.parametrize("rot,inter", [(16, False), (16, True), (6, False), (6, True), (0, False)])
def test_the_oracle_turns_back_what_it_turned(rot, inter):
    """A rotation's transpose is its inverse, and leaves every pair's length."""
    g = torch.Generator().manual_seed(3)
    y = torch.randn(5, 3, 16, generator=g, dtype=torch.float64)
    at, freq = torch.tensor([0, 1, -7, 100, 1 << 20], dtype=torch.int32), st.st_rotary_frequencies(rot) if rot else None
    if rot == 0:
        assert torch.equal(ref.turned(y, at, freq, inter, 1.0), y)
        return
    z = ref.turned(y, at, freq, inter, 1.0)
    assert torch.allclose(ref.turned(z, at, freq, inter, 1.0, back=True), y, rtol=0, atol=1e-12)
    assert torch.allclose(z.norm(dim=-1), y.norm(dim=-1), rtol=1e-12) and torch.equal(z[..., rot:], y[..., rot:]) and torch.equal(z[0], y[0])


@pytest.mark.parametrize("bits", [8, 4])
def test_the_oracle_rounds_to_the_nearest_cell(bits):
    g = torch.Generator().manual_seed(4)
    x = torch.randn(50, 2, 64, generator=g).bfloat16()
    x[3] = 0
    got = sum(ref.parts_of(*ref.quantise(x, bits), bits))
    for c in range(0, 64, 64 if bits == 8 else 32):
        part = x.double()[..., c:c + (64 if bits == 8 else 32)]
        span = part.abs().amax(-1, keepdim=True) / 127 if bits == 8 else (part.amax(-1, keepdim=True) - part.amin(-1, keepdim=True)) / 15
        # half a cell, and what the step's rounding to bf16 (2^-8 of it) and fp32's add up to over 15 or 127 steps
        off = (got[..., c:c + part.shape[-1]] - part).abs()
        assert bool((off <= span * (0.5 + (15 * 2 ** -8 if bits == 4 else 127 * 2 ** -22)) + 1e-30).all())
