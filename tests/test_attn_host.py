"""Refusals of the attention calls: found on the host, before anything touches a device."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

import paper_2211_10482_b200 as st


def tokens(**change):
    t = dict(dtype=st.ST_BF16, reserved=0, nseq=2, nq=100, nk=100, heads=4, kv_heads=2, d=64, dv=64, q_row=256, q_head=64, k_row=128,
             k_head=64, v_row=128, v_head=64)
    t.update(change)
    return ctypes.byref(st.StTokens(*(t[n] for n, _ in st.StTokens._fields_)))


def cache(**change):
    c = dict(dtype=st.ST_BF16, reserved=0, nseq=3, heads=4, kv_heads=2, d=64, pages=10, page=16, table_cols=5, page_stride=2048, token_stride=128,
             head_stride=64)
    c.update(change)
    return ctypes.byref(st.StCache(*(c[n] for n, _ in st.StCache._fields_)))


P = [256 * (i + 1) for i in range(12)]           # addresses that are never read


def window(t=None, q=P[0], k=P[1], v=P[2], qo=P[3], ko=P[4], w=10, sinks=0, out=P[5], lse=P[6], ws=P[7], n=256):
    return st.lib().st_attn_window(t or tokens(), q, k, v, qo, ko, w, sinks, 1.0, out, lse, ws, n, None)


def window_grad(t=None, dout=P[3], qo=P[4], ko=P[5], w=10, ws=P[11], n=1 << 30, dq=P[6], dk=P[7], dv=P[8]):
    return st.lib().st_attn_window_grad(t or tokens(), P[0], P[1], P[2], P[9], P[10], dout, qo, ko, w, 0, 1.0, dq, dk, dv, ws, n, None)


def step(c=None, q=P[0], kp=P[3], table=P[5], lens=P[6], w=10, sinks=0, ws=P[8], n=256):
    return st.lib().st_attn_window_step(c or cache(), q, P[1], P[2], kp, P[4], table, lens, w, sinks, 1.0, P[7], ws, n, None)


EVEN = dict(kv_heads=4, k_row=256, v_row=256)


def decay(t=None, q=P[0], a=P[3], at=P[4], state=None, out=P[5], last=None, ws=P[6], n=1 << 40):
    return st.lib().st_attn_decay(t or tokens(**EVEN), q, P[1], P[2], a, at, state, 1.0, out, last, ws, n, None)


def decay_grad(t=None, dout=P[4], at=P[5], dq=P[6], ws=P[9], n=1 << 40, state=None):
    return st.lib().st_attn_decay_grad(t or tokens(**EVEN), P[0], P[1], P[2], P[3], dout, at, state, None, 1.0, dq, P[7], P[8], None, ws, n, None)


def decay_step(t=None, q=P[0], state=P[4]):
    return st.lib().st_attn_decay_step(t or tokens(nseq=100, **EVEN), q, P[1], P[2], P[3], state, 1.0, P[5], None)


BAD_TOKENS = [
    (dict(dtype=st.ST_F32), st.ST_ERR_DTYPE), (dict(reserved=1), st.ST_ERR_SHAPE), (dict(nseq=0), st.ST_ERR_SHAPE), (dict(d=0), st.ST_ERR_SHAPE),
    (dict(heads=0), st.ST_ERR_SHAPE), (dict(dv=-8), st.ST_ERR_SHAPE), (dict(nq=0, nk=0), st.ST_ERR_SHAPE),
    (dict(d=12, dv=12), st.ST_ERR_UNSUPPORTED), (dict(d=136, dv=136), st.ST_ERR_UNSUPPORTED), (dict(nq=(1 << 29) + 1, nk=(1 << 29) + 1), st.ST_ERR_UNSUPPORTED),
    (dict(q_row=60), st.ST_ERR_SHAPE), (dict(k_head=-64), st.ST_ERR_SHAPE), (dict(v_row=0), st.ST_ERR_SHAPE), (dict(q_row=260), st.ST_ERR_ALIGN),
    (dict(k_head=68), st.ST_ERR_ALIGN), (dict(v_row=1 << 50), st.ST_ERR_UNSUPPORTED)]


@pytest.mark.parametrize("change,status", BAD_TOKENS)
def test_tables_of_tokens_are_checked(change, status):
    assert window(tokens(**change)) == status
    assert window_grad(tokens(**change)) == status
    assert decay(tokens(**{**EVEN, **change})) == status
    assert decay_grad(tokens(**{**EVEN, **change})) == status


def test_window_refusals():
    assert window(q=None) == window(out=None) == window(lse=None) == st.ST_ERR_NULL
    assert window(qo=None) == window(ko=None) == window(qo=None, ko=None) == st.ST_ERR_NULL        # two sequences need both
    assert st.lib().st_attn_window(None, *P[:5], 1, 0, 1.0, *P[5:8], 256, None) == st.ST_ERR_NULL
    assert window(w=0) == window(w=-3) == window(sinks=-1) == window(tokens(dv=32)) == window(tokens(heads=3)) == st.ST_ERR_SHAPE
    assert window(q=264) == window(out=264) == window(qo=260) == window(ws=128 + 256) == st.ST_ERR_ALIGN
    assert window(ws=None) == window(n=255) == st.ST_ERR_WORKSPACE
    assert window_grad(dout=None) == window_grad(dq=None) == window_grad(dk=None) == window_grad(dv=None) == window_grad(qo=None) == st.ST_ERR_NULL
    assert window_grad(w=0) == st.ST_ERR_SHAPE
    assert window_grad(dout=264) == window_grad(dv=264) == st.ST_ERR_ALIGN
    need = st.st_workspace_bytes(st.ST_OP_ATTN_WINDOW_GRAD, 100, 4, 2, 0)
    assert need >= 256 + 1600
    assert window_grad(n=need - 1) == window_grad(ws=None) == st.ST_ERR_WORKSPACE
    assert st.st_workspace_bytes(st.ST_OP_ATTN_WINDOW, 0, 0) == st.st_workspace_bytes(st.ST_OP_ATTN_WINDOW_STEP, 0, 0) == 256
    assert st.st_workspace_bytes(st.ST_OP_ATTN_WINDOW_GRAD, 0, 4, 2) == 0


def test_step_refusals():
    assert step(q=None) == step(kp=None) == step(table=None) == step(lens=None) == st.ST_ERR_NULL
    for change in (dict(nseq=0), dict(pages=0), dict(page=0), dict(table_cols=0), dict(heads=3), dict(reserved=2), dict(token_stride=8), dict(page_stride=-8)):
        assert step(cache(**change)) == st.ST_ERR_SHAPE, change
    for change in (dict(d=20), dict(d=256, token_stride=512, head_stride=256), dict(nseq=1 << 20), dict(page=1 << 20, table_cols=1 << 11)):
        assert step(cache(**change)) == st.ST_ERR_UNSUPPORTED, change
    assert step(cache(dtype=st.ST_F64)) == st.ST_ERR_DTYPE
    assert step(w=0) == step(sinks=-1) == st.ST_ERR_SHAPE
    assert step(cache(page_stride=2052)) == step(kp=264) == step(ws=264) == st.ST_ERR_ALIGN
    assert step(ws=None) == step(n=0) == st.ST_ERR_WORKSPACE


def test_decay_refusals():
    assert decay(q=None) == decay(a=None) == decay(at=None) == decay(out=None) == decay_grad(dout=None) == decay_grad(dq=None) == st.ST_ERR_NULL
    assert decay(tokens()) == decay_grad(tokens()) == decay(tokens(nk=99, **EVEN)) == st.ST_ERR_SHAPE       # shared heads; lengths differ
    assert decay(q=264) == decay(state=264) == decay(last=264) == decay_grad(state=264) == decay(ws=264) == st.ST_ERR_ALIGN
    assert decay(ws=None) == decay(n=8) == decay_grad(ws=None) == decay_grad(n=8) == st.ST_ERR_WORKSPACE
    need = st.st_workspace_bytes(st.ST_OP_ATTN_DECAY, 100, 2, 4, 64)
    assert need >= 256 and decay(n=need - 1) == st.ST_ERR_WORKSPACE
    need = st.st_workspace_bytes(st.ST_OP_ATTN_DECAY_GRAD, 100, 2, 4, 64)
    assert need >= 256 and decay_grad(n=need - 1) == st.ST_ERR_WORKSPACE
    assert st.st_workspace_bytes(st.ST_OP_ATTN_DECAY, 100, 2, 4, 136) == 0
    assert st.lib().st_attn_decay_grad(tokens(**EVEN), *P[:5], P[5], P[9], P[10], 1.0, *P[6:9], P[10], P[11], 1 << 40, None) == st.ST_ERR_UNSUPPORTED
    assert st.lib().st_attn_decay_grad(tokens(**EVEN), *P[:5], P[5], P[9], P[10], 1.0, *P[6:9], P[9], P[11], 1 << 40, None) == st.ST_ERR_UNSUPPORTED
    assert decay_step(q=None) == decay_step(state=None) == st.ST_ERR_NULL
    assert decay_step(tokens(nseq=99, **EVEN)) == decay_step(tokens(nseq=100)) == st.ST_ERR_SHAPE
    assert decay_step(state=264) == st.ST_ERR_ALIGN


@pytest.mark.parametrize("change", [dict(q_row=512), dict(k_row=264), dict(v_row=320), dict(q_head=128, q_row=512), dict(k_head=72, k_row=288), dict(v_head=6400, v_row=64),
                                    dict(q_head=6400, q_row=64)])
def test_a_step_of_the_decay_takes_contiguous_tables_only(change):
    """Its kernel reads them as such: strided ones would be read in the wrong places."""
    assert decay_step(tokens(nseq=100, **{**EVEN, **change})) == st.ST_ERR_SHAPE
    # the stride of an extent of one is never used: these pass, as far as the next refusal
    assert decay_step(tokens(nseq=1, nq=1, nk=1, **{**EVEN, "q_row": 7, "k_row": 9, "v_row": 11}), state=264) == st.ST_ERR_ALIGN
    assert decay_step(tokens(nseq=100, heads=1, kv_heads=1, q_row=64, k_row=64, v_row=64, q_head=0, k_head=3, v_head=5), state=264) == st.ST_ERR_ALIGN


FAR = [(i + 1) << 30 for i in range(14)]         # addresses whose tables do not meet


def test_results_over_operands_are_refused():
    """Calls that would be wrong: another block reads, or another kernel of the call reads again, what a result has replaced.  All tables
    of 100 rows and four heads of 64 bf16 are contiguous; a result lies over an operand from its beginning, its middle or its last byte on."""
    L, t, size, bad = st.lib(), tokens(**EVEN), 100 * 256 * 2, st.ST_ERR_UNSUPPORTED
    q, k, v, out, lse, dout, dq, dk, dv, at, a, s0, s1, ws = FAR
    big = 1 << 40
    shifts = (16, size // 2, size - 16, 16 - size)

    def window(q=q, k=k, v=v, out=out, lse=lse):
        return L.st_attn_window(t, q, k, v, at, at, 10, 0, 1.0, out, lse, ws, big, None)

    def window_grad(q=q, k=k, v=v, out=out, lse=lse, dout=dout, dq=dq, dk=dk, dv=dv):
        return L.st_attn_window_grad(t, q, k, v, out, lse, dout, at, at, 10, 0, 1.0, dq, dk, dv, ws, big, None)

    def decay(q=q, k=k, v=v, out=out, s0=s0, s1=s1):
        return L.st_attn_decay(t, q, k, v, a, at, s0, 1.0, out, s1, ws, big, None)

    def decay_grad(q=q, k=k, v=v, dout=dout, s0=s0, s1=s1, dq=dq, dk=dk, dv=dv, ds=lse):
        return L.st_attn_decay_grad(t, q, k, v, a, dout, at, s0, s1, 1.0, dq, dk, dv, ds, ws, big, None)

    def decay_step(t=tokens(nseq=100, **EVEN), q=q, k=k, v=v, state=s0, out=out):
        return L.st_attn_decay_step(t, q, k, v, a, state, 1.0, out, None)

    def step(q=q, k=k, v=v, out=out):
        return L.st_attn_window_step(cache(), q, k, v, dq, dk, at, a, 10, 0, 1.0, out, ws, big, None)

    for x in (k, v):
        assert window(out=x) == window(lse=x) == bad
    assert window(lse=q) == window(lse=out) == window(lse=out + size - 16) == bad
    for d in shifts:
        assert window(out=q + d) == window(out=k + d) == window(out=v + d) == bad
    for x in (q, k, v, dout, lse, dk, dv):
        assert window_grad(dq=x) == bad
    for d in shifts:
        assert window_grad(dq=q + d) == window_grad(dq=out + d) == window_grad(dk=k + d) == window_grad(dv=k + d) == window_grad(dk=v + d) == bad
    for x in (q, dout, lse):
        assert window_grad(dk=x) == window_grad(dv=x) == bad
    assert window_grad(dv=dk) == window_grad(dv=dk + 32) == bad
    for d in shifts:
        assert decay(out=q + d) == decay(out=k + d) == decay(out=v + d) == bad
    for x in (q, k, v, out):
        assert decay(s1=x) == bad
    assert decay(out=s0) == decay(s1=s0 + 16) == decay(s1=s0 - 16) == bad
    for x in (q, k, v, dout, s0, s1):
        assert decay_grad(dq=x) == decay_grad(dk=x) == decay_grad(dv=x) == decay_grad(ds=x) == bad
    assert decay_grad(dq=dk) == decay_grad(dk=dv) == decay_grad(dv=dq + 16) == decay_grad(ds=dq) == decay_grad(ds=s1 + 64) == bad
    for x in (q, k, v, out):
        assert decay_step(state=x) == bad
    assert decay_step(out=v + 16) == decay_step(out=q + 16) == decay_step(out=s0) == bad
    # the two halves of 128 columns are two blocks', which both read q and k
    wide = tokens(nseq=100, nq=100, nk=100, **{**EVEN, "d": 128, "dv": 128, "q_row": 512, "k_row": 512, "v_row": 512, "q_head": 128, "k_head": 128, "v_head": 128})
    assert decay_step(wide, out=q) == decay_step(wide, out=k) == bad
    t = tokens(**{**EVEN, "d": 128, "dv": 128, "q_row": 512, "k_row": 512, "v_row": 512, "q_head": 128, "k_head": 128, "v_head": 128})
    assert decay(out=q) == decay(out=k) == bad
    assert step(out=k) == step(out=v) == step(out=q + 16) == step(out=v + 3 * 128 * 2 - 16) == bad
    # slices of one projection: out lies over its q, k and v
    t = tokens(kv_heads=4, q_row=768, k_row=768, v_row=768)
    assert window(k=q + 512, v=q + 1024, out=q) == bad


def test_tensors_on_the_host_are_refused_by_name():
    x = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    for f in (lambda: st.st_attn_window(x, x, x, 4), lambda: st.st_attn_window_grad(x, x, x, x, x, x, 4),
              lambda: st.st_attn_window_step(x, x, x, x, x, x, x, 4), lambda: st.st_attn_decay(x, x, x, x),
              lambda: st.st_attn_decay_grad(x, x, x, x, x), lambda: st.st_attn_decay_step(x, x, x, x, x)):
        with pytest.raises(ValueError, match="q must be a CUDA tensor"):
            f()
    with pytest.raises(TypeError, match="q must be a tensor"):
        st.st_attn_decay(None, x, x, x)
