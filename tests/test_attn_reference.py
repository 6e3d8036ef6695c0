"""The attention operators' definitions in 64 bits (attn_reference.py), which the GPU tests hold the kernels against: their gradients against
differences of their results, element by element, on the CPU."""
import math

import pytest

torch = pytest.importorskip("torch")

import attn_reference as ref

STEP = 2.0 ** -14


def normal(seed, *shape):
    return torch.randn(shape, generator=torch.Generator().manual_seed(seed), dtype=torch.float64)


def differences(loss, tables, which):
    """The derivative of loss by each element of tables[which], from five points: off by STEP^4 f^(5) / 30, and by what 64 bits lose."""
    x, out = tables[which], torch.empty_like(tables[which])
    for i in range(x.numel()):
        def at(step):
            y = x.clone()
            y.view(-1)[i] += step
            return float(loss(*tables[:which], y, *tables[which + 1 :]))
        out.view(-1)[i] = (8 * (at(STEP) - at(-STEP)) - (at(2 * STEP) - at(-2 * STEP))) / (12 * STEP)
    return out


def agree(got, want, what):
    # STEP^4 is 1.4e-17, fifth derivatives of sums of some dozen terms are below 10^6; 64 bits lose 2^-53 of sums below 10^3 over STEP: 2e-9
    worst = float((got - want).abs().max())
    assert worst <= 1e-7, (what, worst)
    assert float(want.abs().max()) > 1e-2, "%s: nothing to see" % what


@pytest.mark.parametrize("lq,lk,H,Hk,d,window,sinks,scale", [
    (7, 7, 2, 2, 3, 100, 0, None), (9, 9, 2, 1, 4, 3, 2, None), (5, 11, 4, 2, 2, 4, 1, 0.7), (8, 5, 2, 1, 3, 2, 1, None), (6, 6, 1, 1, 4, 1, 0, None),
    (10, 12, 3, 3, 2, 2, 40, None)])
def test_window_gradients(lq, lk, H, Hk, d, window, sinks, scale):
    q, k, v, dout = normal(1, lq, H, d), normal(2, lk, Hk, d), normal(3, lk, Hk, d), normal(4, lq, H, d)
    out = ref.window(q, k, v, window, sinks, scale)[0]
    got = ref.window_grad(q, k, v, out, dout, window, sinks, scale)

    def loss(q, k, v):
        return (ref.window(q, k, v, window, sinks, scale)[0] * dout).sum()

    for i, name in enumerate(("dq", "dk", "dv")):
        if name != "dv" and window == 1 and sinks == 0:    # one key to a query: its weight is 1 whatever it is
            assert float(got[i][0].abs().max()) <= 1e-12 and float(differences(loss, (q, k, v), i).abs().max()) <= 1e-7
        else:
            agree(got[i][0], differences(loss, (q, k, v), i), name)


def test_window_of_a_query_by_hand():
    """One query, two keys, one value column: weights 1 / (1 + e) and e / (1 + e), and what lies outside the window."""
    q, v = torch.ones(3, 1, 1, dtype=torch.float64), torch.tensor([5.0, 2.0, 7.0], dtype=torch.float64).view(3, 1, 1)
    k = torch.tensor([9.0, 0.0, 1.0], dtype=torch.float64).view(3, 1, 1)
    out, lse, _, _ = ref.window(q[2:], k, v, 2, 0)
    assert abs(float(out) - (2 + 7 * math.e) / (1 + math.e)) < 1e-14 and abs(float(lse) - math.log(1 + math.e)) < 1e-14
    out, lse, _, _ = ref.window(q[2:], k, v, 1, 1)
    assert abs(float(out) - (5 * math.exp(9) + 7 * math.e) / (math.exp(9) + math.e)) < 1e-14
    out, lse, _, _ = ref.window(q, k[:2], v[:2], 1, 0)     # three queries, two keys: the first stands before all
    assert float(out[0]) == 0.0 and float(lse[0]) == -math.inf and out[1:].flatten().tolist() == [5.0, 2.0]


@pytest.mark.parametrize("n,H,d,dv,a,scale", [(7, 2, 3, 2, [-0.3, -0.01], None), (6, 1, 2, 4, [0.0], 0.4), (5, 2, 2, 3, [-math.inf, -2.0], None), (1, 1, 3, 3, [-0.5], None)])
@pytest.mark.parametrize("state", [False, True])
def test_decay_gradients(n, H, d, dv, a, scale, state):
    q, k, v, dout = normal(11, n, H, d), normal(12, n, H, d), normal(13, n, H, dv), normal(14, n, H, dv)
    s, dlast, a = normal(15, H, d, dv), normal(16, H, d, dv) if state else None, torch.tensor(a, dtype=torch.float64)
    if not state:
        s = torch.zeros_like(s)
    got = ref.decay_grad(q, k, v, a, dout, s if state else None, dlast, scale)

    def loss(q, k, v, s):
        out, last, _, _ = ref.decay(q, k, v, a, s, scale)
        return (out * dout).sum() + (0.0 if dlast is None else (last * dlast).sum())

    for i, name in enumerate(("dq", "dk", "dv", "dstate")):
        agree(got[i][0], differences(loss, (q, k, v, s), i), name)


def test_decay_is_its_recurrence():
    """S[t] = e^a S[t-1] + k[t] (x) v[t], out[t] = scale S[t]^T q[t]: token by token."""
    n, H, d, dv = 300, 2, 4, 3
    q, k, v, s = normal(21, n, H, d), normal(22, n, H, d), normal(23, n, H, dv), normal(24, H, d, dv)
    a = torch.tensor([-0.2, -0.001], dtype=torch.float64)
    out, last, _, _ = ref.decay(q, k, v, a, s)
    S = s.clone()
    for t in range(n):
        S = a.exp().view(-1, 1, 1) * S + k[t][..., None] * v[t][:, None]
        assert float((torch.einsum("hd,hde->he", q[t], S) / 2 - out[t]).abs().max()) < 1e-12
    assert float((S - last).abs().max()) < 1e-12
