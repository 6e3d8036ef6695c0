"""The attention operators from their definitions, in 64 bits with torch, dense over all pairs of one sequence, and the error that
the kernels' roundings may leave.

Tolerances count roundings: to bf16 at most half a step, B = 2^-8 of the value.  The rest of the arithmetic is fp32; F = 2^-12 of the
sum of absolute terms stands for it (sums of 128 products: 128 x 2^-24, once in a score, whose error is the relative error of its
weight, and once in a product: 2^-16 of the absolute terms each; the operands' split into two bf16 numbers: 2^-16; scores reach
about 16 times their typical size).  A state is rounded once where it meets a query: B of |query| |state|."""
import math

import torch

B, F = 2.0 ** -8, 2.0 ** -12


def visible(lq, lk, window, sinks, device):
    t = torch.arange(lk - lq, lk, device=device)[:, None]
    s = torch.arange(lk, device=device)[None]
    return (s <= t) & ((s > t - window) | (s < sinks))


def heads_first(x, group=1):
    return x.double().repeat_interleave(group, 1).transpose(0, 1)


def window(q, k, v, window_, sinks, scale=None):
    """out, lse and their tolerances, for one sequence: q [lq, H, d], k and v [lk, Hk, d]."""
    g = q.shape[1] // k.shape[1]
    scale = q.shape[2] ** -0.5 if scale is None else scale
    Q, K, V = heads_first(q), heads_first(k, g), heads_first(v, g)
    see = visible(q.shape[0], k.shape[0], window_, sinks, q.device)
    x = (Q @ K.transpose(1, 2) * scale).masked_fill(~see, -math.inf)
    lse = torch.logsumexp(x, -1) if k.shape[0] else torch.full(x.shape[:2], -math.inf, dtype=torch.float64, device=q.device)
    p = torch.where(see, torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)[..., None]), 0.0)
    out = p @ V
    # weights and result are rounded once each
    tol = (2 * B + F) * (p @ V.abs())
    lse_tol = F * (1 + lse.abs().nan_to_num(posinf=0.0))
    back = lambda z: z.transpose(0, 1)
    return back(out), back(lse), back(tol), back(lse_tol)


def window_grad(q, k, v, out, dout, window_, sinks, scale=None):
    """dq, dk, dv and their tolerances, for one sequence; delta from the rounded out that the call is given."""
    hk = k.shape[1]
    g = q.shape[1] // hk
    scale = q.shape[2] ** -0.5 if scale is None else scale
    Q, K, V, O, D = heads_first(q), heads_first(k, g), heads_first(v, g), heads_first(out), heads_first(dout)
    see = visible(q.shape[0], k.shape[0], window_, sinks, q.device)
    x = (Q @ K.transpose(1, 2) * scale).masked_fill(~see, -math.inf)
    lse = torch.logsumexp(x, -1)
    p = torch.where(see, torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)[..., None]), 0.0)
    ds = p * (D @ V.transpose(1, 2) - (D * O).sum(-1)[..., None]) * scale
    # ds is rounded once, and it is a difference: fp32 errors are relative to what is subtracted
    eds = B * ds.abs() + F * p * (D.abs() @ V.abs().transpose(1, 2) + (D * O).abs().sum(-1)[..., None]) * abs(scale)
    ep = (B + F) * p
    shared = lambda z: z.unflatten(0, (hk, g)).sum(1).transpose(0, 1)
    dq, tq = ds @ K, eds @ K.abs()
    dk, tk = ds.transpose(1, 2) @ Q, eds.transpose(1, 2) @ Q.abs()
    dv, tv = p.transpose(1, 2) @ D, ep.transpose(1, 2) @ D.abs()
    dq, tq, dk, tk, dv, tv = dq.transpose(0, 1), tq.transpose(0, 1), shared(dk), shared(tk), shared(dv), shared(tv)
    return tuple((z, t + B * z.abs()) for z, t in ((dq, tq), (dk, tk), (dv, tv)))


def powers(a, n):
    """exp(a n), 1 where n is 0 whatever a is; [heads, ...]."""
    n = n.double()
    e = a.double().view(-1, *[1] * n.dim()) * n
    return torch.where(n == 0, 1.0, torch.exp(e))


CHUNK = 128


def held(y, z, w, s0, far, x):
    """What the tokens of a chunk (rows of x) take from the state that enters it, in absolute terms, for a state that is rounded before the
    product: sum_i |x_i| |S_ij| with S from the pairs of other chunks (weights w [H, t, s]) and the first state s0 (weights far)."""
    n, out = x.shape[1], [x[:, :0] @ s0]
    for c in range(0, n, CHUNK):
        rows, before = slice(c, min(c + CHUNK, n)), torch.ones(n, dtype=torch.bool, device=x.device)
        before[rows] = False
        # all rows of a chunk take the same state with one factor each: the first row (or the last, backwards) has the largest
        t = c if float(w[:, c, before].sum()) + float(far[:, c].sum()) >= float(w[:, rows.stop - 1, before].sum()) + float(far[:, rows.stop - 1].sum()) else rows.stop - 1
        s = (y[:, before] * w[:, t, before][..., None]).transpose(1, 2) @ z[:, before] + far[:, t, :, None] * s0
        out.append(x[:, rows].abs() @ s.abs())
    return torch.cat(out, 1)


def decay(q, k, v, a, state, scale=None):
    """out and the last state with their tolerances, for one sequence: q and k [n, H, d], v [n, H, dv], state [H, d, dv] or None."""
    n, H, d = q.shape
    scale = d ** -0.5 if scale is None else scale
    Q, K, V = heads_first(q), heads_first(k), heads_first(v)
    S0 = torch.zeros((H, d, v.shape[2]), dtype=torch.float64, device=q.device) if state is None else state.double()
    i = torch.arange(n, device=q.device)
    gap = i[:, None] - i
    w = torch.where(gap >= 0, powers(a, gap.clamp(min=0)), 0.0)
    x = (Q @ K.transpose(1, 2)) * w
    first = powers(a, i + 1)[..., None]
    out = (x @ V + first * (Q @ S0)) * scale
    terms = ((Q.abs() @ K.abs().transpose(1, 2)) * w) @ V.abs() + first * (Q.abs() @ S0.abs())
    tol = B * out.abs() + ((B * x.abs()) @ V.abs() + B * held(K, V, w, S0, first, Q) + F * terms) * abs(scale)
    wl = powers(a, n - 1 - i)[..., None]
    last = (K * wl).transpose(1, 2) @ V + powers(a, torch.tensor(n, device=q.device)).view(-1, 1, 1) * S0
    last_tol = 2.0 ** -14 * ((K * wl).abs().transpose(1, 2) @ V.abs() + powers(a, torch.tensor(n, device=q.device)).view(-1, 1, 1) * S0.abs())
    return out.transpose(0, 1), last, tol.transpose(0, 1), last_tol


def decay_grad(q, k, v, a, dout, state, dlast, scale=None):
    """[(gradient, tolerance)] of q, k, v and the first state, for one sequence."""
    n, H, d = q.shape
    scale = d ** -0.5 if scale is None else scale
    zero = torch.zeros((H, d, v.shape[2]), dtype=torch.float64, device=q.device)
    Q, K, V, D = heads_first(q), heads_first(k), heads_first(v), heads_first(dout)
    S0, R0 = (zero if x is None else x.double() for x in (state, dlast))
    i = torch.arange(n, device=q.device)
    gap = i[:, None] - i
    w = torch.where(gap >= 0, powers(a, gap.clamp(min=0)), 0.0)
    first, rest = powers(a, i + 1)[..., None], powers(a, n - 1 - i)[..., None]
    all_ = powers(a, torch.tensor(n, device=q.device)).view(-1, 1, 1)

    def part(x, y, z, weight, far, first_state, held_scale):
        """sum over pairs of (x.y) weight z, and what the held state brings"""
        s = (x @ y.transpose(1, 2)) * weight
        r = s @ z * scale + far * (x @ first_state) * held_scale
        terms = ((x.abs() @ y.abs().transpose(1, 2)) * weight) @ z.abs() * scale + far * (x.abs() @ first_state.abs()) * held_scale
        taken = held(y * scale, z, weight, first_state * held_scale, far, x)
        return r.transpose(0, 1), (B * r.abs() + (B * s.abs()) @ z.abs() * scale + B * taken + F * terms).transpose(0, 1)

    wt = w.transpose(1, 2)
    dq = part(D, V, K, w, first, S0.transpose(1, 2), scale)
    dk = part(V, D, Q, wt, rest, R0.transpose(1, 2), 1.0)
    dv = part(K, Q, D, wt, rest, R0, 1.0)
    ds = (Q * first).transpose(1, 2) @ D * scale + all_ * R0
    return dq, dk, dv, (ds, 2.0 ** -14 * ((Q * first).abs().transpose(1, 2) @ D.abs() * scale + all_ * R0.abs()))
