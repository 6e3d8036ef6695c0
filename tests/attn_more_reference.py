"""Norms with rotation, cells of a cache and single-token attention over them, from their definitions in 64 bits, and the error that the
kernels' roundings may leave.

Tolerances count roundings as in attn_reference.py: B = 2^-8 of a value for a rounding to bf16.  E = 2^-18 of the sum of absolute terms stands
for fp32 arithmetic of a few operations on each of at most 128 terms: sums of 128 squares or products 2^-24 times 8 (a tree of 16 lanes with
8 terms each: 12 additions), the reciprocal root 2^-22, sine and cosine 2^-22 of 1, products and sums of a rotation 2^-22."""
import torch

from attn_reference import B, F

E = 2.0 ** -18


# ------------------------------------------------------------------------------------ rotation


def pairs_of(rot, interleaved, device):
    i = torch.arange(rot // 2, device=device)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def turned(y, positions, freq, interleaved, factor, back=False):
    """y [n, heads, d] in 64 bits."""
    if freq is None or freq.numel() == 0:
        return y
    a, b = pairs_of(2 * freq.numel(), interleaved, y.device)
    t = positions.double()[:, None] * freq.double()
    c, s = (factor * torch.cos(t))[:, None], (factor * torch.sin(t))[:, None] * (-1 if back else 1)
    out = y.clone()
    out[..., a], out[..., b] = y[..., a] * c - y[..., b] * s, y[..., b] * c + y[..., a] * s
    return out


def pair_sums(y, freq, interleaved, factor):
    """|y_a| + |y_b| in both places of a pair, |y| where there is none: the absolute terms of what is turned."""
    y = y.abs()
    if freq is None or freq.numel() == 0:
        return y
    a, b = pairs_of(2 * freq.numel(), interleaved, y.device)
    out = y.clone()
    out[..., a] = out[..., b] = (y[..., a] + y[..., b]) * abs(factor)
    return out


def normed(x, w, eps):
    if eps is None:
        return x
    n = x / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    return n if w is None else n * w.double()


def rotate(x, w, positions, freq, interleaved, eps, factor):
    """Result and tolerance of one table."""
    y = normed(x.double(), w, eps)
    out = turned(y, positions, freq, interleaved, factor)
    return out, B * out.abs() + E * pair_sums(y, freq, interleaved, factor)


def rotate_grad(x, w, dy, positions, freq, interleaved, eps, factor):
    """((dx, tolerance), (dw, tolerance) or None) of one table."""
    x, dy = x.double(), dy.double()
    g, size = turned(dy, positions, freq, interleaved, factor, back=True), pair_sums(dy, freq, interleaved, factor)
    if eps is None:
        return (g, B * g.abs() + E * size), None
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    n, weight = x * r, 1.0 if w is None else w.double()
    gw, sw = g * weight, size * abs(weight)
    dx = r * (gw - n * (gw * n).mean(-1, keepdim=True))
    tol = B * dx.abs() + E * r * (sw + n.abs() * (sw * n.abs()).mean(-1, keepdim=True))
    # a column's sum: a lane adds up its rows, then 16 lanes' sums, then the blocks' in 32 strands: fewer than 2^8 additions in a row each
    return (dx, tol), ((g * n).sum((0, 1)), 2.0 ** -16 * (size * n.abs()).sum((0, 1)))


# --------------------------------------------------------------------------------------- cells

TINY = 2.0 ** -100


def divided(a, b):
    """A quotient of two tensors, rounded once."""
    return torch.div(a, b)


def quantise(x, bits):
    """Cells and scales as the header defines them, each operation in fp32."""
    x = x.float()
    nan = torch.full((), float("nan"), device=x.device)
    if bits == 8:
        most = x.abs().amax(-1, keepdim=True)
        fine = torch.isfinite(x).all(-1, keepdim=True)
        some = fine & (most >= TINY)
        safe = torch.where(some, most, 1.0)
        scale = torch.where(some, divided(safe, torch.full_like(safe, 127.0)), torch.where(fine, 0.0, nan))
        cells = torch.where(some, torch.round(torch.where(some, x, 0.0) * divided(torch.full_like(safe, 127.0), safe)), 0.0)
        return cells.to(torch.int8), scale.squeeze(-1)
    d = x.shape[-1]
    cells, scales = [], []
    for part in x.split(32, -1):
        lo, hi = part.amin(-1, keepdim=True), part.amax(-1, keepdim=True)
        told = divided(hi - lo, torch.full_like(lo, 15.0)).to(torch.bfloat16).float()
        fine = torch.isfinite(part).all(-1, keepdim=True) & torch.isfinite(told)
        some = fine & (told >= TINY)
        step = torch.where(some, told, 1.0)
        c = torch.round((part - lo) * divided(torch.ones_like(step), step)).clamp(0, 15)
        cells.append(torch.where(some, c, 0.0).nan_to_num(0.0))
        scales.append(torch.cat([torch.where(some, told, torch.where(fine, 0.0, nan)), torch.where(fine, lo, nan)], -1))
    c = torch.cat(cells, -1).to(torch.uint8)
    assert c.shape[-1] == d
    return (c[..., 0::2] | (c[..., 1::2] << 4)).contiguous(), torch.stack(scales, -2).to(torch.bfloat16)


def parts_of(cells, scales, bits):
    """(base, rest) in 64 bits whose sum is what cells stand for; rest is what is multiplied by whole numbers."""
    if bits == 16:
        return torch.zeros_like(cells, dtype=torch.float64), cells.double()
    if bits == 8:
        return torch.zeros(cells.shape, dtype=torch.float64, device=cells.device), cells.double() * scales.double()[..., None]
    q = torch.stack([cells & 15, cells >> 4], -1).flatten(-2).double()
    step, lo = (scales[..., i].double().repeat_interleave(32, -1)[..., : q.shape[-1]] for i in (0, 1))
    return lo, step * q


def values(cells, scales, bits):
    """What cells stand for, rounded to bf16 once: the product and the sum are exact or rounded once in fp32."""
    if bits == 16:
        return cells
    if bits == 8:
        return (cells.float() * scales[..., None]).to(torch.bfloat16)
    lo, rest = parts_of(cells, scales, bits)
    return (lo + rest).float().to(torch.bfloat16)


# --------------------------------------------------------------------------------------- steps


def attend(q, k, v, scale=None):
    """out and tolerance of one token's heads q [H, d] over keys and values given as (base, rest) [n, Hk, d]."""
    H, d = q.shape
    group = H // k[0].shape[1]
    scale = d ** -0.5 if scale is None else scale
    if k[0].shape[0] == 0:
        return torch.zeros((H, d), dtype=torch.float64, device=q.device), torch.zeros((H, d), dtype=torch.float64, device=q.device)
    Q = q.double()[:, None]
    (k0, k1), (v0, v1) = (tuple(z.repeat_interleave(group, 1).transpose(0, 1) for z in x) for x in (k, v))
    x = (Q @ (k0 + k1).transpose(1, 2) * scale).squeeze(1)
    p = torch.softmax(x, -1)[:, None]
    out = p @ (v0 + v1)
    size = p @ (v0.abs() + v1.abs())
    # a score's error is its weight's relative error: fp32 sums of 128 terms, then of up to 4 groups
    off = E * abs(scale) * (Q.abs() @ (k0.abs() + k1.abs()).transpose(1, 2)).amax(-1)
    tol = B * (p @ v1.abs()) + B * out.abs() + (F + 2 * off[..., None]) * size
    return out.squeeze(1), tol.squeeze(1)
