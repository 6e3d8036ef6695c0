"""How far the results of a step may be off in the root mean square, when nothing but the roundings that the kernels state is left.

A result is rounded to bf16 once: of a value between 2^e and 2^(e+1) by an error spread evenly over one step of 2^(e-7), whose mean square is a twelfth of the step's
square.  The weights are rounded before they meet the values: to two bf16 numbers, 2^-16 of a weight at most (2^-8 of a remainder that is 2^-8 of it), or
to one fp16 number, 2^-11.  Errors of that size spread evenly have a third of its square, and those of different keys are independent: they add up to the
sum of the squares of weight times value.  fp32 sums, scores and exponentials, 2^-18 and less of a term, are left out; MORE stands for them, and for
what a mean over some ten thousand results is off by chance (1 % of its root)."""
import torch

TWO_BF16, ONE_FP16, ONE_BF16 = 2.0 ** -16, 2.0 ** -11, 2.0 ** -8
MORE = 1.1


def attend(q, k, v, scale=None):
    """Results of one token's heads q [H, d] in 64 bits, keys and values given as (base, rest) [n, Hk, d], and the sums of (weight times rest)^2."""
    group = q.shape[0] // k[0].shape[1]
    scale = q.shape[1] ** -0.5 if scale is None else scale
    (k0, k1), (v0, v1) = (tuple(z.double().repeat_interleave(group, 1).transpose(0, 1) for z in x) for x in (k, v))
    p = torch.softmax((q.double()[:, None] @ (k0 + k1).transpose(1, 2)) * scale, -1)
    return (p @ (v0 + v1)).squeeze(1), ((p * p) @ (v1 * v1)).squeeze(1)


def step_of(x):
    """The step of bf16 numbers at x."""
    return torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -126))) - 7)


def bound(out, squares, weight):
    """Root mean square that the errors of results `out` stay below."""
    return MORE * float((step_of(out).square().mean() / 12 + weight ** 2 / 3 * squares.mean()).sqrt())


def error(got, out):
    return float((got.double() - out).square().mean().sqrt())
