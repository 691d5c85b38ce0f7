"""How far the head's fp32 results may be from the formulas in the 2-norm, over many elements.

A sum of n contraction indices takes n / 16 steps of the matrix unit, each of which cuts the sum off: by 0.36 2^-23 of it on average (half a unit, which is 0.72
2^-23 of a number in the mean), always towards zero, and the sum grows with the root of the steps, so that 2/3 of n / 16 full ones count. Of the
six passes of fp32 only the last sees a large sum. A sum leaves the matrix unit after 128 indices of an fp32 logit, 768 (128 with few rows) of a bf16 one, 1024 of an fp32 gradient.
Twice the mean is allowed.

An entry of P besides has the error of its exponent, at most (4 |t| + 16) 2^-24 with |t| about 8 where the weight lies: 48 2^-24, a uniform error in the mean 28 2^-24,
below 2^-19; the rest of its way (the row's sum, the factor, the last rounding) as much. So gradients: 2 0.36 2/3 min(n, 1024) / 16 2^-23 + 2^-18, which is 7.5e-6 with long sums.
log p: the same share for its logit and the sum of all, each times its size, and 2^-21 of what is left (exponentials in the sum, logarithm, last rounding)."""
import torch

CUT = 2 * 0.36 * 2 / 3 * 2.0 ** -23


def gradient_bound(n):
    return CUT * min(n, 1024) / 16 + 2.0 ** -18


def logp_bound(n, low, rows):
    """Of |target's logit| + |largest logit| + |log p|, row by row, in the 2-norm."""
    return CUT * min(n, 768 if low and rows > 128 else 128) / 16 + 2.0 ** -21


def off(got, want):
    return float((got.double() - want).norm() / want.norm().clamp(min=1e-300))


def logp_size(x, w, y, want):
    z = want["x"] @ w.double().t()
    live = want["live"]
    size = z.gather(1, torch.where(live, y, 0)[:, None])[:, 0].abs() + z.abs().amax(1) + want["logp"].abs()
    return torch.where(live, size, torch.zeros_like(size))
