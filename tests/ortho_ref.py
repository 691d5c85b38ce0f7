"""The orthogonal update in 64 bits, and the same with the kernels' roundings of the operands."""
import torch

COEFFICIENTS = ((3.4445, -4.7750, 2.0315),) * 5


def _half(x):
    return x.half().double()


def orthogonalised(u, coefficients=COEFFICIENTS, rounded=False):
    """With ``rounded``: operands in fp16, scaled as the kernels scale them; X itself is not rounded."""
    u = u.double()
    norm = u.square().sum().sqrt()
    x = torch.zeros_like(u) if float(norm) == 0 else u / norm
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t()
    power = 0
    while 4 ** (power + 1) <= max(x.shape):
        power += 1
    scale = 2.0 ** power
    for a, b, c in coefficients:
        if rounded:
            op = _half(x * scale) / scale
            s = _half(op @ op.t())
            x = a * x + _half(b * s + c * (s @ s)) @ op
        else:
            s = x @ x.t()
            x = a * x + (b * s + c * (s @ s)) @ x
    return x.t() if tall else x


def updated(g, v, p, beta, nesterov, lr, scale, decay, coefficients=COEFFICIENTS, rounded=False):
    g, v, p = g.double(), v.double(), p.double()
    v = (1 - beta) * g + beta * v
    o = orthogonalised((1 - beta) * g + beta * v if nesterov else v, coefficients, rounded)
    return v, p - lr * (scale * o + decay * p)
