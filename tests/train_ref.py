"""Plain 64-bit implementations of the training operators, for their tests."""
import math

import torch

GROUP = 32
NAN = float("nan")


def two_to(e):
    """2^e in float64 for an int64 tensor e, by its bits."""
    return ((e + 1023) << 52).view(torch.float64)


def act8(x):
    """(codes [rows, 32 G] uint8, exponents [rows, G] uint8, decoded values [rows, cols] float64)."""
    rows, cols = x.shape
    groups = -(-cols // GROUP)
    full = torch.zeros(rows, groups * GROUP, dtype=torch.float64, device=x.device)
    full[:, :cols] = x.double()
    full = full.view(rows, groups, GROUP)
    a = full.abs().amax(2)
    bad = ~(a < 2.0 ** 126) | torch.isnan(full).any(2)
    safe = torch.where(bad, torch.ones_like(a), a)
    e = torch.full(a.shape, -126, dtype=torch.int64, device=x.device)
    for k in range(-126, 121):  # the smallest e with a <= 127 * 2^e
        e = torch.where(safe > 127.0 * 2.0 ** (k - 1), torch.full_like(e, k), e) if k > -126 else e
    unit = two_to(e)[:, :, None]
    q = torch.round(torch.where(bad[:, :, None], torch.zeros_like(full), full) / unit)
    codes = (q.abs().to(torch.int64) | (torch.signbit(full).to(torch.int64) << 7)).to(torch.uint8)
    value = torch.where(bad[:, :, None], torch.full_like(full, NAN), q * unit)
    exps = torch.where(bad, torch.full_like(e, 255), e + 127).to(torch.uint8)
    return codes.view(rows, -1), exps, value.view(rows, -1)[:, :cols], bad


def act(name, x):
    """f(x) and f'(x)."""
    if name == "silu":
        s = torch.sigmoid(x)
        return x * s, s + x * s * (1 - s)
    cdf = 0.5 * torch.special.erfc(-x / math.sqrt(2))
    return x * cdf, cdf + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)


def token_logp(z, targets, weights, c=1.0):
    """(logp with 0 in the rows left out, softmax, rows that count)."""
    vocab = z.shape[1]
    live = (weights != 0) & (targets >= 0) & (targets < vocab)
    y = torch.where(live, targets, torch.zeros_like(targets))
    t = z.double() * c
    if vocab:  # log p does not change with a shift; without it a row of -3e38 would swallow log(vocab), in 64 bits too
        top = t.amax(1, keepdim=True)
        t = torch.where(torch.isfinite(top), t - top, t)
    lse = torch.logsumexp(t, 1) if vocab else torch.zeros(len(z), dtype=torch.float64, device=z.device)
    logp = (t.gather(1, y[:, None])[:, 0] - lse) if vocab else lse
    # a row of nothing but -inf, or with +inf, has no softmax
    p = torch.exp(t - lse[:, None])
    hit = torch.zeros_like(p)
    if vocab:
        hit.scatter_(1, y[:, None], 1.0)
    return torch.where(live, logp, torch.zeros_like(logp)), p, hit, live


def rows_grad(p, hit, live, slope, c):
    d = c * slope[:, None] * (hit - p)
    return torch.where(live[:, None], d, torch.zeros_like(d))


def policy(z, targets, old, ref, adv, w, c, lo, hi, beta):
    logp, p, hit, live = token_logp(z, targets, w, c)
    w, adv = w.double(), adv.double()
    r = torch.exp(logp - old.double())
    plain, held = r * adv, r.clamp(1.0 - lo, 1.0 + hi) * adv
    clipped = plain > held
    kl, dkl = torch.zeros_like(r), torch.zeros_like(r)
    if ref is not None:
        u = torch.exp(ref.double() - logp)
        kl, dkl = u - (ref.double() - logp) - 1, 1 - u
    zero = torch.zeros_like(r)
    each = [w * (beta * kl - torch.minimum(plain, held)), w * kl, w * clipped]
    totals = torch.stack([torch.where(live, v, zero).sum() for v in each])
    slope = torch.where(live, w * (torch.where(clipped, zero, -plain) + beta * dkl), zero)
    return totals, logp, rows_grad(p, hit, live, slope, c)


def preference(z, targets, w, begin, ref, c, kind, beta, smoothing, scale):
    logp, p, hit, live = token_logp(z, targets, w, c)
    w = torch.where(live, w.double(), torch.zeros_like(logp))
    begin = begin.tolist()
    sums = torch.stack([(w[a:b] * logp[a:b]).sum() for a, b in zip(begin, begin[1:])]) if len(begin) > 1 else logp[:0]
    gap = sums - ref.double()
    h = gap[0::2] - gap[1::2]
    m = beta * h
    sp = torch.nn.functional.softplus
    if kind == 0:
        each = (1 - smoothing) * sp(-m) + smoothing * sp(m)
        slope = beta * (smoothing * torch.sigmoid(m) - (1 - smoothing) * torch.sigmoid(-m))
    elif kind == 1:
        each, slope = (1 - m).clamp(min=0), torch.where(m < 1, -beta, 0.0).double()
    else:
        each, slope = (h - 1 / (2 * beta)) ** 2, 2 * (h - 1 / (2 * beta))
    per_row = torch.zeros_like(w)
    for k, (a, b) in enumerate(zip(begin, begin[1:])):
        per_row[a:b] = scale * slope[k // 2] * (1 if k % 2 == 0 else -1)
    return scale * each.sum(), m, sums, logp, rows_grad(p, hit, live, per_row * w, c)
