"""The cross entropy at the head in 64 bits, and how far its kernels may be from it."""
import torch


def head(x, w, y, k, c=1.0, z_coef=0.0, scale=1.0):
    x, w, k = x.double(), w.double(), k.double()
    vocab = w.shape[0]
    live = (k != 0) & (y >= 0) & (y < vocab)
    x = torch.where(live[:, None], x, torch.zeros_like(x))
    at = torch.where(live, y, torch.zeros_like(y))
    z = x @ w.t()
    lse = torch.logsumexp(c * z, 1)
    logp = torch.where(live, c * z.gather(1, at[:, None])[:, 0] - lse, 0.0)
    k = torch.where(live, k, 0.0)
    p = torch.exp(c * z - lse[:, None])
    hit = torch.zeros_like(p).scatter_(1, at[:, None], 1.0)
    grad = scale * c * k[:, None] * ((1 + 2 * z_coef * lse)[:, None] * p - hit)
    square = (k * lse * lse).sum()
    return {"totals": torch.stack([z_coef * square - (k * logp).sum(), square]), "logp": logp, "lse": lse, "live": live,
            "p": p, "hit": hit, "grad": grad, "dx": grad @ w, "dw": grad.t() @ x, "x": x, "k": k}


def head_bounds(x, w, y, k, want, c, z_coef, scale, dw_half):
    low = x.dtype == torch.bfloat16
    half = torch.finfo(x.dtype).eps / 2
    passes = 1 if low else 6
    ax, aw = want["x"].abs(), w.double().abs()
    rows, (vocab, width), unit = x.shape[0], w.shape, 2.0 ** -23
    size = (ax @ aw.t()).amax(1)
    n = passes * width
    e = 4 * (min(n, 1024) / 16 + n / 1024) * unit * size
    logp = 2 * c * e + 2.0 ** -15 + 2.0 ** -22 * want["lse"].abs()
    kk = want["k"].abs()
    totals = torch.stack([(kk * logp).sum() + abs(z_coef) * (kk * 2 * want["lse"].abs() * logp).sum(), (kk * 2 * want["lse"].abs() * logp).sum()])
    totals = totals + unit * want["totals"].abs()
    factor = abs(scale) * c * kk * (1 + 2 * abs(z_coef) * want["lse"].abs())
    rel = logp + (2.0 ** -11 + 2.0 ** -8 if low else 0.0) + 2.0 ** -20
    p = factor[:, None] * (rel[:, None] * want["p"] + (2.0 ** -25 if low else 0.0) + 2 * logp[:, None] * want["hit"])
    p = p + half * want["grad"].abs() + (0 if z_coef == 0 else abs(scale) * c * (kk * 2 * abs(z_coef) * logp)[:, None] * want["p"])
    size_p = want["grad"].abs() + p
    steps = lambda n: 4 * (min(passes * n, 16384) / 16 + passes * n / 2048 + 8) * unit  # noqa: E731
    dx = p @ aw + steps(vocab) * (size_p @ aw) + half * want["dx"].abs()
    dw = p.t() @ ax + steps(rows) * (size_p.t() @ ax) + dw_half * want["dw"].abs()
    tiny = 1e-37  # sums that the memory adds may lose subnormals
    return {"logp": torch.where(want["live"], logp, tiny), "totals": totals + tiny, "dx": dx + tiny, "dw": dw + tiny}
