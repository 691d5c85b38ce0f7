"""What is measured of the two ends of a training step: the loss at a language model's head, and the
update of its matrices.

``run`` computes an operator from ``prepare``'s state, in plain elementary torch operations in 32
bits (``own`` false) or through the package's entry points (``own`` true). ``exact`` gives the same
outputs from the definitions in 64 bits, written apart from the plain form.

Two operators:

``head``   softmax cross entropy of x W^T over a large vocabulary, from the hidden states x and the
           head W, with the gradients of both (or the loss alone)
``ortho``  the update of matrices by their momentum with all singular values drawn towards 1:
           X <- a X + (b X X^T + c (X X^T)^2) X, some steps, from the momentum over its norm; alone,
           or with the momentum's and the parameter's update around it
"""
import math

import torch

own = False

DEV = "cuda"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
COEFFICIENTS = (3.4445, -4.7750, 2.0315)
STEPS = 5
BETA, LR, DECAY = 0.95, 3e-4, 0.1


# ---- cases ----------------------------------------------------------------------------------------

def listed():
    return [
        # a short answer in a small model: latency counts
        dict(name="head 64 x 1024 over 32000 bf16", op="head", rows=64, width=1024, vocab=32000, pad=0, dtype="bf16", grad=True, masked=0.0, z=0.0),
        # a batch scored without a gradient, odd vocabulary
        dict(name="head loss 2048 x 2048 over 50257 bf16", op="head", rows=2048, width=2048, vocab=50257, pad=0, dtype="bf16", grad=False, masked=0.0, z=0.0),
        # everything in 32 bits, odd sizes
        dict(name="head 1021 x 770 over 32001 f32", op="head", rows=1021, width=770, vocab=32001, pad=0, dtype="f32", grad=True, masked=0.1, z=0.0),
        # prompts and answers: positions of the prompts carry no weight; hidden states a part of wider rows; the z term
        dict(name="head 4100 x 2048 over 65536 bf16", op="head", rows=4100, width=2048, vocab=65536, pad=64, dtype="bf16", grad=True, masked=0.4, z=1e-4),
        # a whole micro-batch over a large vocabulary
        dict(name="head 8192 x 4096 over 131072 bf16", op="head", rows=8192, width=4096, vocab=131072, pad=0, dtype="bf16", grad=True, masked=0.0, z=0.0),
        # one small matrix: latency counts
        dict(name="ortho 128 x 128 f32", op="ortho", count=1, rows=128, cols=128, dtype="f32", step=False, nesterov=False),
        # the classifier of the ResNet-50 that the framework is measured with, whole step
        dict(name="ortho step 1000 x 2048 f32", op="ortho", count=1, rows=1000, cols=2048, dtype="f32", step=True, nesterov=True),
        # its three largest convolutions, 512 x 512 x 3 x 3, whole step
        dict(name="ortho step 3 of 512 x 4608 f32", op="ortho", count=3, rows=512, cols=4608, dtype="f32", step=True, nesterov=False),
        # an odd tall matrix
        dict(name="ortho 2731 x 1001 bf16", op="ortho", count=1, rows=2731, cols=1001, dtype="bf16", step=False, nesterov=False),
        # the same projection of twelve layers, whole step
        dict(name="ortho step 12 of 4096 x 1024 bf16", op="ortho", count=12, rows=4096, cols=1024, dtype="bf16", step=True, nesterov=True),
        # one large square projection
        dict(name="ortho 4096 x 4096 bf16", op="ortho", count=1, rows=4096, cols=4096, dtype="bf16", step=False, nesterov=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.5:
        dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
        vocab = _log_int(rng, 300, 131072)
        width = _log_int(rng, 32, 4096 if dtype == "bf16" else 1024)
        if rng.random() < 0.8:  # most are multiples of something
            width = min(4096, width + -width % 64)
        most = (1 << 42) // (4 if dtype == "f32" else 1)
        rows = _log_int(rng, 1, max(2, min(8192, most // (vocab * width))))
        return dict(op="head", rows=rows, width=width, vocab=vocab, pad=rng.choice([0, 0, 64, 3]), dtype=dtype,
                    grad=rng.random() < 0.8, masked=rng.choice([0.0, 0.0, 0.1, 0.5]), z=rng.choice([0.0, 1e-4]))
    rows, cols = _log_int(rng, 32, 4096), _log_int(rng, 32, 4096)
    if rng.random() < 0.6:
        rows, cols = rows + -rows % 32, cols + -cols % 32
    count = _log_int(rng, 1, max(1, min(12, (1 << 25) // (rows * cols))))
    return dict(op="ortho", count=count, rows=min(rows, 4096), cols=min(cols, 4096), dtype=rng.choice(["bf16", "f32"]),
                step=rng.random() < 0.5, nesterov=rng.random() < 0.5)


# ---- inputs ---------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _prepare_head(case, g, s):
    rows, width, vocab, dt = case["rows"], case["width"], case["vocab"], DTYPES[case["dtype"]]
    s["w"] = torch.randn(vocab, width, generator=g, device=DEV, dtype=dt).mul_(2 * width ** -0.5)
    s["targets"] = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    # hidden states of a trained model: normal logits, the right token's well above the rest
    taken = s["w"][s["targets"]].float()
    lift = (math.log(vocab) + 2 + torch.randn(rows, generator=g, device=DEV)) / taken.square().sum(1).clamp(min=1e-3)
    wide = torch.randn(rows, width + case["pad"], generator=g, device=DEV, dtype=dt)
    wide[:, :width] = (wide[:, :width].float() + lift[:, None] * taken).to(dt)
    s["x"] = wide[:, :width]
    keep = (torch.rand(rows, generator=g, device=DEV) >= case["masked"]).float()
    keep[-1] = 1
    s["weights"] = keep / keep.sum()
    s["totals"], s["logp"] = torch.empty(2, device=DEV), torch.empty(rows, device=DEV)
    s["dx"] = torch.empty(rows, width, dtype=dt, device=DEV) if case["grad"] else None
    s["dw"] = torch.empty(vocab, width, dtype=dt, device=DEV) if case["grad"] else None


def _prepare_ortho(case, g, s):
    count, rows, cols, dt = case["count"], case["rows"], case["cols"], DTYPES[case["dtype"]]

    def gradients(size):
        """A few strong directions over noise, as gradients of matrices have them."""
        k = min(16, rows, cols)
        u, v = (torch.randn(count, n, k, generator=g, device=DEV) for n in (rows, cols))
        strength = 3 * size / torch.arange(1, k + 1, device=DEV)
        return [m.to(dt) for m in (u * strength) @ v.transpose(1, 2) + size * torch.randn(count, rows, cols, generator=g, device=DEV)]

    s["in"] = gradients(1e-3)
    if case["step"]:
        s["v"] = [m.float() for m in gradients(5e-4)]
        s["p"] = list(torch.randn(count, rows, cols, generator=g, device=DEV) * cols ** -0.5)
        s["v_out"], s["p_out"] = ([torch.empty(rows, cols, device=DEV) for _ in range(count)] for _ in range(2))
        s["scale"] = 0.2 * max(rows, cols) ** 0.5
    else:
        s["out"] = [torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV) for _ in range(count)]


def prepare(case, seed):
    s = dict(case)
    (_prepare_head if case["op"] == "head" else _prepare_ortho)(case, _generator(seed), s)
    return s


# ---- plain forms ----------------------------------------------------------------------------------

def _plain_head(s):
    x, w, weights = s["x"].float(), s["w"].float(), s["weights"]
    live = weights != 0
    z = x @ w.t()
    top = z.amax(1, keepdim=True)
    e = (z - top).exp()
    total = e.sum(1, keepdim=True)
    lse = (top + total.log())[:, 0]
    logp = torch.where(live, (z.gather(1, s["targets"][:, None]) - top)[:, 0] - total.log()[:, 0], 0.0)
    del z
    square = torch.where(live, weights * lse * lse, 0.0).sum()
    out = {"totals": torch.stack([s["z"] * square - (weights * logp).sum(), square]), "logp": logp}
    if s["grad"]:
        p = e.div_(total)
        p.mul_((weights * (1 + 2 * s["z"] * lse))[:, None])
        p.scatter_add_(1, s["targets"][:, None], -weights[:, None])
        p = torch.where(live[:, None], p, 0.0)
        out["dx"], out["dw"] = (p @ w).to(s["x"].dtype), (p.t() @ x).to(s["w"].dtype)
    return out


def _plain_orthogonal(u):
    a, b, c = COEFFICIENTS
    x = u / u.square().sum().sqrt()
    tall = x.shape[0] > x.shape[1]
    if tall:
        x = x.t()
    for _ in range(STEPS):
        s = x @ x.t()
        x = a * x + (b * s + c * (s @ s)) @ x
    return x.t() if tall else x


def _plain_ortho(s):
    if not s["step"]:
        return {"out": [_plain_orthogonal(m.float()).to(torch.bfloat16) for m in s["in"]]}
    out = {"v": [], "p": []}
    for g, v, p in zip(s["in"], s["v"], s["p"]):
        g = g.float()
        v = BETA * v + (1 - BETA) * g
        o = _plain_orthogonal(BETA * v + (1 - BETA) * g if s["nesterov"] else v)
        out["v"].append(v)
        out["p"].append(p - LR * (s["scale"] * o + DECAY * p))
    return out


# ---- the package's operators ----------------------------------------------------------------------

def _own_head(ss, s):
    ss.ss_linear_cross_entropy(s["x"], s["w"], s["targets"], s["weights"], s["totals"], s["logp"], s["dx"], s["dw"], z_coef=s["z"])
    out = {"totals": s["totals"], "logp": s["logp"]}
    if s["grad"]:
        out["dx"], out["dw"] = s["dx"], s["dw"]
    return out


def _own_ortho(ss, s):
    coefficients = [COEFFICIENTS] * STEPS
    if not s["step"]:
        ss.ss_orthogonalise(s["in"], s["out"], coefficients)
        return {"out": s["out"]}
    ss.ss_orthogonal_update(s["in"], s["v"], s["v_out"], s["p"], s["p_out"], beta=BETA, nesterov=s["nesterov"],
                            coefficients=coefficients, lr=LR, scale=s["scale"], weight_decay=DECAY)
    return {"v": s["v_out"], "p": s["p_out"]}


def run(state):
    if own:
        from paper_1810_05291_b200 import binding as ss
        return (_own_head if state["op"] == "head" else _own_ortho)(ss, state)
    return (_plain_head if state["op"] == "head" else _plain_ortho)(state)


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    eb = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "head":
        rows, width, vocab = case["rows"], case["width"], case["vocab"]
        live = max(1.0, rows * (1 - case["masked"]))  # positions without weight need not be read
        moved = (live + vocab) * width * eb + rows * 16 + 8
        if case["grad"]:
            moved += (rows + vocab) * width * eb
        return {"bytes": moved, "flops": (6.0 if case["grad"] else 2.0) * live * vocab * width}
    n = case["count"] * case["rows"] * case["cols"]
    small, large = sorted((case["rows"], case["cols"]))
    # both symmetric products by half, the third whole
    flops = case["count"] * STEPS * (3.0 * small * small * large + small ** 3)
    return {"bytes": n * (eb + 16) if case["step"] else n * (eb + 2), "flops": flops}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def _exact_head(s):
    w, c = s["w"].double(), s["weights"].double()
    rows, vocab = s["rows"], s["vocab"]
    logp, lse = torch.zeros(rows, dtype=torch.float64, device=DEV), torch.zeros(rows, dtype=torch.float64, device=DEV)
    dx = torch.zeros(rows, s["width"], dtype=torch.float64, device=DEV)
    dw = torch.zeros_like(w)
    at = torch.nonzero(c)[:, 0]
    for part in at.split(max(1, (1 << 26) // vocab)):
        x, y, k = s["x"][part].double(), s["targets"][part], c[part]
        logits = torch.einsum("td,vd->tv", x, w)
        lse[part] = torch.logsumexp(logits, 1)
        own_place = torch.arange(len(part), device=DEV)
        logp[part] = logits[own_place, y] - lse[part]
        if s["grad"]:
            d = torch.exp(logits - lse[part][:, None])
            d *= (1 + 2 * s["z"] * lse[part])[:, None]
            d[own_place, y] -= 1
            d *= k[:, None]
            dx[part] = d @ w
            dw += d.t() @ x
    square = (c * lse * lse).sum()
    out = {"totals": torch.stack([s["z"] * square - (c * logp).sum(), square]), "logp": logp}
    if s["grad"]:
        # float64 of the largest would not fit beside the rest: 32 bits are far below its type's own rounding
        out["dx"], out["dw"] = dx, dw.float() if s["dtype"] == "bf16" else dw
    return out


def _exact_orthogonal(m):
    a, b, c = COEFFICIENTS
    m = m / torch.linalg.vector_norm(m)
    for _ in range(STEPS):
        if m.shape[0] <= m.shape[1]:
            s = m @ m.t()
            m = a * m + b * (s @ m) + c * (s @ (s @ m))
        else:
            s = m.t() @ m
            m = a * m + b * (m @ s) + c * ((m @ s) @ s)
    return m


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "head":
        return _exact_head(s)
    if not case["step"]:
        return {"out": [_exact_orthogonal(m.double()) for m in s["in"]]}
    v = [0.95 * v.double() + 0.05 * g.double() for g, v in zip(s["in"], s["v"])]
    u = [0.95 * m + 0.05 * g.double() for g, m in zip(s["in"], v)] if case["nesterov"] else v
    p = [p.double() * (1 - LR * DECAY) - LR * s["scale"] * _exact_orthogonal(m) for p, m in zip(s["p"], u)]
    return {"v": v, "p": p}
