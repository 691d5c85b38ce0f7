"""What is measured of the training operators: the 8-bit activation checkpoints and the two losses.

``run`` computes an operator from ``prepare``'s state, in plain elementary torch operations in 32
bits (``own`` false) or through the package's entry points (``own`` true). ``exact`` gives the same
outputs from the definitions in 64 bits, written apart from the plain form.

Four operators, three listed cases each:

``policy``      clipped policy loss with a KL term over logits [rows, vocab], with its gradient
``preference``  paired preference loss over packed sequences, with its gradient
``act``         a (gated) activation whose inputs are kept in 8 bits, forward and backward
``wgrad``       a linear layer's input kept in 8 bits, and the weight gradient formed from it

The 8-bit format: groups of 32 neighbouring columns of a row share a power of two 2^e, e the
smallest integer >= -126 for which the group's largest magnitude is at most 127 * 2^e; a value is
kept as the integer round-half-even(x / 2^e). One byte for each value and one for each group.
"""
import math

import torch

own = False

DEV = "cuda"
GROUP = 32
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ---- cases ----------------------------------------------------------------------------------------

def listed():
    return [
        # one short sampled answer scored for its update: latency counts
        dict(name="policy 16 x 32768 bf16", op="policy", rows=16, vocab=32768, pad=0, dtype="bf16", kl=True, masked=0.0),
        # a micro-batch of answers, odd vocabulary so that rows start on no particular boundary, fp32 logits, no KL term
        dict(name="policy 2053 x 32001 f32", op="policy", rows=2053, vocab=32001, pad=0, dtype="f32", kl=False, masked=0.3),
        # a whole batch of answers over a large vocabulary
        dict(name="policy 8192 x 131072 bf16", op="policy", rows=8192, vocab=131072, pad=0, dtype="bf16", kl=True, masked=0.1),
        # one pair of short answers
        dict(name="preference 1 pair f32", op="preference", rows=96, pairs=1, vocab=32768, pad=0, dtype="f32", kind="sigmoid", masked=0.0),
        # pairs of different lengths whose prompts carry no weight, vocabulary padded in memory
        dict(name="preference 12 pairs bf16", op="preference", rows=4100, pairs=12, vocab=32001, pad=63, dtype="bf16", kind="squared", masked=0.4),
        # a large batch of pairs
        dict(name="preference 32 pairs bf16", op="preference", rows=16384, pairs=32, vocab=65536, pad=0, dtype="bf16", kind="sigmoid", masked=0.25),
        # a small layer, few tokens
        dict(name="act gelu 48 x 1024 f32", op="act", rows=48, cols=1024, dtype="f32", f="gelu", gated=False, fused=False),
        # gate and up from two projections, odd sizes
        dict(name="act silu*up 4099 x 2731 bf16", op="act", rows=4099, cols=2731, dtype="bf16", f="silu", gated=True, fused=False),
        # gate and up as the two halves of one projection's output, and their gradients likewise
        dict(name="act silu*up 16384 x 8192 bf16", op="act", rows=16384, cols=8192, dtype="bf16", f="silu", gated=True, fused=True),
        # a small projection, few tokens
        dict(name="wgrad 160 x 512 x 512 bf16", op="wgrad", rows=160, n_out=512, n_in=512, pad=0, dtype="bf16"),
        # fp32 activations, sizes that fill no tile
        dict(name="wgrad 4099 x 1000 x 2050 f32", op="wgrad", rows=4099, n_out=1000, n_in=2050, pad=0, dtype="f32"),
        # a square projection over a long batch, its output gradient a slice of a wider one
        dict(name="wgrad 16384 x 4096 x 4096 bf16", op="wgrad", rows=16384, n_out=4096, n_in=4096, pad=2048, dtype="bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["policy", "preference", "act", "wgrad"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    most = 1 << (30 if dtype == "bf16" else 29)
    if op == "policy":
        vocab = _log_int(rng, 300, 131072)
        rows = _log_int(rng, 1, min(8192, most // vocab))
        return dict(op=op, rows=rows, vocab=vocab, pad=rng.choice([0, 0, -vocab % 64]), dtype=dtype,
                    kl=rng.random() < 0.5, masked=rng.choice([0.0, 0.1, 0.5]))
    if op == "preference":
        vocab = _log_int(rng, 300, 65536)
        rows = _log_int(rng, 4, min(16384, most // vocab))
        return dict(op=op, rows=rows, pairs=_log_int(rng, 1, min(32, max(1, rows // 4))), vocab=vocab,
                    pad=rng.choice([0, 0, -vocab % 64]), dtype=dtype, kind=rng.choice(["sigmoid", "squared"]),
                    masked=rng.choice([0.0, 0.25, 0.5]))
    if op == "act":
        cols = _log_int(rng, 16, 8192)
        rows = _log_int(rng, 1, min(16384, (1 << (27 if dtype == "bf16" else 26)) // cols))
        gated = rng.random() < 0.6
        return dict(op=op, rows=rows, cols=cols, dtype=dtype, f=rng.choice(["gelu", "silu"]), gated=gated,
                    fused=gated and rng.random() < 0.5)
    rows, n_out, n_in = _log_int(rng, 1, 16384), _log_int(rng, 8, 4096), _log_int(rng, 8, 4096)
    if rng.random() < 0.6:  # most layers are multiples of something
        n_out, n_in = n_out + -n_out % 8, n_in + -n_in % 8
    if dtype == "f32":
        rows = max(1, rows // 3)
    return dict(op=op, rows=rows, n_out=n_out, n_in=n_in, pad=rng.choice([0, 0, 128]), dtype=dtype)


# ---- inputs ---------------------------------------------------------------------------------------

def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _logits(case, g):
    """Logits of a trained model: normal over the vocabulary, the taken token well above the rest."""
    rows, vocab, pitch = case["rows"], case["vocab"], case["vocab"] + case["pad"]
    whole = torch.randn(rows, pitch, generator=g, device=DEV, dtype=DTYPES[case["dtype"]])
    whole.mul_(2)
    logits = whole[:, :vocab]
    targets = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    near = math.log(vocab) + 2 + torch.randn(rows, generator=g, device=DEV)
    logits[torch.arange(rows, device=DEV), targets] = near.to(logits.dtype)
    return logits, targets


def _weights(case, g):
    keep = torch.rand(case["rows"], generator=g, device=DEV) >= case["masked"]
    keep[-1] = True
    return keep.float()


def _logp_now(logits, targets):
    """The policy's present log probabilities, a block of rows at a time."""
    out = []
    for z, y in zip(logits.split(512), targets.split(512)):
        z = z.float()
        top = z.amax(1, keepdim=True)
        out.append((z.gather(1, y[:, None]) - top)[:, 0] - (z - top).exp().sum(1).log())
    return torch.cat(out)


def prepare(case, seed):
    g = _generator(seed)
    dt = DTYPES[case["dtype"]]
    s = dict(case)
    if case["op"] in ("policy", "preference"):
        rows = case["rows"]
        s["logits"], s["targets"] = _logits(case, g)
        s["weights"] = _weights(case, g)
        logp = _logp_now(s["logits"], s["targets"])
        s["dlogits"] = torch.empty_strided(s["logits"].shape, s["logits"].stride(), dtype=dt, device=DEV)
        s["logp"] = torch.empty(rows, device=DEV)
        if case["op"] == "policy":
            s["weights"] /= s["weights"].sum()  # the mean over the answer's tokens
            # the policy that sampled was a few updates older; no ratio sits on the edge of the clip range, where rounding decides
            step = 0.15 * torch.randn(rows, generator=g, device=DEV)
            edge = ((step.exp() - 1).abs() - 0.2).abs() < 2e-3
            s["old_logp"] = logp - torch.where(edge, 0.5 * step, step)
            s["ref_logp"] = logp + 0.3 * torch.randn(rows, generator=g, device=DEV) if case["kl"] else None
            s["advantages"] = torch.randn(rows, generator=g, device=DEV)
            s["kl_coef"] = 0.05 if case["kl"] else 0.0
            s["totals"] = torch.empty(3, device=DEV)
        else:
            pairs = case["pairs"]
            cuts = torch.randint(0, rows + 1, (2 * pairs - 1,), generator=g, device=DEV)
            ends = torch.arange(1, 2 * pairs, device=DEV) * rows / (2 * pairs)  # lengths vary about the mean
            cuts = (0.5 * cuts + 0.5 * ends).long().sort().values
            edges = [torch.zeros(1, dtype=torch.long, device=DEV), cuts, torch.full((1,), rows, device=DEV)]
            s["seq_begin"] = torch.cat(edges)
            in_seq = _in_sequence(rows, s["seq_begin"])
            now = (in_seq * (s["weights"] * logp)).sum(1)
            s["ref_seq_logp"] = now + 4 * torch.randn(2 * pairs, generator=g, device=DEV)
            s["loss"] = torch.empty(1, device=DEV)
            s["margins"] = torch.empty(pairs, device=DEV)
            s["seq_logp"] = torch.empty(2 * pairs, device=DEV)
    elif case["op"] == "act":
        rows, cols = case["rows"], case["cols"]
        wide = 2 * cols if case["fused"] else cols
        scale = 1 + 3 * (torch.rand(wide, generator=g, device=DEV) < 0.02)  # a few loud channels
        s["x"] = (torch.randn(rows, wide, generator=g, device=DEV, dtype=dt) * scale).to(dt)
        s["dx"] = torch.empty(rows, wide, dtype=dt, device=DEV)
        s["up"] = s["dup"] = None
        if case["fused"]:
            s["x"], s["up"] = s["x"][:, :cols], s["x"][:, cols:]
            s["dx"], s["dup"] = s["dx"][:, :cols], s["dx"][:, cols:]
        elif case["gated"]:
            s["up"] = torch.randn(rows, cols, generator=g, device=DEV, dtype=dt)
            s["dup"] = torch.empty(rows, cols, dtype=dt, device=DEV)
        s["dy"] = 0.01 * torch.randn(rows, cols, generator=g, device=DEV, dtype=dt)
        s["y"] = torch.empty(rows, cols, dtype=dt, device=DEV)
        size = rows * (GROUP + 1) * -(-cols // GROUP)
        s["kept"] = torch.empty(size, dtype=torch.uint8, device=DEV)
        s["kept_up"] = torch.empty(size, dtype=torch.uint8, device=DEV) if case["gated"] else None
    else:
        rows, n_out, n_in = case["rows"], case["n_out"], case["n_in"]
        s["x"] = torch.randn(rows, n_in, generator=g, device=DEV, dtype=dt)
        dy = torch.randn(rows, n_out + case["pad"], generator=g, device=DEV, dtype=dt)
        s["dy"] = dy[:, :n_out]
        s["dw"] = torch.empty(n_out, n_in, device=DEV)
        s["kept"] = torch.empty(rows * (GROUP + 1) * -(-n_in // GROUP), dtype=torch.uint8, device=DEV)
    return s


# ---- plain forms ----------------------------------------------------------------------------------

def _in_sequence(rows, begin):
    at = torch.arange(rows, device=begin.device)
    return ((at >= begin[:-1, None]) & (at < begin[1:, None])).float()


def _plain_logp(s):
    z = s["logits"].float()
    top = z.amax(1, keepdim=True)
    e = (z - top).exp()
    total = e.sum(1, keepdim=True)
    picked = (z.gather(1, s["targets"][:, None]) - top)[:, 0]
    live = s["weights"] != 0
    return torch.where(live, picked - total.log()[:, 0], 0.0), e / total


def _plain_dlogits(s, probs, coef):
    d = -coef[:, None] * probs
    d.scatter_add_(1, s["targets"][:, None], coef[:, None])
    return torch.where((s["weights"] != 0)[:, None], d, 0.0).to(s["logits"].dtype)


def _plain_policy(s):
    logp, probs = _plain_logp(s)
    w, adv, beta = s["weights"], s["advantages"], s["kl_coef"]
    ratio = (logp - s["old_logp"]).exp()
    held = ratio.clamp(0.8, 1.2)
    gain, gain_held = ratio * adv, held * adv
    clipped = gain > gain_held
    slope = torch.where(clipped, 0.0, -gain)
    loss = -torch.minimum(gain, gain_held)
    kl = torch.zeros_like(loss)
    if s["ref_logp"] is not None:
        back = s["ref_logp"] - logp
        kl = back.exp() - back - 1
        slope = slope + beta * (1 - back.exp())
    live = w != 0
    totals = torch.stack([torch.where(live, w * v, 0.0).sum() for v in (loss + beta * kl, kl, clipped.float())])
    return {"totals": totals, "logp": logp, "dlogits": _plain_dlogits(s, probs, torch.where(live, w * slope, 0.0))}


def _plain_preference(s):
    logp, probs = _plain_logp(s)
    inside = _in_sequence(s["rows"], s["seq_begin"])
    seq_logp = (inside * (s["weights"] * logp)).sum(1)
    gap = seq_logp - s["ref_seq_logp"]
    h = gap[0::2] - gap[1::2]
    margin = 0.1 * h
    if s["kind"] == "sigmoid":
        each = torch.log1p((-margin.abs()).exp()) + (-margin).clamp(min=0)
        slope = -0.1 / (1 + margin.exp())
    else:
        each = (h - 5.0) ** 2
        slope = 2 * (h - 5.0)
    slope = slope / s["pairs"]
    per_seq = torch.stack([slope, -slope], 1).reshape(-1)
    coef = (inside * per_seq[:, None]).sum(0) * s["weights"]
    return {"loss": each.mean().reshape(1), "margins": margin, "seq_logp": seq_logp, "logp": logp,
            "dlogits": _plain_dlogits(s, probs, coef)}


def _plain_kept(x):
    """The values that a row's 8-bit groups stand for, in 32 bits."""
    rows, cols = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -cols % GROUP)).view(rows, -1, GROUP)
    frac, power = torch.frexp(x.abs().amax(2, keepdim=True))
    e = (power - 6 - (frac <= 127 / 128).int()).clamp(min=-126)
    unit, inverse = (((127 + k) << 23).view(torch.float32) for k in (e, -e))  # powers of two, exactly
    return ((x * inverse).round() * unit).view(rows, -1)[:, :cols]


def _plain_act(s):
    f = s["f"]

    def value_and_slope(x):
        if f == "silu":
            sig = 1 / (1 + (-x).exp())
            return x * sig, sig * (1 + x * (1 - sig))
        cdf = 0.5 * (1 + torch.erf(x * math.sqrt(0.5)))
        return x * cdf, cdf + x * (-0.5 * x * x).exp() * (1 / math.sqrt(2 * math.pi))

    dt, dy = s["x"].dtype, s["dy"].float()
    y = value_and_slope(s["x"].float())[0]
    kept, slope = value_and_slope(_plain_kept(s["x"]))
    if s["up"] is None:
        return {"y": y.to(dt), "dx": (dy * slope).to(dt)}
    up = _plain_kept(s["up"])
    return {"y": (y * s["up"].float()).to(dt), "dx": (dy * up * slope).to(dt), "dup": (dy * kept).to(dt)}


def _plain_wgrad(s):
    return {"dw": s["dy"].float().t() @ _plain_kept(s["x"])}


# ---- the package's operators ----------------------------------------------------------------------

def _own_policy(ss, s):
    ss.ss_policy_loss(s["logits"], s["targets"], s["old_logp"], s["ref_logp"], s["advantages"], s["weights"],
                      s["totals"], s["logp"], s["dlogits"], clip_low=0.2, clip_high=0.2, kl_coef=s["kl_coef"])
    return {"totals": s["totals"], "logp": s["logp"], "dlogits": s["dlogits"]}


def _own_preference(ss, s):
    kind = ss.SS_PREF_SIGMOID if s["kind"] == "sigmoid" else ss.SS_PREF_SQUARED
    ss.ss_preference_loss(s["logits"], s["targets"], s["weights"], s["seq_begin"], s["ref_seq_logp"], s["loss"],
                          s["margins"], s["seq_logp"], s["logp"], s["dlogits"], kind=kind, beta=0.1,
                          scale=1.0 / s["pairs"])
    return {k: s[k] for k in ("loss", "margins", "seq_logp", "logp", "dlogits")}


def _own_act(ss, s):
    f = ss.SS_ACT_SILU if s["f"] == "silu" else ss.SS_ACT_GELU
    ss.ss_act8_forward(s["x"], s["up"], f, s["y"], s["kept"], s["kept_up"])
    ss.ss_act8_backward(s["dy"], s["kept"], s["kept_up"], f, s["dx"], s["dup"])
    out = {"y": s["y"], "dx": s["dx"]}
    if s["dup"] is not None:
        out["dup"] = s["dup"]
    return out


def _own_wgrad(ss, s):
    ss.ss_act8_pack(s["x"], s["kept"])
    ss.ss_weight_grad8(s["dy"], s["kept"], s["dw"])
    return {"dw": s["dw"]}


def run(state):
    if own:
        from paper_1810_05291_b200 import binding as ss
        return {"policy": _own_policy, "preference": _own_preference, "act": _own_act, "wgrad": _own_wgrad}[state["op"]](ss, state)
    return {"policy": _plain_policy, "preference": _plain_preference, "act": _plain_act, "wgrad": _plain_wgrad}[state["op"]](state)


# ---- what a pass cannot do without ----------------------------------------------------------------

def work(case):
    eb = 2 if case["dtype"] == "bf16" else 4
    rows = case["rows"]
    if case["op"] in ("policy", "preference"):
        n = rows * case["vocab"]
        # rows of no weight need not be read; every row of the gradient is written
        per_row = 8 + 4 + 4 + (16 if case["op"] == "policy" else 0)
        return {"bytes": n * (1 - case["masked"]) * eb + n * eb + rows * per_row, "flops": 8.0 * n * (1 - case["masked"])}
    if case["op"] == "act":
        n = rows * case["cols"]
        tensors = 2 if case["gated"] else 1
        kept = tensors * n * (GROUP + 1) / GROUP
        # forward: inputs in, y and checkpoints out; backward: dy and checkpoints in, gradients out
        return {"bytes": n * eb * (tensors + 1) + kept + n * eb * (1 + tensors) + kept, "flops": 40.0 * n}
    n_out, n_in = case["n_out"], case["n_in"]
    kept = rows * n_in * (GROUP + 1) / GROUP
    return {"bytes": rows * n_in * eb + 2 * kept + rows * n_out * eb + 4 * n_out * n_in, "flops": 2.0 * rows * n_out * n_in}


# ---- the definitions in 64 bits -------------------------------------------------------------------

def _exact_rows(s, coef_of=None):
    """Log probabilities, and with `coef_of` (a coefficient for each row) the gradient, some rows at a time."""
    logp, grads = [], []
    block = max(1, (1 << 27) // s["vocab"])
    for at in range(0, s["rows"], block):
        rows = slice(at, at + block)
        z = s["logits"][rows].double()
        lse = torch.logsumexp(z, 1)
        y = s["targets"][rows]
        if coef_of is None:
            logp.append(z[torch.arange(len(y), device=z.device), y] - lse)
        else:
            p = torch.exp(z - lse[:, None])
            hit = torch.zeros_like(p)
            hit[torch.arange(len(y), device=z.device), y] = 1
            # float64 of the largest would not fit beside the rest: 32 bits are far below its type's own rounding
            d = coef_of[rows, None] * (hit - p)
            grads.append(d.float() if s["dtype"] == "bf16" else d)
    return torch.cat(logp) if coef_of is None else torch.cat(grads)


def _exact_kept(x):
    x = x.double()
    rows, cols = x.shape
    full = torch.zeros(rows, cols + -cols % GROUP, dtype=torch.float64, device=x.device)
    full[:, :cols] = x
    groups = full.view(rows, -1, GROUP)
    big = groups.abs().max(2, keepdim=True).values

    def two_to(e):
        return ((e + 1023) << 52).view(torch.float64)

    e = torch.floor(torch.log2(big.clamp(min=1e-300))).long() - 8  # too small by up to three steps
    for _ in range(4):
        e = torch.where(big > 127 * two_to(e), e + 1, e)
    unit = two_to(e.clamp(min=-126))
    return (torch.round(groups / unit) * unit).view(rows, -1)[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("policy", "preference"):
        w = s["weights"].double()
        logp = torch.where(w != 0, _exact_rows(s), 0)
        if case["op"] == "policy":
            adv, beta = s["advantages"].double(), s["kl_coef"]
            r = torch.exp(logp - s["old_logp"].double())
            gain = torch.min(r * adv, torch.clip(r, 0.8, 1.2) * adv)
            open_ = gain == r * adv
            kl, dkl = torch.zeros_like(r), torch.zeros_like(r)
            if case["kl"]:
                u = torch.exp(s["ref_logp"].double() - logp)
                kl, dkl = u - torch.log(u) - 1, 1 - u
            coef = w * (beta * dkl - open_ * adv * r)
            totals = torch.stack([(w * (beta * kl - gain)).sum(), (w * kl).sum(), (w * ~open_).sum()])
            return {"totals": totals, "logp": logp, "dlogits": _exact_rows(s, coef)}
        begin = s["seq_begin"].tolist()
        sums = torch.stack([(w[a:b] * logp[a:b]).sum() for a, b in zip(begin, begin[1:])])
        gap = sums - s["ref_seq_logp"].double()
        h = gap[::2] - gap[1::2]
        if case["kind"] == "sigmoid":
            each, slope = -torch.log(torch.sigmoid(0.1 * h)), -0.1 * torch.sigmoid(-0.1 * h)
        else:
            each, slope = (h - 5) ** 2, 2 * (h - 5)
        coef = torch.zeros_like(w)
        for k, (a, b) in enumerate(zip(begin, begin[1:])):
            coef[a:b] = w[a:b] * slope[k // 2] / case["pairs"] * (1 if k % 2 == 0 else -1)
        return {"loss": each.mean().reshape(1), "margins": 0.1 * h, "seq_logp": sums, "logp": logp,
                "dlogits": _exact_rows(s, coef)}
    kept = _exact_kept(s["x"])
    if case["op"] == "wgrad":
        return {"dw": torch.einsum("tn,tk->nk", s["dy"].double(), kept)}

    def value(x):
        return x * torch.sigmoid(x) if case["f"] == "silu" else x * torch.special.ndtr(x)

    def slope(x):
        if case["f"] == "silu":
            return torch.sigmoid(x) + x * torch.sigmoid(x) * torch.sigmoid(-x)
        return torch.special.ndtr(x) + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi)

    dy, y = s["dy"].double(), value(s["x"].double())
    if not case["gated"]:
        return {"y": y, "dx": dy * slope(kept)}
    up = _exact_kept(s["up"])
    return {"y": y * s["up"].double(), "dx": dy * up * slope(kept), "dup": dy * value(kept)}
