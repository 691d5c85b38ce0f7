"""The training operators on the GPU against plain 64-bit implementations.

Tolerances, derived from the arithmetic:
* 8-bit checkpoints are exact: the scales are powers of two and the rounding is the definition's.
* An fp32 result formed by a handful of rounded operations (each 2^-24, functions a few units in
  the last place) is within 1e-6 of the terms it is made of; a bf16 result adds half a unit of its
  last place, at most 2^-8 of the value (8 significant bits).
* dW: products of a bf16 value (or of the three bf16 terms of an fp32 one) with a decoded value
  are exact in fp32. Sums in the matrix unit truncate: at most 2^-23 of the partial sum for each
  of the 32 steps of 16 rows between two promotions, and 2^-23 of the largest term in the
  alignment of each step, so 64 * 2^-23 of sum |dy x^| bounds an element. (Written when a promotion
  came every 32 steps. It comes every 128 now; the tolerance is kept, though the worst case
  is four times as large: terms of both signs come nowhere near it.)
* log probabilities: a difference of numbers of the size of the row's largest |c z| and of
  log(vocab), each rounded to 2^-24 a few times: 1e-6 * (max |c z| + log(vocab) + 1).
"""
import math

import pytest
import torch

from paper_1810_05291_b200 import binding as B
from tests import train_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16_HALF = 2.0 ** -8
DTYPES = [torch.float32, torch.bfloat16]
IDS = ["f32", "bf16"]
ACTS = {"gelu": B.SS_ACT_GELU, "silu": B.SS_ACT_SILU}


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


class Guarded:
    """A [rows, cols] view inside a larger filled buffer; check() finds writes outside the view."""

    def __init__(self, rows, cols, dtype, stride=None, offset=0, fill=77.0):
        stride = cols if stride is None else stride
        self.full = torch.full((rows * stride + offset + 64,), fill, dtype=dtype, device=DEV)
        self.view = self.full[32 + offset:].as_strided((rows, cols), (stride, 1))
        self.inside = torch.zeros_like(self.full, dtype=torch.bool)
        self.inside[32 + offset:].as_strided((rows, cols), (stride, 1)).fill_(True)
        self.fill = fill

    def check(self):
        assert bool((self.full[~self.inside] == self.fill).all()), "write outside the output"


def guarded_bytes(n):
    full = torch.full((n + 64,), 0xA5, dtype=torch.uint8, device=DEV)
    return full, full[32: 32 + n]


def check_bytes(full, n):
    assert bool((full[:32] == 0xA5).all()) and bool((full[32 + n:] == 0xA5).all()), "write outside the checkpoint"


def close(got, want, tol, what=""):
    got = got.double()
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan), "%s: NaNs at other places" % what
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), "%s: infinities differ" % what
    ok = ~(nan | inf)
    tol = torch.as_tensor(tol, dtype=torch.float64, device=DEV).expand_as(want)
    over = ((got - want).abs() - tol)[ok]
    assert over.numel() == 0 or float(over.max()) <= 0, "%s: beyond its tolerance by %g" % (what, float(over.max()))


def half_unit(dtype, want):
    return torch.nan_to_num(want.abs(), 0.0, 0.0, 0.0) * (BF16_HALF if dtype == torch.bfloat16 else 2.0 ** -24) + 1e-38


# ---- 8-bit checkpoints ------------------------------------------------------------------------------

def special_rows(cols, dtype):
    """Rows whose groups sit at the edges of the format."""
    rows = []
    base = torch.linspace(-1, 1, cols, device=DEV, dtype=torch.float64)
    for top in (127.0, 126.99999, 127.00001, 128.0, 127.5, 1.0, 2.0 ** -126, 2.0 ** -133, 1e-45, 2.0 ** 120 * 127,
                2.0 ** 126 * 0.9999, 2.0 ** 126, 3.0e38):
        r = base * top
        r[0] = top
        rows.append(r)
    rows.append(torch.zeros_like(base))
    rows.append(-torch.zeros_like(base))
    ties = torch.arange(cols, device=DEV, dtype=torch.float64) % 127 + 0.5
    ties[0] = 127
    rows.append(ties)
    for bad in (float("inf"), -float("inf"), float("nan")):
        r = base.clone()
        r[cols // 2] = bad
        rows.append(r)
    return torch.stack(rows).to(dtype)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("cols", [1, 31, 32, 33, 64, 200, 1024, 1027])
def test_pack_and_unpack_are_exact(cols, dtype):
    x = torch.cat([special_rows(cols, dtype), (3 * torch.randn(37, cols, generator=gen(cols), device=DEV)).to(dtype)])
    for stride, offset in ((cols, 0), (cols + 5, 1), (-(-cols // 16) * 16, 0)):
        src = Guarded(len(x), cols, dtype, stride, offset)
        src.view.copy_(x)
        n = B.ss_act8_bytes(*x.shape)
        full, ck = guarded_bytes(n)
        B.ss_act8_pack(src.view, ck)
        codes, exps, value, bad = ref.act8(x)
        got_codes, got_exps = ck[:codes.numel()].view_as(codes), ck[codes.numel():].view_as(exps)
        assert torch.equal(got_exps, exps)
        marked = bad.repeat_interleave(32, 1)
        assert torch.equal(got_codes[~marked], codes[~marked])
        check_bytes(full, n)
        for out_dtype in DTYPES:
            out = Guarded(len(x), cols, out_dtype, stride, offset)
            B.ss_act8_unpack(ck, out.view)
            assert torch.equal(torch.isnan(out.view), torch.isnan(value))
            assert torch.equal(torch.nan_to_num(out.view.double()), torch.nan_to_num(value))
            out.check()


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("name", list(ACTS))
@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
@pytest.mark.parametrize("rows,cols,layout", [(1, 1, "dense"), (3, 31, "dense"), (5, 32, "odd"), (129, 200, "dense"),
                                              (17, 1024, "halves"), (9, 1000, "halves"), (67, 2731, "dense"), (33, 96, "odd")])
def test_activation_forward_and_backward(rows, cols, layout, gated, name, dtype):
    g = gen(rows * 7 + cols)
    x0 = (4 * torch.randn(rows, cols, generator=g, device=DEV)).to(dtype)
    u0 = torch.randn(rows, cols, generator=g, device=DEV).to(dtype)
    dy = torch.randn(rows, cols, generator=g, device=DEV).to(dtype)
    if layout == "halves":  # two halves of one wider matrix, in and out
        src, grad = Guarded(rows, 2 * cols, dtype), Guarded(rows, 2 * cols, dtype)
        x, up = src.view[:, :cols], src.view[:, cols:]
        dx, dup = grad.view[:, :cols], grad.view[:, cols:]
        outs = [grad]
    else:
        pad, off = (0, 0) if layout == "dense" else (3, 1)
        srcs = [Guarded(rows, cols, dtype, cols + pad, off) for _ in range(2)]
        outs = [Guarded(rows, cols, dtype, cols + pad, off) for _ in range(2)]
        (x, up), (dx, dup) = (s.view for s in srcs), (o.view for o in outs)
    x.copy_(x0)
    up.copy_(u0)
    y = Guarded(rows, cols, dtype)
    n = B.ss_act8_bytes(rows, cols)
    kept = [guarded_bytes(n) for _ in range(3)]
    B.ss_act8_forward(x, up if gated else None, ACTS[name], y.view, kept[0][1], kept[1][1] if gated else None, kept[2][1])
    B.ss_act8_backward(dy, kept[0][1], kept[1][1] if gated else None, ACTS[name], dx, dup if gated else None)

    def same_as_packed(ck, of):
        alone = torch.zeros_like(ck)
        B.ss_act8_pack(of, alone)
        assert torch.equal(ck, alone)

    same_as_packed(kept[0][1], x0)
    same_as_packed(kept[2][1], y.view)
    xd, ud = x0.double(), u0.double() if gated else torch.ones_like(x0, dtype=torch.float64)
    want = ref.act(name, xd)[0] * ud
    close(y.view, want, half_unit(dtype, want) + 1e-6 * (want.abs() + xd.abs() * ud.abs()), "y")
    xk = ref.act8(x0)[2]
    uk = torch.ones_like(xk)
    if gated:
        same_as_packed(kept[1][1], u0)
        uk = ref.act8(u0)[2]
    f, slope = ref.act(name, xk)
    d = dy.double()
    want = d * uk * slope
    close(dx, want, half_unit(dtype, want) + 1e-6 * (d * uk).abs() * (1 + xk.abs()), "dx")
    if gated:
        want = d * f
        close(dup, want, half_unit(dtype, want) + 1e-6 * d.abs() * (f.abs() + xk.abs()), "dup")
    for o in outs + [y]:
        o.check()
    for full, _ in kept:
        check_bytes(full, n)


def test_activation_at_extreme_values():
    big = torch.tensor([[-1e30, -200.0, -90.0, -20.0, -0.0, 0.0, 1e-40, 20.0, 90.0, 200.0, 1e30]], device=DEV)
    big = big.t().contiguous()  # a group each
    for name in ACTS:
        y = torch.empty_like(big)
        ck = B.act8_checkpoint(*big.shape, DEV)
        B.ss_act8_forward(big, None, ACTS[name], y, ck)
        want = ref.act(name, big.double())[0]
        close(y, want, 1e-6 * big.abs().double().clamp(max=1e3) + 1e-6 * want.abs() + 1e-38, name)
        dx = torch.empty_like(big)
        B.ss_act8_backward(torch.ones_like(big), ck, None, ACTS[name], dx)
        want = ref.act(name, ref.act8(big)[2])[1]
        close(dx, want, 2e-6, name + " slope")


def test_a_group_that_blew_up_shows_in_the_gradients():
    x = torch.randn(4, 96, generator=gen(1), device=DEV)
    x[1, 40] = float("inf")
    x[2, 0] = float("nan")
    ck = B.act8_checkpoint(4, 96, DEV)
    B.ss_act8_pack(x, ck)
    dx = torch.empty_like(x)
    B.ss_act8_backward(torch.ones_like(x), ck, None, B.SS_ACT_SILU, dx)
    want = torch.zeros(4, 96, dtype=torch.bool, device=DEV)
    want[1, 32:64] = True
    want[2, :32] = True
    assert torch.equal(torch.isnan(dx), want)
    dw = torch.empty(8, 96, device=DEV)
    B.ss_weight_grad8(torch.ones(4, 8, device=DEV), ck, dw)
    assert torch.equal(torch.isnan(dw), want.any(0).expand(8, 96))


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_activation_in_place(dtype):
    rows, cols = 37, 130
    x = torch.randn(rows, cols, generator=gen(2), device=DEV).to(dtype)
    up = torch.randn(rows, cols, generator=gen(3), device=DEV).to(dtype)
    dy = torch.randn(rows, cols, generator=gen(4), device=DEV).to(dtype)
    cx, cu = (B.act8_checkpoint(rows, cols, DEV) for _ in range(2))
    y, dx, du = (torch.empty_like(x) for _ in range(3))
    B.ss_act8_forward(x, up, B.SS_ACT_SILU, y, cx, cu)
    B.ss_act8_backward(dy, cx, cu, B.SS_ACT_SILU, dx, du)
    for over in ("x", "up"):
        t = {"x": x.clone(), "up": up.clone()}
        c1, c2 = B.act8_checkpoint(rows, cols, DEV), B.act8_checkpoint(rows, cols, DEV)
        B.ss_act8_forward(t["x"], t["up"], B.SS_ACT_SILU, t[over], c1, c2)
        assert torch.equal(t[over], y) and torch.equal(c1, cx) and torch.equal(c2, cu)
    for over in ("dx", "dup"):
        t, other = dy.clone(), torch.empty_like(dy)
        B.ss_act8_backward(t, cx, cu, B.SS_ACT_SILU, *((t, other) if over == "dx" else (other, t)))
        assert torch.equal(t, dx if over == "dx" else du) and torch.equal(other, du if over == "dx" else dx)


def test_activation_slope_against_differences():
    """f' at a decoded point against (f(x+h) - f(x-h)) / 2h by the forward kernel. With h = 2^-6:
    truncation h^2/6 max|f'''| (below 1.3 for both) = 5.3e-5, rounding 2 * 2^-23 |f| / 2h = 1.6e-5 for |f| <= 2."""
    h = 2.0 ** -6
    x = (torch.arange(-126, 127, device=DEV).float() / 64).reshape(-1, 1)  # every row a group that decodes to itself
    ck = B.act8_checkpoint(*x.shape, DEV)
    for name in ACTS:
        B.ss_act8_pack(x, ck)
        back = torch.empty_like(x)
        B.ss_act8_unpack(ck, back)
        assert torch.equal(back, x)
        dx, hi, lo = (torch.empty_like(x) for _ in range(3))
        B.ss_act8_backward(torch.ones_like(x), ck, None, ACTS[name], dx)
        spare = torch.empty_like(ck)
        B.ss_act8_forward(x + h, None, ACTS[name], hi, spare)
        B.ss_act8_forward(x - h, None, ACTS[name], lo, spare)
        assert float((dx - (hi - lo) / (2 * h)).abs().max()) < 7e-5


# ---- weight gradient --------------------------------------------------------------------------------

def weight_grad_case(rows, n_out, n_in, dtype, dy_pad=0, dy_off=0, dw_pad=0, dw_off=0, accumulate=False, seed=0, tail=False):
    g = gen(rows + 3 * n_out + 5 * n_in + seed)
    x = torch.randn(rows, n_in, generator=g, device=DEV)
    if tail:
        x = x * torch.exp(2 * torch.randn(rows, 1, generator=g, device=DEV))
    dy0 = torch.randn(rows, n_out, generator=g, device=DEV).to(dtype)
    src = Guarded(rows, n_out, dtype, n_out + dy_pad, dy_off, fill=float("nan"))  # what lies between the rows must not be used
    src.view.copy_(dy0)
    ck = B.act8_checkpoint(rows, n_in, DEV)
    B.ss_act8_pack(x, ck)
    xk = ref.act8(x)[2]
    out = Guarded(n_out, n_in, torch.float32, n_in + dw_pad, dw_off)
    start = torch.randn(n_out, n_in, generator=g, device=DEV)
    out.view.copy_(start)
    B.ss_weight_grad8(src.view, ck, out.view, accumulate=accumulate)
    want = dy0.double().t() @ xk
    scale = dy0.double().abs().t() @ xk.abs()
    if accumulate:
        want = want + start.double()
        scale = scale + start.double().abs()
    close(out.view, want, 64 * 2.0 ** -23 * scale + 1e-38, "dw")
    if rows >= 64 and not accumulate and not tail:
        rel = float((out.view.double() - want).norm() / want.norm())
        assert rel < 1.5e-6, rel
    out.check()


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("rows,n_out,n_in", [
    (1, 1, 1), (1, 8, 32), (2, 128, 256), (63, 64, 64), (64, 128, 256), (65, 129, 257), (100, 1000, 48), (512, 256, 256),
    (513, 264, 520), (1023, 8, 2050), (1500, 640, 33), (4099, 136, 200), (257, 1, 512), (2048, 2056, 1), (9000, 64, 96)])
def test_weight_grad(rows, n_out, n_in, dtype):
    weight_grad_case(rows, n_out, n_in, dtype)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("dy_pad,dy_off,dw_pad,dw_off", [(8, 0, 0, 0), (1, 0, 0, 0), (0, 1, 0, 0), (24, 8, 4, 0), (8, 3, 1, 1), (0, 0, 3, 2)])
def test_weight_grad_strides_and_alignment(dy_pad, dy_off, dw_pad, dw_off, dtype):
    for accumulate in (False, True):
        weight_grad_case(700, 200, 328, dtype, dy_pad, dy_off, dw_pad, dw_off, accumulate)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_weight_grad_with_rows_of_very_different_size(dtype):
    weight_grad_case(1100, 136, 264, dtype, tail=True)


def test_weight_grad_of_a_long_batch_keeps_its_precision():
    """The sums in the matrix unit truncate; promoted every few hundred rows, the whole stays within 1.5e-6."""
    weight_grad_case(16384, 256, 512, torch.bfloat16)


def test_weight_grad_of_no_rows():
    ck = B.act8_checkpoint(0, 40, DEV)
    dw = torch.ones(24, 40, device=DEV)
    B.ss_weight_grad8(torch.empty(0, 24, device=DEV), ck, dw, accumulate=True)
    assert bool((dw == 1).all())
    B.ss_weight_grad8(torch.empty(0, 24, device=DEV), ck, dw)
    assert bool((dw == 0).all())


def test_weight_grad_twice_is_the_same():
    rows, n_out, n_in = 3000, 264, 520
    dy = torch.randn(rows, n_out, generator=gen(5), device=DEV).bfloat16()
    ck = B.act8_checkpoint(rows, n_in, DEV)
    B.ss_act8_pack(torch.randn(rows, n_in, generator=gen(6), device=DEV), ck)
    outs = []
    for _ in range(3):
        dw = torch.empty(n_out, n_in, device=DEV)
        B.ss_weight_grad8(dy, ck, dw)
        outs.append(dw)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


def test_weight_grad_against_differences():
    """sum_t dy . (x^ W^T) is linear in W: with W moved by a direction D it moves by <dW, D>, to fp32 rounding of the sum."""
    rows, n_out, n_in = 300, 40, 72
    x, dy = torch.randn(rows, n_in, generator=gen(7), device=DEV), torch.randn(rows, n_out, generator=gen(8), device=DEV)
    ck, xk = B.act8_checkpoint(rows, n_in, DEV), torch.empty(rows, n_in, device=DEV)
    B.ss_act8_pack(x, ck)
    B.ss_act8_unpack(ck, xk)
    dw = torch.empty(n_out, n_in, device=DEV)
    B.ss_weight_grad8(dy, ck, dw)
    w, d = (torch.randn(n_out, n_in, generator=gen(s), device=DEV).double() for s in (9, 10))
    loss = lambda m: float((dy.double() * (xk.double() @ m.t())).sum())  # noqa: E731
    moved = (loss(w + d) - loss(w - d)) / 2
    size = float((dy.double().abs().t() @ xk.double().abs() * d.abs()).sum())
    assert abs(moved - float((dw.double() * d).sum())) <= 64 * 2.0 ** -23 * size


# ---- losses -----------------------------------------------------------------------------------------

def loss_inputs(rows, vocab, dtype, pad=0, off=0, seed=0, spread=2.0, masked=0.25):
    g = gen(1000 * seed + rows + vocab)
    buf = Guarded(rows, vocab, dtype, vocab + pad, off, fill=float("nan"))
    buf.view.copy_(spread * torch.randn(rows, vocab, generator=g, device=DEV))
    targets = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    w = torch.rand(rows, generator=g, device=DEV) + 0.1
    w[torch.rand(rows, generator=g, device=DEV) < masked] = 0
    logp = ref.token_logp(buf.view, targets, torch.ones_like(w))[0].float()
    old = logp + 0.2 * torch.randn(rows, generator=g, device=DEV)
    # no ratio where rounding decides whether it is clipped
    r = (logp - old).exp()
    old = torch.where(((r - 0.8).abs() < 1e-3) | ((r - 1.2).abs() < 1e-3), logp, old)
    rlp = logp + 0.5 * torch.randn(rows, generator=g, device=DEV)
    adv = torch.randn(rows, generator=g, device=DEV)
    return buf.view, targets, w, old, rlp, adv


def logp_tol(z, vocab, c):
    top = torch.nan_to_num(z.double().abs() * c, 0.0, 0.0, 0.0)
    top = torch.where(top < 1e30, top, torch.zeros_like(top)).amax(1) if vocab else torch.zeros(len(z), device=DEV, dtype=torch.float64)
    return 1e-6 * (top + math.log(max(vocab, 1)) + 1)


def run_policy(z, targets, old, rlp, adv, w, dz, c=1.0, lo=0.2, hi=0.2, beta=0.05, grad_scale=None):
    totals, logp = torch.full((3,), 9.0, device=DEV), torch.full((len(z),), 9.0, device=DEV)
    B.ss_policy_loss(z, targets, old, rlp, adv, w, totals, logp, dz, inv_temperature=c, clip_low=lo, clip_high=hi,
                     kl_coef=beta, grad_scale=grad_scale)
    return totals, logp


def check_policy(z, targets, old, rlp, adv, w, c=1.0, lo=0.2, hi=0.2, beta=0.05, out=None, scale=1.0):
    rows, vocab = z.shape
    z0 = z.clone()
    dz = Guarded(rows, vocab, z.dtype) if out is None else out
    gs = None if scale == 1.0 else torch.full((1,), scale, device=DEV)
    totals, logp = run_policy(z, targets, old, rlp, adv, w, dz.view, c, lo, hi, beta, gs)
    want_t, want_l, want_d = ref.policy(z0, targets, old, rlp, adv, w, c, lo, hi, beta)
    want_d = want_d * scale
    tol = logp_tol(z0, vocab, c)
    close(logp, want_l, tol, "logp")
    # a log probability off by tol moves r and u by that share of themselves
    r = torch.exp(want_l - old.double())
    u = torch.exp(rlp.double() - want_l) if rlp is not None else torch.zeros_like(r)
    live = (w != 0) & (targets >= 0) & (targets < vocab)
    size = torch.where(live, w.double().abs() * (r * adv.double().abs() + beta * (u + 1)), torch.zeros_like(r))
    kl_size = torch.where(live, w.double().abs() * (u + 1 + (want_l.abs() + old.abs().double())), torch.zeros_like(r))
    fine = torch.nan_to_num(2 * size * (tol + 4e-7), 0.0, 0.0, 0.0)
    t_tol = fine.sum() + torch.nan_to_num(kl_size, 0.0, 0.0, 0.0).sum() * beta * 1e-6 + 1e-30
    close(totals[:1], want_t[:1], t_tol, "loss")
    close(totals[1:2], want_t[1:2], torch.nan_to_num(kl_size * (tol + 1e-6), 0.0, 0.0, 0.0).sum() + 1e-30, "kl")
    close(totals[2:], want_t[2:], 1e-6 * want_t[2].abs() + 1e-30, "clipped")
    p_part = torch.nan_to_num(want_d.abs(), 0.0, 0.0, 0.0)
    err = (2 * torch.nan_to_num(size, 0.0, 0.0, 0.0) * (tol + 1e-6) * c * abs(scale))[:, None] + p_part * (2 * tol[:, None] + 2e-6)
    close(dz.view, want_d, err + half_unit(z.dtype, want_d), "dlogits")
    assert bool((dz.view[~live] == 0).all())
    if out is None:
        dz.check()
    return totals, logp


SHAPES = [(1, 1), (1, 2), (3, 7), (5, 33), (2, 1000), (70, 257), (1, 32768), (33, 4099), (300, 1024), (7, 50001), (3, 140001), (2, 300007), (1, 900001), (150, 3000), (301, 9001)]


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("rows,vocab", SHAPES)
def test_policy_loss(rows, vocab, dtype):
    z, y, w, old, rlp, adv = loss_inputs(rows, vocab, dtype)
    check_policy(z, y, old, rlp, adv, w)
    check_policy(z, y, old, None, adv, w, c=0.7, lo=0.1, hi=0.3, beta=0.0)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("pad,off,out_pad,out_off", [(1, 0, 1, 0), (0, 1, 0, 0), (3, 2, 5, 1), (8, 0, 16, 0), (7, 1, 7, 1)])
def test_policy_loss_strides_and_alignment(pad, off, out_pad, out_off, dtype):
    for vocab in (5, 1001, 4096):
        z, y, w, old, rlp, adv = loss_inputs(19, vocab, dtype, pad, off)
        out = Guarded(19, vocab, dtype, vocab + out_pad, out_off)
        check_policy(z, y, old, rlp, adv, w, out=out, scale=-2.5)
        out.check()


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("rows,vocab", [(9, 1000), (64, 32001), (2, 150000)])
def test_losses_in_place_and_without_gradient(rows, vocab, dtype):
    """The bits are those of the same call: with the same layout, in place or not, they are equal. Without a
    gradient, or with rows that start elsewhere against 16 bytes, sums may be taken in another order: within the tolerances."""
    z, y, w, old, rlp, adv = loss_inputs(rows, vocab, dtype, pad=3)
    like = lambda: torch.empty_strided(z.shape, z.stride(), dtype=dtype, device=DEV)  # noqa: E731
    in_place = lambda t: type("Out", (), {"view": t})  # noqa: E731
    begin, ref2 = torch.tensor([0, rows // 2, rows], device=DEV), torch.zeros(2, device=DEV)
    zs = like().copy_(z)
    dz = like()
    totals, logp = run_policy(zs, y, old, rlp, adv, w, dz)
    over = like().copy_(z)
    t2, l2 = run_policy(over, y, old, rlp, adv, w, over)
    assert torch.equal(over, dz) and torch.equal(totals, t2) and torch.equal(logp, l2)
    first = run_preference(zs, y, w, begin, ref2, dz)
    over = like().copy_(z)
    second = run_preference(over, y, w, begin, ref2, over)
    assert torch.equal(over, dz) and all(torch.equal(a, b) for a, b in zip(first, second))
    dense = z.contiguous()  # another layout
    check_policy(dense, y, old, rlp, adv, w, out=in_place(dense))
    dense = z.contiguous()
    check_preference(dense, y, w, begin, ref2, out=in_place(dense))
    want = ref.policy(z, y, old, rlp, adv, w, 1.0, 0.2, 0.2, 0.05)
    t3, l3 = run_policy(z, y, old, rlp, adv, w, None)
    close(l3, want[1], logp_tol(z, vocab, 1.0), "logp")
    close(t3, totals.double(), 1e-5 * (totals.abs().double() + w.double().sum()), "totals")
    alone = run_preference(z, y, w, begin, ref2, None)
    close(alone[3], want[1], logp_tol(z, vocab, 1.0), "logp")


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
def test_rows_left_out_are_not_read(dtype):
    rows, vocab = 12, 333
    z, y, w, old, rlp, adv = loss_inputs(rows, vocab, dtype, masked=0.0)
    w[2], w[5] = 0, 0
    z[2] = float("nan")
    z[5] = float("inf")
    z[7] = float("nan")
    y[7] = -100
    y[8] = vocab
    old[2], adv[5], rlp[5] = float("nan"), float("nan"), float("inf")
    check_policy(z, y, old, rlp, adv, w)
    begin = torch.tensor([0, 6, 12], device=DEV)
    check_preference(z, y, w, begin, torch.zeros(2, device=DEV))
    # nothing left at all
    check_policy(z, y, old, rlp, adv, torch.zeros_like(w))
    check_preference(z, y, torch.zeros_like(w), begin, torch.zeros(2, device=DEV))


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("vocab", [40, 5000])
def test_masked_vocabulary_and_rows_without_a_softmax(vocab, dtype):
    rows = 8
    z, y, w, old, rlp, adv = loss_inputs(rows, vocab, dtype, masked=0.0)
    y[:] = torch.arange(rows, device=DEV)
    z[:, vocab // 2:] = float("-inf")                    # half of the vocabulary cannot be taken
    z[1, 10:] = torch.finfo(dtype).min                   # the type's lowest value as a mask
    z[2, :] = torch.finfo(dtype).min                     # nothing but lowest values: uniform
    z[3, :] = float("-inf")
    z[3, 3] = -1.0                                       # one token left
    check_policy(z[:4], y[:4], old[:4], rlp[:4], adv[:4], w[:4])
    z[4, :] = float("-inf")                              # nothing left
    z[5, 0] = float("inf")
    z[6, 1] = float("nan")
    dz = torch.empty_like(z)
    totals, logp = run_policy(z, y, old, rlp, adv, w, dz)
    assert torch.isnan(logp).tolist() == [False] * 4 + [True] * 3 + [False]
    assert bool(torch.isnan(dz[4:7]).all()) and not bool(torch.isnan(dz[:4]).any()) and not bool(torch.isnan(dz[7]).any())
    assert bool(torch.isnan(totals[:2]).all())


def test_policy_loss_is_clipped_on_both_sides():
    vocab, deltas = 64, [-0.5, -0.1, 0.1, 0.5]
    z = torch.randn(8, vocab, generator=gen(3), device=DEV)
    y = torch.arange(8, device=DEV)
    w = torch.full((8,), 0.125, device=DEV)
    logp = ref.token_logp(z, y, w)[0].float()
    old = logp - torch.tensor(deltas * 2, device=DEV)
    adv = torch.tensor([1.0] * 4 + [-1.0] * 4, device=DEV)
    totals, _ = check_policy(z, y, old, None, adv, w, beta=0.0, lo=0.2, hi=0.2)
    dz = torch.empty_like(z)
    run_policy(z, y, old, None, adv, w, dz, beta=0.0)
    still = (dz.abs().sum(1) == 0).tolist()
    assert still == [False, False, False, True, True, False, False, False]  # a gain beyond the range counts no further
    assert abs(float(totals[2]) - 0.25) < 1e-6


def test_policy_gradient_against_differences():
    """<dz, D> against (L(z + hD) - L(z - hD)) / 2h on the kernel's own loss, h = 2^-7: rounding
    about 8 * 2^-24 |L| / 2h = 4e-5 for |L| <= 1.2, truncation h^2/6 |L'''| with |L'''| <= 4 sum w = 4: 4e-5."""
    rows, vocab, h = 40, 50, 2.0 ** -7
    z, y, w, old, rlp, adv = loss_inputs(rows, vocab, torch.float32, masked=0.2, seed=4, spread=1.0)
    w = w / w.sum()
    old = torch.where((old - ref.token_logp(z, y, torch.ones_like(w))[0]).abs().sub(0.2).abs() < 0.06, rlp * 0 + ref.token_logp(z, y, torch.ones_like(w))[0].float(), old)
    d = torch.randn(rows, vocab, generator=gen(5), device=DEV)
    d = d / d.norm(dim=1, keepdim=True)
    dz = torch.empty_like(z)
    run_policy(z, y, old, rlp, adv, w, dz)
    up = run_policy(z + h * d, y, old, rlp, adv, w, None)[0][0]
    down = run_policy(z - h * d, y, old, rlp, adv, w, None)[0][0]
    assert abs(float(up - down) / (2 * h) - float((dz * d).sum())) < 1e-4


# ---- preference loss --------------------------------------------------------------------------------

def run_preference(z, y, w, begin, rlp, dz, c=1.0, kind=0, beta=0.1, smoothing=0.0, scale=1.0, grad_scale=None):
    pairs = (len(begin) - 1) // 2
    loss, margins = torch.full((1,), 9.0, device=DEV), torch.full((pairs,), 9.0, device=DEV)
    seq, logp = torch.full((2 * pairs,), 9.0, device=DEV), torch.full((len(z),), 9.0, device=DEV)
    B.ss_preference_loss(z, y, w, begin, rlp, loss, margins, seq, logp, dz, inv_temperature=c, kind=kind, beta=beta,
                         label_smoothing=smoothing, scale=scale, grad_scale=grad_scale)
    return loss, margins, seq, logp


def check_preference(z, y, w, begin, rlp, c=1.0, kind=0, beta=0.1, smoothing=0.0, scale=0.5, out=None, gs=1.0):
    rows, vocab = z.shape
    z0 = z.clone()
    dz = Guarded(rows, vocab, z.dtype) if out is None else out
    got = run_preference(z, y, w, begin, rlp, dz.view, c, kind, beta, smoothing, scale,
                         None if gs == 1.0 else torch.full((1,), gs, device=DEV))
    want = ref.preference(z0, y, w, begin, rlp, c, kind, beta, smoothing, scale)
    tol = logp_tol(z0, vocab, c)
    close(got[3], want[3], tol, "logp")
    live = (w != 0) & (y >= 0) & (y < vocab)
    b = begin.tolist()
    wt = torch.where(live, w.double().abs() * tol, torch.zeros_like(tol))
    s_tol = torch.stack([wt[p:q].sum() for p, q in zip(b, b[1:])]) if len(b) > 1 else wt[:0]
    close(got[2], want[2], s_tol + want[2].abs() * 2.0 ** -23 + 1e-30, "seq_logp")
    h_tol = s_tol[0::2] + s_tol[1::2]
    close(got[1], want[1], beta * h_tol + want[1].abs() * 2.0 ** -22 + 1e-30, "margins")
    steep = 2 * (want[1] / beta - 0.5 / beta).abs() + 1 if kind == 2 else torch.full_like(h_tol, beta)
    l_tol = scale * (steep * (h_tol + want[1].abs() / beta * 2.0 ** -22)).sum() + 4e-7 * want[0].abs() + 2e-7 * scale * len(b) / 2
    close(got[0].reshape(()), want[0], l_tol + 1e-30, "loss")
    # the coefficient of a pair moves with its margin, by at most `bend` for each unit of h
    bend = 2.0 if kind == 2 else beta * beta
    c_tol = torch.zeros(rows, dtype=torch.float64, device=DEV)
    for k in range(len(b) - 1):
        c_tol[b[k]:b[k + 1]] = scale * (bend * (h_tol[k // 2] + want[1][k // 2].abs() / beta * 2.0 ** -22)) + 1e-6 * scale * steep[k // 2]
    err = (c_tol * w.double().abs() * c * abs(gs))[:, None] + want[4].abs() * abs(gs) * (2 * tol[:, None] + 2e-6)
    close(dz.view, want[4] * gs, torch.nan_to_num(err, 0.0, 0.0, 0.0) + half_unit(z.dtype, want[4] * gs), "dlogits")
    if out is None:
        dz.check()
    return got


def cuts(rows, pairs, seed):
    c = torch.randint(0, rows + 1, (2 * pairs + 1,), generator=gen(seed), device=DEV).sort().values
    return c


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("kind", [0, 1, 2], ids=["sigmoid", "hinge", "squared"])
@pytest.mark.parametrize("rows,vocab,pairs", [(1, 1, 1), (2, 40, 1), (31, 257, 3), (200, 1024, 7), (24, 32001, 2), (600, 97, 40), (5, 140001, 1), (4, 300007, 2)])
def test_preference_loss(rows, vocab, pairs, kind, dtype):
    z, y, w, _, _, _ = loss_inputs(rows, vocab, dtype)
    begin = cuts(rows, pairs, rows + pairs)  # some sequences empty, some rows in none
    now = ref.preference(z, y, w, begin, torch.zeros(2 * pairs, device=DEV), 1.0, 0, 0.1, 0.0, 1.0)[2]
    rlp = (now + 3 * torch.randn(2 * pairs, generator=gen(rows), device=DEV)).float()
    check_preference(z, y, w, begin, rlp, kind=kind)
    check_preference(z, y, w, begin, rlp, kind=kind, c=1.5, beta=0.3, smoothing=0.1 if kind == 0 else 0.0, scale=1.0 / pairs, gs=3.0)


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("begin", [[3, 100, 190, 190, 190, 400, 650, 651, 652, 680, 690], [0, 0, 0, 350, 700, 700, 700], [0, 1, 2] + [700] * 6,
                                   [10] * 7, list(range(0, 701, 25))], ids=["rows of none", "empty", "short", "all empty", "even"])
def test_preference_loss_over_many_logits(begin, dtype):
    """Logits too large for the L2 cache, sequences cut in every way. In place too, and the same bits again."""
    rows, vocab = 700, 50001
    pairs = (len(begin) - 1) // 2
    z, y, w, _, _, _ = loss_inputs(rows, vocab, dtype, pad=2)
    begin = torch.tensor(begin, device=DEV)
    now = ref.preference(z, y, w, begin, torch.zeros(2 * pairs, device=DEV), 1.0, 0, 0.1, 0.0, 1.0)[2]
    rlp = (now + 3 * torch.randn(2 * pairs, generator=gen(rows), device=DEV)).float()
    for kind in (0, 2):
        check_preference(z, y, w, begin, rlp, kind=kind, scale=1.0 / pairs)
    like = lambda: torch.empty_strided(z.shape, z.stride(), dtype=dtype, device=DEV)  # noqa: E731
    zs, dz, over = like().copy_(z), like(), like().copy_(z)
    first, second = run_preference(zs, y, w, begin, rlp, dz), run_preference(over, y, w, begin, rlp, over)
    assert torch.equal(dz, over) and all(torch.equal(p, q) for p, q in zip(first, second))


@pytest.mark.parametrize("dtype", DTYPES, ids=IDS)
@pytest.mark.parametrize("pad,off,out_pad,out_off", [(1, 0, 1, 0), (0, 1, 0, 0), (3, 2, 5, 1), (7, 1, 7, 1)])
def test_preference_loss_strides_and_alignment(pad, off, out_pad, out_off, dtype):
    for vocab in (5, 1001, 4096):
        z, y, w, _, _, _ = loss_inputs(23, vocab, dtype, pad, off)
        out = Guarded(23, vocab, dtype, vocab + out_pad, out_off)
        check_preference(z, y, w, torch.tensor([0, 9, 23], device=DEV), torch.zeros(2, device=DEV), out=out)
        out.check()


def test_preference_loss_far_margins():
    """Margins of +-hundreds: no overflow, the right branch."""
    z, y, w, _, _, _ = loss_inputs(20, 30, torch.float32, masked=0.0)
    begin = torch.tensor([0, 5, 10, 15, 20], device=DEV)
    for shift in (5e3, -5e3):
        rlp = torch.tensor([shift, 0.0, 0.0, shift], device=DEV)
        for kind in (0, 1, 2):
            check_preference(z, y, w, begin, rlp, kind=kind)


def test_preference_loss_of_nothing():
    z, y, w, _, _, _ = loss_inputs(6, 50, torch.float32)
    empty = torch.zeros(0, device=DEV)
    dz = torch.full_like(z, 5.0)
    loss, logp = torch.full((1,), 9.0, device=DEV), torch.full((6,), 9.0, device=DEV)
    B.ss_preference_loss(z, y, w, torch.zeros(1, dtype=torch.int64, device=DEV), empty, loss, empty, empty, logp, dz)
    assert float(loss) == 0 and bool((dz == 0).all())
    no_rows = torch.empty(0, 50, device=DEV)
    no_y = torch.empty(0, dtype=torch.int64, device=DEV)
    margins, seq, totals = torch.ones(1, device=DEV), torch.ones(2, device=DEV), torch.ones(3, device=DEV)
    B.ss_preference_loss(no_rows, no_y, empty, torch.zeros(3, dtype=torch.int64, device=DEV), torch.zeros(2, device=DEV),
                         loss, margins, seq, empty, None)
    assert abs(float(loss) - math.log(2)) < 1e-6 and float(margins) == 0 and bool((seq == 0).all())
    B.ss_policy_loss(no_rows, no_y, empty, None, empty, empty, totals, empty)
    assert bool((totals == 0).all())


def test_a_table_of_sequences_out_of_range_reads_nothing_beyond():
    z, y, w, _, _, _ = loss_inputs(10, 40, torch.float32, masked=0.0)
    begin = torch.tensor([-5, 4, 1 << 40], device=DEV)
    clean = torch.tensor([0, 4, 10], device=DEV)
    rlp = torch.zeros(2, device=DEV)
    a, b = torch.empty_like(z), torch.empty_like(z)
    for got, want in zip(run_preference(z, y, w, begin, rlp, a), run_preference(z, y, w, clean, rlp, b)):
        assert torch.equal(got, want)
    assert torch.equal(a, b)


def test_preference_gradient_against_differences():
    """As for the policy loss: h = 2^-7, |L| <= 2, and a third derivative along a direction of norm 1 in each row of
    at most 4 a row times |dL/dlogp| <= beta: truncation below 1e-4 for 40 rows."""
    rows, vocab, h = 40, 50, 2.0 ** -7
    z, y, w, _, _, _ = loss_inputs(rows, vocab, torch.float32, masked=0.2, seed=6, spread=1.0)
    begin = torch.tensor([0, 8, 20, 31, 40], device=DEV)
    now = ref.preference(z, y, w, begin, torch.zeros(4, device=DEV), 1.0, 0, 0.1, 0.0, 1.0)[2]
    rlp = (now + torch.randn(4, generator=gen(8), device=DEV)).float()
    d = torch.randn(rows, vocab, generator=gen(5), device=DEV)
    d = d / d.norm(dim=1, keepdim=True)
    dz = torch.empty_like(z)
    run_preference(z, y, w, begin, rlp, dz, scale=0.5)
    up = run_preference(z + h * d, y, w, begin, rlp, None, scale=0.5)[0]
    down = run_preference(z - h * d, y, w, begin, rlp, None, scale=0.5)[0]
    assert abs(float(up - down) / (2 * h) - float((dz * d).sum())) < 2e-4


# ---- streams, repetition ----------------------------------------------------------------------------

def test_another_stream_and_the_same_bits_every_time():
    rows, vocab = 130, 9001
    z, y, w, old, rlp, adv = loss_inputs(rows, vocab, torch.bfloat16)
    begin, seq_ref = cuts(rows, 3, 4), torch.zeros(6, device=DEV)
    a, b = torch.empty(rows, vocab, dtype=z.dtype, device=DEV), torch.empty(rows, vocab, dtype=z.dtype, device=DEV)
    first = run_policy(z, y, old, rlp, adv, w, a), run_preference(z, y, w, begin, seq_ref, b)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c, d = torch.empty_like(a), torch.empty_like(b)
        second = run_policy(z, y, old, rlp, adv, w, c), run_preference(z, y, w, begin, seq_ref, d)
        x = torch.randn(50, 96, device=DEV)
        ck, back = B.act8_checkpoint(50, 96, DEV), torch.empty_like(x)
        B.ss_act8_pack(x, ck)
        B.ss_act8_unpack(ck, back)
    side.synchronize()
    assert torch.equal(a, c) and torch.equal(b, d)
    for p, q in zip(first, second):
        for s, t in zip(p, q):
            assert torch.equal(s, t)
    assert torch.equal(back.double(), ref.act8(x)[2])


@pytest.mark.parametrize("as_handle", [False, True], ids=["stream", "handle"])
def test_scratch_memory_belongs_to_the_call_s_stream(as_handle):
    """A call that is given a stream other than the current one, and no workspace, while that stream is busy:
    what the current stream allocates and fills in the meantime must not be the call's workspace."""
    rows, vocab = 40, 9001
    z, y, w, old, rlp, adv = loss_inputs(rows, vocab, torch.bfloat16)
    dy, x = torch.randn(700, 130, device=DEV), torch.randn(700, 96, device=DEV)
    ck = B.act8_checkpoint(700, 96, DEV)
    B.ss_act8_pack(x, ck)
    begin, seq_ref = cuts(rows, 2, 4), torch.zeros(4, device=DEV)

    def outputs():
        return {"totals": torch.empty(3, device=DEV), "logp": torch.empty(rows, device=DEV), "dlogits": torch.empty_like(z)}

    def calls(stream):
        a, b = outputs(), outputs()
        loss, margins, seq = torch.empty(1, device=DEV), torch.empty(2, device=DEV), torch.empty(4, device=DEV)
        dw = torch.empty(130, 96, device=DEV)
        torch.cuda.synchronize()
        if stream is not None:
            with torch.cuda.stream(side):
                torch.cuda._sleep(20_000_000)  # cycles: about 10 ms
        B.ss_policy_loss(z, y, old, rlp, adv, w, a["totals"], a["logp"], a["dlogits"], kl_coef=0.05, stream=stream)
        B.ss_preference_loss(z, y, w, begin, seq_ref, loss, margins, seq, b["logp"], b["dlogits"], stream=stream)
        B.ss_weight_grad8(dy, ck, dw, stream=stream)
        sizes = (B.ss_loss_workspace(rows, 0), B.ss_loss_workspace(rows, 2), B.ss_weight_grad8_workspace(dy, 96))
        kept = [torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV) for n in sizes for _ in range(2)]
        torch.cuda.synchronize()
        assert all(bool((k == 0xFF).all()) for k in kept)
        return [a["totals"], a["logp"], a["dlogits"], loss, margins, seq, b["logp"], b["dlogits"], dw]

    want = calls(None)
    side = torch.cuda.Stream()
    for got, expected in zip(calls(side.cuda_stream if as_handle else side), want):
        assert torch.equal(got, expected)


def test_calls_in_a_cuda_graph():
    """Captured once, replayed on new contents of the same buffers: the bits of plain calls."""
    rows, vocab = 40, 9001
    z, y, w, old, rlp, adv = loss_inputs(rows, vocab, torch.bfloat16)
    dy, x = torch.randn(700, 130, device=DEV), torch.randn(700, 96, device=DEV)
    ck = B.act8_checkpoint(700, 96, DEV)
    begin, seq_ref = cuts(rows, 2, 4), torch.zeros(4, device=DEV)
    ws = torch.empty(max(B.ss_loss_workspace(rows, 2), B.ss_weight_grad8_workspace(dy, 96)), dtype=torch.uint8, device=DEV)
    new = lambda n: torch.empty(n, device=DEV)  # noqa: E731
    totals, logp, loss, margins, seq, dw = new(3), new(rows), new(1), new(2), new(4), new((130, 96))
    dz, dp = torch.empty_like(z), torch.empty_like(z)
    outs = [totals, logp, loss, margins, seq, dw, dz, dp]

    def calls():
        B.ss_policy_loss(z, y, old, rlp, adv, w, totals, logp, dz, kl_coef=0.05, workspace=ws)
        B.ss_preference_loss(z, y, w, begin, seq_ref, loss, margins, seq, logp, dp, workspace=ws)
        B.ss_act8_pack(x, ck)
        B.ss_weight_grad8(dy, ck, dw, workspace=ws)

    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for scale in (1.0, 0.5):
        z.mul_(scale), x.mul_(scale)
        for t in outs:
            t.fill_(-7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        calls()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, outs))
