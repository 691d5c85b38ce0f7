"""Softmax cross entropy at the head on the GPU, against the formulas in 64 bits.

Tolerances. With T the largest sum |x| |w| of a row's logits: the matrix unit truncates each of the 64 steps of a
chunk of 1024 contraction indices, by less than 2^-23 of what it has summed (four times that is allowed for its inner
alignment), and a chunk is added with half a unit; so a logit is off by E = 4 (min(n, 1024) / 16 + n / 1024) 2^-23 T, n the
contraction indices of all passes. log p adds the hardware's exponentials (2^-22 each) and sums of up to 128 of
them, then of parts: 2^-15. An entry of P is off by 2^-11 (e in fp16) and 2^-8 (P in bf16) of itself for bf16
inputs, and by 2^-25 of the row's factor where e is below fp16's normal range; the target's by log p's error.
dx and dW carry these through |W| and |x|, add a truncation for each 16 contraction indices of a chunk, and half a
unit of their own type."""
import pytest
import torch

from paper_1810_05291_b200 import binding as B
from tests import head_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16
NAN = float("nan")


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def case(rows, width, vocab, dtype, seed=0, masked=0.2, pad=0, offset=0):
    """x and w as slices of wider matrices where pad is given, off 16 bytes with an odd offset."""
    g = gen(seed)
    x = torch.randn(rows, width + pad, generator=g, device=DEV).to(dtype)[:, offset:offset + width]
    w = (torch.randn(vocab, width + pad, generator=g, device=DEV) * width ** -0.5 * 2).to(dtype)[:, offset:offset + width]
    y = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    k = torch.rand(rows, generator=g, device=DEV) + 0.5
    k[torch.rand(rows, generator=g, device=DEV) < masked] = 0
    return x, w, y, k


def run(x, w, y, k, dw_dtype=None, accumulate=None, want=(True, True), **options):
    rows = x.shape[0]
    totals, logp = torch.full((2,), NAN, device=DEV), torch.full((rows,), NAN, device=DEV)
    dx = torch.full_like(x, NAN) if want[0] else None
    dw = None
    if want[1]:
        dw = torch.full(w.shape, NAN, dtype=dw_dtype or w.dtype, device=DEV) if accumulate is None else accumulate.clone()
    B.ss_linear_cross_entropy(x, w, y, k, totals, logp, dx, dw, accumulate=accumulate is not None, **options)
    return totals, logp, dx, dw


def within(name, got, want, bound):
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert not bool(bad.any()), "%s: %d of %d outside, worst %.3g of its bound, at %s" % (
        name, int(bad.sum()), bad.numel(), float((off / bound).nan_to_num(1e9).max()), bad.nonzero()[0].tolist())


def check(x, w, y, k, got, c=1.0, z_coef=0.0, scale=1.0, base=None):
    totals, logp, dx, dw = got
    want = ref.head(x, w, y, k, c, z_coef, scale)
    bound = ref.head_bounds(x, w, y, k, want, c, z_coef, scale, dw_half=0.0 if dw is None else torch.finfo(dw.dtype).eps / 2)
    within("logp", logp, want["logp"], bound["logp"])
    within("totals", totals, want["totals"], bound["totals"])
    if dx is not None:
        within("dx", dx, want["dx"], bound["dx"])
    if dw is not None:
        more = 0 if base is None else base.double()
        within("dw", dw, want["dw"] + more, bound["dw"] + 0 if base is None else bound["dw"] + 2.0 ** -22 * base.abs())


SHAPES = [(1, 64, 300), (1, 1, 1), (3, 7, 129), (64, 256, 257), (127, 96, 1000), (128, 64, 128), (129, 72, 2049), (256, 512, 256), (300, 130, 5003), (515, 1000, 4099)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=["%dx%dx%d" % s for s in SHAPES])
def test_loss_and_gradients(shape, dtype):
    c = case(*shape, dtype, seed=sum(shape), masked=0.0 if shape[0] == 1 else 0.2)
    check(*c, run(*c))


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("pad,offset", [(64, 0), (8, 8), (3, 1), (5, 0)])
def test_rows_of_wider_matrices(dtype, pad, offset):
    c = case(90, 200, 700, dtype, seed=pad, pad=pad, offset=offset)
    check(*c, run(*c))


@pytest.mark.parametrize("want", [(False, False), (True, False), (False, True)], ids=["loss", "dx", "dw"])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_what_is_not_asked_for_changes_nothing(dtype, want):
    c = case(200, 160, 1111, dtype, seed=5)
    whole, part = run(*c), run(*c, want=want)
    for a, b in zip(whole, part):
        assert b is None or torch.equal(a, b)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_temperature_z_term_and_scale(dtype):
    c = case(150, 128, 900, dtype, seed=9)
    gs = torch.tensor([-2.5], device=DEV)
    check(*c, run(*c, inv_temperature=0.7, z_coef=0.01, grad_scale=gs), c=0.7, z_coef=0.01, scale=-2.5)


def test_a_weight_gradient_in_fp32_of_bf16_inputs_written_and_added_to():
    c = case(260, 192, 1500, BF16, seed=11)
    check(*c, run(*c, dw_dtype=F32))
    base = torch.randn(1500, 192, generator=gen(1), device=DEV)
    check(*c, run(*c, accumulate=base), base=base)
    c = case(260, 192, 1500, F32, seed=12)
    check(*c, run(*c, accumulate=base), base=base)


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_positions_that_do_not_count(dtype):
    """Their hidden states may hold anything; outside targets count as little as weights of 0."""
    x, w, y, k = case(70, 64, 333, dtype, seed=3, masked=0.0)
    k[:20] = 0
    y[20:30], y[30:35] = -100, 333
    y[35] = 1 << 40
    x[:36] = NAN
    x[7] = float("inf")
    got = run(x, w, y, k)
    clean = x.clone()
    clean[:36] = 0
    check(clean, w, y, k, got)
    assert not bool(got[2][:36].any()) and not bool(got[1][:36].any())
    k[:] = 0
    totals, logp, dx, dw = run(x, w, y, k)
    for t in (totals, logp, dx, dw):
        assert not bool(t.any())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_values_that_are_not_finite(dtype):
    x, w, y, k = case(40, 64, 500, dtype, seed=4, masked=0.0)
    x[3] = NAN
    totals, logp, dx, dw = run(x, w, y, k)
    assert bool(totals.isnan().all()) and bool(logp[3].isnan()) and bool(dx[3].isnan().all()) and bool(dw.isnan().all())
    rest = torch.arange(40, device=DEV) != 3
    assert bool(logp[rest].isfinite().all()) and bool(dx[rest].isfinite().all())


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_logits_far_apart(dtype):
    """Certain, hopeless and equal: logits of +-300, all the same."""
    x, w, y, k = case(64, 64, 400, dtype, seed=6, masked=0.0)
    x.zero_()
    w.zero_()
    w[:, 0] = torch.where(torch.arange(400, device=DEV) == 7, 1.0, -1.0).to(dtype)
    x[:32, 0] = 300.0
    y[:16], y[16:32] = 7, 8
    totals, logp, dx, dw = run(x, w, y, k)
    assert torch.equal(logp[:16], torch.zeros(16, device=DEV)) and torch.allclose(logp[16:32], torch.full((16,), -600.0, device=DEV))
    check(x, w, y, k, (totals, logp, dx, dw))


def test_nothing_to_do():
    x, w = torch.empty(0, 64, dtype=BF16, device=DEV), torch.ones(30, 64, dtype=BF16, device=DEV)
    y, k = torch.empty(0, dtype=torch.int64, device=DEV), torch.empty(0, device=DEV)
    totals, _, _, dw = run(x, w, y, k)
    assert not bool(totals.any()) and not bool(dw.any())
    base = torch.ones(30, 64, device=DEV)
    assert torch.equal(run(x, w, y, k, accumulate=base)[3], base)


def test_dx_in_place():
    x, w, y, k = case(333, 96, 800, BF16, seed=8)
    want = run(x, w, y, k)
    totals, logp = torch.empty(2, device=DEV), torch.empty(333, device=DEV)
    B.ss_linear_cross_entropy(x, w, y, k, totals, logp, x)
    assert torch.equal(x, want[2]) and torch.equal(logp, want[1])


def test_the_same_call_gives_the_same_bits():
    c = case(1000, 512, 9000, BF16, seed=10)
    for a, b in zip(run(*c), run(*c)):
        assert torch.equal(a, b)
