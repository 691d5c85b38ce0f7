"""The losses over logits where the earlier tests do not look: terms near their zero, terms left out by their
coefficient. Tolerances are derived beside each test."""
import pytest
import torch

from paper_1810_05291_b200 import binding as B
from tests.test_gpu_train_ops import Guarded, check_policy, loss_inputs

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def confident(rows, vocab, seed):
    """Logits whose target has about the probability 1/2: a logp near -0.7, so that differences of 1e-7 exist."""
    z = torch.randn(rows, vocab, generator=gen(seed), device=DEV)
    y = torch.randint(0, vocab, (rows,), generator=gen(seed + 1), device=DEV)
    z.scatter_(1, y[:, None], torch.logsumexp(z, 1, keepdim=True))
    return z, y


def policy(z, y, old, rlp, adv, w, dz, **options):
    totals, logp = torch.empty(3, device=DEV), torch.empty(len(z), device=DEV)
    B.ss_policy_loss(z, y, old, rlp, adv, w, totals, logp, dz, **options)
    return totals, logp


@pytest.mark.parametrize("vocab", [257, 5000, 20001])
@pytest.mark.parametrize("size", [1e-6, 1e-4, 1e-3, 0.03, 0.4, 0.6, 3.0])
def test_the_kl_term_near_its_zero(size, vocab):
    """ref_logp is set from the kernel's own logp, so that their difference d is exact in fp32 (or, from 0.4 on, rounded to
    2^-24 of the larger) and kl = exp(d) - 1 - d can be had from it in 64 bits. No term is negative, and each is formed
    from d by a few operations: a rounding of d moves it by at most 2^-24 |d kl'| / kl <= 2^-24 (2 + |d|) of itself, every other one by
    2^-24 |d| / kl of itself where it is a difference (|d| >= 1/2: 2^-24 * 5 at most) and 2^-24 where it is not. 16 * 2^-24 covers them, 1e-6. The slope,
    1 - exp(d), likewise; the logits' gradient has the softmax's rounding on top, 1e-6 at logits of this size, and 2^-24 of (1 - p)."""
    rows = 64
    z, y = confident(rows, vocab, 3)
    one, zero, dz = torch.ones(rows, device=DEV), torch.zeros(rows, device=DEV), torch.empty_like(z)
    logp = policy(z, y, zero - 0.7, None, zero, one, dz)[1]
    rlp = logp + size * torch.randn(rows, generator=gen(5), device=DEV)
    totals, again = policy(z, y, logp, rlp, zero, one, dz, kl_coef=1.0)
    assert torch.equal(again, logp)
    d = rlp.double() - logp.double()
    kl = torch.expm1(d) - d
    assert abs(float(totals[1]) - float(kl.sum())) <= 1e-6 * float(kl.sum())
    assert abs(float(totals[0]) - float(kl.sum())) <= 1e-6 * float(kl.sum())
    p = torch.softmax(z.double(), 1).gather(1, y[:, None])[:, 0]
    got, want = dz.gather(1, y[:, None])[:, 0].double(), -torch.expm1(d) * (1 - p)
    assert bool(((got - want).abs() <= 4e-6 * want.abs()).all())
    for k in range(4):  # alone: never below zero
        w = zero.clone()
        w[k] = 1.0
        alone = policy(z, y, logp, rlp, zero, w, None, kl_coef=1.0)[0]
        assert float(alone[1]) >= 0.0


def test_a_kl_coefficient_of_zero_leaves_the_term_out():
    """A reference given for the figure alone: where the KL term is infinite, loss and gradient are those without it."""
    z, y = confident(6, 300, 7)
    z[2, y[2]] = float("-inf")                       # a token that this policy cannot take: logp is -inf, the term has no end
    one = torch.ones(6, device=DEV)
    old, rlp, adv = -one, -one, torch.tensor([1.0, -1.0] * 3, device=DEV)
    rlp[4] = 200.0                                   # the term overflows
    dz, plain = torch.empty_like(z), torch.empty_like(z)
    totals, logp = policy(z, y, old, rlp, adv, one, dz, kl_coef=0.0)
    want, _ = policy(z, y, old, None, adv, one, plain)
    assert torch.equal(totals[[0, 2]], want[[0, 2]]) and torch.equal(dz, plain) and bool(torch.isfinite(dz).all())
    assert not bool(torch.isfinite(totals[1]))       # the figure says what it is


@pytest.mark.parametrize("smoothing", [0.0, 0.25])
def test_a_label_smoothing_of_zero_leaves_the_term_out(smoothing):
    """A rejected answer with a token that cannot be taken: the margin is +inf, -log sigma of it is 0."""
    z, y = confident(8, 300, 8)
    z[5, y[5]] = float("-inf")
    begin, w = torch.tensor([0, 4, 8], device=DEV), torch.ones(8, device=DEV)
    loss, margins, seq, logp = torch.empty(1, device=DEV), torch.empty(1, device=DEV), torch.empty(2, device=DEV), torch.empty(8, device=DEV)
    dz = torch.empty_like(z)
    B.ss_preference_loss(z, y, w, begin, torch.zeros(2, device=DEV), loss, margins, seq, logp, dz, label_smoothing=smoothing)
    assert float(margins) == float("inf") and float(seq[1]) == float("-inf")
    if smoothing == 0.0:
        assert float(loss) == 0.0 and not bool(dz.any())
    else:
        assert float(loss) == float("inf")


# ---- rows of a cluster one after another ----------------------------------------------------------------
# For 148 SMs. A cluster takes more than one row where rows times blocks of a row come to 4440 or more (2664 for the rows
# whose threads hold 128 logits): the comments give the blocks and rows of a cluster for bf16.

@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,vocab,pad,off", [
    (9000, 5001, 0, 0),       # 1 block, 4 rows
    (13001, 4104, 0, 0),      # 1 block, 5 rows, aligned rows in bf16
    (5000, 9001, 3, 1),       # 2 blocks, 4 rows
    (2300, 32001, 0, 0),      # 4 blocks, 4 rows
    (2500, 50001, 7, 0),      # 8 blocks, 8 rows (fp32: 128 logits to a thread)
    (500, 100001, 0, 3),      # 8 blocks, 128 logits to a thread, 3 rows
    (340, 131072, 0, 0),      # the longest row there is room for
])
def test_policy_rows_one_after_another(rows, vocab, pad, off, dtype):
    z, y, w, old, rlp, adv = loss_inputs(rows, vocab, dtype, pad, off)
    w[5:9], w[20:37], w[-3:] = 0.0, 0.0, 0.0                     # runs of rows left out, longer than a cluster's share
    y[41], y[43], y[44] = -100, vocab, -1
    w[50:70] = 0.0
    w[60] = 1.0
    z[21:25] = float("nan")
    check_policy(z, y, old, rlp, adv, w)
    out = Guarded(rows, vocab, dtype, vocab + 5, 1)              # gradients that lie otherwise against 16 bytes
    check_policy(z, y, old, None, adv, w, beta=0.0, out=out, scale=0.5)
    out.check()
    like = lambda: torch.empty_strided(z.shape, z.stride(), dtype=dtype, device=DEV)  # noqa: E731
    apart, over = like().copy_(z), like().copy_(z)               # in place: the same bits
    dz = like()
    first = policy(apart, y, old, rlp, adv, w, dz, kl_coef=0.05)
    second = policy(over, y, old, rlp, adv, w, over, kl_coef=0.05)
    assert torch.equal(over, dz) and all(torch.equal(a, b) for a, b in zip(first, second))


def test_policy_rows_all_left_out():
    for rows, vocab in ((9000, 5001), (2300, 32001)):
        z, y, w, old, rlp, adv = loss_inputs(rows, vocab, torch.bfloat16)
        z.fill_(float("nan"))
        check_policy(z, y, old, rlp, adv, torch.zeros_like(w))
