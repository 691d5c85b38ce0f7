"""The losses over logits where the earlier tests do not look: terms near their zero, terms left out by their
coefficient. Tolerances are derived beside each test."""
import pytest
import torch

from paper_1810_05291_b200 import binding as B

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
