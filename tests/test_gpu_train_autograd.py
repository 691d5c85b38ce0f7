"""The autograd forms of the training operators on the GPU: gradients against PyTorch's own of the
same formulas on the decoded values, accumulation into a flat buffer, and the example that runs them
together."""
import importlib.util
import os

import pytest
import torch

from paper_1810_05291_b200 import binding as B
from paper_1810_05291_b200 import train_ops as T
from paper_1810_05291_b200.optim import SignumVote
from tests import train_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rand(shape, seed, dtype=torch.float32, scale=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (scale * torch.randn(*shape, generator=g, device=DEV)).to(dtype)


@pytest.mark.parametrize("shape", [(70, 96), (3, 5, 33)])
def test_linear8_gradients(shape):
    """dW is the formula's on the decoded input, to the fp32 sums' 1.5e-6; dx is PyTorch's product."""
    x, w = rand(shape, 1).requires_grad_(), rand((40, shape[-1]), 2).requires_grad_()
    dy = rand(shape[:-1] + (40,), 3)
    y = T.linear8(x, w)
    y.backward(dy)
    assert torch.equal(y, (x.detach().reshape(-1, shape[-1]) @ w.detach().t()).view_as(y))
    kept = ref.act8(x.detach().reshape(-1, shape[-1]))[2]
    want = dy.reshape(-1, 40).double().t() @ kept
    assert float((w.grad.double() - want).norm() / want.norm()) < 1.5e-6
    assert torch.equal(x.grad, (dy.reshape(-1, 40) @ w.detach()).view_as(x))


def test_linear8_adds_into_the_gradient_that_is_there():
    x, w = rand((50, 64), 4, torch.bfloat16), rand((24, 64), 5).requires_grad_()
    start = rand((24, 64), 6)
    w.grad = start.clone()
    at = w.grad.data_ptr()
    dy = rand((50, 24), 7, torch.bfloat16)
    T.linear8(x, w).backward(dy)
    T.linear8(x, w).backward(dy)  # the same layer used twice
    want = start.double() + 2 * dy.double().t() @ ref.act8(x)[2]
    assert w.grad.data_ptr() == at
    assert float((w.grad.double() - want).norm() / want.norm()) < 1.5e-6


def test_linear8_hands_the_gradient_on_when_asked():
    x, w = rand((50, 64), 4), rand((24, 64), 5).requires_grad_()
    w.grad = torch.zeros_like(w)
    dy = rand((50, 24), 7)
    got, = torch.autograd.grad(T.linear8(x, w, into_grad=False), w, dy)
    want = dy.double().t() @ ref.act8(x)[2]
    assert float((got.double() - want).norm() / want.norm()) < 1.5e-6 and not bool(w.grad.any())


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("name", ["gelu", "silu"])
def test_act8_gradients(name, gated):
    x, up = rand((37, 130), 8).requires_grad_(), rand((37, 130), 9).requires_grad_()
    dy = rand((37, 130), 10)
    y, kept = T.act8(x, up if gated else None, name, keep_output=True)
    y.backward(dy)
    alone = B.act8_checkpoint(37, 130, DEV)
    B.ss_act8_pack(y.detach(), alone)
    assert torch.equal(kept, alone) and not kept.requires_grad
    xk = ref.act8(x.detach())[2]
    f, slope = ref.act(name, xk)
    uk = ref.act8(up.detach())[2] if gated else torch.ones_like(xk)
    for got, want in ((x.grad, dy.double() * uk * slope), (up.grad, dy.double() * f if gated else None)):
        if want is None:
            assert got is None
        else:
            assert float((got.double() - want).abs().max()) <= 1e-6 * float((dy.double() * uk).abs().max()) * 8


def test_losses_carry_the_gradient_that_arrives():
    """Twice the loss plus nothing else: the logits' gradient is twice the formula's."""
    rows, vocab = 24, 301
    z = rand((rows, vocab), 11).requires_grad_()
    y = torch.randint(0, vocab, (rows,), device=DEV, generator=torch.Generator(device=DEV).manual_seed(12))
    w = torch.full((rows,), 1.0 / rows, device=DEV)
    old = ref.token_logp(z.detach(), y, w)[0].float() + 0.05
    adv = rand((rows,), 13)
    loss, figures, logp = T.policy_loss(z, y, old, adv, w, ref_logp=old, kl_coef=0.1)
    (2 * loss).backward()
    want_t, want_l, want_d = ref.policy(z.detach(), y, old, old, adv, w, 1.0, 0.2, 0.2, 0.1)
    assert abs(float(loss.detach()) - float(want_t[0])) < 1e-5 and float((logp - want_l).abs().max()) < 2e-5
    assert abs(float(figures[0]) - float(want_t[1])) < 1e-5
    assert float((z.grad.double() - 2 * want_d).norm() / want_d.norm()) < 4e-5
    z.grad = None
    begin, rlp = torch.tensor([0, 5, 11, 20, 24], device=DEV), torch.zeros(4, device=DEV)
    loss, margins, seq, logp = T.preference_loss(z, y, torch.ones_like(w), begin, rlp, beta=0.2)
    (2 * loss).backward()
    want = ref.preference(z.detach(), y, torch.ones_like(w), begin, rlp, 1.0, 0, 0.2, 0.0, 0.5)
    assert abs(float(loss.detach()) - float(want[0])) < 1e-4 and float((margins - want[1]).abs().max()) < 1e-3
    assert float((z.grad.double() - 2 * want[4]).norm() / want[4].norm()) < 1e-3


def test_a_step_of_the_optimiser_takes_the_gradient_where_it_was_formed():
    """Under SignumVote the weight's grad is a view of the flat buffer: the layer adds into it, and the vote moves
    each weight by lr against the sign of its gradient."""
    w = torch.nn.Parameter(rand((48, 80), 14))
    before = w.detach().clone()
    opt = SignumVote([w], lr=0.25, momentum=None)
    x, dy = rand((200, 80), 15, torch.bfloat16), rand((200, 48), 16, torch.bfloat16)
    T.linear8(x, w).backward(dy)
    assert w.grad.data_ptr() == opt.flat_grad.data_ptr()
    want = dy.double().t() @ ref.act8(x)[2]
    clear = want.abs() > 1e-3
    opt.step()
    assert torch.equal((w.detach() - before)[clear], -0.25 * torch.sign(want[clear]).float()) or bool(
        ((w.detach() - before)[clear] + 0.25 * torch.sign(want[clear]).float()).abs().max() < 1e-6)


def test_the_example_learns():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "preference_then_policy.py")
    spec = importlib.util.spec_from_file_location("preference_then_policy", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    history = example.train(steps=40, say=lambda *_: None)
    assert history["preference"][-1] < 0.5 * history["preference"][0]
    assert sum(history["reward"][-5:]) / 5 > sum(history["reward"][:5]) / 5 + 0.05
