"""The cross entropy at the head as an autograd function, and the optimiser of matrices, on plain CPU stand-ins for the kernels."""
import copy

import pytest
import torch

from paper_1810_05291_b200 import train_ops as T
from paper_1810_05291_b200.optim import OrthogonalMomentum
from tests import head_ref, head_stand_ins, ortho_ref

BF16 = torch.bfloat16


@pytest.fixture
def calls(monkeypatch):
    return head_stand_ins.install(monkeypatch)


def case(rows=9, width=12, vocab=20, dtype=torch.float32, wdtype=torch.float32):
    g = torch.Generator().manual_seed(rows * vocab)
    x = torch.randn(rows, width, generator=g).to(dtype).requires_grad_()
    w = torch.randn(vocab, width, generator=g).to(wdtype).requires_grad_()
    y = torch.randint(0, vocab, (rows,), generator=g)
    y[2] = -100
    return x, w, y, torch.rand(rows, generator=g)


def near(got, want, tol=1e-6):
    assert float((got.double() - want.double()).norm() / want.double().norm().clamp(min=1e-30)) < tol


@pytest.mark.parametrize("z_coef", [0.0, 0.02])
def test_gradients_are_the_formulas(calls, z_coef):
    x, w, y, k = case()
    loss, square, logp = T.linear_cross_entropy(x, w, y, k, 0.8, z_coef)
    (3 * loss).backward()
    z = 0.8 * x.detach().double() @ w.detach().double().t()
    live = (y >= 0).double() * k.double()
    lp = torch.log_softmax(z, 1)[torch.arange(9), y.clamp(min=0)]
    lse = torch.logsumexp(z, 1)
    near(loss.detach(), (live * (z_coef * lse ** 2 - lp)).sum())
    near(square, (live * lse ** 2).sum())
    xx, ww = x.detach().double().requires_grad_(), w.detach().double().requires_grad_()
    z = 0.8 * xx @ ww.t()
    lse = torch.logsumexp(z, 1)
    (3 * (live * (lse - z[torch.arange(9), y.clamp(min=0)] + z_coef * lse ** 2)).sum()).backward()
    near(x.grad, xx.grad)
    near(w.grad, ww.grad)


def test_gradients_are_differences(calls):
    x, w, y, k = case(4, 5, 7)
    loss = lambda a, b: head_ref.head(a, b, y, k)["totals"][0]  # noqa: E731
    T.linear_cross_entropy(x, w, y, k)[0].backward()
    for t, grad, f in ((x, x.grad, lambda d: loss(x.detach().double() + d, w.detach().double())),
                       (w, w.grad, lambda d: loss(x.detach().double(), w.detach().double() + d))):
        for at in ((0, 1), (2, 3), (3, 4)):
            d = torch.zeros(t.shape, dtype=torch.float64)
            d[at] = 1e-5
            assert abs(float((f(d) - f(-d)) / 2e-5 - grad[at])) < 1e-6


def test_nothing_is_formed_that_no_gradient_can_be_asked_for(calls):
    x, w, y, k = case()
    with torch.no_grad():
        T.linear_cross_entropy(x, w, y, k)
    T.linear_cross_entropy(x.detach(), w, y, k)[0].backward()
    T.linear_cross_entropy(x, w.detach(), y, k)[0].backward()
    T.linear_cross_entropy(x.detach(), w.detach(), y, k)
    assert [c[1:] for c in calls] == [(False, False), (False, True), (True, False), (False, False)]


def test_shapes_types_and_autocast(calls):
    x, w, y, k = case(12, 8, 10, BF16)
    loss, _, logp = T.linear_cross_entropy(x.view(3, 4, 8), w, y.view(3, 4), k.view(3, 4))
    assert logp.shape == (12,) and loss.shape == ()
    loss.backward()
    assert x.grad.dtype == BF16 and w.grad.dtype == torch.float32
    x, w, y, k = case(12, 8, 10, BF16, BF16)
    T.linear_cross_entropy(x, w, y, k)[0].backward()
    assert w.grad.dtype == BF16
    x, w, y, k = case(12, 8, 10)
    with torch.autocast("cpu", BF16):
        loss = T.linear_cross_entropy(x, w, y, k)[0]
    loss.backward()
    assert x.grad.dtype == w.grad.dtype == torch.float32
    want = head_ref.head(x.detach().to(BF16), w.detach().to(BF16), y, k)
    near(loss.detach(), want["totals"][0])


def test_a_gradient_that_arrives_is_not_rounded_before_the_product(calls):
    x, w, y, k = case(12, 8, 10, BF16, BF16)
    (T.linear_cross_entropy(x, w, y, k)[0] / 3).backward()
    want = head_ref.head(x.detach(), w.detach(), y, k)
    once = (want["dx"].to(BF16).double() / 3).float()
    assert torch.equal(x.grad, (want["dx"].to(BF16).float() * torch.tensor(1.0).div(3)).to(BF16))
    near(x.grad, once, 2.0 ** -8)


def test_into_grad(calls):
    x, w, y, k = case()
    T.linear_cross_entropy(x, w, y, k)[0].backward()
    want = w.grad.clone()
    w.grad.zero_()
    buffer = w.grad
    T.linear_cross_entropy(x, w, y, k, into_grad=True)[0].backward()
    assert w.grad is buffer and torch.equal(w.grad, want)
    T.linear_cross_entropy(x, w, y, k, into_grad=True)[0].backward()
    near(w.grad, 2 * want)
    w.grad = None                                            # nowhere to add: through autograd
    T.linear_cross_entropy(x, w, y, k, into_grad=True)[0].backward()
    near(w.grad, want)
    (dw,) = torch.autograd.grad(T.linear_cross_entropy(x, w, y, k, into_grad=True)[0], w)
    near(dw, want)
    near(w.grad, want)


def test_twice_through_the_same_graph_and_second_derivatives(calls):
    x, w, y, k = case()
    loss = T.linear_cross_entropy(x, w, y, k)[0]
    loss.backward(retain_graph=True)
    first = x.grad.clone()
    loss.backward()
    near(x.grad, 2 * first)
    (dx,) = torch.autograd.grad(T.linear_cross_entropy(x, w, y, k)[0], x, create_graph=True)
    with pytest.raises(RuntimeError, match="second derivatives"):
        dx.sum().backward()


# ---- the optimiser

def optimiser(params, **options):
    kernels = head_stand_ins.Kernels()
    return OrthogonalMomentum(params, kernels=kernels, **options), kernels


def params(shapes, seed=0):
    g = torch.Generator().manual_seed(seed)
    out = [torch.nn.Parameter(torch.randn(s, generator=g)) for s in shapes]
    for p in out:
        p.grad = torch.randn(p.shape, generator=g)
    return out


@pytest.mark.parametrize("scale,factor", [("rms", lambda r, c: 0.2 * max(r, c) ** 0.5), ("spectral", lambda r, c: max(1.0, r / c) ** 0.5), (0.3, lambda r, c: 0.3)])
@pytest.mark.parametrize("nesterov", [False, True])
def test_steps_are_the_formulas(nesterov, scale, factor):
    ps = params([(6, 9), (9, 6), (4, 2, 3, 2)])
    want = [(p.detach().clone().view(p.shape[0], -1), torch.zeros(p.shape).view(p.shape[0], -1)) for p in ps]
    opt, _ = optimiser(ps, lr=0.01, momentum=0.9, nesterov=nesterov, weight_decay=0.1, scale=scale)
    for _ in range(3):
        opt.step()
        want = [tuple(t.float() for t in ortho_ref.updated(p.grad.view(m.shape), v, m, 0.9, nesterov, 0.01, factor(*m.shape), 0.1)[::-1]) for p, (m, v) in zip(ps, want)]
    for p, (m, v) in zip(ps, want):
        near(p.detach().view(m.shape), m)
        near(opt.state[p]["momentum_buffer"].view(m.shape), v)


def test_matrices_alike_go_together_and_no_more_than_fit():
    ps = params([(6, 9)] * 6 + [(9, 6)] * 2 + [(3, 2, 3)])
    opt, kernels = optimiser(ps)
    ps[0].grad = None
    opt.step()
    assert sorted(kernels.calls) == [(1, (3, 6)), (1, (6, 9)), (2, (9, 6)), (4, (6, 9))]
    assert "momentum_buffer" not in opt.state[ps[0]]


def test_groups_schedules_and_checkpoints():
    ps = params([(5, 7), (7, 5)])
    opt, _ = optimiser([dict(params=[ps[0]], lr=0.5), dict(params=[ps[1]], weight_decay=0.5)], lr=0.1)
    opt.step()
    other = [torch.nn.Parameter(p.detach().clone()) for p in ps]
    for a, b in zip(other, ps):
        a.grad = b.grad.clone()
    again, _ = optimiser([dict(params=[other[0]]), dict(params=[other[1]])])
    again.load_state_dict(copy.deepcopy(opt.state_dict()))
    for o in (opt, again):
        o.param_groups[0]["lr"] = 0.25
        o.step()
    for a, b in zip(other, ps):
        assert torch.equal(a, b)


def test_gradients_and_parameters_of_other_layouts():
    whole = torch.randn(8, 20, generator=torch.Generator().manual_seed(3))
    p = torch.nn.Parameter(whole[:, 3:13])                   # columns of a wider matrix, stepped where they are
    p.grad = torch.ones(10, 8).t()                           # column major
    opt, kernels = optimiser([p], lr=0.1)
    before = whole.clone()
    opt.step()
    assert torch.equal(whole[:, :3], before[:, :3]) and not torch.equal(whole[:, 3:13], before[:, 3:13])
    bad = torch.nn.Parameter(torch.randn(5, 6).t())
    with pytest.raises(ValueError):
        optimiser([bad])


def test_refusals():
    p = torch.nn.Parameter(torch.randn(3, 4))
    for options in (dict(lr=-1.0), dict(momentum=1.0), dict(weight_decay=-0.1), dict(scale="x"), dict(lr=float("nan"))):
        with pytest.raises(ValueError):
            optimiser([p], **options)
    with pytest.raises(ValueError):
        optimiser([torch.nn.Parameter(torch.randn(4))])
    with pytest.raises(ValueError):
        optimiser([torch.nn.Parameter(torch.randn(4, 4).bfloat16())])


def test_closure():
    ps = params([(4, 4)])
    opt, _ = optimiser(ps)
    assert float(opt.step(lambda: torch.tensor(2.0))) == 2.0
