"""The autograd side of the training operators on the CPU, with stand-ins for the kernels: what a backward pass
changes, and what it refuses."""
import pytest
import torch

from paper_1810_05291_b200 import train_ops as T
from tests import train_ref as ref
from tests import train_stand_ins


@pytest.fixture
def calls(monkeypatch):
    return train_stand_ins.install(monkeypatch)


def rand(*shape, seed=0, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator().manual_seed(seed)).to(dtype)


def layer(seed=0, rows=6, n_in=40, n_out=8):
    x, w, dy = rand(rows, n_in, seed=seed), rand(n_out, n_in, seed=seed + 1), rand(rows, n_out, seed=seed + 2)
    want = (dy.double().t() @ ref.act8(x)[2]).float()
    return x.requires_grad_(), w.requires_grad_(), dy, want


# ---- whose gradient a backward pass changes ---------------------------------------------------------
# A stand-in's product is rounded once and so is its sum with what is there: 2^-23 of the terms.

@pytest.mark.parametrize("options", [{}, {"into_grad": True}], ids=["default", "into_grad"])
def test_a_gradient_of_the_input_alone_leaves_the_weight_s_as_it_is(calls, options):
    x, w, dy, _ = layer()
    w.grad = rand(8, 40, seed=9)
    before = w.grad.clone()
    torch.autograd.grad(T.linear8(x, w, **options), [x], dy)
    assert torch.equal(w.grad, before)
    T.linear8(x, w, **options).backward(dy, inputs=[x])
    assert torch.equal(w.grad, before) and x.grad is not None


@pytest.mark.parametrize("options", [{}, {"into_grad": True}], ids=["default", "into_grad"])
def test_a_gradient_of_the_weight_is_returned_and_not_added(calls, options):
    x, w, dy, want = layer()
    w.grad = rand(8, 40, seed=9)
    before = w.grad.clone()
    got = torch.autograd.grad(T.linear8(x, w, **options), [x, w], dy)[1]
    assert torch.equal(got, want) and torch.equal(w.grad, before)


@pytest.mark.parametrize("options", [{}, {"into_grad": True}], ids=["default", "into_grad"])
@pytest.mark.parametrize("where", ["before", "after"])
def test_a_hook_on_the_weight_acts(calls, options, where):
    x, w, dy, want = layer()
    w.grad = torch.zeros_like(w)
    at, seen = w.grad.data_ptr(), []
    if where == "before":
        w.register_hook(lambda g: 0.5 * g)
        want = 0.5 * want
    else:
        w.register_post_accumulate_grad_hook(lambda p: seen.append(p.grad.clone()))
    T.linear8(x, w, **options).backward(dy)
    assert torch.equal(w.grad, want) and w.grad.data_ptr() == at
    assert where == "before" or (len(seen) == 1 and torch.equal(seen[0], want))


@pytest.mark.parametrize("options", [{}, {"into_grad": True}], ids=["default", "into_grad"])
def test_the_weight_s_gradient_is_added_in_place(calls, options):
    x, w, dy, want = layer()
    start = rand(8, 40, seed=9)
    w.grad = start.clone()
    at = w.grad.data_ptr()
    T.linear8(x, w, **options).backward(dy)
    T.linear8(x, w, **options).backward(dy, inputs=[w])
    assert torch.equal(w.grad, (start + want) + want) and w.grad.data_ptr() == at
    w.grad = None
    T.linear8(x, w, **options).backward(dy)
    assert torch.equal(w.grad, want)


def test_into_grad_forms_no_second_buffer(calls, monkeypatch):
    x, w, dy, want = layer()
    w.grad = torch.zeros_like(w)
    y, made = T.linear8(x, w, into_grad=True), []
    monkeypatch.setattr(torch, "empty", lambda *a, **k: made.append(a))
    y.backward(dy)
    monkeypatch.undo()
    assert made == [] and torch.equal(w.grad, want)


# ---- second derivatives -------------------------------------------------------------------------------

def losses(z):
    rows = z.shape[0]
    y, w, zero = torch.arange(rows) % z.shape[1], torch.ones(rows), torch.zeros(rows)
    begin = torch.tensor([0, rows // 2, rows])
    return {"policy": lambda: T.policy_loss(z, y, zero - 2, torch.ones(rows), w)[0],
            "preference": lambda: T.preference_loss(z, y, w, begin, torch.zeros(2))[0]}


@pytest.mark.parametrize("what", ["linear8", "act8", "gated act8", "sum of act8", "policy", "preference"])
def test_a_second_derivative_is_refused(calls, what):
    """The kernels have none. A first derivative that passed for a constant would leave terms out of the second."""
    x, w = rand(6, 40).requires_grad_(), rand(8, 40, seed=1).requires_grad_()
    out = {"linear8": lambda: T.linear8(x, w).square().sum(), "act8": lambda: T.act8(x)[0].square().sum(),
           "gated act8": lambda: T.act8(x, w[:6] * 2)[0].square().sum(), "sum of act8": lambda: T.act8(x)[0].sum(),
           **losses(x)}[what]()
    g, = torch.autograd.grad(out, [x], create_graph=True)
    with pytest.raises(RuntimeError, match="second derivative"):
        (g.square().sum() + x.square().sum()).backward()


def test_create_graph_alone_is_no_error(calls):
    x, w, dy, want = layer()
    gx, gw = torch.autograd.grad(T.linear8(x, w), [x, w], dy, create_graph=True)
    assert torch.equal(gw, want) and torch.equal(gx, dy @ w.detach())
    T.linear8(x, w).backward(dy, create_graph=True)
    assert torch.equal(w.grad, want)
    (x * 2).sum().backward()                         # and what else the graph holds goes on


def test_a_second_derivative_through_the_weight_s_grad_is_refused(calls):
    x, w, dy, want = layer()
    w.grad = torch.zeros_like(w)
    T.linear8(x, w, into_grad=True).backward(dy, create_graph=True)
    assert torch.equal(w.grad, want)
    with pytest.raises(RuntimeError, match="second derivative"):
        w.grad.square().sum().backward()


# ---- checkpoints that a caller brings -------------------------------------------------------------------

def test_a_checkpoint_of_other_sizes_is_refused_at_once(calls):
    x, w, _, _ = layer()
    for rows, cols in ((6, 64 + 1), (5, 40), (7, 40)):
        with pytest.raises(ValueError):
            T.linear8(x, w, torch.empty(rows * 33 * -(-cols // 32), dtype=torch.uint8))
    with pytest.raises(TypeError):
        T.linear8(x, w, torch.empty(6 * 66, dtype=torch.int8))
    with pytest.raises(ValueError):
        T.linear8(x, w, torch.empty(12 * 66, dtype=torch.uint8)[::2])


def test_a_checkpoint_written_again_in_between_is_refused(calls):
    x, w, dy, want = layer()
    kept = torch.empty(6 * 66, dtype=torch.uint8)
    T.B.ss_act8_pack(x.detach(), kept)
    y = T.linear8(x, w, kept)
    y.backward(dy)
    assert torch.equal(w.grad, want)
    y = T.linear8(x, w, kept)
    kept.zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward(dy)


# ---- strides --------------------------------------------------------------------------------------------

@pytest.mark.parametrize("shape,over", [((6, 40), 0), ((2, 3, 40), (0, 1)), ((1, 6, 40), 1)], ids=["rows", "both", "batch of one"])
def test_the_gradient_of_a_sum_over_rows(calls, shape, over):
    """It arrives with a row stride of 0."""
    x, w = rand(*shape).requires_grad_(), rand(8, 40, seed=1).requires_grad_()
    v = rand(8, seed=2)
    (T.linear8(x, w).sum(over) * v).sum().backward()
    flat = x.detach().reshape(6, 40)
    assert torch.equal(w.grad, (v.expand(6, 8).double().t() @ ref.act8(flat)[2]).float())
    assert torch.equal(x.grad.reshape(6, 40), (v.expand(6, 8) @ w.detach()))
    up, u = rand(*shape, seed=3).requires_grad_(), rand(40, seed=4)
    x.grad = None
    (T.act8(x, up)[0].sum(over) * u).sum().backward()
    f, slope = ref.act("silu", ref.act8(flat)[2])
    assert torch.equal(x.grad.reshape(6, 40), (u.double() * ref.act8(up.detach().reshape(6, 40))[2] * slope).float())
    assert torch.equal(up.grad.reshape(6, 40), (u.double() * f).float())


def test_expanded_and_overlapping_inputs(calls):
    w, dy = rand(8, 40, seed=1).requires_grad_(), rand(6, 8, seed=2)
    base = rand(1, 40).requires_grad_()
    T.linear8(base.expand(6, 40), w).backward(dy)
    want = dy.double().t() @ ref.act8(base.detach())[2].expand(6, 40)
    assert torch.equal(w.grad, want.float())
    assert torch.allclose(base.grad, (dy @ w.detach()).sum(0, keepdim=True), rtol=1e-5, atol=1e-5)
    window = rand(64).as_strided((6, 40), (4, 1))           # rows overlap
    assert torch.equal(T.act8(window)[0], ref.act("silu", window.double())[0].float())
    gate, up = rand(6, 40, seed=5).requires_grad_(), rand(1, 40, seed=6).requires_grad_()
    T.act8(gate, up.expand(6, 40))[0].sum().backward()
    f = ref.act("silu", ref.act8(gate.detach())[2])[0]
    assert torch.allclose(up.grad.double(), f.sum(0, keepdim=True), rtol=1e-5, atol=1e-6)
    column = rand(6, 1).requires_grad_()
    T.act8(column)[0].sum().backward()
    assert column.grad.shape == (6, 1)


def test_losses_of_expanded_logits(calls):
    z = rand(1, 40).requires_grad_()
    for loss in losses(z.expand(6, 40)).values():
        z.grad = None
        loss().backward()
        assert bool(torch.isfinite(z.grad).all()) and bool(z.grad.any())


@pytest.mark.parametrize("shape", [(0, 40), (2, 0, 40), (3, 0), (2, 3, 0)])
def test_empty_inputs(calls, shape):
    x, w = rand(*shape).requires_grad_(), rand(8, shape[-1], seed=1).requires_grad_()
    y = T.linear8(x, w)
    assert y.shape == shape[:-1] + (8,) and not bool(y.any())
    y.sum().backward()
    assert w.grad.shape == w.shape and not bool(w.grad.any()) and x.grad.shape == shape
    x.grad = None
    T.act8(x, torch.ones(shape))[0].sum().backward()
    assert x.grad.shape == shape


# ---- autocast -------------------------------------------------------------------------------------------

def test_linear8_under_autocast_is_a_bf16_layer(calls):
    x, w, dy, _ = layer()
    start = rand(8, 40, seed=9)
    low = x.detach().bfloat16()
    want = dy.bfloat16().double().t() @ ref.act8(low)[2]
    for options in ({}, {"into_grad": True}):
        x.grad, w.grad = None, start.clone()
        with torch.autocast("cpu", torch.bfloat16):
            y = T.linear8(x, w, **options)
        assert y.dtype == torch.bfloat16 and torch.equal(y, low @ w.detach().bfloat16().t())
        y.backward(dy.bfloat16())
        assert torch.equal(w.grad, start + want.float())
        assert x.grad.dtype == torch.float32 and torch.equal(x.grad, (dy.bfloat16() @ w.detach().bfloat16()).float())


def test_linear8_backward_under_autocast(calls):
    """A backward pass inside the region computes in the types of its forward pass, as one outside does."""
    x, w, dy, want = layer()
    y = T.linear8(x, w)
    with torch.autocast("cpu", torch.bfloat16):
        y.backward(dy)
    assert torch.equal(x.grad, dy @ w.detach()) and torch.equal(w.grad, want)


# ---- work that nobody asked for -------------------------------------------------------------------------

def test_the_checkpoint_of_the_result_gets_no_gradient(calls, monkeypatch):
    """PyTorch fills one with zeros unless it is told not to."""
    made = []
    for name, f in (("act8", T._Act8), ("linear8", T._Linear8), ("policy", T._PolicyLoss), ("preference", T._PreferenceLoss)):
        def watch(ctx, *grads, _run=f.backward, _name=name):
            made.append((_name, [g is None for g in grads]))
            return _run(ctx, *grads)
        monkeypatch.setattr(f, "backward", staticmethod(watch))
    x, up, w = rand(6, 40).requires_grad_(), rand(6, 40, seed=1).requires_grad_(), rand(8, 40, seed=2).requires_grad_()
    y, kept = T.act8(x, up, keep_output=True)
    z = T.linear8(y, w, kept)
    (losses(z)["policy"]() + losses(z)["preference"]()).backward()
    assert sorted(made) == [("act8", [False, True]), ("linear8", [False]), ("policy", [False, True, True]),
                            ("preference", [False, True, True, True])]


def test_a_result_without_a_gradient(calls):
    """A Function whose result is left out of the loss, beside one that is not."""
    class Both(torch.autograd.Function):
        @staticmethod
        def forward(ctx, a, b):
            ctx.set_materialize_grads(False)
            return a * 2, b * 2

        @staticmethod
        def backward(ctx, da, db):
            return None, db * 2

    x, w = rand(6, 40).requires_grad_(), rand(8, 40, seed=2).requires_grad_()
    y, other = T.act8(T.linear8(x, w))[0], rand(6, 8, seed=3).requires_grad_()
    Both.apply(y, other)[1].sum().backward()
    assert x.grad is None and w.grad is None and torch.equal(other.grad, torch.full((6, 8), 2.0))
    z = rand(6, 40, seed=4).requires_grad_()
    for loss in losses(z).values():
        Both.apply(loss(), other.sum())[1].backward()
        assert z.grad is None


def test_no_gradients_no_checkpoints(calls):
    x, up, w = rand(6, 40).requires_grad_(), rand(6, 40, seed=1).requires_grad_(), rand(8, 40, seed=2).requires_grad_()
    with torch.no_grad():
        y, kept = T.act8(x, up)
        T.linear8(y, w)
    assert kept is None and calls == ["forward"]
    del calls[:]
    T.act8(x.detach(), up.detach())
    T.linear8(x, w.detach()).sum().backward()        # a frozen weight: the input's gradient alone
    assert calls == ["forward"] and x.grad is not None
    with torch.no_grad():                            # asked for: made
        y, kept = T.act8(x, keep_output=True)
    assert calls == ["forward", "forward", "kept"]
    w.grad = None
    T.linear8(y, w, kept).sum().backward()
    assert torch.equal(w.grad, (torch.ones(6, 8).double().t() @ ref.act8(y)[2]).float())


def test_a_gradient_of_one_input_alone(calls):
    x, up, dy = rand(6, 40), rand(6, 40, seed=1), rand(6, 40, seed=2)
    f, slope = ref.act("silu", ref.act8(x)[2])
    a, b = x.clone().requires_grad_(), up.clone().requires_grad_()
    T.act8(a, up)[0].backward(dy)
    assert torch.equal(a.grad, (dy.double() * ref.act8(up)[2] * slope).float())
    T.act8(x, b)[0].backward(dy)
    assert torch.equal(b.grad, (dy.double() * f).float())


def test_what_a_layer_holds_until_its_backward_pass(calls):
    """The weight in the input's type for the input's gradient, the checkpoint for the weight's: no more than is needed."""
    x, w = rand(6, 40, dtype=torch.bfloat16), rand(8, 40, seed=1)
    kept = torch.empty(6 * 66, dtype=torch.uint8)
    T.B.ss_act8_pack(x, kept)
    held = lambda y: [t is not None for t in y.grad_fn.saved_tensors]  # noqa: E731
    assert held(T.linear8(x, w.requires_grad_(), kept)) == [False, True]
    assert held(T.linear8(x.requires_grad_(), w.detach(), kept)) == [True, False]
    assert held(T.linear8(x, w)) == [True, True]
