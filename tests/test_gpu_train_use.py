"""The autograd forms of the training operators on the GPU: what they refuse, and calls as users make them."""
import pytest
import torch

from paper_1810_05291_b200 import binding as B
from paper_1810_05291_b200 import train_ops as T
from tests import train_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rand(shape, seed, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


def near(got, want, tol=1.5e-6):
    assert float((got.double() - want).norm() / want.norm()) < tol


@pytest.mark.parametrize("by", ["pack", "forward", "torch"])
def test_a_checkpoint_written_again_before_the_backward_pass_is_refused(by):
    x, w, dy = rand((50, 64), 1), rand((24, 64), 2).requires_grad_(), rand((50, 24), 3)
    kept = B.act8_checkpoint(50, 64, DEV)
    B.ss_act8_pack(x, kept)
    y = T.linear8(x, w, kept)
    other, spare = rand((50, 64), 4), B.act8_checkpoint(50, 64, DEV)
    if by == "pack":
        B.ss_act8_pack(other, kept)
    elif by == "forward":
        B.ss_act8_forward(other, None, B.SS_ACT_SILU, torch.empty_like(other), spare, None, kept)
    else:
        kept.zero_()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward(dy)


def test_checkpoints_under_inference_mode():
    with torch.inference_mode():
        x, ck, back = rand((5, 64), 1), B.act8_checkpoint(5, 64, DEV), torch.empty(5, 64, device=DEV)
        B.ss_act8_pack(x, ck)
        B.ss_act8_unpack(ck, back)
        y, kept = T.act8(x, keep_output=True)
        T.linear8(y, rand((8, 64), 2), kept)
    assert torch.equal(back.double(), ref.act8(x)[2])


@pytest.mark.parametrize("shape", [(0, 40), (2, 0, 40), (3, 0), (2, 3, 0)])
def test_empty_inputs(shape):
    """The gradient of a sum of nothing has column stride 0."""
    x, w = rand(shape, 1).requires_grad_(), rand((8, shape[-1]), 2).requires_grad_()
    T.linear8(x, w).sum().backward()
    assert w.grad.shape == w.shape and not bool(w.grad.any()) and x.grad.shape == shape
    x.grad = None
    T.act8(x, torch.ones(shape, device=DEV))[0].sum().backward()
    assert x.grad.shape == shape
    z, none = rand((0, 40), 3).requires_grad_(), torch.empty(0, device=DEV)
    loss = T.policy_loss(z, none.long(), none, none, none)[0]
    loss.backward()
    assert float(loss.detach()) == 0 and z.grad.shape == z.shape


@pytest.mark.parametrize("shape,over", [((70, 96), 0), ((2, 35, 96), (0, 1)), ((1, 70, 96), 1)], ids=["rows", "both", "batch of one"])
def test_the_gradient_of_a_sum_over_rows(shape, over):
    x, w, v = rand(shape, 1).requires_grad_(), rand((24, 96), 2).requires_grad_(), rand((24,), 3)
    (T.linear8(x, w).sum(over) * v).sum().backward()
    flat = x.detach().reshape(70, 96)
    near(w.grad, v.expand(70, 24).double().t() @ ref.act8(flat)[2])
    u, up = rand((96,), 4), rand((96,), 5).requires_grad_()
    x.grad = None
    (T.act8(x, up.expand(shape))[0].sum(over) * u).sum().backward()
    f, slope = ref.act("silu", ref.act8(flat)[2])
    near(x.grad.reshape(70, 96), u.double() * ref.act8(up.detach().expand(70, 96))[2] * slope)
    near(up.grad, (u.double() * f).sum(0))


def test_layers_under_autocast():
    """An fp32 input is taken in the region's type, as other linear layers take it; gradients come back in fp32."""
    x, w, dy = rand((70, 96), 1).requires_grad_(), rand((24, 96), 2).requires_grad_(), rand((70, 24), 3, torch.bfloat16)
    low = x.detach().bfloat16()
    with torch.autocast("cuda", torch.bfloat16):
        y = T.linear8(x, w)
        h, _ = T.act8(T.linear8(x, w), act="gelu")
        loss = T.policy_loss(h, torch.zeros(70, dtype=torch.int64, device=DEV), *[torch.ones(70, device=DEV) for _ in range(3)])[0]
    assert y.dtype == h.dtype == torch.bfloat16 and torch.equal(y, low @ w.detach().bfloat16().t())
    y.backward(dy)
    assert x.grad.dtype == torch.float32 and torch.equal(x.grad, (dy @ w.detach().bfloat16()).float())
    near(w.grad, dy.double().t() @ ref.act8(low)[2])
    loss.backward()
    assert bool(torch.isfinite(w.grad).all())


def test_the_backward_pass_of_an_activation_makes_no_buffer_for_the_checkpoint():
    """At its peak it holds its two gradients beside what was there; a gradient of kept_y would be 1056 bytes a row more."""
    rows, cols = 4096, 1024
    x, up = (rand((rows, cols), k, torch.bfloat16).requires_grad_() for k in (1, 2))
    dy = rand((rows, cols), 3, torch.bfloat16)
    y, kept = T.act8(x, up, keep_output=True)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    y.backward(dy)
    assert torch.cuda.max_memory_allocated() - before <= 2 * rows * cols * 2 + 4096


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
@pytest.mark.parametrize("shape", [(1, 1), (37, 130), (64, 256)])
def test_an_activation_that_keeps_nothing(shape, gated, dtype):
    """The bits of the one that does, and, where asked for, the same checkpoint of the result."""
    x, up = rand(shape, 1, dtype), rand(shape, 2, dtype) if gated else None
    new = lambda: B.act8_checkpoint(*shape, DEV)  # noqa: E731
    y, ck = torch.empty_like(x), new()
    B.ss_act8_forward(x, up, B.SS_ACT_GELU, y, new(), new() if gated else None, ck)
    alone, only = torch.empty_like(x), new()
    B.ss_act8_forward(x, up, B.SS_ACT_GELU, alone)
    assert torch.equal(alone, y)
    B.ss_act8_forward(x, up, B.SS_ACT_GELU, alone.zero_(), None, None, only)
    assert torch.equal(alone, y) and torch.equal(only, ck)
    with torch.no_grad():
        assert torch.equal(T.act8(x, up, "gelu")[0], y)
    if gated:
        for kept in ((new(), None), (None, new())):
            with pytest.raises(B.SignSGDError):
                B.ss_act8_forward(x, up, B.SS_ACT_GELU, alone, *kept)
