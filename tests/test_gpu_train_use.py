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
