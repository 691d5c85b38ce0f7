"""A step of the matrices' optimiser tells autograd that it wrote to the parameters, as torch's optimisers do."""
import pytest
import torch

from paper_1810_05291_b200.optim import OrthogonalMomentum
from tests import head_stand_ins


@pytest.mark.parametrize("shape", [(6, 9), (4, 2, 3, 2)])
def test_a_backward_pass_after_a_step_is_refused(shape):
    p = torch.nn.Parameter(torch.randn(shape))
    p.grad = torch.randn(shape)
    opt = OrthogonalMomentum([p], kernels=head_stand_ins.Kernels())
    x = torch.randn(5, p[0].numel(), requires_grad=True)
    y = (x @ p.view(shape[0], -1).t()).sum()
    opt.step()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()
