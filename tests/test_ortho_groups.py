"""Groups of the matrices' optimiser are checked however they come: by themselves, with options of their own, added later."""
import pytest
import torch

from paper_1810_05291_b200.optim import OrthogonalMomentum
from tests import head_stand_ins


def optimiser(params, **options):
    return OrthogonalMomentum(params, kernels=head_stand_ins.Kernels(), **options)


def matrix(*shape):
    return torch.nn.Parameter(torch.randn(*(shape or (4, 5))))


BAD = [dict(lr=-1.0), dict(lr=float("nan")), dict(momentum=1.0), dict(momentum=-0.1), dict(weight_decay=-0.1), dict(scale="x"), dict(scale=None)]


@pytest.mark.parametrize("options", BAD)
def test_options_of_a_group(options):
    with pytest.raises(ValueError):
        optimiser([dict(params=[matrix()], **options)])
    opt = optimiser([matrix()])
    with pytest.raises(ValueError):
        opt.add_param_group(dict(params=[matrix()], **options))
    assert len(opt.param_groups) == 1


@pytest.mark.parametrize("bad", [torch.randn(4), torch.randn(4, 5).bfloat16(), torch.randn(5, 4).t(), torch.randn(2, 3, 4, 5).transpose(0, 1)])
def test_parameters_of_a_group_that_is_added(bad):
    opt = optimiser([matrix()])
    with pytest.raises(ValueError):
        opt.add_param_group(dict(params=[matrix(), torch.nn.Parameter(bad)]))
    assert len(opt.param_groups) == 1
    for g in opt.param_groups:                               # what was there before still steps
        for p in g["params"]:
            p.grad = torch.randn_like(p)
    opt.step()


def test_a_group_that_is_added_steps():
    opt, p = optimiser([matrix()]), matrix(3, 2, 2)
    opt.add_param_group(dict(params=p, lr=0.5, scale=1))
    p.grad = torch.randn_like(p)
    before = p.detach().clone()
    opt.step()
    assert not torch.equal(before, p)


def test_a_parameter_without_elements():
    ps = [matrix(0, 3, 3), matrix(3, 0, 2), matrix(0, 4)]
    opt = optimiser(ps)
    for p in ps:
        p.grad = torch.zeros_like(p)
    opt.step()


def test_a_group_whose_options_cannot_be_compared():
    opt = optimiser([matrix()])
    with pytest.raises(TypeError):
        opt.add_param_group(dict(params=[matrix()], lr="0.1"))
    assert len(opt.param_groups) == 1
