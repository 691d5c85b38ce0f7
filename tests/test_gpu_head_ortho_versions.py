"""What the kernels of the cross entropy at the head and of the orthogonal update write, autograd is told of."""
import pytest
import torch

from paper_1810_05291_b200 import binding as B
from paper_1810_05291_b200.optim import OrthogonalMomentum

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def test_a_backward_pass_after_a_step_is_refused():
    p = torch.nn.Parameter(torch.randn(40, 60, device=DEV))
    x = torch.randn(5, 60, device=DEV, requires_grad=True)
    opt = OrthogonalMomentum([p])
    y = (x @ p.t()).square().sum()
    y.backward(retain_graph=True)
    opt.step()
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


def raised(call, *tensors):
    before = [t._version for t in tensors]
    call()
    return all(t._version > v for t, v in zip(tensors, before))


@pytest.mark.parametrize("inference", [False, True])
def test_versions_of_outputs(inference):
    with torch.inference_mode(inference):
        g, v, vo, p, po = ([torch.randn(20, 30, device=DEV)] for _ in range(5))
        x, w = torch.randn(6, 32, device=DEV).to(BF16), torch.randn(50, 32, device=DEV).to(BF16)
        y, k = torch.arange(6, device=DEV), torch.ones(6, device=DEV)
        totals, logp, dw = torch.empty(2, device=DEV), torch.empty(6, device=DEV), torch.zeros(50, 32, device=DEV)
        update = lambda: B.ss_orthogonal_update(g, v, vo, p, po, 0.9)  # noqa: E731
        alone = lambda: B.ss_orthogonalise(g, po)  # noqa: E731
        head = lambda: B.ss_linear_cross_entropy(x, w, y, k, totals, logp, x, dw, accumulate=True)  # noqa: E731
        if inference:                                        # these have no versions
            update(), alone(), head()
        else:
            untouched = [t._version for t in (g[0], v[0], p[0], w, y, k)]
            assert raised(update, vo[0], po[0]) and raised(alone, po[0]) and raised(head, totals, logp, x, dw)
            assert untouched == [t._version for t in (g[0], v[0], p[0], w, y, k)]
