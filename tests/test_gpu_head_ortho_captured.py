"""A whole step captured into a graph and replayed with other inputs: the cross entropy at the head forward and backward through autograd, both ways that its
weight's gradient goes, and the matrices' optimiser."""
import pytest
import torch

from paper_1810_05291_b200 import train_ops as T
from paper_1810_05291_b200.optim import OrthogonalMomentum

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def rand(*shape, seed, size=1.0):
    return size * torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)


class Step:
    def __init__(self, into_grad):
        self.into_grad = into_grad
        self.body = torch.nn.Parameter(rand(96, 64, seed=1, size=0.1))
        self.head = torch.nn.Parameter(rand(500, 96, seed=2, size=0.1))
        for p in (self.body, self.head):
            p.grad = torch.zeros_like(p)
        self.opt = OrthogonalMomentum([self.body], lr=0.01)
        self.x, self.y, self.k = rand(130, 64, seed=3), torch.zeros(130, dtype=torch.int64, device=DEV), torch.ones(130, device=DEV)
        self.loss = torch.zeros((), device=DEV)

    def __call__(self):
        for p in (self.body, self.head):
            p.grad.zero_()
        hidden = (self.x @ self.body.t()).bfloat16()
        loss = T.linear_cross_entropy(hidden, self.head, self.y, self.k / 130, z_coef=1e-4, into_grad=self.into_grad)[0]
        (2.5 * loss).backward()
        self.opt.step()
        with torch.no_grad():
            self.head.sub_(0.1 * self.head.grad)
        self.loss.copy_(loss.detach())

    def feed(self, seed):
        self.x.copy_(rand(130, 64, seed=seed))
        self.y.copy_(torch.randint(0, 500, (130,), generator=torch.Generator().manual_seed(seed)))
        self.k.fill_(1.0)
        self.k[: 10 * (seed % 5)] = 0

    def state(self):
        return [t.clone() for t in (self.loss, self.body, self.head, self.body.grad, self.head.grad, self.opt.state[self.body]["momentum_buffer"])]


@pytest.mark.parametrize("into_grad", [False, True])
def test_a_captured_step_is_the_eager_one(into_grad):
    eager, captured = Step(into_grad), Step(into_grad)
    side = torch.cuda.Stream()
    for step in (eager, captured):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step.feed(7)
            step()
        torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured()
    for seed in (11, 12, 13):
        eager.feed(seed)
        eager()
        captured.feed(seed)
        graph.replay()
        for a, b in zip(eager.state(), captured.state()):
            assert torch.equal(a, b)
