"""The training operators on several streams: a backward pass, and what reads its results on the stream that called it."""
import threading

import pytest
import torch

from paper_1810_05291_b200 import binding as B
from paper_1810_05291_b200 import train_ops as T
from tests import train_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
CYCLES = 20_000_000  # of _sleep: about 10 ms, far longer than the host takes to return


def rand(shape, seed, dtype=torch.float32):
    return torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV).to(dtype)


def slow(y):
    """The gradient that arrives at y comes late on the stream of y's backward pass."""
    def wait(g):
        torch.cuda._sleep(CYCLES)
        return g.clone()
    y.register_hook(wait)
    return y


def near(got, want):
    assert float((got.double() - want).norm() / want.norm()) < 1.5e-6


@pytest.mark.filterwarnings("ignore:The AccumulateGrad node's stream does not match")
@pytest.mark.parametrize("options", [{}, {"into_grad": True}], ids=["default", "into_grad"])
@pytest.mark.parametrize("forward,older,caller", [("side", "main", "main"), ("main", "side", "side"), ("side", "other", "main"), ("side", "side", "main")])
def test_the_caller_s_stream_waits_for_the_weight_s_gradient(options, forward, older, caller):
    """Forward pass, node that accumulates (kept alive from before) and backward() on streams of their own."""
    streams = {"main": torch.cuda.current_stream(), "side": torch.cuda.Stream(), "other": torch.cuda.Stream()}
    x, w, dy = rand((700, 96), 1), rand((130, 96), 2).requires_grad_(), rand((700, 130), 3)
    w.grad = rand((130, 96), 4)
    want = w.grad.double() + dy.double().t() @ ref.act8(x)[2]
    torch.cuda.synchronize()
    with torch.cuda.stream(streams[older]):
        node = torch.autograd.graph.get_gradient_edge(w).node
    with torch.cuda.stream(streams[forward]):
        y = slow(T.linear8(x, w, **options))
    torch.cuda.synchronize()
    with torch.cuda.stream(streams[caller]):
        y.backward(dy)
        got = w.grad.clone()
    torch.cuda.synchronize()
    near(got, want)
    near(w.grad, want)
    del node


@pytest.mark.parametrize("options", [{}, {"into_grad": True}], ids=["default", "into_grad"])
@pytest.mark.parametrize("late", [0, 1])
def test_a_weight_used_on_two_streams(options, late):
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    xs, dys = [rand((4000, 256), k) for k in (1, 2)], [rand((4000, 130), k) for k in (3, 4)]
    w = rand((130, 256), 5).requires_grad_()
    w.grad = torch.zeros_like(w)
    want = sum(dy.double().t() @ ref.act8(x)[2] for x, dy in zip(xs, dys))
    torch.cuda.synchronize()
    ys = []
    for k, s in enumerate(streams):
        with torch.cuda.stream(s):
            y = T.linear8(xs[k], w, **options)
            ys.append(slow(y) if k == late else y)
    torch.cuda.synchronize()
    torch.autograd.backward(ys, dys)
    got = w.grad.clone()
    torch.cuda.synchronize()
    near(got, want)


def test_calls_from_two_threads():
    """Every operator from two host threads at once, each on its own stream and buffers: the bits of one thread's calls."""
    g = torch.Generator(device=DEV).manual_seed(11)
    rows, vocab = 300, 20001
    sets = []
    for _ in range(2):
        z = torch.randn(rows, vocab, generator=g, device=DEV, dtype=torch.bfloat16)
        x, dy = torch.randn(rows, 200, generator=g, device=DEV), torch.randn(rows, 136, generator=g, device=DEV)
        sets.append((z, x, dy))
    y, one = torch.arange(rows, device=DEV), torch.ones(rows, device=DEV)
    begin, zero = torch.tensor([0, 100, 300], device=DEV), torch.zeros(2, device=DEV)

    def calls(z, x, dy):
        new = lambda *n: torch.empty(*n, device=DEV)  # noqa: E731
        totals, logp, dz, loss, margins, seq, dp = new(3), new(rows), torch.empty_like(z), new(1), new(1), new(2), torch.empty_like(z)
        ck, ck_y, out, dx, dw = B.act8_checkpoint(rows, 200, DEV), B.act8_checkpoint(rows, 200, DEV), torch.empty_like(x), torch.empty_like(x), new(136, 200)
        B.ss_policy_loss(z, y, one, None, one, one, totals, logp, dz)
        B.ss_preference_loss(z, y, one, begin, zero, loss, margins, seq, logp, dp)
        B.ss_act8_forward(x, None, B.SS_ACT_GELU, out, ck, None, ck_y)
        B.ss_act8_backward(out, ck, None, B.SS_ACT_GELU, dx)
        B.ss_weight_grad8(dy, ck_y, dw)
        return totals, logp, dz, loss, margins, seq, dp, out, dx, dw, ck, ck_y

    want = [calls(*s) for s in sets]
    torch.cuda.synchronize()
    got = [[], []]

    def work(k):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                got[k].append(calls(*sets[k]))
            torch.cuda.current_stream().synchronize()

    threads = [threading.Thread(target=work, args=(k,)) for k in (0, 1)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    for k in (0, 1):
        assert len(got[k]) == 20
        for outs in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(outs, want[k]))
