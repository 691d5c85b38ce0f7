"""The cross entropy at the head and the orthogonal update as users run them on the GPU: through autograd and the optimiser,
on other streams, captured and replayed, from two threads, with a workspace of their own, on more than 2^31 elements, together."""
import threading

import pytest
import torch

from paper_1810_05291_b200 import binding as B
from paper_1810_05291_b200 import train_ops as T
from paper_1810_05291_b200.optim import OrthogonalMomentum
from tests import head_ref, ortho_ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def rand(shape, seed, dtype=F32, size=1.0):
    return (size * torch.randn(*shape, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV)).to(dtype)


def head_case(rows, width, vocab, dtype=BF16, seed=0):
    g = torch.Generator(device=DEV).manual_seed(seed + 77)
    y = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    return rand((rows, width), seed, dtype), rand((vocab, width), seed + 1, dtype, width ** -0.5), y, torch.rand(rows, generator=g, device=DEV) + 0.1


def head_run(x, w, y, k, grads=True, **options):
    out = [torch.empty(2, device=DEV), torch.empty(x.shape[0], device=DEV)]
    if grads:
        out += [torch.empty_like(x), torch.empty_like(w)]
    B.ss_linear_cross_entropy(x, w, y, k, *out, **options)
    return out


def near(got, want, tol):
    assert float((got.double() - want.double()).norm() / want.double().norm()) < tol


# bf16 gradients carry P's rounding (2^-8 at most for each term, 2^-9 in the mean) and their own (2^-8 at most)
@pytest.mark.parametrize("dtype,wdtype,tol", [(F32, F32, 2e-5), (BF16, F32, 2.0 ** -8), (BF16, BF16, 2.0 ** -7)])
def test_autograd(dtype, wdtype, tol):
    x, w, y, k = head_case(300, 128, 1000, dtype)
    w = w.to(wdtype)
    x, w = x.requires_grad_(), w.requires_grad_()
    want = head_ref.head(x.detach(), w.detach().to(dtype), y, k, 0.9, 0.01, 2.5)
    loss, square, logp = T.linear_cross_entropy(x, w, y, k, 0.9, 0.01)
    (2.5 * loss).backward()
    near(loss.detach(), want["totals"][0], 1e-5)
    near(logp, want["logp"], 1e-4)
    near(x.grad, want["dx"], max(tol, 2.0 ** -7 if dtype == BF16 else tol))
    near(w.grad, want["dw"], tol)
    assert x.grad.dtype == dtype and w.grad.dtype == wdtype
    again = w.grad.clone()
    if wdtype == F32:
        w.grad.zero_()
        (2.5 * T.linear_cross_entropy(x, w, y, k, 0.9, 0.01, into_grad=True)[0]).backward()
        near(w.grad, again, 1e-6)


def test_autograd_on_another_stream():
    x, w, y, k = head_case(256, 256, 4000)
    x, w = x.requires_grad_(), w.float().requires_grad_()
    T.linear_cross_entropy(x, w, y, k)[0].backward()
    want_x, want_w = x.grad.clone(), w.grad.clone()
    x.grad = None
    w.grad.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        with torch.cuda.stream(side):
            loss = T.linear_cross_entropy(x, w, y, k, into_grad=True)[0]
        loss.backward()
    torch.cuda.synchronize()
    near(w.grad, 3 * want_w, 1e-6)
    near(x.grad, 3 * want_x, 2.0 ** -7)


@pytest.mark.parametrize("grads", [False, True])
def test_head_with_a_stream_and_workspace_of_ones_own(grads):
    c = head_case(700, 192, 3001)
    want = head_run(*c, grads=grads)
    need = B.ss_linear_cross_entropy_workspace(c[1], 700, grads, BF16 if grads else None)
    ws = torch.full((need,), 255, dtype=torch.uint8, device=DEV)   # NaN throughout: it needs no initial content
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = head_run(*c, grads=grads, workspace=ws, stream=side)
    also = head_run(*c, grads=grads, stream=side.cuda_stream)
    torch.cuda.synchronize()
    for a, b, d in zip(want, got, also):
        assert torch.equal(a, b) and torch.equal(a, d)
    with pytest.raises(B.SignSGDError):
        head_run(*c, grads=grads, workspace=ws[:need - 256])


@pytest.mark.parametrize("shape", [(100, 200), (300, 700)])
def test_ortho_with_a_stream_and_workspace_of_ones_own(shape):
    u = [rand(shape, i) for i in range(3)]
    want = [torch.empty_like(m) for m in u]
    B.ss_orthogonalise(u, want)
    ws = torch.full((B.ss_orthogonal_workspace(3, *shape),), 255, dtype=torch.uint8, device=DEV)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = [torch.empty_like(m) for m in u]
    B.ss_orthogonalise(u, got, workspace=ws, stream=side)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert torch.equal(a, b)
    with pytest.raises(B.SignSGDError):
        B.ss_orthogonalise(u, got, workspace=ws[:-256])


def test_captured_and_replayed_with_other_inputs():
    """One graph with both operators; its inputs change between replays, the number of positions that count among them."""
    x, w, y, k = head_case(400, 128, 2000)
    u = [rand((300, 200), i) for i in range(2)] + [rand((300, 200), 9)]
    small = [rand((64, 500), 5)]
    outs = [torch.empty(2, device=DEV), torch.empty(400, device=DEV), torch.empty_like(x), torch.empty_like(w)]
    o, os_ = [torch.empty_like(m) for m in u], [torch.empty_like(m) for m in small]

    def run():
        B.ss_linear_cross_entropy(x, w, y, k, *outs)
        B.ss_orthogonalise(u, o)
        B.ss_orthogonalise(small, os_)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in (11, 12):
        c = head_case(400, 128, 2000, seed=seed)
        for a, b in zip((x, w, y, k), c):
            a.copy_(b)
        k[: 100 * (seed - 10)] = 0
        for i, m in enumerate(u + small):
            m.copy_(rand(tuple(m.shape), seed + i))
        graph.replay()
        got = [t.clone() for t in outs + o + os_]
        for t in outs + o + os_:
            t.fill_(-7)
        run()
        for a, b in zip(got, outs + o + os_):
            assert torch.equal(a, b)


def test_two_graphs_share_a_pool():
    """Their workspaces may lie in the same memory: each replay is whole before the next begins."""
    cases = [head_case(300, 96, 1500, seed=s) for s in (1, 2)]
    outs = [[torch.empty(2, device=DEV), torch.empty(300, device=DEV), torch.empty_like(c[0]), torch.empty_like(c[1])] for c in cases]
    want = [head_run(*c) for c in cases]
    torch.cuda.synchronize()
    graphs, pool = [], None
    for c, out in zip(cases, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=pool):
            B.ss_linear_cross_entropy(*c, *out)
        pool = g.pool()
        graphs.append(g)
    for g in (graphs[0], graphs[1], graphs[0]):
        g.replay()
    for a, b in zip(want, outs):
        for s, t in zip(a, b):
            assert torch.equal(s, t)


def test_two_host_threads():
    cases = [head_case(200 + 50 * i, 128, 1000, seed=i) for i in range(2)]
    mats = [[rand((150, 160), i)] for i in range(2)]
    want = [head_run(*c) for c in cases]
    want_o = [[torch.empty_like(m[0])] for m in mats]
    for m, o in zip(mats, want_o):
        B.ss_orthogonalise(m, o)
    torch.cuda.synchronize()
    bad = []

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                got, o = head_run(*cases[i]), [torch.empty_like(mats[i][0])]
                B.ss_orthogonalise(mats[i], o)
                stream.synchronize()
                if not all(torch.equal(a, b) for a, b in zip(got + o, want[i] + want_o[i])):
                    bad.append(i)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


def test_head_in_several_pieces():
    """More rows than a piece has: the rows' results are those of a call of their own, the weight gradient the sum of theirs."""
    rows, width, vocab = 9000, 64, 70000                     # 140 KB a row: pieces of 7424 rows
    x, w, y, k = head_case(rows, width, vocab, seed=3)
    k[5000:5600] = 0
    totals, logp, dx, dw = head_run(x, w, y, k)
    sums = torch.zeros(vocab, width, dtype=torch.float64, device=DEV)
    for a, b in ((0, 4000), (4000, rows)):
        t, lp, d, g = (torch.empty(2, device=DEV), torch.empty(b - a, device=DEV), torch.empty(b - a, width, dtype=BF16, device=DEV),
                       torch.empty(vocab, width, device=DEV))
        B.ss_linear_cross_entropy(x[a:b], w, y[a:b], k[a:b], t, lp, d, g)
        assert torch.equal(lp, logp[a:b])
        near(dx[a:b], d, 2.0 ** -9)                          # sums in other parts round otherwise here and there
        sums += g.double()
    near(dw, sums, 2.0 ** -8)
    acc = torch.ones(vocab, width, device=DEV)
    B.ss_linear_cross_entropy(x, w, y, k, totals, logp, None, acc, accumulate=True)
    near(acc - 1, sums, 1e-5)
    k[:] = 0                                                 # pieces of which none counts
    for t in head_run(x, w, y, k):
        assert not bool(t.any())


def test_loss_alone_in_several_pieces():
    c = head_case(40000, 64, 500, seed=4)
    totals, logp = head_run(*c, grads=False)
    for a, b in ((0, 700), (700, 17000), (17000, 40000)):
        assert torch.equal(head_run(c[0][a:b], c[1], c[2][a:b], c[3][a:b], grads=False)[1], logp[a:b])
    assert abs(float(totals[0]) + float((c[3].double() * logp.double()).sum())) < 1e-6 * float(totals[0].abs())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,width,vocab", [(1, 64, 300), (200, 160, 1111), (256, 64, 70000), (257, 130, 5003), (8000, 64, 70000)])
def test_head_writes_nothing_behind_its_workspace(rows, width, vocab, dtype):
    x, w, y, k = head_case(rows, width, vocab, dtype)
    for dwt in {dtype, F32}:
        need = B.ss_linear_cross_entropy_workspace(w, rows, True, dwt)
        ws = torch.full((need + 8192,), 171, dtype=torch.uint8, device=DEV)
        dx, dw = torch.empty_like(x), torch.empty(vocab, width, dtype=dwt, device=DEV)
        B.ss_linear_cross_entropy(x, w, y, k, torch.empty(2, device=DEV), torch.empty(rows, device=DEV), dx, dw, workspace=ws)
        assert bool((ws[need:] == 171).all())


@pytest.mark.parametrize("shape", [(3, 5), (129, 1), (130, 130), (100, 2049), (333, 257), (2000, 1999), (4100, 140)])
def test_ortho_writes_nothing_behind_its_workspace(shape):
    u = [rand(shape, i) for i in range(2)]
    need = B.ss_orthogonal_workspace(2, *shape)
    ws = torch.full((need + 8192,), 171, dtype=torch.uint8, device=DEV)
    B.ss_orthogonalise(u, [torch.empty_like(m) for m in u], workspace=ws)
    assert bool((ws[need:] == 171).all())


def test_head_beyond_2_31_elements():
    """Logits of 2.4e9 and a weight gradient behind 2^31 elements of a wider buffer: a few rows and columns against the formula."""
    rows, width, vocab = 18432, 64, 131072
    x, w, y, k = head_case(rows, width, vocab, seed=5)
    wide = torch.zeros(vocab, 17000, dtype=BF16, device=DEV)
    dw = wide[:, 16900:16964]
    totals, logp, dx = torch.empty(2, device=DEV), torch.empty(rows, device=DEV), torch.empty_like(x)
    B.ss_linear_cross_entropy(x, w, y, k, totals, logp, dx, dw)
    at = torch.tensor([0, 1, 8191, 8192, 16383, 16384, rows - 1], device=DEV)
    z = x[at].double() @ w.double().t()
    lse = torch.logsumexp(z, 1)
    near(logp[at], z.gather(1, y[at, None])[:, 0] - lse, 1e-5)
    p = torch.exp(z - lse[:, None])
    p[torch.arange(len(at), device=DEV), y[at]] -= 1
    near(dx[at], (k[at, None].double() * p) @ w.double(), 2.0 ** -7)
    cols = torch.tensor([0, 65535, vocab - 1, int(y[rows - 1])], device=DEV)
    z = x.double() @ w[cols].double().t()
    lse = []
    for part in x.split(2048):
        lse.append(torch.logsumexp(part.double() @ w.double().t(), 1))
    p = torch.exp(z - torch.cat(lse)[:, None]) - (y[:, None] == cols).double()
    near(dw[cols], (k.double()[:, None] * p).t() @ x.double(), 2.0 ** -7)
    assert not bool(wide[:, :16900].any()) and not bool(wide[:, 16964:].any())


def test_ortho_beyond_2_31_elements():
    """Matrices far into one buffer, rows of a stride that passes 2^31 elements in all."""
    whole = torch.zeros(200, 11_000_000, dtype=BF16, device=DEV)
    whole[:, -300:] = rand((200, 300), 1, BF16)
    u = whole[:, -300:]
    out = torch.empty(200, 300, device=DEV)
    B.ss_orthogonalise([u], [out])
    want = torch.empty_like(out)
    B.ss_orthogonalise([u.contiguous()], [want])
    assert torch.equal(out, want)
    whole[:, :300].fill_(3)
    B.ss_orthogonalise([u], [u])
    assert torch.equal(u, want.to(BF16)) and bool((whole[:, :300] == 3).all()) and not bool(whole[:, 300:600].any())


def test_large_matrices_in_pairs_of_blocks():
    for shape in ((2600, 2500), (1200, 5000), (5000, 1100)):
        u = rand(shape, sum(shape), BF16)
        out = torch.empty(shape, device=DEV)
        B.ss_orthogonalise([u, u], [out, torch.empty_like(out)])
        want, model = ortho_ref.orthogonalised(u), ortho_ref.orthogonalised(u, rounded=True)
        assert float((out.double() - want).norm()) <= 2 * float((model - want).norm()) + 2e-5 * float(want.norm())


def test_optimiser_steps_and_keeps_parameters_in_place():
    shapes = [(300, 200)] * 3 + [(64, 3, 3, 3), (64, 64), (200, 300)]
    ps = [torch.nn.Parameter(rand(s, i, size=0.1)) for i, s in enumerate(shapes)]
    opt = OrthogonalMomentum(ps, lr=0.01, weight_decay=0.1)
    at = [p.data_ptr() for p in ps]
    want = [(p.detach().view(p.shape[0], -1).double(), torch.zeros(p.shape[0], p[0].numel(), device=DEV)) for p in ps]
    for step in range(2):
        for i, p in enumerate(ps):
            p.grad = rand(p.shape, 100 * step + i, size=1e-3)
        opt.step()
        for i, (p, (m, v)) in enumerate(zip(ps, want)):
            nv, np_ = ortho_ref.updated(p.grad.view(m.shape), v, m, 0.95, True, 0.01, 0.2 * max(m.shape) ** 0.5, 0.1)
            want[i] = (np_, nv)
    assert at == [p.data_ptr() for p in ps]
    for p, (m, v) in zip(ps, want):
        near(opt.state[p]["momentum_buffer"].view(m.shape), v, 1e-6)
        # a step is 0.01 * 0.2 a coordinate, of which 5e-3 at most is rounding, against parameters of 0.1
        near(p.detach().view(m.shape), m, 2 * 0.002 * 5e-3 / 0.1)


def test_the_example_runs_and_its_gradients_are_the_formulas():
    from examples import next_token
    model, history = next_token.train(steps=3, say=lambda s: None)
    assert len(history) == 3 and all(h == h and abs(h) < 100 for h in history)
    gen = torch.Generator().manual_seed(5)
    now, previous, targets, weights = next_token.batch_of(97, 16, gen, DEV)
    hidden = model(now, previous)
    x = hidden.detach().requires_grad_()
    model.head.grad.zero_()
    T.linear_cross_entropy(x, model.head, targets, weights, z_coef=1e-4, into_grad=True)[0].backward()
    want = head_ref.head(x.detach(), model.head.detach().to(BF16), targets, weights, 1.0, 1e-4)
    near(model.head.grad, want["dw"], 2.0 ** -8)
    near(x.grad, want["dx"], 2.0 ** -7)


def test_tensors_must_share_a_device_and_shapes():
    x, w, y, k = head_case(10, 64, 100)
    t, lp = torch.empty(2, device=DEV), torch.empty(10, device=DEV)
    for bad in (dict(weight=w.cpu()), dict(targets=y.cpu()), dict(weights=k[:5]), dict(targets=y.int()), dict(weight=w.float()),
                dict(weight=w[:, :32]), dict(dx=torch.empty(10, 32, dtype=BF16, device=DEV)), dict(dw=torch.empty(100, 64, dtype=torch.half, device=DEV)),
                dict(totals=torch.empty(3, device=DEV)), dict(x=x.t())):
        args = dict(x=x, weight=w, targets=y, weights=k, totals=t, logp=lp)
        args.update(bad)
        with pytest.raises((ValueError, TypeError)):
            B.ss_linear_cross_entropy(**args) if "x" not in bad else B.ss_linear_cross_entropy(args.pop("x"), **args)
    u = [rand((5, 6), 1), rand((5, 6), 2)]
    for ins, outs in (([u[0], u[1][:, :5]], u), (u, [u[0].cpu(), u[1]]), ([u[0], rand((5, 8), 1)[:, :6]], u), (u, u[:1])):
        with pytest.raises((ValueError, TypeError)):
            B.ss_orthogonalise(ins, outs)
    with pytest.raises(B.SignSGDError):
        B.ss_orthogonalise(u, [u[0].clone(), u[0].clone()], coefficients=[(float("nan"), 1.0, 1.0)])
    with pytest.raises(B.SignSGDError):
        B.ss_orthogonalise(u, [u[1], u[0]])                   # each over the other's input
