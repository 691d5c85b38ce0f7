"""Workers that average their gradients before they step the matrices' optimiser stay one model; that is all it asks of a group."""
import socket

import torch
import torch.distributed as dist
import torch.multiprocessing as mp

from paper_1810_05291_b200.optim import OrthogonalMomentum
from tests import head_stand_ins


def gradients(rank, step):
    g = torch.Generator().manual_seed(100 * step + rank)
    return [torch.randn(s, generator=g) for s in ((6, 9), (4, 3, 2))]


def model():
    g = torch.Generator().manual_seed(0)
    ps = [torch.nn.Parameter(torch.randn(s, generator=g)) for s in ((6, 9), (4, 3, 2))]
    return ps, OrthogonalMomentum(ps, lr=0.1, weight_decay=0.1, kernels=head_stand_ins.Kernels())


def _worker(rank, world, port):
    dist.init_process_group("gloo", init_method="tcp://127.0.0.1:%d" % port, rank=rank, world_size=world)
    try:
        (ps, opt), (alone, one) = model(), model()
        for step in range(3):
            for p, g in zip(ps, gradients(rank, step)):
                p.grad = g
                dist.all_reduce(p.grad)
                p.grad /= world
            opt.step()
            for p, *gs in zip(alone, *(gradients(r, step) for r in range(world))):
                p.grad = sum(gs) / world
            one.step()
        for p, q in zip(ps, alone):
            everyone = [torch.zeros_like(p) for _ in range(world)]
            dist.all_gather(everyone, p.detach())
            assert all(torch.equal(e, p) for e in everyone)  # the replicas never drifted apart
            assert torch.equal(p, q)                         # one process with the mean of all gradients (of two, in either order)
    finally:
        dist.destroy_process_group()


def test_workers_over_gloo_stay_one_model():
    with socket.socket() as s:
        s.bind(("127.0.0.1", 0))
        port = s.getsockname()[1]
    mp.spawn(_worker, args=(2, port), nprocs=2, join=True)
