"""The training operators' entry points without a GPU: sizes, and refusals before any CUDA call."""
import ctypes

import pytest
import torch

from paper_1810_05291_b200 import binding as B
from paper_1810_05291_b200 import build as libbuild

vp = ctypes.c_void_p
BAD, MIS = B.SS_ERR_INVALID_ARG, B.SS_ERR_MISALIGNED
NAN, INF = float("nan"), float("inf")
BIG = 1 << 31


@pytest.fixture(scope="module")
def L():
    libbuild.build()
    return B.lib()


def test_checkpoint_sizes(L):
    assert B.ss_act8_bytes(0, 10) == 0 and B.ss_act8_bytes(10, 0) == 0
    assert B.ss_act8_bytes(1, 1) == 33 and B.ss_act8_bytes(3, 32) == 99 and B.ss_act8_bytes(3, 33) == 198
    assert B.ss_act8_bytes(BIG - 1, BIG - 1) == (BIG - 1) * (BIG // 32) * 33
    assert B.ss_act8_bytes(-1, 4) == -1 and B.ss_act8_bytes(4, BIG) == -1


def pack(L, x=0x10000, stride=40, dt=0, rows=3, cols=40, ck=0x20000):
    return L.ss_act8_pack(vp(x), stride, dt, rows, cols, vp(ck), None)


def unpack(L, ck=0x20000, rows=3, cols=40, out=0x10000, stride=40, dt=0):
    return L.ss_act8_unpack(vp(ck), rows, cols, vp(out), stride, dt, None)


@pytest.mark.parametrize("call,big", [(pack, "x"), (unpack, "out")])
def test_pack_and_unpack_refusals(L, call, big):
    assert call(L, **{big: 0}) == BAD and call(L, ck=0) == BAD
    assert call(L, dt=5) == BAD and call(L, rows=-1) == BAD and call(L, cols=BIG) == BAD
    assert call(L, stride=39) == BAD and call(L, stride=1 << 40) == BAD
    assert call(L, **{big: 0x10002}) == MIS and call(L, ck=0x20008) == MIS
    assert call(L, ck=0x10010) == BAD                         # overlap
    assert call(L, rows=0, ck=0, **{big: 0}) == B.SS_OK and call(L, cols=0, stride=0) == B.SS_OK


def forward(L, x=0x10000, xs=40, up=0x20000, us=40, dt=0, act=1, rows=3, cols=40, y=0x30000, ys=40, cx=0x40000,
            cu=0x50000, cy=0x60000):
    return L.ss_act8_forward(vp(x), xs, vp(up), us, dt, act, rows, cols, vp(y), ys, vp(cx), vp(cu), vp(cy), None)


def test_forward_refusals(L):
    for k in ("x", "y", "cx", "cu"):
        assert forward(L, **{k: 0}) == BAD
    assert forward(L, up=0) == BAD                            # checkpoint of up without up
    assert forward(L, act=2) == BAD and forward(L, dt=2) == BAD and forward(L, rows=BIG) == BAD
    for k in ("xs", "us", "ys"):
        assert forward(L, **{k: 39}) == BAD
    for k in ("x", "up", "y"):
        assert forward(L, **{k: 0x30002 if k == "y" else 0x70002}) == MIS
    for k in ("cx", "cu", "cy"):
        assert forward(L, **{k: 0x70004}) == MIS
    assert forward(L, y=0x10004) == BAD                       # over x, but not in place
    assert forward(L, y=0x10000, ys=48) == BAD                # in place with another stride
    assert forward(L, y=0x20004) == BAD
    assert forward(L, cx=0x10010) == BAD and forward(L, cu=0x20010) == BAD and forward(L, cy=0x30010) == BAD
    assert forward(L, cx=0x40000, cu=0x40010) == BAD and forward(L, cy=0x50000) == BAD
    assert forward(L, rows=0, x=0, y=0) == B.SS_OK


def backward(L, dy=0x10000, dys=40, cx=0x40000, cu=0x50000, dt=0, act=1, rows=3, cols=40, dx=0x20000, dxs=40,
             du=0x30000, dus=40):
    return L.ss_act8_backward(vp(dy), dys, vp(cx), vp(cu), dt, act, rows, cols, vp(dx), dxs, vp(du), dus, None)


def test_backward_refusals(L):
    for k in ("dy", "cx", "dx", "cu", "du"):
        assert backward(L, **{k: 0}) == BAD
    for k in ("dys", "dxs", "dus"):
        assert backward(L, **{k: 8}) == BAD
    for k in ("dy", "dx", "du"):
        assert backward(L, **{k: 0x70002}) == MIS
    assert backward(L, cx=0x70008) == MIS
    assert backward(L, act=-1) == BAD and backward(L, dt=9) == BAD
    assert backward(L, dx=0x10004) == BAD and backward(L, du=0x10004) == BAD
    assert backward(L, dx=0x10000, du=0x10000) == BAD         # both in place
    assert backward(L, du=0x20000) == BAD
    assert backward(L, dx=0x40010) == BAD and backward(L, du=0x50010) == BAD
    # columns of one wider matrix interleave; too close they overlap
    assert backward(L, dx=0x20000, dxs=80, du=0x20000 + 39 * 4, dus=80) == BAD


def grad(L, dy=0x100000, dys=24, dt=0, ck=0x200000, rows=5, n_out=24, n_in=40, dw=0x300000, dws=40, acc=0, ws=0x400000,
         bytes_=1 << 20):
    return L.ss_weight_grad8(vp(dy), dys, dt, vp(ck), rows, n_out, n_in, vp(dw), dws, acc, vp(ws), bytes_, None)


def test_weight_grad_refusals(L):
    for k in ("dy", "ck", "dw"):
        assert grad(L, **{k: 0}) == BAD
    assert grad(L, dys=23) == BAD and grad(L, dws=39) == BAD and grad(L, dt=3) == BAD
    assert grad(L, rows=-1) == BAD and grad(L, n_out=BIG) == BAD and grad(L, n_in=-3) == BAD
    assert grad(L, dy=0x100001) == MIS and grad(L, dw=0x300002) == MIS and grad(L, ck=0x200001) == MIS
    assert grad(L, dw=0x100010) == BAD and grad(L, dw=0x200010) == BAD
    assert grad(L, n_out=0) == B.SS_OK
    for dt, dy, stride in ((0, 0x100000, 24), (1, 0x100000, 24), (1, 0x100002, 25)):
        need = L.ss_weight_grad8_workspace(vp(dy), stride, dt, 5, 24, 40)
        assert need >= 0
        if need:
            assert grad(L, dt=dt, dy=dy, dys=stride, bytes_=need - 1) == BAD
            assert grad(L, dt=dt, dy=dy, dys=stride, ws=0) == BAD
            assert grad(L, dt=dt, dy=dy, dys=stride, ws=0x400010) == MIS
            assert grad(L, dt=dt, dy=dy, dys=stride, ws=0x300000) == BAD
    assert L.ss_weight_grad8_workspace(vp(0x100000), 24, 7, 5, 24, 40) == -1
    assert L.ss_weight_grad8_workspace(vp(0x100000), 24, 0, BIG, 24, 40) == -1


def policy(L, z=0x100000, zs=64, dt=0, rows=4, vocab=64, y=0x200000, old=0x210000, ref=0x220000, adv=0x230000,
           w=0x240000, c=1.0, lo=0.2, hi=0.2, beta=0.1, gs=0x250000, totals=0x260000, logp=0x270000, dz=0x300000,
           dzs=64, ws=0x400000, bytes_=1 << 20):
    return L.ss_policy_loss(vp(z), zs, dt, rows, vocab, vp(y), vp(old), vp(ref), vp(adv), vp(w), c, lo, hi, beta, vp(gs),
                            vp(totals), vp(logp), vp(dz), dzs, vp(ws), bytes_, None)


def preference(L, z=0x100000, zs=64, dt=0, rows=4, vocab=64, y=0x200000, w=0x240000, begin=0x210000, pairs=2,
               ref=0x220000, c=1.0, kind=0, beta=0.1, eps=0.0, scale=1.0, gs=0x250000, loss=0x260000, margins=0x270000,
               seq=0x280000, logp=0x290000, dz=0x300000, dzs=64, ws=0x400000, bytes_=1 << 20):
    return L.ss_preference_loss(vp(z), zs, dt, rows, vocab, vp(y), vp(w), vp(begin), pairs, vp(ref), c, kind, beta, eps,
                                scale, vp(gs), vp(loss), vp(margins), vp(seq), vp(logp), vp(dz), dzs, vp(ws), bytes_, None)


@pytest.mark.parametrize("call", [policy, preference])
def test_refusals_that_the_losses_share(L, call):
    for k in ("z", "y", "w", "logp", "ws"):
        assert call(L, **{k: 0}) == BAD
    assert call(L, dt=2) == BAD and call(L, rows=-1) == BAD and call(L, vocab=BIG) == BAD
    assert call(L, zs=63) == BAD and call(L, dzs=63) == BAD and call(L, zs=1 << 39) == BAD
    for c in (0.0, -1.0, NAN, INF):
        assert call(L, c=c) == BAD
    for k, v in (("z", 0x100002), ("dz", 0x300002), ("y", 0x200004), ("w", 0x240002), ("gs", 0x250002),
                 ("logp", 0x270002), ("ws", 0x400080)):
        assert call(L, **{k: v}) == MIS
    assert call(L, dz=0x100004) == BAD                       # over the logits, but not in place
    assert call(L, dz=0x100000, dzs=128) == BAD
    assert call(L, logp=0x100010) == BAD and call(L, logp=0x300010) == BAD and call(L, logp=0x240004) == BAD
    assert call(L, ws=0x300000) == BAD and call(L, ws=0x200000) == BAD
    assert call(L, dz=0x240000) == BAD                       # over an input
    pairs = 2 if call is preference else 0
    assert call(L, bytes_=L.ss_loss_workspace(4, pairs) - 1) == BAD


def test_policy_refusals(L):
    for k in ("old", "adv", "totals"):
        assert policy(L, **{k: 0}) == BAD
    assert policy(L, ref=0) == BAD                           # a KL term needs a reference
    assert policy(L, lo=-0.1) == BAD and policy(L, lo=1.1) == BAD and policy(L, hi=-0.1) == BAD
    assert policy(L, lo=NAN) == BAD and policy(L, hi=INF) == BAD and policy(L, beta=NAN) == BAD
    assert policy(L, totals=0x230004) == BAD and policy(L, totals=0x270004) == BAD


def test_preference_refusals(L):
    for k in ("begin", "ref", "loss", "margins", "seq"):
        assert preference(L, **{k: 0}) == BAD
    assert preference(L, kind=3) == BAD and preference(L, kind=-1) == BAD and preference(L, pairs=-1) == BAD
    assert preference(L, beta=0.0) == BAD and preference(L, beta=NAN) == BAD and preference(L, beta=INF) == BAD
    assert preference(L, eps=-0.1) == BAD and preference(L, eps=0.6) == BAD and preference(L, eps=0.1, kind=1) == BAD
    assert preference(L, scale=NAN) == BAD and preference(L, scale=INF) == BAD
    assert preference(L, begin=0x210004) == MIS
    assert preference(L, seq=0x270004) == BAD and preference(L, loss=0x220004) == BAD


def test_loss_workspace_sizes(L):
    assert L.ss_loss_workspace(-1, 0) == -1 and L.ss_loss_workspace(0, -1) == -1 and L.ss_loss_workspace(BIG, 0) == -1
    assert L.ss_loss_workspace(100, 10) > 0


def test_binding_refuses_what_it_cannot_marshal(L):
    x, ck = torch.zeros(4, 32), torch.zeros(132, dtype=torch.uint8)
    for call in (lambda: B.ss_act8_pack(x, ck), lambda: B.ss_act8_unpack(ck, x),
                 lambda: B.ss_act8_forward(x, None, B.SS_ACT_GELU, x, ck), lambda: B.ss_weight_grad8(x, ck, x),
                 lambda: B.ss_policy_loss(x, x, x, None, x, x, x, x),
                 lambda: B.ss_preference_loss(x, x, x, x, x, x, x, x, x)):
        with pytest.raises(ValueError):                      # tensors on the host
            call()
    with pytest.raises(TypeError):
        B.ss_act8_pack(x.half(), ck)
