"""The cross entropy at the head and the orthogonal update without a GPU: sizes, and refusals before any CUDA call."""
import ctypes

import pytest
import torch

from paper_1810_05291_b200 import binding as B
from paper_1810_05291_b200 import build as libbuild

vp = ctypes.c_void_p
OK, BAD, MIS, UNS = B.SS_OK, B.SS_ERR_INVALID_ARG, B.SS_ERR_MISALIGNED, B.SS_ERR_UNSUPPORTED
NAN, INF = float("nan"), float("inf")
BIG = 1 << 31


@pytest.fixture(scope="module")
def L():
    libbuild.build()
    return B.lib()


def head(L, x=0x1000000, xs=64, w=0x2000000, ws=64, dt=0, rows=4, width=64, vocab=100, y=0x3000000, k=0x3100000, c=1.0,
         z=0.0, gs=0x3200000, totals=0x3300000, logp=0x3400000, dx=0x4000000, dxs=64, dw=0x5000000, dws=64, dwt=0, acc=0,
         scratch=0x10000000, bytes_=1 << 28):
    return L.ss_linear_cross_entropy(vp(x), xs, vp(w), ws, dt, rows, width, vocab, vp(y), vp(k), c, z, vp(gs), vp(totals),
                                     vp(logp), vp(dx), dxs, vp(dw), dws, dwt, acc, vp(scratch), bytes_, None)


def test_head_refusals(L):
    for name in ("x", "w", "y", "k", "totals", "logp", "scratch"):
        assert head(L, **{name: 0}) == BAD, name
    assert head(L, dt=2) == BAD and head(L, dwt=5) == BAD and head(L, dwt=1) == BAD    # a bf16 dw of fp32 inputs
    assert head(L, dt=1, dwt=1, acc=1) == BAD                                           # added to in fp32 only
    for name in ("rows", "width", "vocab"):
        assert head(L, **{name: -1}) == BAD and head(L, **{name: BIG}) == BAD
    assert head(L, width=0) == BAD and head(L, vocab=0) == BAD
    for name in ("xs", "ws", "dxs", "dws"):
        assert head(L, **{name: 63}) == BAD and head(L, **{name: 1 << 40}) == BAD
    for v in (0.0, -1.0, NAN, INF):
        assert head(L, c=v) == BAD
    assert head(L, z=NAN) == BAD and head(L, z=INF) == BAD
    for name, at in (("x", 0x1000002), ("w", 0x2000002), ("y", 0x3000004), ("k", 0x3100002), ("gs", 0x3200001), ("totals", 0x3300002),
                     ("logp", 0x3400002), ("dx", 0x4000002), ("dw", 0x5000002), ("scratch", 0x10000080)):
        assert head(L, **{name: at}) == MIS, name
    assert head(L, dx=0x1000010) == BAD and head(L, dx=0x1000000, dxs=128) == BAD       # over x, but not in place
    assert head(L, dx=0x2000000) == BAD and head(L, dw=0x2000000) == BAD and head(L, dw=0x1000000) == BAD and head(L, dw=0x4000010) == BAD
    for out in ("dx", "dw"):
        for other in (0x3000000, 0x3100000, 0x3200000, 0x3300000, 0x3400000):
            assert head(L, **{out: other}) == BAD
    for other in (0x1000000, 0x2000000, 0x3000000, 0x3100000, 0x3200000):
        assert head(L, totals=other) == BAD and head(L, logp=other) == BAD
    assert head(L, totals=0x3400004) == BAD
    for other in (0x1000000, 0x2000000, 0x3000000, 0x3100000, 0x3300000, 0x3400000, 0x4000000, 0x5000000):
        assert head(L, scratch=other) == BAD
    far = dict(x=1 << 44, w=2 << 44, y=3 << 44, k=4 << 44, logp=5 << 44, dx=6 << 44, dw=7 << 44)
    assert head(L, rows=(1 << 24) + 1, **far) == UNS
    assert head(L, vocab=(1 << 31) - 1, rows=1024, **far) == UNS


@pytest.mark.parametrize("dt", [0, 1])
def test_head_workspace(L, dt):
    size = lambda rows=4, width=64, vocab=100, w=0x2000000, ws=64, dx=1, dw=1, dwt=0: \
        L.ss_linear_cross_entropy_workspace(vp(w), ws, dt, rows, width, vocab, dx, dw, dwt)  # noqa: E731
    need = size()
    assert need > 0 and head(L, dt=dt, bytes_=need - 1) == BAD
    assert size(rows=0) == 0 and size(rows=-1) == -1 and size(width=0) == -1 and size(ws=3) == -1
    assert size(dx=0, dw=0) < need
    if dt == 1:
        assert size(w=0x2000002) > need                      # a copy of w
        assert size(dwt=1) == need
    # what does not depend on the rows is bounded: the pieces are at most a GiB
    big = size(rows=1 << 20, width=1024, vocab=131072, ws=1024, dw=0)
    assert big < (2 << 30) + (1 << 20) * 1024 * 2 * (3 if dt == 0 else 1) + (131072 * 1024 * 6 if dt == 0 else 0)


def ptrs(at, n=2, step=0x100000):
    return (vp * n)(*[at + i * step if at else None for i in range(n)])


CO = (ctypes.c_float * 6)(3.4, -4.7, 2.0, 3.4, -4.7, 2.0)


def ortho(L, a=0x1000000, a_s=40, at=0, b=0x2000000, bs=40, bt=0, n=2, rows=30, cols=40, co=CO, steps=2, scratch=0x10000000, bytes_=1 << 24, arrays=None):
    x, y = arrays or (ptrs(a), ptrs(b))
    return L.ss_orthogonalise(x, a_s, at, y, bs, bt, n, rows, cols, co, steps, vp(scratch), bytes_, None)


def test_orthogonalise_refusals(L):
    assert ortho(L, a=0) == BAD and ortho(L, b=0) == BAD and ortho(L, scratch=0) == BAD and ortho(L, co=None) == BAD
    assert ortho(L, arrays=(None, ptrs(0x2000000))) == BAD and ortho(L, arrays=(ptrs(0x1000000), None)) == BAD
    assert ortho(L, at=2) == BAD and ortho(L, bt=-1) == BAD
    assert ortho(L, n=65) == BAD and ortho(L, n=-1) == BAD and ortho(L, rows=-1) == BAD and ortho(L, cols=BIG) == BAD
    assert ortho(L, steps=0) == BAD and ortho(L, steps=33) == BAD
    for v in (NAN, INF):
        assert ortho(L, co=(ctypes.c_float * 6)(3.4, -4.7, 2.0, 3.4, v, 2.0)) == BAD
    assert ortho(L, a_s=39) == BAD and ortho(L, bs=39) == BAD and ortho(L, bs=1 << 40) == BAD
    assert ortho(L, a=0x1000002) == MIS and ortho(L, b=0x2000001) == MIS and ortho(L, scratch=0x10000010) == MIS
    assert ortho(L, b=0x1000010) == BAD and ortho(L, b=0x1000000, bs=48) == BAD and ortho(L, b=0x1000000, bt=1) == BAD
    assert ortho(L, b=0x1100000) == BAD                       # out_0 over in_1
    assert ortho(L, arrays=(ptrs(0x1000000), ptrs(0x2000000, step=16))) == BAD
    assert ortho(L, scratch=0x1000000) == BAD and ortho(L, scratch=0x2100000) == BAD
    assert ortho(L, bytes_=L.ss_orthogonal_workspace(2, 30, 40) - 1) == BAD
    assert ortho(L, n=0) == OK and ortho(L, rows=0) == OK and ortho(L, cols=0, a=0, b=0) == OK
    assert ortho(L, n=1, b=0x100000000, rows=(1 << 20) + 1) == UNS


def test_orthogonal_workspace(L):
    w = L.ss_orthogonal_workspace
    assert w(-1, 3, 3) == -1 and w(65, 3, 3) == -1 and w(1, -1, 3) == -1 and w(1, 3, (1 << 20) + 1) == -1
    assert w(0, 3, 3) == 0 and w(2, 0, 3) == 0 and w(1, 1, 1) > 0 and w(3, 100, 70) > w(2, 100, 70)


def update(L, g=0x1000000, gs=40, dt=0, v=0x2000000, vo=0x3000000, vs=40, p=0x4000000, po=0x5000000, ps=40, n=2, rows=30, cols=40,
           beta=0.9, co=CO, steps=2, lr=0.1, scale=1.0, wd=0.0, scratch=0x10000000, bytes_=1 << 24):
    return L.ss_orthogonal_update(ptrs(g), gs, dt, ptrs(v), ptrs(vo), vs, ptrs(p), ptrs(po), ps, n, rows, cols, beta, 1, co, steps,
                                  lr, scale, wd, vp(scratch), bytes_, None)


def test_update_refusals(L):
    for name in ("g", "v", "vo", "p", "po", "scratch"):
        assert update(L, **{name: 0}) == BAD, name
    for name in ("gs", "vs", "ps"):
        assert update(L, **{name: 39}) == BAD
    for name, at in (("g", 0x1000002), ("v", 0x2000002), ("vo", 0x3000002), ("p", 0x4000002), ("po", 0x5000001), ("scratch", 0x10000020)):
        assert update(L, **{name: at}) == MIS, name
    for beta in (-0.1, 1.0, NAN):
        assert update(L, beta=beta) == BAD
    for name in ("lr", "scale", "wd"):
        assert update(L, **{name: NAN}) == BAD and update(L, **{name: INF}) == BAD
    assert update(L, dt=3) == BAD and update(L, n=65) == BAD and update(L, steps=0) == BAD and update(L, co=None) == BAD
    for out in ("vo", "po"):
        for other in (0x1000000, 0x2000010, 0x4000010, 0x2100000):
            assert update(L, **{out: other}) == BAD, (out, hex(other))
    assert update(L, vo=0x4000000) == BAD and update(L, po=0x2000000) == BAD and update(L, vo=0x5000000) == BAD
    for other in (0x1000000, 0x2000000, 0x3000000, 0x4000000, 0x5000000):
        assert update(L, scratch=other) == BAD
    assert update(L, bytes_=L.ss_orthogonal_workspace(2, 30, 40) - 1) == BAD
    assert update(L, n=0) == OK and update(L, rows=0) == OK


def test_binding_refuses_what_it_cannot_marshal(L):
    m, y, k = torch.zeros(4, 32), torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    for call in (lambda: B.ss_linear_cross_entropy(m, m, y, k, k[:2], k), lambda: B.ss_orthogonalise([m], [m.clone()]),
                 lambda: B.ss_orthogonal_update([m], [m], [m], [m], [m], 0.9)):
        with pytest.raises(ValueError):                      # tensors on the host
            call()
    with pytest.raises(TypeError):
        B.ss_orthogonalise([m.half()], [m])
    with pytest.raises(ValueError):
        B.ss_orthogonalise([m, m], [m])                      # counts
    with pytest.raises(ValueError):
        B._coefficients(((1.0, 2.0),))
