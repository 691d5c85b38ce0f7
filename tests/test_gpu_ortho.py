"""The orthogonal update on the GPU, against the formula in 64 bits.

Tolerances. A result differs from the formula's by what the rounding of the operands to fp16 makes of it, which
depends on the matrix (each step enlarges it where singular values are small), and by the rounding of the result. The first is what
the reference gives with the same roundings in 64 bits (``rounded``): a kernel's may differ from that, since a sum
that lies near a rounding's edge falls on the other side, so twice its 2-norm is allowed, and 2e-5 where the reference happens to round nothing.
The second is half a unit of the result's type for each element."""
import pytest
import torch

from paper_1810_05291_b200 import binding as B
from tests import ortho_ref as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def matrix(rows, cols, seed=0, kind="strong", dtype=F32, size=1e-3):
    g = gen(seed)
    m = torch.randn(rows, cols, generator=g, device=DEV)
    if kind == "strong":  # a few directions far above the rest
        k = min(8, rows, cols)
        m = m + 4 * torch.randn(rows, k, generator=g, device=DEV) @ torch.randn(k, cols, generator=g, device=DEV)
    return (size * m).to(dtype)


def near(name, got, u, coefficients=ref.COEFFICIENTS):
    want = ref.orthogonalised(u, coefficients)
    model = ref.orthogonalised(u, coefficients, rounded=True)
    norm = float(want.norm())
    half = torch.finfo(got.dtype).eps / 2
    allowed = 2 * float((model - want).norm()) + 2e-5 * norm + half * norm
    off = float((got.double() - want).norm())
    assert off <= allowed, "%s: off by %.3g, allowed %.3g" % (name, off / norm, allowed / norm)


def run(mats, out_dtype=F32, coefficients=ref.COEFFICIENTS):
    out = [torch.full(m.shape, float("nan"), dtype=out_dtype, device=DEV) for m in mats]
    B.ss_orthogonalise(mats, out, coefficients)
    return out


SHAPES = [(1, 1), (1, 40), (40, 1), (2, 3), (17, 33), (64, 64), (33, 17), (100, 257), (257, 100), (128, 640), (300, 300), (511, 513), (700, 260), (1000, 2048),
          (5, 256), (256, 5), (128, 257), (257, 128), (77, 1000), (1025, 128), (128, 2048), (2048, 100), (2049, 128), (129, 129), (64, 4000), (4096, 128), (128, 4097), (1, 3000)]


@pytest.mark.parametrize("kind", ["strong", "noise"])
@pytest.mark.parametrize("shape", SHAPES, ids=["%dx%d" % s for s in SHAPES])
def test_orthogonalise(shape, kind):
    for dtype in (F32, BF16):
        u = matrix(*shape, seed=sum(shape), kind=kind, dtype=dtype)
        for out in (F32, BF16):
            near("%s -> %s" % (dtype, out), run([u], out)[0], u)


@pytest.mark.parametrize("shape", [(96, 200), (200, 96), (120, 900), (600, 50), (300, 150)])
def test_several_matrices_are_each_their_own(shape):
    mats = [matrix(*shape, seed=i, size=10.0 ** (i - 3)) for i in range(7)]
    for got, u in zip(run(mats), mats):
        assert torch.equal(got, run([u])[0])
        near("one of several", got, u)


def test_as_many_as_a_call_takes():
    mats = [matrix(20, 30, seed=i) for i in range(64)]
    for got, u in zip(run(mats), mats):
        near("of 64", got, u)


@pytest.mark.parametrize("steps", [1, 2, 9])
def test_coefficients_of_each_step(steps):
    co = tuple((2.0 - 0.1 * k, -1.5 + 0.05 * k, 0.5) for k in range(steps))
    u = matrix(150, 220, seed=steps)
    near("%d steps" % steps, run([u], coefficients=co)[0], u, co)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("pad,offset", [(8, 0), (4, 4), (3, 1)])
@pytest.mark.parametrize("rows", [90, 190])
def test_slices_of_wider_matrices(rows, dtype, pad, offset):
    u = matrix(rows, 130 + pad, seed=pad, dtype=dtype)[:, offset:offset + 130]
    whole = torch.full((rows, 130 + pad), 7.0, dtype=dtype, device=DEV)
    out = whole[:, offset:offset + 130]
    B.ss_orthogonalise([u], [out])
    assert torch.equal(out, run([u.contiguous()], dtype)[0])
    out.fill_(7)
    assert bool((whole == 7).all())


def test_in_place():
    for dtype in (F32, BF16):
        mats = [matrix(70, 90, seed=i, dtype=dtype) for i in range(3)]
        want = run(mats, dtype)
        B.ss_orthogonalise(mats, mats)
        for a, b in zip(mats, want):
            assert torch.equal(a, b)


@pytest.mark.parametrize("shape", [(48, 80), (80, 48), (100, 700), (200, 160)])
def test_zeros_and_values_that_are_not_finite(shape):
    zero, nan, inf, fine = (matrix(*shape, seed=i) for i in range(4))
    zero.zero_()
    nan[3, 5], inf[0, 0] = float("nan"), float("inf")
    out = run([zero, nan, inf, fine])
    assert not bool(out[0].any()) and bool(out[1].isnan().all()) and bool(out[2].isnan().all())
    near("the one between", out[3], fine)


@pytest.mark.parametrize("size", [1e-38, 1e-25, 1e30, 3e37])
@pytest.mark.parametrize("shape", [(60, 70), (150, 170)])
def test_the_whole_range_of_fp32(shape, size):
    u = matrix(*shape, seed=2, kind="noise", size=1.0) * size
    near("size %g" % size, run([u])[0], u)


def update(g, v, p, beta=0.95, nesterov=True, lr=0.02, scale=0.7, decay=0.1, in_place=False):
    vo, po = (v, p) if in_place else ([torch.full_like(m, float("nan")) for m in v], [torch.full_like(m, float("nan")) for m in p])
    B.ss_orthogonal_update(g, v, vo, p, po, beta, nesterov, ref.COEFFICIENTS, lr, scale, decay)
    return vo, po


@pytest.mark.parametrize("dtype", [F32, BF16], ids=["f32", "bf16"])
@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("shape", [(1, 1), (130, 70), (65, 259), (900, 33), (512, 512), (140, 1111)])
def test_update(shape, nesterov, dtype):
    g, v, p = ([matrix(*shape, seed=10 * k + i, size=s).to(dt) for i in range(2)] for k, s, dt in ((1, 1e-3, dtype), (2, 1e-3, F32), (3, 1e-2, F32)))
    vo, po = update(g, v, p, nesterov=nesterov)
    for i in range(2):
        want_v, want_p = ref.updated(g[i], v[i], p[i], 0.95, nesterov, 0.02, 0.7, 0.1)
        model = ref.updated(g[i], v[i], p[i], 0.95, nesterov, 0.02, 0.7, 0.1, rounded=True)[1]
        # two products and a sum: three roundings of at most half a unit of the larger term (five allowed). And 0.95 reaches the
        # kernel in fp32, off by up to half its unit there, 2^-25, and 1 - beta, formed exactly from it, by the same
        gv = g[i].double().abs() + v[i].double().abs()
        bound = 5 * 2.0 ** -24 * (0.95 * v[i].double().abs() + 0.05 * g[i].double().abs()) + 2.0 ** -25 * gv
        assert bool(((vo[i].double() - want_v).abs() <= bound).all())
        allowed = 2 * float((model - want_p).norm()) + 0.02 * 0.7 * 2e-5 * float(ref.orthogonalised(want_v).norm()) + 4 * 2.0 ** -24 * float(want_p.norm())
        assert float((po[i].double() - want_p).norm()) <= allowed
    again_v, again_p = update(g, [m.clone() for m in v], [m.clone() for m in p], nesterov=nesterov, in_place=True)
    for a, b in zip(vo + po, again_v + again_p):
        assert torch.equal(a, b)


def test_update_of_slices():
    """Parameters and momenta as columns of wider ones, gradients of another stride, at odd places."""
    g = [matrix(50, 90, seed=i)[:, 3:73] for i in range(2)]
    v, p = ([matrix(50, 80, seed=10 * k + i)[:, 1:71] for i in range(2)] for k in (1, 2))
    want = update([m.contiguous() for m in g], [m.contiguous() for m in v], [m.contiguous() for m in p])
    got = update(g, v, p, in_place=True)
    for a, b in zip(want[0] + want[1], got[0] + got[1]):
        assert torch.equal(a, b)


def test_nothing_to_do():
    B.ss_orthogonalise([], [])
    empty = [torch.empty(0, 5, device=DEV)]
    B.ss_orthogonalise(empty, [torch.empty(0, 5, device=DEV)])
    B.ss_orthogonal_update(empty, empty, empty, empty, empty, 0.9)


def test_the_same_call_gives_the_same_bits():
    mats = [matrix(600, 900, seed=i) for i in range(3)]
    for a, b in zip(run(mats), run(mats)):
        assert torch.equal(a, b)
