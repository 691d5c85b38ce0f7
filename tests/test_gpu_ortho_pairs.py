"""The step of momentum and parameter where its products go through pairs of blocks on 256 x 256 tiles; tolerances as in tests/test_gpu_ortho.py."""
import pytest
import torch

from tests import ortho_ref as ref
from tests.test_gpu_ortho import BF16, F32, matrix, update

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("nesterov", [False, True])
@pytest.mark.parametrize("count,shape,dtype", [(2, (2600, 2500), F32), (1, (5000, 1100), BF16), (8, (1300, 4100), BF16)])
def test_update(count, shape, dtype, nesterov):
    rows, cols = shape
    make = lambda k, size, dt, pad: [matrix(rows, cols + pad, seed=10 * k + i, size=size).to(dt)[:, pad // 2:pad // 2 + cols] for i in range(count)]  # noqa: E731
    g, v, p = make(1, 1e-3, dtype, 3), make(2, 1e-3, F32, 5), make(3, 1e-2, F32, 3)  # columns of wider ones, rows off 16 bytes
    own = [[m.contiguous() for m in ms] for ms in (g, v, p)]
    vo, po = update(*own, nesterov=nesterov)
    for i in {0, count - 1}:
        want_v, want_p = ref.updated(g[i], v[i], p[i], 0.95, nesterov, 0.02, 0.7, 0.1)
        model = ref.updated(g[i], v[i], p[i], 0.95, nesterov, 0.02, 0.7, 0.1, rounded=True)[1]
        gv = g[i].double().abs() + v[i].double().abs()
        bound = 5 * 2.0 ** -24 * (0.95 * v[i].double().abs() + 0.05 * g[i].double().abs()) + 2.0 ** -25 * gv
        assert bool(((vo[i].double() - want_v).abs() <= bound).all())
        allowed = 2 * float((model - want_p).norm()) + 0.02 * 0.7 * 2e-5 * float(ref.orthogonalised(want_v).norm()) + 4 * 2.0 ** -24 * float(want_p.norm())
        assert float((po[i].double() - want_p).norm()) <= allowed
    for a, b in zip(v + p, own[1] + own[2]):
        assert torch.equal(a, b)
    again_v, again_p = update(g, v, p, nesterov=nesterov, in_place=True)  # where they are
    for a, b in zip(vo + po, again_v + again_p):
        assert torch.equal(a, b)
