"""The orthogonal update on the GPU with coefficients up to the limits of what it takes, each way that it goes by size.

Tolerances: twice the 2-norm that the operands' roundings make in 64 bits, and 2e-5, as in tests/test_gpu_ortho.py; and what the model does not have. The
norm of u and the factor are fp32 (2^-22 of a singular value s), and the matrix unit truncates each of n / 16 steps of a sum, by less than 2^-23 of it: with n the
longest side t = n / 16 2^-23, twice in b s^3 (S, Q X) and four times in c s^5 (S twice, S S, Q X). A step hands an error on times |f'(s)|, with f = a s + b s^3 +
c s^5. With the set that begins with 8.29 and a matrix of one direction (s = 1) the five f' are 24, 12, 11, 8 and 2.5: 7e4 in all, so that 2^-22 becomes a
percent, and t of the first step, times 40 for its terms and 2800 for the steps behind it, as much again."""
import math

import pytest
import torch

from paper_1810_05291_b200 import binding as B
from tests import ortho_ref as ref
from tests.test_gpu_ortho import DEV, gen, run
from tests.test_ortho_coefficients import REFUSED, TAKEN

pytestmark = pytest.mark.gpu


def drift(u, sets):
    s = torch.linalg.svdvals(u.double())
    s = s / s.square().sum().sqrt()
    t = math.ceil(max(u.shape) / 16) * 2.0 ** -23
    e = 2.0 ** -22 * s
    for a, b, c in sets:
        e = (a + 3 * b * s ** 2 + 5 * c * s ** 4).abs() * e + t * (2 * abs(b) * s.abs() ** 3 + 4 * abs(c) * s.abs() ** 5)
        s = a * s + b * s ** 3 + c * s ** 5
    return float(e.norm())


@pytest.mark.parametrize("shape", [(60, 70), (100, 700), (150, 170), (700, 300)])
@pytest.mark.parametrize("co", [s for s in TAKEN if len(s) < 30 and sum(s[-1]) != 0], ids=lambda s: "%dx%g,%g,%g" % (len(s), *s[0]))
def test_taken(co, shape):
    g = gen(sum(shape))
    noise = torch.randn(shape, generator=g, device=DEV)
    one = torch.randn(shape[0], 1, generator=g, device=DEV) @ torch.randn(1, shape[1], generator=g, device=DEV)
    for u in (noise, one):
        out = run([u], coefficients=co)[0].double()
        want, model = ref.orthogonalised(u, co), ref.orthogonalised(u, co, rounded=True)
        assert bool(out.isfinite().all())
        assert float((out - want).norm()) <= 2 * float((model - want).norm()) + 2e-5 * float(want.norm()) + drift(u, co)


@pytest.mark.parametrize("co", REFUSED)
def test_a_refused_call_writes_nothing(co):
    u, out = torch.ones(6, 7, device=DEV), torch.full((6, 7), 5.0, device=DEV)
    with pytest.raises(B.SignSGDError):
        B.ss_orthogonalise([u], [out], coefficients=co)
    with pytest.raises(B.SignSGDError):
        B.ss_orthogonal_update([u], [out], [out], [u.clone()], [u.clone()], 0.9, coefficients=co)
    assert bool((out == 5).all())
