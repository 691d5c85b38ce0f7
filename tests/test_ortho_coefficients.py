"""Which coefficients the orthogonal update takes: those whose steps stay inside the range of its operands (fp16). The check
comes before everything else, so a call of no matrices shows it without a GPU."""
import ctypes

import pytest
import torch

from paper_1810_05291_b200 import binding as B
from paper_1810_05291_b200 import build as libbuild
from tests import ortho_ref as ref

DEFAULT = ((3.4445, -4.7750, 2.0315),)
# taken: sets that people use, a sign, a shrinking one, the limits
TAKEN = [DEFAULT * 5, DEFAULT * 32, ((1.5, -0.5, 0.0),) * 32, ((15 / 8, -10 / 8, 3 / 8),) * 10, ((-3.4445, 4.7750, -2.0315),) * 5, ((0.5, 0.0, 0.0),) * 32,
         ((8.2872, -23.5959, 17.3004), (4.1071, -2.9478, 0.5448), (3.9487, -2.9089, 0.5518), (3.3184, -2.4885, 0.51), (2.3007, -1.6689, 0.4188)), ((0.0, 0.0, 0.0),) * 2,
         ((31.0, 0.0, 0.0), (1.0, 0.0, 0.0)), ((50.0, 0.0, 0.0),), ((4.0, 0.0, 0.0), (4.0, 0.0, 0.0), (1.0, 0.25, 0.0625)), ((0.02, 1.0, 0.0),) * 2, ((1.0, -32.0, 31.0),)]
# refused: values or Q beyond fp16, nothing but a power that loses small singular values, a result beyond fp32
REFUSED = [((50.0, 0.0, 0.0),) * 3, ((50.0, 0.0, 0.0),) * 2, ((2.0, 1.0, 1.0),) * 4, ((30.0, 0.0, 0.0), (900.0, 40.0, 0.0)), ((0.0, 1.0, 0.0),) * 2, ((0.0, 0.0, 1.0),),
           ((0.01, 1.0, 0.0),), ((1.0, -40.0, 41.0),), ((1.0, 40000.0, -40000.0),), ((1e35, 0.0, 0.0),), ((3e38, 3e38, 3e38),), ((-50.0, 0.0, 0.0),) * 2,
           # one that looks like a set above, but takes 1 to 2, 2.04, 2.9 and 48
           ((8.3, -23.6, 17.3), (4.1, -2.95, 0.545), (3.95, -2.91, 0.552), (3.32, -2.49, 0.51), (2.3, -1.67, 0.419))]


@pytest.fixture(scope="module")
def L():
    libbuild.build()
    return B.lib()


def status(L, sets):
    flat = [v for s in sets for v in s]
    co, none = (ctypes.c_float * len(flat))(*flat), (ctypes.c_void_p * 1)()
    alone = L.ss_orthogonalise(none, 5, 0, none, 5, 0, 0, 4, 5, co, len(sets), None, 0, None)
    step = L.ss_orthogonal_update(none, 5, 0, none, none, 5, none, none, 5, 0, 4, 5, 0.9, 1, co, len(sets), 0.1, 1.0, 0.0, None, 0, None)
    assert alone == step
    return alone


@pytest.mark.parametrize("sets", TAKEN)
def test_taken(L, sets):
    assert status(L, sets) == B.SS_OK


@pytest.mark.parametrize("sets", REFUSED)
def test_refused(L, sets):
    assert status(L, sets) == B.SS_ERR_UNSUPPORTED


@pytest.mark.parametrize("shape", [(1, 1), (64, 64), (40, 900), (200, 150)])
@pytest.mark.parametrize("sets", TAKEN)
def test_what_is_taken_stays_inside_the_operands_range(sets, shape):
    """With the kernels' roundings of the operands in 64 bits: for a matrix of one direction, whose singular value is 1 at the start,
    the largest there is, and for noise. An operand has eleven bits, off by 2^-11 at most; S, Q and X are three in a row, four such are allowed a step, of the terms
    |a| s, |b| s^3 and |c| s^5 (their sum may be 0, as that of the last set is for s = 1)."""
    g = torch.Generator().manual_seed(sum(shape))
    for u in (torch.randn(shape, generator=g), torch.randn(shape[0], 1, generator=g) @ torch.randn(1, shape[1], generator=g)):
        want, model = ref.orthogonalised(u, sets), ref.orthogonalised(u, sets, rounded=True)
        assert bool(model.isfinite().all())
        x = ref.orthogonalised(u, sets[:-1])
        a, b, c = map(abs, sets[-1])
        s = torch.linalg.svdvals(x)
        terms = float((a * s + b * s ** 3 + c * s ** 5).norm())
        # in the steps before the last none of these sets' sums is below a fifth of its terms
        assert float((model - want).norm()) <= len(sets) * 5 * 4 * 2.0 ** -11 * terms
