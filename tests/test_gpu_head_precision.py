"""The cross entropy at the head on the GPU: how far it is off in the 2-norm (head_precision has the bounds' derivation), and its values
where other tests have none: fp32 with more than 1024 rows, with rows in several pieces, with at most 1024 rows in several pieces. Element by element the
bounds of head_ref hold there too."""
import pytest
import torch

from tests import head_precision as hp
from tests import head_ref as ref
from tests.test_gpu_train_head import BF16, DEV, F32, case, check, gen, run

pytestmark = pytest.mark.gpu


def precise(c, got, base=None):
    x, w, y, k = c
    want = ref.head(x, w, y, k)
    low = x.dtype == BF16
    size = hp.logp_size(x, w, y, want)
    assert float((got[1].double() - want["logp"]).norm()) <= hp.logp_bound(x.shape[1], low, x.shape[0]) * float(size.norm())
    if not low:
        assert hp.off(got[2], want["dx"]) <= hp.gradient_bound(w.shape[0])
        dw = got[3].double() if base is None else got[3].double() - base.double()
        more = 0 if base is None else 2.0 ** -23 * float(base.double().norm())  # it is added to in fp32, a few times
        assert float((dw - want["dw"]).norm()) <= hp.gradient_bound(x.shape[0]) * float(want["dw"].norm()) + more


SHAPES = [(64, 256, 257), (127, 96, 1000), (129, 72, 2049), (256, 512, 256), (300, 130, 5003), (515, 1000, 4099), (700, 1600, 2000)]


@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("shape", SHAPES, ids=["%dx%dx%d" % s for s in SHAPES])
def test_error_in_the_2_norm(shape, dtype):
    c = case(*shape, dtype, seed=sum(shape))
    precise(c, run(*c))


@pytest.mark.parametrize("shape", [(2500, 200, 1300), (3333, 130, 777), (1100, 1025, 2049)], ids=lambda s: "%dx%dx%d" % s)
def test_fp32_with_more_rows(shape):
    """Rows found by a kernel of their own, a weight gradient summed over several blocks of 1024 rows, written and added to."""
    c = case(*shape, F32, seed=sum(shape))
    got = run(*c)
    check(*c, got)
    precise(c, got)
    base = torch.randn(c[1].shape, generator=gen(1), device=DEV)
    got = run(*c, accumulate=base)
    check(*c, got, base=base)
    precise(c, got, base)


@pytest.mark.parametrize("dtype,rows,vocab", [(F32, 2500, 70000), (F32, 1000, 131072), (BF16, 900, 700000)], ids=["f32", "f32-few", "bf16-few"])
def test_in_several_pieces(dtype, rows, vocab):
    c = case(rows, 72, vocab, dtype, seed=rows)
    c[3][rows // 2:rows // 2 + 100] = 0
    got = run(*c)
    check(*c, got)
    precise(c, got)
    if dtype == F32:
        base = torch.randn(c[1].shape, generator=gen(1), device=DEV)
        got = run(*c, accumulate=base)
        check(*c, got, base=base)
        precise(c, got, base)
    only_loss = run(*c, want=(False, False))                 # the statistics by another kernel, of as many pieces
    check(*c, only_loss)
    c[3][rows // 3:] = 0                                     # a last piece of which no row counts
    check(*c, run(*c))
