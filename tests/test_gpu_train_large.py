"""The training operators on tensors of more than 2^31 elements (more than 2^32 bytes): the rows on either side of an offset that
no longer fits 32 bits. Up to 18 GB on the device."""
import pytest
import torch

from paper_1810_05291_b200 import binding as B
from tests import train_ref as ref
from tests.test_gpu_train_ops import check_preference, close, half_unit, logp_tol

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
ROWS, COLS = 40000, 65543                                # 2^31 elements end in row 32764, 2^32 bytes too
SAMPLE = [0, 1, 16382, 16383, 32763, 32764, 32765, 32766, 39998, 39999]


def normal(rows, cols, seed):
    return torch.randn(rows, cols, generator=torch.Generator(device=DEV).manual_seed(seed), device=DEV, dtype=torch.bfloat16)


def test_losses():
    z, y = normal(ROWS, COLS, 1), torch.arange(ROWS, device=DEV)
    one, adv = torch.ones(ROWS, device=DEV), torch.linspace(-1, 1, ROWS, device=DEV)
    old, w = -11 * one, one / 64
    sample = torch.tensor(SAMPLE, device=DEV)
    zs, few = z[sample], [t[sample] for t in (y, old, adv, w)]
    totals, logp, dz = torch.empty(3, device=DEV), torch.empty(ROWS, device=DEV), torch.empty_like(z)
    B.ss_policy_loss(z, y, old, None, adv, w, totals, logp, dz)
    _, want_l, want_d = ref.policy(zs, few[0], few[1], None, few[2], few[3], 1.0, 0.2, 0.2, 0.0)
    tol = logp_tol(zs, COLS, 1.0)
    close(logp[sample], want_l, tol, "logp")
    # an r off by tol, the softmax by 1e-6 of itself (as in the other tests of this loss)
    r = torch.exp(want_l - few[1].double())
    err = (2 * few[3].double() * r * few[2].double().abs() * (tol + 1e-6))[:, None] + want_d.abs() * (2 * tol[:, None] + 2e-6)
    close(dz[sample], want_d, err + half_unit(z.dtype, want_d), "dlogits")

    # a pair over the last rows; those before it are in no sequence
    begin, zero = torch.tensor([ROWS - 8, ROWS - 5, ROWS], device=DEV), torch.zeros(2, device=DEV)
    loss, margins, seq = torch.empty(1, device=DEV), torch.empty(1, device=DEV), torch.empty(2, device=DEV)
    B.ss_preference_loss(z, y, one, begin, zero, loss, margins, seq, logp, dz)
    assert not bool(dz[:ROWS - 8].any())
    last = z[ROWS - 8:].clone()
    got = check_preference(last, y[ROWS - 8:], one[:8], begin - (ROWS - 8), zero, scale=1.0)
    alone = torch.empty_like(last)
    B.ss_preference_loss(last, y[ROWS - 8:], one[:8], begin - (ROWS - 8), zero, *[torch.empty_like(t) for t in got], alone)
    # the same rows in a smaller call: sums in another order (8 rows have more threads each)
    assert abs(float(margins) - float(got[1])) < 1e-4
    scale = float(alone.float().abs().max())
    assert float((dz[ROWS - 8:].float() - alone.float()).abs().max()) <= 2.0 ** -7 * scale


def test_activations():
    x = normal(ROWS, COLS, 2)
    y, back = torch.empty_like(x), torch.empty_like(x)
    ck, ck_y = B.act8_checkpoint(ROWS, COLS, DEV), B.act8_checkpoint(ROWS, COLS, DEV)
    B.ss_act8_forward(x, None, B.SS_ACT_SILU, y, ck, None, ck_y)
    B.ss_act8_unpack(ck, back)
    dx = torch.empty_like(x)
    B.ss_act8_backward(y, ck, None, B.SS_ACT_SILU, dx)
    other = torch.empty_like(ck)
    B.ss_act8_pack(x, other)
    assert torch.equal(ck, other)
    for k in SAMPLE:
        xd, yd = x[k:k + 1].double(), y[k:k + 1].double()
        kept = ref.act8(x[k:k + 1])[2]
        assert torch.equal(back[k:k + 1].double(), kept)
        want = ref.act("silu", xd)[0]
        close(y[k:k + 1], want, half_unit(x.dtype, want) + 1e-6 * (want.abs() + xd.abs()), "y")
        want = yd * ref.act("silu", kept)[1]
        close(dx[k:k + 1], want, half_unit(x.dtype, want) + 1e-6 * yd.abs() * (1 + kept.abs()), "dx")


@pytest.mark.parametrize("n_out,n_in", [(24, 1029), (1029, 24)], ids=["wide x", "wide dy"])
def test_weight_gradient(n_out, n_in):
    """2.2 million rows: codes, or dy, beyond 2^31 elements. Tolerance as in the other tests of it, with a chunk for every 2048 rows."""
    rows = 2_200_003
    x, dy = normal(rows, n_in, 3), normal(rows, n_out, 4)
    ck, dw = B.act8_checkpoint(rows, n_in, DEV), torch.empty(n_out, n_in, device=DEV)
    B.ss_act8_pack(x, ck)
    B.ss_weight_grad8(dy, ck, dw)
    want, size = (torch.zeros(n_out, n_in, dtype=torch.float64, device=DEV) for _ in range(2))
    for a, b in zip(x.split(100_000), dy.split(100_000)):
        kept, d = ref.act8(a)[2], b.double()
        want += d.t() @ kept
        size += d.abs().t() @ kept.abs()
    close(dw, want, (256 + (rows / 2048 + 74) / 2) * 2.0 ** -23 * size, "dw")
    assert float((dw.double() - want).norm() / want.norm()) < 5.2e-6
