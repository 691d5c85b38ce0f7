"""Entries of the head's gradient that are small beside the largest of their row, one by one.

Row t of x is twice the t-th unit vector, so dw[v, t] = 2 P_t[v], a sum of one term, and the logits are exact. What is left
are the roundings of P's way, each at most half a step. With t = log2 of an entry's ratio to the row's largest: the exponent (z - m) log2(e)
is formed in two roundings, with a constant that has one, and once more between a part's maximum and the row's: 4 |t| 2^-24 in all; the hardware's exponentials and the sum
of the row: 16 times 2^-24. For bf16 inputs the exponential that is kept has 11 bits (2^-11) and P 8 (2^-8). An fp32 P is carried exactly."""
import pytest
import torch

from paper_1810_05291_b200 import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
F32, BF16 = torch.float32, torch.bfloat16


@pytest.mark.parametrize("above", [2.0, 12.0, 18.0, 27.0, 36.0])
@pytest.mark.parametrize("rows", [40, 1100])  # with statistics formed with the gradient, and by a launch of their own
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_small_entries_beside_a_certain_one(dtype, rows, above):
    vocab, g = 333, torch.Generator(device=DEV).manual_seed(rows + int(above))
    y = torch.randint(0, vocab, (rows,), generator=g, device=DEV)
    z = torch.randn(vocab, rows, generator=g, device=DEV).clamp(-3, 3)
    at = torch.arange(rows, device=DEV)
    z[y, at] = above
    w, x = (z / 2).to(dtype), (2 * torch.eye(rows, device=DEV)).to(dtype)
    k = torch.rand(rows, generator=g, device=DEV) + 0.5
    dw = torch.full((vocab, rows), float("nan"), device=DEV)
    B.ss_linear_cross_entropy(x, w, y, k, torch.empty(2, device=DEV), torch.empty(rows, device=DEV), None, dw)
    z = 2 * w.double()
    want = 2 * k.double() * torch.softmax(z, 0)
    bits = (z.amax(0) - z) * 1.4426950408889634
    bound = (4 * bits + 16) * 2.0 ** -24 + (2.0 ** -11 + 2.0 ** -8 if dtype == BF16 else 0.0)
    off = (dw.double() - want).abs() / want
    off[y, at] = 0                                           # the target's, a difference, has a bound of its own elsewhere
    assert bool((off <= bound).all()), "worst %.3g of its bound" % float((off / bound).nan_to_num(1e9).max())
