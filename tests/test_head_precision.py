"""The bounds of the head's fp32 gradients are narrow enough to tell three terms of an operand from two: operands cut to two bf16 terms
(16 significant bits), in the oracle, are outside them."""
import pytest
import torch

from tests import head_precision, head_ref


def cut(t, terms):
    """The first `terms` bf16 terms of fp32 values, each cut off."""
    rest, out = t.float(), torch.zeros_like(t, dtype=torch.float32)
    for _ in range(terms):
        part = (rest.view(torch.int32) & -65536).view(torch.float32)
        out, rest = out + part, rest - part
    return out


@pytest.mark.parametrize("shape", [(64, 256, 257), (129, 72, 2049), (300, 130, 5003), (515, 1000, 4099)])
def test_two_terms_are_outside(shape):
    rows, width, vocab = shape
    g = torch.Generator().manual_seed(sum(shape))
    x, w = torch.randn(rows, width, generator=g), 2 * width ** -0.5 * torch.randn(vocab, width, generator=g)
    y, k = torch.randint(0, vocab, (rows,), generator=g), torch.rand(rows, generator=g) + 0.5
    want = head_ref.head(x, w, y, k)
    for terms in (2, 3):
        cx, cw = cut(x, terms), cut(w, terms)
        p = cut(head_ref.head(cx, cw, y, k)["grad"], terms).double()
        dx, dw = p @ cw.double(), p.t() @ cx.double()
        for got, name, n in ((dx, "dx", vocab), (dw, "dw", rows)):
            assert (head_precision.off(got, want[name]) > head_precision.gradient_bound(n)) == (terms == 2)
