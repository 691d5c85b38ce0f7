"""Scratch of the cross entropy at the head: what of it grows with the vocabulary is for the rows that there are, not for 256."""
import ctypes

import pytest

from paper_1810_05291_b200 import binding as B
from paper_1810_05291_b200 import build as libbuild

vp = ctypes.c_void_p


@pytest.fixture(scope="module")
def L():
    libbuild.build()
    return B.lib()


def up(n, m):
    return (n + m - 1) // m * m


@pytest.mark.parametrize("rows,width,vocab", [(1, 64, 131072), (64, 64, 1 << 20), (64, 64, 1 << 22), (65, 100, 50257), (200, 64, 32000), (1000, 64, 131072), (5000, 64, 70000)])
@pytest.mark.parametrize("dt", [B.SS_F32, B.SS_BF16])
def test_what_grows_with_the_vocabulary(L, dt, rows, width, vocab):
    need = L.ss_linear_cross_entropy_workspace(vp(1 << 24), up(width, 8), dt, rows, width, vocab, 1, 1, dt)
    a_logit = 10 if dt == B.SS_F32 else 2                    # e and P: fp32 and three bf16, or 16 bits in one place
    cols, here = up(vocab, 64), up(rows, 64)
    piece = max(256, (1 << 30) // (a_logit * cols) // 256 * 256)
    here = min(here, piece)
    pieces = -(-rows // here)
    e_and_p = here * cols * a_logit
    statistics = here * up(vocab, 256) // 128 * 8
    copy = 3 * vocab * up(width, 64) * 2 if dt == B.SS_F32 else 0
    sums = vocab * up(width, 64) * 4 if dt == B.SS_BF16 and pieces > 1 else 0
    gathered = pieces * here * (up(width, 64) * (6 if dt == B.SS_F32 else 2) + 64) + here * up(width, 64) * 4
    parts = 2 * 74 * 256 * 256 * 4                           # of tiles that come in parts: 74 pairs of blocks, for dx and for dw
    assert need <= e_and_p + statistics + copy + sums + gathered + parts + 65536
