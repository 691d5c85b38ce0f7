"""Few rows at the head, whose scratch is for those alone: values against the formulas, and nothing written behind it."""
import pytest
import torch

from paper_1810_05291_b200 import binding as B
from tests.test_gpu_train_head import BF16, DEV, F32, case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [1, 63, 64, 65, 128, 130, 192, 257, 1025, 1100])
@pytest.mark.parametrize("dtype", [BF16, F32], ids=["bf16", "f32"])
def test_rows_that_fill_no_tile(dtype, rows):
    x, w, y, k = case(rows, 72, 1300, dtype, seed=rows, masked=0.3 if rows > 1 else 0.0)
    need = B.ss_linear_cross_entropy_workspace(w, rows, True, dtype)
    ws = torch.full((need + 8192,), 171, dtype=torch.uint8, device=DEV)
    out = [torch.full((2,), float("nan"), device=DEV), torch.full((rows,), float("nan"), device=DEV), torch.full_like(x, float("nan")), torch.full_like(w, float("nan"))]
    B.ss_linear_cross_entropy(x, w, y, k, *out, workspace=ws)
    check(x, w, y, k, out)
    assert bool((ws[need:] == 171).all())
