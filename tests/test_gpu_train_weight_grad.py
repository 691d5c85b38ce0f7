"""The weight gradient beyond one tile to a pair of blocks and one chunk of rows to a tile.

Sizes are chosen for 148 SMs, 74 pairs of blocks, 256 x 256 tiles, stages of 64 rows and chunks of 32 stages: the comments
say how a case is cut. Tolerances, from the arithmetic:
* An element. A chunk is 128 steps of 16 rows in the matrix unit. A step truncates the sum, at most 2^-23 of it, and what it adds is
  aligned with truncation, at most 2^-23 of the largest term: 256 * 2^-23 of the chunk's sum |dy x^|. A chunk, and a part, is
  then added with rounding to nearest: 2^-24 of the whole sum |dy x^| each.
* All of them, for inputs of mean 0. The sum after i steps is about sqrt(i / 128) of the chunk's; a truncation takes 2^-24 of it on average,
  always towards zero: 2^-24 * 128 * 2/3 = 5.1e-6 of the chunk's sum, and as much of the total. (Not promoted, 16384 rows would lose eight
  times that; a chunk that is lost or added twice shows in the first digit.)
"""
import pytest
import torch

from paper_1810_05291_b200 import binding as B
from tests import train_ref as ref
from tests.test_gpu_train_ops import Guarded, close

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
CHUNK_ROWS = 2048


def check(rows, n_out, n_in, dtype, accumulate=False, dy_pad=0, dy_off=0, dw_pad=0, dw_off=0):
    g = torch.Generator(device=DEV).manual_seed(rows + n_out + n_in)
    x = torch.randn(rows, n_in, generator=g, device=DEV)
    src = Guarded(rows, n_out, dtype, n_out + dy_pad, dy_off, fill=float("nan"))
    src.view.copy_(torch.randn(rows, n_out, generator=g, device=DEV))
    out = Guarded(n_out, n_in, torch.float32, n_in + dw_pad, dw_off)
    start = torch.randn(n_out, n_in, generator=g, device=DEV)
    out.view.copy_(start)
    ck = B.act8_checkpoint(rows, n_in, DEV)
    B.ss_act8_pack(x, ck)
    xk, dy = ref.act8(x)[2], src.view.double()
    B.ss_weight_grad8(src.view, ck, out.view, accumulate=accumulate)
    want, size = dy.t() @ xk, dy.abs().t() @ xk.abs()
    error = out.view.double() - want - (start.double() if accumulate else 0)
    if not accumulate:
        assert float(error.norm() / want.norm()) < 5.2e-6
    planes = 3 if dtype == torch.float32 else 1
    adds = planes * -(-rows // CHUNK_ROWS) + 74  # chunks, and parts at most
    if accumulate:
        want, size = want + start.double(), size + start.double().abs()
    close(out.view, want, (256 + adds / 2) * 2.0 ** -23 * size + 1e-38, "dw")
    out.check()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("accumulate", [False, True], ids=["written", "added"])
@pytest.mark.parametrize("rows,n_out,n_in", [
    (4500, 2560, 2304),   # 90 tiles of 71 stages (213 fp32): 74 whole in 3 chunks (7), 16 in four parts; two units to a pair
    (6500, 1537, 1793),   # 56 tiles, not cut, 4 chunks, ragged on both sides
    (2100, 4999, 1001),   # 80 tiles of 33 stages: a second chunk of one stage
    (9000, 2560, 2048),   # 80 tiles, 6 of them in twelve parts
])
def test_tiles_of_several_chunks(rows, n_out, n_in, accumulate, dtype):
    check(rows, n_out, n_in, dtype, accumulate)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("rows,n_out,n_in", [
    (700, 4300, 6000),    # 408 tiles of 11 stages: six units to a pair, 38 tiles left over and not cut
    (130, 5000, 5000),    # 400 of 3: a unit is shorter than the round of the decoding groups
    (64, 4999, 5003),     # 400 of one
    (1, 5121, 3841),
])
def test_several_short_units_to_a_pair(rows, n_out, n_in, dtype):
    check(rows, n_out, n_in, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["f32", "bf16"])
@pytest.mark.parametrize("accumulate", [False, True], ids=["written", "added"])
@pytest.mark.parametrize("dy_pad,dy_off,dw_pad,dw_off", [(1, 1, 0, 0), (8, 0, 3, 1), (3, 2, 4, 0)])
def test_several_chunks_with_strides(dy_pad, dy_off, dw_pad, dw_off, accumulate, dtype):
    check(4500, 2560, 2300, dtype, accumulate, dy_pad, dy_off, dw_pad, dw_off)


def test_a_long_batch_summed_whole():
    """16384 rows: 90 tiles, 74 of them in 8 chunks of their own, 16 in four parts of two chunks."""
    check(16384, 2560, 2304, torch.bfloat16)


def test_several_chunks_twice_are_the_same():
    rows, n_out, n_in = 5000, 2600, 1900
    g = torch.Generator(device=DEV).manual_seed(1)
    dy = torch.randn(rows, n_out, generator=g, device=DEV)
    ck = B.act8_checkpoint(rows, n_in, DEV)
    B.ss_act8_pack(torch.randn(rows, n_in, generator=g, device=DEV), ck)
    outs = []
    for _ in range(3):
        dw = torch.empty(n_out, n_in, device=DEV)
        B.ss_weight_grad8(dy, ck, dw)
        outs.append(dw)
    assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
