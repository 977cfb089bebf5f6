"""The sum of squares and clipping of lists whose tensors lie in other ways than one buffer each.

Bounds as in test_gpu_list.py: 2^-24 of a device's sum, and of a clipped element half the k roundings of the norm's parts, three of the root, the division and the product, and
its own rounding U, all relative."""
import math

import pytest
import torch

import paper_2110_15032_amd as sbp
from train_harness import CODE, TYPE, column, room

pytestmark = pytest.mark.gpu
E = 2.0 ** -24


@pytest.mark.parametrize("kind", ["bf16", "f32"])
@pytest.mark.parametrize("short", [2, 4, 7])
def test_rows_that_end_just_below_two_to_the_31(kind, short):
    """the last columns of rows at a pitch, whose place plus eight is past 2^31"""
    rows, pitch = 2, 2 ** 31 - 1
    cols = 2 ** 31 - short
    raw = torch.zeros((rows - 1) * pitch + cols, dtype=TYPE[kind], device="cuda")
    x = raw.as_strided((rows, cols), (pitch, 1))
    tail = torch.tensor([[3.0, 8, 1, 12, 5, 2, 7, 4, 9, 6, 11, 10], [2.0, 5, 9, 1, 7, 12, 3, 8, 10, 4, 6, 11]], device="cuda")
    x[:, -12:] = tail
    lst = sbp.SbpList([sbp.SbpTensor([raw], rows, cols, CODE[kind], 0, pitch)], [sbp.B])
    out, norm = column(1, "f32", "B", 1), column(1, "f32", "B", 1)
    sbp.sbp_square_sum(lst, out.desc, room(sbp.sbp_square_sum_workspace(lst, 1)), 1)
    total = float((tail ** 2).sum())
    assert float(out.host()[0][0, 0]) == total                                             # whole numbers
    sbp.sbp_clip(lst, out.desc, sbp.B, 0.5 * math.sqrt(total), lst, norm.desc, 1)
    got = x[:, -12:].float()
    assert bool(((got - 0.5 * tail).abs() <= 4 * E * tail).all()), got
    assert int(raw.count_nonzero()) == 24
