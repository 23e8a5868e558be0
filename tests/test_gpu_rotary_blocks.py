"""Rotary positions of large prompts: a block takes one, two or four of 2048 rows and more, by the
items of a row (heads times pieces of a head): below 256 four, to 511 two, else one.  An odd number of rows
leaves the last block of two half full.  Tolerances: test_gpu_rotary.py's."""
import numpy as np
import pytest
import torch

from paper_2608_13524_amd import dartree as D
from tests.test_gpu_rotary import BF, FP, HALF, INTER, Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("b,rows,hq,hkv,rot,layout,dtype,items", [
    (3, 683, 32, 8, 128, HALF, BF, 320), (3, 683, 16, 4, 128, INTER, BF, 320), (3, 683, 12, 4, 128, HALF, FP, 256),
    (3, 683, 7, 2, 128, INTER, FP, 288), (3, 683, 2, 1, 36, HALF, BF, 330), (3, 683, 31, 0, 128, INTER, BF, 496),
    (3, 683, 32, 8, 128, INTER, BF, 640), (2, 1024, 60, 4, 128, HALF, BF, 512), (3, 683, 20, 12, 96, HALF, FP, 640)])
def test_rows_of_a_block(b, rows, hq, hkv, rot, layout, dtype, items):
    vector = (8 if dtype is BF else 4) * (2 if layout == HALF else 1)
    each = vector // 2 if layout == HALF else vector
    assert items == (hq + hkv) * (rot // vector + (128 - rot) // each if rot % vector == 0 else 128 - rot // 2)
    counts = [rows - 1, 0, rows // 2 + 1][:b]
    case = lambda **kw: Case(b, rows, hq, hkv, 128, rot, layout, dtype, start=[5, 100000, 77][:b], seed=rows + items, **kw)
    case().check()
    case(fused=True).check("in")
    case(fused=True, counts=counts).check("in")
    case(counts=counts, inverse=1, amplitude=1.25).check("wide")
