"""dw and dx in one launch, whose CTAs finish tiles of both products through the same staged tiles: each gradient has
the bits that it has in a launch of its own, time after time (a store that reads a tile late would show in
some of them), and is right."""

import pytest
import torch

import test_gpu_linear_ce as L

pytestmark = pytest.mark.gpu
agn = L.agn


def joint(agn, rows, inner, classes, dtype, ignored, times=25):
    x, w, b, labels = L.make(rows, inner, classes, dtype, ignored=ignored)
    _, lse, both = L.check(agn, x, w, b, labels, dtype, scale=1.0 / rows)
    for k, without in (("dx", ("dw", "dbias")), ("dw", ("dx", "dbias"))):
        alone = L.backward(agn, x, w, b, labels, lse, dtype, scale=1.0 / rows, without=without)
        assert torch.equal(alone[k], both[k])
    for _ in range(times):
        again = L.backward(agn, x, w, b, labels, lse, dtype, scale=1.0 / rows)
        for k in both:
            assert torch.equal(again[k], both[k]), k


# rows without a label (dx leaves row by row, dw by bulk stores), rows whose bytes are no multiple of 16 (dw
# leaves row by row, dx as ranges' sums); a second product of few steps
@pytest.mark.parametrize("rows,inner,classes,dtype,ignored", [
    (700, 1000, 520, 1, 0.1), (2048, 1000, 1000, 0, 0.1), (4000, 512, 300, 1, 0.3), (2048, 264, 2000, 0, 0.02),
    (300, 1001, 20000, 1, 0.0), (300, 1001, 20000, 1, 0.2), (257, 601, 9000, 0, 0.0), (1500, 333, 5000, 1, 0.0)])
def test_rows_after_bulk_stores(agn, rows, inner, classes, dtype, ignored):
    joint(agn, rows, inner, classes, dtype, ignored)


# bf16 dw by halves of a tile after dx as fp32 sums of ranges or of pieces of the classes; K of few steps, so that
# its sums are there at once; and the other way round
@pytest.mark.parametrize("rows,inner,classes,dtype,ignored", [
    (777, 1000, 10007, 1, 0.0), (256, 2048, 8000, 1, 0.0), (300, 1000, 20000, 1, 0.0), (300, 1000, 20000, 1, 0.3),
    (256, 520, 30000, 1, 0.0), (9000, 200, 20000, 1, 0.0), (2000, 2048, 300, 1, 0.0), (300, 264, 20000, 0, 0.0)])
def test_stores_of_both_kinds(agn, rows, inner, classes, dtype, ignored):
    joint(agn, rows, inner, classes, dtype, ignored)
