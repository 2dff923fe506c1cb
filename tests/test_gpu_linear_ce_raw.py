"""The output layer's loss for fp32 and up to 128 rows of a large w, whose products read w as it is: the
checks of test_gpu_linear_ce and of test_gpu_linear_ce_waits at such sizes (3 M elements of w and more)."""

import math

import pytest
import torch

import test_gpu_linear_ce as C
import test_gpu_linear_ce_waits as W
from test_gpu_linear_ce import agn            # noqa: F401 (fixtures)
from test_gpu_linear_ce_waits import waits    # noqa: F401

pytestmark = pytest.mark.gpu

# rows about 8, 64 and 128; w's rows aligned or not; tiles and steps of 64 whole or not; few tiles with many ranges
SIZES = [(9, 1000, 4001), (16, 520, 6100), (17, 4097, 800), (33, 64, 50001), (63, 777, 4200), (64, 48, 70000),
         (64, 4096, 1024), (65, 778, 4199), (100, 8192, 400), (128, 30000, 130), (127, 2049, 1601), (128, 2048, 1664),
         (90, 13, 260000), (40, 100000, 33), (128, 128, 25000), (12, 1000003, 4)]


@pytest.mark.parametrize("rows,inner,classes", SIZES)
def test_sizes(agn, rows, inner, classes):
    x, w, b, labels = C.make(rows, inner, classes, 0, bias=(rows + inner) % 2 == 0)
    C.check(agn, x, w, b, labels, 0, scale=1.0 / rows)


@pytest.mark.parametrize("ignored", [0.3, 0.97, 1.0])
@pytest.mark.parametrize("rows,inner,classes", [(30, 1000, 3300), (120, 601, 5301)])
def test_rows_left_out(agn, rows, inner, classes, ignored):
    C.test_rows_left_out(agn, rows, inner, classes, ignored, 0)


@pytest.mark.parametrize("rows,inner,classes", [(40, 1024, 3200), (100, 129, 25000)])
def test_masked_classes_and_rows_that_are_not_finite(agn, rows, inner, classes):
    C.test_masked_classes(agn, rows, inner, classes, 0)
    C.test_rows_that_are_not_finite(agn, rows, inner, classes, 0)


@pytest.mark.parametrize("size", [(20, 1001, 3300), (128, 1024, 3201)])
def test_calls_repeat_stay_inside_and_may_be_captured(agn, size):
    C.test_equal_calls_give_equal_bits_and_stay_inside(agn, size, 0)
    C.test_in_a_graph_and_on_another_stream(agn, size)


@pytest.mark.parametrize("without", [("dx",), ("dw", "dbias"), ("dw", "dx")])
def test_outputs_not_wanted(agn, without):
    x, w, b, labels = C.make(70, 600, 5300, 0, ignored=0.2)
    _, lse = C.forward(agn, x, w, b, labels, 0)
    want = C.backward(agn, x, w, b, labels, lse, 0)
    got = C.backward(agn, x, w, b, labels, lse, 0, without=without)
    for k, v in got.items():
        assert (v is None) == (k in without)
        assert v is None or torch.equal(v, want[k])


def test_values_far_apart(agn):
    """x and w whose pieces differ by many binades, columns that cancel."""
    x, w, b, labels = C.make(50, 1024, 3200, 0)
    s = torch.exp2(torch.randint(-20, 21, (1024,), device="cuda").float())
    C.check(agn, x * s, w / s, b, labels, 0, scale=math.pi)


@pytest.mark.parametrize("rows,inner,classes,ignored", [(60, 64, 50000, 0.0), (100, 3000, 1100, 0.2), (30, 20000, 160, 0.1)])
def test_withheld_load(agn, waits, rows, inner, classes, ignored):
    W.test_withheld_load(agn, waits, 0, rows, inner, classes, ignored, [0])
