"""The bounded waits of the output layer's products, made to run out on purpose without faulting or
hanging the GPU: one CTA of each tile leaves out a load (agn_debug_linear_ce_waits) under a 2 ms limit.
What could not be computed is NaN, *err is 1, and calls after it give what they gave before, bit for bit."""

import time

import pytest
import torch

from test_gpu_linear_ce import make

pytestmark = pytest.mark.gpu
LIMIT = 2_000_000


@pytest.fixture(scope="module")
def agn():
    import paper_1710_02368_gb300 as agn
    return agn


@pytest.fixture
def waits(agn):
    yield agn.agn_debug_linear_ce_waits
    agn.agn_debug_linear_ce_waits(0, -1)


# one CTA a tile: K of one stage and of more than the ring has; pairs: the same, several tiles for each,
# ranges along K, rows gathered
SHAPES = [(60, 64, 600, 0.0, [0]), (100, 3000, 130, 0.2, [0]), (200, 64, 700, 0.0, [0, 1]), (300, 3000, 400, 0.3, [0, 1]),
          (1500, 520, 9000, 0.0, [0, 1]), (9000, 64, 140, 0.1, [0, 1]),
          (4096, 640, 5000, 0.1, [0, 1])]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,inner,classes,ignored,ranks", SHAPES, ids=str)
def test_withheld_load(agn, waits, dtype, rows, inner, classes, ignored, ranks):
    x, w, b, labels = make(rows, inner, classes, dtype, ignored=ignored)
    known = labels >= 0
    known &= labels < classes
    n = max(agn.agn_linear_ce_bytes(rows, inner, classes, dtype, k) for k in (0, 1))
    work = torch.zeros(n, dtype=torch.uint8, device="cuda")
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    sizes = (dtype, rows, inner, classes)

    def forward():
        loss, lse = (torch.full((rows,), 7.0, device="cuda") for _ in range(2))
        agn.agn_linear_ce(x, w, labels, *sizes, loss, lse, work, n, bias=b, err=err)
        return [loss, lse]

    def backward(lse):
        out = [torch.full_like(x, 7.0), torch.full_like(w, 7.0), torch.full_like(b, 7.0)]
        agn.agn_linear_ce_backward(x, w, labels, lse, *sizes, work, n, dx=out[0], dw=out[1], dbias=out[2], bias=b,
                                   err=err)
        return out

    good = forward()
    good += backward(good[1])
    assert int(err) == 0 and all(torch.all(torch.isfinite(t)) for t in good)
    for rank in ranks:
        for call in (forward, lambda: backward(good[1])):
            waits(LIMIT, rank)
            torch.cuda.synchronize()
            t0 = time.monotonic()
            bad = call()
            torch.cuda.synchronize()
            # far less than 2 s: every copy in flight was accounted for, none waited for to its own limit
            assert time.monotonic() - t0 < 1.0
            assert int(err) == 1
            assert any(torch.any(torch.isnan(t)) for t in bad)
            for t in bad:   # NaN, or right: nothing in between in a loss, no value left as it was
                assert not torch.any(t == 7.0)
            if len(bad) == 2:
                assert torch.all(torch.isnan(bad[0]) | (bad[0] == good[0]))
                assert torch.all(bad[0][~known] == 0)
            bad = call()   # without a host wait between: the next call does not inherit anything
            waits(0, -1)
            again = forward()
            again += backward(again[1])
            assert all(torch.equal(s, t) for s, t in zip(again, good))
            assert int(err) == 1   # never cleared by a call
            err.zero_()


def test_err_may_be_null_and_other_threads_are_not_touched(agn, waits):
    import threading
    x, w, b, labels = make(300, 64, 700, 1)
    n = agn.agn_linear_ce_bytes(300, 64, 700, 1)
    outs = [torch.full((2, 300), 7.0, device="cuda") for _ in range(2)]
    work = [torch.zeros(n, dtype=torch.uint8, device="cuda") for _ in range(2)]

    def call(i):
        agn.agn_linear_ce(x, w, labels, 1, 300, 64, 700, outs[i][0], outs[i][1], work[i], n)
    waits(LIMIT, 0)
    call(0)
    t = threading.Thread(target=call, args=(1,))
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert torch.all(outs[0].isnan()) and torch.all(outs[1].isfinite())
