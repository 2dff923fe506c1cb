"""The 4-bit product's bounded waits, made to run out on purpose without faulting or hanging the GPU:
one CTA of each cluster (or pair) leaves out a load (agn_debug_linear_waits, agn_debug_waits) under a
2 ms limit.  The values are NaN, *err is 1, agn_evaluate_mx4 returns AGN_E_TIMEOUT, and calls after
it give what they gave before, bit for bit."""

import time

import numpy as np
import pytest

import agn_inputs as I

LIMIT = 2_000_000


@pytest.fixture(scope="module")
def agn():
    import __graft_entry__ as g
    g.build()
    import paper_1710_02368_gb300 as agn
    return agn


@pytest.fixture
def waits(agn):
    yield agn.agn_debug_linear_waits
    agn.agn_debug_linear_waits(0, -1)


def test_hook_validates_its_arguments(agn):
    for bad in ((-1, 0), (2_000_000_001, 0), (0, -2), (0, 65535)):
        with pytest.raises(agn.AGNError) as e:
            agn.agn_debug_linear_waits(*bad)
        assert e.value.code == agn.AGN_E_INVALID
    agn.agn_debug_linear_waits(0, -1)


# one CTA a tile: K in one stage, in fewer stages than the ring has, over clusters, in more than the
# ring has; pairs: one stage, a few, more than the ring, half units alone, several tiles for each pair
SHAPES = [(5, 64, 130, [0]), (16, 1000, 256, [0, 3]), (30, 8192, 4500, [0]), (64, 2000, 128, [0, 7]), (100, 4096, 1000, [0, 1]), (128, 5000, 7000, [0]),
          (600, 96, 300, [0]), (900, 96, 300, [0, 1]), (700, 1000, 520, [0, 1]), (1500, 2600, 384, [0, 1]), (9800, 65, 257, [0, 1]), (2433, 1500, 2111, [0, 1])]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [0, 1, 2])
@pytest.mark.parametrize("rows,inner,out,ranks", SHAPES, ids=str)
def test_withheld_load_gives_nan_and_err(agn, waits, dtype, rows, inner, out, ranks):
    import torch
    g = torch.Generator(device="cuda").manual_seed(rows)
    m = []
    for r in (rows, out):
        c, s = (torch.empty(n, dtype=torch.uint8, device="cuda") for n in agn.agn_mx4_bytes(r, inner))
        agn.agn_mx4_quantize(torch.randn(r, inner, generator=g, device="cuda"), 0, r, inner, c, s)
        m += [c, s]
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    nc, ns = agn.agn_mx4_bytes(rows, out)

    def call():
        """The output's values as floats (and, in 4 bits, its codes)."""
        if dtype != 2:
            y = torch.full((rows, out), 7.0, device="cuda").to(torch.bfloat16 if dtype else torch.float32)
            agn.agn_mx4_linear(*m, rows, inner, out, y, dtype, err=err)
            return y.float()
        c, s = torch.zeros(nc, dtype=torch.uint8, device="cuda"), torch.zeros(ns, dtype=torch.uint8, device="cuda")
        agn.agn_mx4_linear(*m, rows, inner, out, c, dtype, y_scales=s, err=err)
        y = torch.empty(rows, out, device="cuda")
        agn.agn_mx4_dequantize(c, s, rows, out, y, 0)
        return y

    want = call()
    assert int(err) == 0 and torch.all(want.isfinite())
    for rank in ranks:
        waits(LIMIT, rank)
        torch.cuda.synchronize()
        t0 = time.monotonic()
        bad = call()
        torch.cuda.synchronize()
        # far less than 2 s: every copy in flight was accounted for, none waited for to its own limit
        assert time.monotonic() - t0 < 1.0
        assert int(err) == 1 and torch.all(bad.isnan())
        bad = call()   # without a host wait between: the next call does not inherit anything
        waits(0, -1)
        good = call()
        assert torch.all(bad.isnan()) and torch.equal(good, want)
        assert int(err) == 1   # never cleared by a call
        err.zero_()
    waits(LIMIT, 60000)   # no such rank: nothing is left out
    assert torch.equal(call(), want) and int(err) == 0


@pytest.mark.gpu
def test_err_may_be_null_and_other_threads_are_not_touched(agn, waits):
    import threading

    import torch
    c, s = (torch.zeros(n, dtype=torch.uint8, device="cuda") for n in agn.agn_mx4_bytes(64, 64))
    ys = [torch.full((64, 64), 7.0, device="cuda") for _ in range(2)]
    waits(LIMIT, 0)
    agn.agn_mx4_linear(c, s, c, s, 64, 64, 64, ys[0], 0)
    t = threading.Thread(target=lambda: agn.agn_mx4_linear(c, s, c, s, 64, 64, 64, ys[1], 0))
    t.start()
    t.join()
    torch.cuda.synchronize()
    assert torch.all(ys[0].isnan()) and torch.all(ys[1] == 0)


@pytest.mark.gpu
@pytest.mark.parametrize("n_eval", [12, 70, 900])
@pytest.mark.parametrize("rank", [0, 1])
def test_evaluation_in_4_bits_times_out_and_the_handle_goes_on(agn, n_eval, rank):
    dims, n, seed, m = (600, 520, 264, 10), 2, 31, 64
    w, tau = I.make_schedule(n, 4 + n, 0, 1, seed)

    def handle():
        return agn.AGN(dims, n, 2, 0.05, seed, batch=m, n_samples=n * 4 * m, n_eval=n_eval, eval_mx4=1)

    def use(h):
        first = h.evaluate_mx4(with_pred=True)
        h.run(4, w, tau)
        return [*first, h.central(), *h.evaluate_mx4(with_pred=True), *h.evaluate()]
    with handle() as h:
        want = use(h)
    with handle() as h:
        agn.agn_debug_waits(h.h, LIMIT, rank)
        for _ in range(2):
            with pytest.raises(agn.AGNError) as e:
                h.evaluate_mx4()
            assert e.value.code == agn.AGN_E_TIMEOUT
        agn.agn_debug_waits(h.h, 0, -1)
        for g, r in zip(use(h), want):
            assert np.array_equal(g, r)
    assert np.isfinite(want[0])
