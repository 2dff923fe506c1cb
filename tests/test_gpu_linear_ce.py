"""The output layer's softmax cross-entropy over many classes and its gradients against 64-bit
references on the same inputs, with bounds from the arithmetic (train_ops_ref)."""

import math

import pytest
import torch

import train_ops_ref as T

pytestmark = pytest.mark.gpu
DT = {0: torch.float32, 1: torch.bfloat16}


@pytest.fixture(scope="module")
def agn():
    import paper_1710_02368_gb300 as agn
    return agn


def make(rows, inner, classes, dtype, bias=True, ignored=0.0, masked=0, seed=0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    x = torch.randn(rows, inner, generator=g, device="cuda").to(DT[dtype])
    w = (torch.randn(classes, inner, generator=g, device="cuda") * 2 / math.sqrt(inner)).to(DT[dtype])
    b = None
    if bias:
        b = 0.5 * torch.randn(classes, generator=g, device="cuda")
        if masked:
            b[classes - masked:] = -math.inf
    labels = torch.randint(0, max(1, classes - masked), (rows,), generator=g, device="cuda", dtype=torch.int32)
    drop = torch.rand(rows, generator=g, device="cuda") < ignored
    bad = torch.where(torch.rand(rows, generator=g, device="cuda") < 0.5, -100, classes).to(torch.int32)
    return x, w, b, torch.where(drop, bad, labels)


def work_of(agn, x, w, dtype, backward):
    n = agn.agn_linear_ce_bytes(x.shape[0], x.shape[1], w.shape[0], dtype, backward)
    return torch.full((n,), 255, dtype=torch.uint8, device="cuda"), n   # (NaN in any type)


def forward(agn, x, w, b, labels, dtype, **kw):
    rows = x.shape[0]
    loss, lse = (torch.full((rows,), math.nan, device="cuda") for _ in range(2))
    work, n = work_of(agn, x, w, dtype, 0)
    agn.agn_linear_ce(x, w, labels, dtype, rows, x.shape[1], w.shape[0], loss, lse, work, n, bias=b,
                      stream=torch.cuda.current_stream().cuda_stream, **kw)
    return loss, lse


def backward(agn, x, w, b, labels, lse, dtype, **kw):
    out = dict(dx=torch.full_like(x, math.nan), dw=torch.full_like(w, math.nan),
               dbias=torch.full((w.shape[0],), math.nan, device="cuda"))
    for k in kw.pop("without", ()):
        out[k] = None
    work, n = work_of(agn, x, w, dtype, 1)
    agn.agn_linear_ce_backward(x, w, labels, lse, dtype, x.shape[0], x.shape[1], w.shape[0], work, n, bias=b,
                               stream=torch.cuda.current_stream().cuda_stream, **out, **kw)
    return out


def close(got, want, bound, what):
    got, want = got.double(), want.double()
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    err = torch.where(same, 0.0, (got - want).abs())
    bad = ~(err <= bound)
    assert not bad.any(), (f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float(torch.nan_to_num(err, nan=math.inf).max()):.3g}, "
                           f"bound there {float(bound.max()):.3g}, first at {bad.nonzero()[0].tolist()}")


def check(agn, x, w, b, labels, dtype, scale=1.0, dloss=None, dlse=None):
    inner = x.shape[1]
    ref = T.linear_ce(x, w, b, labels, dloss, dlse, scale)
    loss, lse = forward(agn, x, w, b, labels, dtype)
    bl, bs = T.loss_bounds(ref, inner, dtype)
    close(lse, ref["lse"], bs, "lse")
    close(loss, ref["loss"], bl, "loss")
    out = backward(agn, x, w, b, labels, lse, dtype, scale=scale, dloss=dloss, dlse=dlse)
    for k, bound in zip(("dbias", "dx", "dw"), (lambda t: (t[2], t[0], t[1]))(T.grad_bounds(ref, inner, dtype))):
        close(out[k], ref[k], bound, k)
    return loss, lse, out


SIZES = [(1, 16, 2), (1, 1, 1), (33, 100, 10), (32, 128, 10), (512, 33, 60),        # plain kernels
         (513, 64, 100), (600, 1, 3), (257, 64, 257), (130, 72, 1000),              # pairs
         (1, 4096, 3001), (2, 100, 2000), (3, 1000, 777), (8, 520, 999), (7, 35, 4001),   # few rows
         (9, 2048, 515), (16, 1600, 301), (16, 4100, 100), (15, 33, 5000), (12, 8, 70000),
         (100, 80, 5000), (128, 1000, 999), (17, 8, 70000), (20, 4096, 640),              # a CTA a tile
         (777, 1000, 1500), (300, 130, 700), (1000, 257, 515),                      # ragged, packed rows
         (4096, 200, 10), (64, 64, 20000), (16000, 40, 5), (300, 3000, 200),        # ranges along K
         (60, 5000, 600), (63, 19, 1365), (700, 2100, 15), (2, 5000, 900),
         (4096, 600, 5000), (5000, 64, 2600), (3001, 1025, 3000)]                   # many tiles


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,inner,classes", SIZES)
def test_sizes(agn, rows, inner, classes, dtype):
    x, w, b, labels = make(rows, inner, classes, dtype, bias=(rows + inner) % 2 == 0)
    check(agn, x, w, b, labels, dtype, scale=1.0 / rows)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,inner,classes", [(70, 30, 20), (7, 80, 3000), (16, 50, 900), (700, 96, 333), (1300, 100, 130), (90, 64, 3000)])
@pytest.mark.parametrize("ignored", [0.3, 0.97, 1.0])
def test_rows_left_out(agn, rows, inner, classes, ignored, dtype):
    """They hold NaN and infinities and touch nothing; their dx is zero."""
    x, w, b, labels = make(rows, inner, classes, dtype, ignored=ignored, seed=3)
    out = (labels < 0) | (labels >= classes)
    x[out] = torch.where(torch.rand(int(out.sum()), inner, device="cuda") < 0.5, math.nan, math.inf).to(x.dtype)
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    dloss = torch.where(out, math.nan, torch.randn(rows, generator=g, device="cuda"))
    dlse = torch.where(out, math.inf, 0.1 * torch.randn(rows, generator=g, device="cuda"))
    _, _, got = check_masked(agn, x, w, b, labels, dtype, out, dloss, dlse)
    assert torch.all(got["dx"][out] == 0)
    if ignored == 1.0:
        assert torch.all(got["dw"] == 0) and torch.all(got["dbias"] == 0)


def check_masked(agn, x, w, b, labels, dtype, out, dloss, dlse):
    ref = T.linear_ce(x, w, b, labels, torch.where(out, 0.0, dloss), torch.where(out, 0.0, dlse), 0.01)
    inner = x.shape[1]
    loss, lse = forward(agn, x, w, b, labels, dtype)
    bl, bs = T.loss_bounds(ref, inner, dtype)
    close(lse, ref["lse"], bs, "lse")
    close(loss, ref["loss"], bl, "loss")
    got = backward(agn, x, w, b, labels, lse, dtype, scale=0.01, dloss=dloss, dlse=dlse)
    bx, bw, bb = T.grad_bounds(ref, inner, dtype)
    close(got["dbias"], ref["dbias"], bb, "dbias")
    close(got["dx"], ref["dx"], bx, "dx")
    close(got["dw"], ref["dw"], bw, "dw")
    return loss, lse, got


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,inner,classes", [(40, 24, 30), (8, 64, 900), (700, 64, 300)])
def test_masked_classes(agn, rows, inner, classes, dtype):
    """Classes with a bias of minus infinity (some of them labels, then the loss is infinite) and all of them."""
    x, w, b, labels = make(rows, inner, classes, dtype, masked=classes // 3)
    labels[::7] = classes - 1
    check(agn, x, w, b, labels, dtype)
    b[:] = -math.inf
    loss, lse, out = check(agn, x, w, b, labels, dtype)
    assert torch.all(lse == -math.inf) and torch.all(loss == math.inf)
    assert all(torch.all(out[k] == 0) for k in out)
    b[:] = torch.finfo(torch.float32).min   # the type's lowest value: all classes alike
    loss, lse = forward(agn, x, w, b, labels, dtype)
    assert torch.all(torch.isfinite(lse)) and torch.all(lse <= torch.finfo(torch.float32).min)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,inner,classes", [(40, 24, 30), (8, 64, 900), (700, 64, 300)])
def test_rows_that_are_not_finite(agn, rows, inner, classes, dtype):
    """A NaN row that has a label is NaN; the other rows' losses and dx are what they are without it."""
    x, w, b, labels = make(rows, inner, classes, dtype)
    loss0, lse0 = forward(agn, x, w, b, labels, dtype)
    dx0 = backward(agn, x, w, b, labels, lse0, dtype)["dx"]
    x[7, 3] = math.nan
    loss, lse = forward(agn, x, w, b, labels, dtype)
    rest = torch.arange(rows, device="cuda") != 7
    assert torch.isnan(loss[7]) and torch.isnan(lse[7])
    assert torch.equal(loss[rest], loss0[rest]) and torch.equal(lse[rest], lse0[rest])
    dx = backward(agn, x, w, b, labels, lse, dtype)["dx"]
    assert torch.all(torch.isnan(dx[7])) and torch.equal(dx[rest], dx0[rest])


@pytest.mark.parametrize("dtype,rows", [(1, 16384), (0, 6000)])
@pytest.mark.parametrize("ignored", [0.0, 0.2])
def test_pieces_of_the_classes(agn, dtype, rows, ignored):
    """More than one piece: dx is summed over them."""
    x, w, b, labels = make(rows, 24, 6001, dtype, ignored=ignored)
    assert rows * 6001 * (2 if dtype else 6) > 128 << 20
    check(agn, x, w, b, labels, dtype, scale=1.0 / rows)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("inner", [16, 13])
@pytest.mark.parametrize("ignored", [0.0, 0.4])
def test_more_rows_than_one_launch_prepares(agn, dtype, inner, ignored):
    rows = 40_001
    x, w, b, labels = make(rows, inner, 37, dtype, ignored=ignored)
    out = (labels < 0) | (labels >= 37)
    x[out] = math.nan
    _, _, got = check(agn, x, w, b, labels, dtype, scale=1.0 / rows)
    assert torch.all(got["dx"][out] == 0)


@pytest.mark.parametrize("dtype", [0, 1])
def test_outputs_not_wanted(agn, dtype):
    for size in ((40, 24, 30), (6, 64, 900), (700, 64, 300)):
        x, w, b, labels = make(*size, dtype)
        _, lse = forward(agn, x, w, b, labels, dtype)
        full = backward(agn, x, w, b, labels, lse, dtype)
        for without in (("dx",), ("dw",), ("dbias",), ("dx", "dw"), ("dw", "dbias"), ("dx", "dw", "dbias")):
            got = backward(agn, x, w, b, labels, lse, dtype, without=without)
            for k in full:
                assert got[k] is None if k in without else torch.equal(got[k], full[k])


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("size", [(40, 24, 30), (7, 70, 3000), (700, 64, 3000), (90, 200, 900), (3000, 264, 24)])
def test_equal_calls_give_equal_bits_and_stay_inside(agn, size, dtype):
    """Also in a workspace with other contents; what lies around the buffers stays as it was."""
    rows, inner, classes = size
    x, w, b, labels = make(*size, dtype, ignored=0.1)
    loss, lse = forward(agn, x, w, b, labels, dtype)
    full = backward(agn, x, w, b, labels, lse, dtype)
    n = [agn.agn_linear_ce_bytes(rows, inner, classes, dtype, k) for k in (0, 1)]
    work = torch.zeros(max(n) + 512, dtype=torch.uint8, device="cuda")
    pad = torch.full((2, rows + 8), 7.0, device="cuda")
    agn.agn_linear_ce(x, w, labels, dtype, rows, inner, classes, pad[0], pad[1], work, n[0], bias=b)
    assert torch.equal(pad[0, :rows], loss) and torch.equal(pad[1, :rows], lse) and torch.all(pad[:, rows:] == 7)
    assert torch.all(work[n[0]:] == 0)
    big = [torch.full((r * inner + 64,), 7.0, dtype=x.dtype, device="cuda") for r in (rows, classes)]
    db = torch.full((classes + 8,), 7.0, device="cuda")
    work[:] = 3
    agn.agn_linear_ce_backward(x, w, labels, lse, dtype, rows, inner, classes, work, n[1], dx=big[0], dw=big[1],
                               dbias=db, bias=b)
    for t, k in zip(big, ("dx", "dw")):
        assert torch.equal(t[:-64].view_as(full[k]), full[k]) and torch.all(t[-64:] == 7)
    assert torch.equal(db[:classes], full["dbias"]) and torch.all(db[classes:] == 7)
    assert torch.all(work[n[1]:] == 3)


def test_gradient_against_differences(agn):
    """dx and dw of the sum of losses (with a term of lse) against central differences of the forward call."""
    rows, inner, classes = 600, 24, 60
    x, w, b, labels = make(rows, inner, classes, 0)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    dloss, dlse = (torch.randn(rows, generator=g, device="cuda") for _ in range(2))
    _, lse = forward(agn, x, w, b, labels, 0)
    out = backward(agn, x, w, b, labels, lse, 0, dloss=dloss, dlse=dlse)

    def value(x, w, b):
        loss, lse = forward(agn, x, w, b, labels, 0)
        return float((dloss.double() * loss.double()).sum() + (dlse.double() * lse.double()).sum())

    for t, k in ((x, "dx"), (w, "dw"), (b, "dbias")):
        d = torch.randn(t.shape, generator=g, device="cuda")
        h = 2.0 ** -7
        args = dict(x=x, w=w, b=b)
        name = {"dx": "x", "dw": "w", "dbias": "b"}[k]
        hi, lo = (value(**dict(args, **{name: t + s * h * d})) for s in (1, -1))
        want = float((out[k].double() * d.double()).sum())
        # a row's curvature along d gives h^2 / 6 times a third derivative of order |dz|^3 (|dz| ~ 5 for dx and dw);
        # the values' own error is 1200 terms of 2^-20
        size = float((out[k].double().abs() * d.double().abs()).sum())
        assert abs((hi - lo) / (2 * h) - want) <= 0.02 * size + 1200 * 2.0 ** -20 / h


@pytest.mark.parametrize("size", [(40, 24, 30), (700, 64, 300), (100, 1000, 3000)])
def test_in_a_graph_and_on_another_stream(agn, size):
    """Loss and gradients captured (the first calls among them) and replayed on other contents."""
    rows, inner, classes = size
    x, w, b, labels = make(*size, 1, ignored=0.2)
    loss, lse, db = (torch.zeros(n, device="cuda") for n in (rows, rows, classes))
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    n = max(agn.agn_linear_ce_bytes(*size, 1, k) for k in (0, 1))
    work = torch.zeros(n, dtype=torch.uint8, device="cuda")

    def calls():
        st = torch.cuda.current_stream().cuda_stream
        agn.agn_linear_ce(x, w, labels, 1, *size, loss, lse, work, n, bias=b, stream=st)
        agn.agn_linear_ce_backward(x, w, labels, lse, 1, *size, work, n, dx=dx, dw=dw, dbias=db, bias=b, stream=st)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        calls()
    for seed in (1, 2):
        x2, w2, b2, l2 = make(*size, 1, ignored=0.4 * seed, seed=seed)
        for t, s in ((x, x2), (w, w2), (b, b2), (labels, l2)):
            t.copy_(s)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (loss, lse, dx, dw, db)]
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            calls()
        side.synchronize()
        for t, s in zip((loss, lse, dx, dw, db), got):
            assert torch.equal(t, s)
        ref = T.linear_ce(x2, w2, b2, l2)
        close(loss, ref["loss"], T.loss_bounds(ref, inner, 1)[0], "loss")
