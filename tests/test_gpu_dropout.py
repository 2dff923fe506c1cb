"""agn_dropout and agn_dropout_backward against their formulas in 64 bits: types, odd sizes,
strides, alignment, masked values that are not finite, captured and concurrent calls."""

import numpy as np
import pytest

import ops_ref as R

pytestmark = pytest.mark.gpu
HALF = {0: 2.0 ** -24, 1: 2.0 ** -8}   # half a step, relative


@pytest.fixture(scope="module")
def agn():
    import paper_1710_02368_gb300 as agn
    return agn


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


def dt(torch, d):
    return torch.float32 if d == 0 else torch.bfloat16


def strided(torch, d, rows, ld, start, rng, fill=None):
    """A [rows][ld] matrix that starts `start` elements into its buffer; (buffer, view)."""
    v = rng.standard_normal(start + rows * ld + 16) if fill is None else np.full(start + rows * ld + 16, fill)
    buf = torch.tensor(v, dtype=torch.float32, device="cuda").to(dt(torch, d))
    return buf, buf[start:start + rows * ld].view(rows, ld)


def f64(t):
    return t.double().cpu().numpy()


def check(got, want, tol):
    """Elementwise |got - want| <= tol."""
    assert got.shape == want.shape
    far = np.abs(got - want) - tol
    assert np.all(far <= 0), f"{np.sum(far > 0)} values off, worst {np.max(far)}"


SIZES = [(1, 1), (1, 3), (2, 4), (3, 5), (5, 8), (7, 31), (32, 128), (33, 1000), (40, 1003), (1, 4096),
         (257, 10), (1000, 12), (300, 257), (2049, 64)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("bias,relu,residual", [(0, 0, 0), (1, 1, 0), (0, 1, 1), (1, 0, 1)])
def test_forward(agn, torch, dtype, rows, cols, bias, relu, residual):
    rng = np.random.default_rng(rows * 7919 + cols)
    p, seed, offset = 0.3, 0xFEDCBA9876543210, (1 << 64) - 3   # the numbers wrap
    x = torch.tensor(rng.standard_normal((rows, cols)), device="cuda").to(dt(torch, dtype))
    b = torch.tensor(rng.standard_normal(cols), dtype=torch.float32, device="cuda") if bias else None
    res = torch.tensor(rng.standard_normal((rows, cols)), device="cuda").to(dt(torch, dtype)) if residual else None
    y = torch.full_like(x, 7.0)
    agn.agn_dropout(x, y, dtype, rows, cols, p, seed, offset, bias=b, residual=res, relu=relu)
    v = f64(x) + (f64(b) if bias else 0.0)
    t = np.where(R.keep_mask(rows, cols, p, seed, offset), (np.maximum(v, 0) if relu else v) * R.gain(p), 0.0)
    want = t + (f64(res) if residual else 0.0)
    # the sum with the bias, the scale (itself rounded) and its product: 3 roundings of 2^-24 of the
    # term; the sum with the residual 2^-24 of its value (of the term's error too: (1 + 2^-24)); the
    # output's half step of what is rounded.  1.01: second orders.
    term = 3 * 2.0 ** -24 * np.abs(t)
    tol = 1.01 * (term + 2.0 ** -24 * np.abs(want) + HALF[dtype] * (np.abs(want) + term)) + 1e-45
    check(f64(y), want, tol)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,cols", SIZES + [(5000, 24), (9000, 3)])
@pytest.mark.parametrize("relu,sums", [(0, 1), (1, 1), (1, 0)])
def test_backward(agn, torch, dtype, rows, cols, relu, sums):
    rng = np.random.default_rng(rows * 31 + cols)
    p, seed, offset = 0.6, 99, 1 << 40
    x = torch.tensor(rng.standard_normal((rows, cols)), device="cuda").to(dt(torch, dtype))
    b = torch.tensor(rng.standard_normal(cols), dtype=torch.float32, device="cuda")
    dy = torch.tensor(rng.standard_normal((rows, cols)), device="cuda").to(dt(torch, dtype))
    dx = torch.full_like(dy, 7.0)
    db = torch.full((cols,), 7.0, device="cuda") if sums else None
    agn.agn_dropout_backward(dy, dx, dtype, rows, cols, p, seed, offset, x=x if relu else None,
                             bias=b if relu else None, dbias=db, relu=relu)
    live = R.keep_mask(rows, cols, p, seed, offset)
    if relu:
        live = live & (f64(x) + f64(b) > 0)
    want = np.where(live, f64(dy) * R.gain(p), 0.0)
    check(f64(dx), want, 1.01 * (2 * 2.0 ** -24 + HALF[dtype]) * np.abs(want))
    if sums:
        # each term two roundings (scale, product), then rows - 1 additions, each of at most 2^-24 of the
        # sum of the magnitudes
        tol = 1.01 * (rows + 1) * 2.0 ** -24 * np.abs(want).sum(0) + 1e-45
        check(f64(db), want.sum(0), tol)
        again = torch.empty_like(db)
        agn.agn_dropout_backward(dy, dx, dtype, rows, cols, p, seed, offset, x=x if relu else None,
                                 bias=b if relu else None, dbias=again, relu=relu)
        assert torch.equal(db, again)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,cols", [(40000, 8), (33001, 4), (20011, 16), (17000, 33), (65536, 2)])
@pytest.mark.parametrize("relu", [0, 1])
def test_sums_of_tall_matrices(agn, torch, dtype, rows, cols, relu):
    """Wide clusters down the rows."""
    test_backward(agn, torch, dtype, rows, cols, relu, 1)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("ldx,ldr,ldy,start", [(20, 20, 20, 0), (21, 17, 19, 0), (24, 24, 24, 1), (17, 32, 24, 3)])
def test_strides_and_alignment(agn, torch, dtype, ldx, ldr, ldy, start):
    rng = np.random.default_rng(5)
    rows, cols = 37, 17
    _, x = strided(torch, dtype, rows, ldx, start, rng)
    _, res = strided(torch, dtype, rows, ldr, start, rng)
    buf, y = strided(torch, dtype, rows, ldy, start, rng, fill=7.0)
    agn.agn_dropout(x, y, dtype, rows, cols, 0.5, 3, residual=res, ldx=ldx, ldr=ldr, ldy=ldy)
    # the same values from packed rows: the same bits
    a, r2 = x[:, :cols].contiguous(), res[:, :cols].contiguous()
    z = torch.empty_like(a)
    agn.agn_dropout(a, z, dtype, rows, cols, 0.5, 3, residual=r2)
    assert torch.equal(y[:, :cols], z)
    buf[start:start + rows * ldy].view(rows, ldy)[:, :cols] = 7.0
    assert torch.all(buf == 7.0)   # nothing else was written
    # backward through other strides
    db, db2 = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    buf, dx = strided(torch, dtype, rows, ldy, start, rng, fill=7.0)
    agn.agn_dropout_backward(res, dx, dtype, rows, cols, 0.5, 3, x=x, dbias=db, relu=1, lddy=ldr,
                             ldx=ldx, lddx=ldy)
    agn.agn_dropout_backward(r2, z, dtype, rows, cols, 0.5, 3, x=a, dbias=db2, relu=1)
    assert torch.equal(dx[:, :cols], z)
    np.testing.assert_allclose(f64(db), f64(db2), rtol=0, atol=1.01 * 38 * 2.0 ** -24 * 2 * f64(r2.abs()).sum(0).max())
    buf[start:start + rows * ldy].view(rows, ldy)[:, :cols] = 7.0
    assert torch.all(buf == 7.0)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,cols,ld,start", [(1, 9, 9, 5), (70, 3, 5, 1), (211, 24, 24, 3), (530, 63, 67, 2), (1030, 287, 287, 0),
                                                (95, 1001, 1002, 7), (64, 260, 264, 4), (2050, 121, 125, 6)])
@pytest.mark.parametrize("two,sums", [(0, 0), (1, 0), (0, 1), (1, 1)])
def test_rows_that_start_alike_but_unaligned(agn, torch, dtype, rows, cols, ld, start, two, sums):
    """Every matrix's rows lie the same way to 16 bytes; what is between and around the rows stays."""
    rng = np.random.default_rng(rows + cols)
    p, seed, offset = 0.4, 77, 5
    _, a = strided(torch, dtype, rows, ld, start, rng)
    _, b = strided(torch, dtype, rows, ld, start, rng)
    buf, y = strided(torch, dtype, rows, ld, start, rng, fill=7.0)
    bias = torch.tensor(rng.standard_normal(cols), dtype=torch.float32, device="cuda")
    live = R.keep_mask(rows, cols, p, seed, offset)
    x, other = f64(a)[:, :cols], f64(b)[:, :cols]
    if sums:   # backward: dy a, the ReLU's input b
        db = torch.full((cols + 2,), 7.0, device="cuda")
        agn.agn_dropout_backward(a, y, dtype, rows, cols, p, seed, offset, x=b if two else None, bias=bias if two else None,
                                 dbias=db[1:], relu=two, lddy=ld, ldx=ld, lddx=ld)
        if two:
            live = live & (other + f64(bias) > 0)
        want = np.where(live, x * R.gain(p), 0.0)
        tol = 1.01 * (2 * 2.0 ** -24 + HALF[dtype]) * np.abs(want)
        # as in test_backward
        check(f64(db)[1:-1], want.sum(0), 1.01 * (rows + 1) * 2.0 ** -24 * np.abs(want).sum(0) + 1e-45)
        assert db[0] == 7 and db[-1] == 7
    else:
        agn.agn_dropout(a, y, dtype, rows, cols, p, seed, offset, bias=bias, residual=b if two else None, relu=1,
                        ldx=ld, ldr=ld, ldy=ld)
        t = np.where(live, np.maximum(x + f64(bias), 0) * R.gain(p), 0.0)
        want = t + (other if two else 0.0)
        # as in test_forward
        term = 3 * 2.0 ** -24 * np.abs(t)
        tol = 1.01 * (term + 2.0 ** -24 * np.abs(want) + HALF[dtype] * (np.abs(want) + term)) + 1e-45
    check(f64(y)[:, :cols], want, tol)
    if sums:   # in place: the same bits
        c, db2 = a.clone(), torch.empty_like(db[1:])
        agn.agn_dropout_backward(a, a, dtype, rows, cols, p, seed, offset, x=b if two else None, bias=bias if two else None,
                                 dbias=db2, relu=two, lddy=ld, ldx=ld, lddx=ld)
        assert torch.equal(a[:, :cols], y[:, :cols]) and torch.equal(a[:, cols:], c[:, cols:])
        check(f64(db2)[:-1], want.sum(0), 1.01 * (rows + 1) * 2.0 ** -24 * np.abs(want).sum(0) + 1e-45)
    rest = f64(buf)
    rest[start:start + rows * ld].reshape(rows, ld)[:, :cols] = 7.0
    assert np.all(rest == 7.0)


@pytest.mark.parametrize("dtype", [0, 1])
def test_in_place(agn, torch, dtype):
    rng = np.random.default_rng(6)
    x = torch.tensor(rng.standard_normal((65, 133)), device="cuda").to(dt(torch, dtype))
    r = torch.tensor(rng.standard_normal((65, 133)), device="cuda").to(dt(torch, dtype))
    y = torch.empty_like(x)
    agn.agn_dropout(x, y, dtype, 65, 133, 0.5, 3, residual=r, relu=1)
    a, b = x.clone(), r.clone()
    agn.agn_dropout(a, a, dtype, 65, 133, 0.5, 3, residual=r, relu=1)
    agn.agn_dropout(x, b, dtype, 65, 133, 0.5, 3, residual=b, relu=1)
    assert torch.equal(a, y) and torch.equal(b, y)
    d1, d2, d3 = torch.empty_like(x), r.clone(), x.clone()
    agn.agn_dropout_backward(r, d1, dtype, 65, 133, 0.5, 3, x=x, relu=1)
    agn.agn_dropout_backward(d2, d2, dtype, 65, 133, 0.5, 3, x=x, relu=1)
    agn.agn_dropout_backward(r, d3, dtype, 65, 133, 0.5, 3, x=d3, relu=1)
    assert torch.equal(d1, d2) and torch.equal(d1, d3)


def test_probabilities_at_the_ends(agn, torch):
    x = torch.randn(64, 100, device="cuda")
    y = torch.empty_like(x)
    for p in (0.0, 2.0 ** -18):                       # T = 0: nothing is dropped, scale 1
        agn.agn_dropout(x, y, 0, 64, 100, p, 1)
        assert torch.equal(x, y)
    agn.agn_dropout(x, y, 0, 64, 100, 0.9999999, 1)   # T = 65535: one in 65536 is kept
    keep = torch.tensor(R.keep_mask(64, 100, 0.9999999, 1), device="cuda")
    assert torch.equal(y != 0, keep)


@pytest.mark.parametrize("dtype", [0, 1])
def test_values_that_are_not_finite(agn, torch, dtype):
    """Dropped places are zero whatever they held; kept ones pass on (NaN through the ReLU too)."""
    rows, cols, p = 16, 40, 0.5
    x = torch.randn(rows, cols, device="cuda").to(dt(torch, dtype))
    x[0], x[1], x[2] = float("nan"), float("inf"), -float("inf")
    dy = torch.full_like(x, float("inf"))
    dy[3] = float("nan")
    y, dx = torch.empty_like(x), torch.empty_like(x)
    keep = torch.tensor(R.keep_mask(rows, cols, p, 8), device="cuda")
    agn.agn_dropout(x, y, dtype, rows, cols, p, 8, relu=1)
    assert torch.all(y[~keep] == 0)
    assert torch.all(y[0][keep[0]].isnan()) and torch.all(y[1][keep[1]] == float("inf"))
    assert torch.all(y[2] == 0)
    agn.agn_dropout_backward(dy, dx, dtype, rows, cols, p, 8, x=x, relu=1)
    live = keep & ~(x <= 0)
    assert torch.all(dx[~live] == 0) and torch.all(~dx[live].isfinite())


def test_gradient_against_differences(agn, torch):
    """d/dt of sum(w y(x + t d)) by central differences in 64 bits from the forward call itself: with
    steps of 2^-6 and inputs on a grid of 2^-10, sums and products here are exact in fp32."""
    rows, cols, p = 24, 36, 0.5
    rng = np.random.default_rng(9)
    grid = lambda *s: torch.tensor(rng.integers(-1024, 1025, s) / 1024.0, dtype=torch.float32, device="cuda")  # noqa: E731
    x, w, b, d, e = grid(rows, cols), grid(rows, cols), grid(cols), grid(rows, cols).sign(), grid(cols).sign()
    h = 2.0 ** -6
    x[(x + b).abs() < 4 * h] = 0.5   # away from the kink ...
    x[(x + b).abs() < 4 * h] = 1.0
    dx, db = torch.empty_like(x), torch.empty_like(b)
    agn.agn_dropout_backward(w, dx, 0, rows, cols, p, 5, x=x, bias=b, dbias=db, relu=1)

    def loss(xx, bb):
        y = torch.empty_like(xx)
        agn.agn_dropout(xx, y, 0, rows, cols, p, 5, bias=bb, relu=1)
        return float((y.double() * w.double()).sum())
    assert abs((loss(x + h * d, b) - loss(x - h * d, b)) / (2 * h) - float((dx.double() * d.double()).sum())) < 1e-9
    assert abs((loss(x, b + h * e) - loss(x, b - h * e)) / (2 * h) - float((db.double() * e.double()).sum())) < 1e-9


def test_empty_rows_give_zero_sums(agn, torch):
    db = torch.full((100,), 7.0, device="cuda")
    agn.agn_dropout_backward(None, None, 1, 0, 100, 0.5, 1, dbias=db)
    assert torch.all(db == 0)


def test_streams_and_graphs(agn, torch):
    """Two graphs and an eager call with other masks at once; a replay after the inputs changed."""
    rows, cols = 700, 1000
    x = torch.randn(rows, cols, device="cuda")
    outs = [torch.empty_like(x) for _ in range(3)]
    dbs = [torch.empty(cols, device="cuda") for _ in range(2)]
    graphs = []
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s = torch.cuda.current_stream().cuda_stream
            agn.agn_dropout(x, outs[i], 0, rows, cols, 0.5, 10 + i, relu=1, stream=s)
            agn.agn_dropout_backward(outs[i], outs[i], 0, rows, cols, 0.5, 10 + i, dbias=dbs[i], stream=s)
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(3)]
    x.copy_(torch.randn(rows, cols, device="cuda"))
    torch.cuda.synchronize()
    for i, g in enumerate(graphs):
        with torch.cuda.stream(streams[i]):
            g.replay()
            g.replay()
    agn.agn_dropout(x, outs[2], 0, rows, cols, 0.5, 12, relu=1, stream=streams[2].cuda_stream)
    torch.cuda.synchronize()
    for i in range(3):
        t = torch.empty_like(x)
        agn.agn_dropout(x, t, 0, rows, cols, 0.5, 10 + i, relu=1)
        if i < 2:
            db = torch.empty(cols, device="cuda")
            agn.agn_dropout_backward(t, t, 0, rows, cols, 0.5, 10 + i, dbias=db)
            assert torch.equal(db, dbs[i])
        assert torch.equal(t, outs[i])


def test_offsets_past_32_bits(agn, torch):
    """A matrix of 2.2 G elements: the last rows and their mask."""
    rows, cols = 270000, 8192
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    agn.agn_dropout(x, x, 1, rows, cols, 0.5, 4)
    tail = f64(x[-3:])
    groups = cols // 4
    want = R.keep_mask(3, cols, 0.5, 4, offset=(rows - 3) * groups) * 2.0
    assert np.array_equal(tail, want)
    del x
    torch.cuda.empty_cache()


def test_wide_clusters_first_called_in_a_capture():
    """A process whose first call is a captured one that needs clusters of more than eight blocks."""
    import os
    import subprocess
    import sys
    code = """
import torch, paper_1710_02368_gb300 as agn
x, y = torch.randn(40000, 8, device="cuda"), torch.empty(40000, 8, device="cuda")
db, again = torch.empty(8, device="cuda"), torch.empty(8, device="cuda")
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    agn.agn_dropout_backward(x, y, 0, 40000, 8, 0.5, 1, dbias=db, stream=torch.cuda.current_stream().cuda_stream)
g.replay(); torch.cuda.synchronize()
z = y.clone()
agn.agn_dropout_backward(x, y, 0, 40000, 8, 0.5, 1, dbias=again)
assert torch.equal(db, again) and torch.equal(y, z) and float(db.abs().sum()) > 0
print("same")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=root)
    assert r.returncode == 0 and "same" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]
