"""Microscaled 4-bit quantisation and product against their definitions in 64 bits: odd sizes,
strides, blocks that are empty, huge, tiny or not finite, every tile and split, captured calls."""

import numpy as np
import pytest

import ops_ref as R

pytestmark = pytest.mark.gpu


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


def buffers(agn, torch, rows, cols, fill=0xEE):
    c, s = agn.agn_mx4_bytes(rows, cols)
    return tuple(torch.full((max(n, 16),), fill, dtype=torch.uint8, device="cuda") for n in (c, s))


def quantize(agn, torch, x, dtype=0, ldx=None, cols=None, fill=0xEE):
    rows, cols = x.shape[0], x.shape[1] if cols is None else cols
    c, s = buffers(agn, torch, rows, cols, fill)
    agn.agn_mx4_quantize(x, dtype, rows, cols, c, s, ldx=ldx)
    return c, s


def padding(rows, cols):
    """Scale bytes that belong to a row, blocks past the row's last included; and those past it."""
    nb, k = R.blocks(cols), -(-R.blocks(cols) // 4)
    idx = np.arange(-(-rows // 128) * k * 512).reshape(-1, k, 32, 4, 4)
    by_row = idx.transpose(0, 3, 2, 1, 4).reshape(-1, 4 * k)
    return by_row[:rows, :nb], by_row[:rows, nb:], by_row[rows:]


def check_quantized(torch, x64, rows, cols, c, s):
    code, scale = R.mx4_quantize(x64)
    own, pad, beyond = padding(rows, cols)
    c, s = c.cpu().numpy(), s.cpu().numpy()
    assert np.array_equal(s[own], scale)
    assert np.array_equal(c[:code.size // 2].reshape(rows, -1), code[:, 0::2] | (code[:, 1::2] << 4))
    assert np.all(s[pad] == 0) and np.all(s[beyond] == 0xEE)


def hard_rows(rng, rows, cols):
    """Rows over 30 binades, with empty blocks, ties and saturated values among them."""
    x = rng.standard_normal((rows, cols)) * np.exp2(rng.integers(-15, 15, (rows, 1)))
    x[::3, : cols // 2] = 0
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.99, -0.25, -2.5, -5.0, 4.0])
    if cols >= 12:
        x[rows // 2, :12] = ties
        x[rows // 2, 12:] = np.clip(x[rows // 2, 12:], -7, 7)
    return x


SIZES = [(1, 1), (1, 31), (2, 32), (3, 33), (5, 100), (33, 127), (129, 128), (64, 129), (7, 784), (300, 250),
         (128, 1000), (1, 5000), (700, 40)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_quantize(agn, torch, dtype, rows, cols):
    x = torch.tensor(hard_rows(np.random.default_rng(cols), rows, cols), device="cuda").to(dt(torch, dtype))
    c, s = quantize(agn, torch, x, dtype)
    check_quantized(torch, x.double().cpu().numpy(), rows, cols, c, s)
    # and back, exact in either dtype
    for d in (0, 1):
        y = torch.full((rows, cols + 3), 7.0, device="cuda").to(dt(torch, d))
        agn.agn_mx4_dequantize(c, s, rows, cols, y, d, ldy=cols + 3)
        assert np.array_equal(y[:, :cols].double().cpu().numpy(),
                              R.mx4_unpack(c.cpu().numpy()[:rows * R.blocks(cols) * 16], s.cpu().numpy(), rows, cols))
        assert torch.all(y[:, cols:] == 7.0)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("ldx,start", [(104, 0), (101, 0), (104, 3), (120, 8)])
def test_quantize_strides(agn, torch, dtype, ldx, start):
    rng = np.random.default_rng(1)
    rows, cols = 50, 100
    buf = torch.tensor(rng.standard_normal(start + rows * ldx), device="cuda").to(dt(torch, dtype))
    x = buf[start:].view(rows, ldx)
    c, s = quantize(agn, torch, x, dtype, ldx=ldx, cols=cols)
    check_quantized(torch, x[:, :cols].double().cpu().numpy(), rows, cols, c, s)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,cols,ld,start", [(1, 1, 1, 1), (3, 16, 17, 3), (130, 33, 33, 0), (70, 95, 96, 7), (257, 1001, 1003, 5),
                                                (40, 4095, 4095, 2), (600, 17, 18, 1)])
def test_rows_that_are_not_aligned(agn, torch, dtype, rows, cols, ld, start):
    """Quantised and back; what is between and around the rows stays."""
    x = hard_rows(np.random.default_rng(rows), rows, cols)
    buf = torch.full((start + rows * ld + 9,), float("nan"), device="cuda").to(dt(torch, dtype))
    m = buf[start:start + rows * ld].view(rows, ld)
    m[:, :cols] = torch.tensor(x, device="cuda").to(dt(torch, dtype))
    c, s = quantize(agn, torch, m, dtype, ldx=ld, cols=cols)
    check_quantized(torch, m[:, :cols].double().cpu().numpy(), rows, cols, c, s)
    buf.fill_(7.0)
    agn.agn_mx4_dequantize(c, s, rows, cols, m, dtype, ldy=ld)
    want = R.mx4_unpack(c.cpu().numpy()[:rows * R.blocks(cols) * 16], s.cpu().numpy(), rows, cols)
    assert np.array_equal(m[:, :cols].double().cpu().numpy(), want)
    m[:, :cols] = 7.0
    assert torch.all(buf == 7.0)


def test_quantize_extremes(agn, torch):
    """Subnormal, smallest, largest and signed zero blocks; blocks that are not finite are NaN."""
    x = torch.zeros(8, 64, device="cuda")
    x[0, :32] = 2.0 ** -149
    x[0, 32:] = 1.5 * 2.0 ** -126
    x[1] = torch.finfo(torch.float32).max
    x[2, 5] = -2.0 ** -127
    x[3] = -0.0
    x[4, 3], x[5, 40], x[6, 63] = float("nan"), float("inf"), -float("inf")
    x[4:7] += 0.0
    x[7] = torch.linspace(-1e-38, 1e-38, 64)
    c, s = quantize(agn, torch, x)
    check_quantized(torch, x.double().cpu().numpy(), 8, 64, c, s)
    y = torch.empty_like(x)
    agn.agn_mx4_dequantize(c, s, 8, 64, y, 0)
    assert torch.all(y[4, :32].isnan()) and torch.all(y[4, 32:] == 0)
    assert torch.all(y[5, 32:].isnan()) and torch.all(y[5, :32] == 0)
    assert torch.all(y[6, 32:].isnan())
    assert torch.all(torch.signbit(y[3]))


# -------------------------------------------------------------------- product

def operands(agn, torch, rng, rows, inner, out, spread=0):
    """4-bit x and w and their values in 64 bits; spread: binades between the rows' sizes."""
    x = np.maximum(rng.standard_normal((rows, inner)), 0) * np.exp2(rng.integers(0, spread + 1, (rows, 1)))
    w = rng.uniform(-1, 1, (out, inner)) * np.exp2(rng.integers(0, spread + 1, (out, 1)))
    res = []
    for m in (x, w):
        code, scale = R.mx4_quantize(m)
        c, s = R.mx4_pack(code, scale)
        s = s.copy()
        s[padding(*m.shape)[2].ravel()] = 0xFF    # rows past the last one: NaN scales must not matter
        res.append((torch.tensor(c.reshape(-1), device="cuda"), torch.tensor(s, device="cuda"),
                    R.mx4_values(code, scale)[:, :inner]))
    return res


def linear(agn, torch, x, w, rows, inner, out, dtype=0, ldy=None, fill=7.0, **kw):
    ldy = out if ldy is None else ldy
    y = torch.full((rows, ldy), fill, device="cuda").to(dt(torch, dtype))
    agn.agn_mx4_linear(x[0], x[1], w[0], w[1], rows, inner, out, y, dtype, ldy=ldy, **kw)
    return y


def units(x, w):
    """Every product of a row of x and one of w is a multiple of the smallest last bits of the two; whether
    the sum of the magnitudes stays below 2^24 of it, where fp32 sums are exact in any order."""
    def unit(m):
        # a value is 1 or 1.5 times a power of two: its last bit is at least half its leading one
        _, ex = np.frexp(np.where(m == 0, np.inf, m))
        return np.where(m == 0, np.inf, np.exp2(ex - 2.0)).min(1)
    ux, uw = (np.where(np.isinf(u), 1.0, u) for u in (unit(x), unit(w)))
    u = np.outer(ux, uw)
    return u, np.abs(x) @ np.abs(w).T / u < 2 ** 24


LINEAR = [(1, 32, 1), (1, 1, 4), (2, 33, 10), (1, 784, 128), (5, 100, 31), (16, 256, 129), (17, 257, 128),
          (32, 64, 33), (33, 1000, 127), (64, 320, 300), (65, 784, 96), (128, 128, 128), (129, 65, 257),
          (200, 2048, 100), (257, 512, 260), (300, 96, 520), (1, 8192, 64), (3, 4096, 1000), (1030, 160, 140),
          (1100, 300, 388), (70, 5000, 40), (9800, 65, 257), (2500, 640, 1030), (2433, 1100, 1111)]


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,inner,out", LINEAR)
def test_linear_exact(agn, torch, rows, inner, out, dtype):
    """Sums that fp32 holds exactly have to come out exact (bf16: their one rounding)."""
    x, w = operands(agn, torch, np.random.default_rng(rows + inner + out), rows, inner, out)
    y = linear(agn, torch, x, w, rows, inner, out, dtype)
    want = x[2] @ w[2].T
    _, exact = units(x[2], w[2])
    assert exact.mean() > 0.9
    want32 = torch.tensor(want, dtype=torch.float32).to(dt(torch, dtype)).double().numpy()
    got = y.double().cpu().numpy()
    assert np.array_equal(got[exact], want32[exact])
    # elsewhere: every addition (at most inner) at most a step of 2^-23 of the sum of the magnitudes, twice the half
    # step that rounding to nearest takes, as tensor cores may cut off; then the output's rounding
    half = 2.0 ** -24 if dtype == 0 else 2.0 ** -8
    tol = inner * 2.0 ** -23 * (np.abs(x[2]) @ np.abs(w[2]).T) + half * np.abs(want)
    assert np.all(np.abs(got - want) <= 1.01 * tol)


@pytest.mark.parametrize("rows,inner,out", [(3, 200, 70), (40, 1000, 130), (150, 600, 260), (1500, 500, 200), (2433, 500, 1030)])
def test_linear_spread(agn, torch, rows, inner, out):
    """Rows 20 binades apart."""
    x, w = operands(agn, torch, np.random.default_rng(3), rows, inner, out, spread=20)
    got = linear(agn, torch, x, w, rows, inner, out).double().cpu().numpy()
    tol = 1.01 * inner * 2.0 ** -23 * (np.abs(x[2]) @ np.abs(w[2]).T)
    assert np.all(np.abs(got - x[2] @ w[2].T) <= tol)


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,inner,out", [(1, 64, 10), (20, 300, 131), (100, 257, 130), (1200, 128, 72), (9800, 65, 140)])
def test_bias_relu_strides(agn, torch, rows, inner, out, dtype):
    rng = np.random.default_rng(4)
    x, w = operands(agn, torch, rng, rows, inner, out)
    b = torch.tensor(rng.integers(-8, 9, out) / 4.0, dtype=torch.float32, device="cuda")
    want = np.maximum(x[2] @ w[2].T + b.double().cpu().numpy(), 0)
    want = torch.tensor(want, dtype=torch.float32).to(dt(torch, dtype)).double().numpy()
    _, exact = units(x[2], w[2])
    for ldy in (out, out + 1, (out + 7) // 4 * 4):
        y = linear(agn, torch, x, w, rows, inner, out, dtype, ldy=ldy, bias=b, relu=1)
        assert np.array_equal(y[:, :out].double().cpu().numpy()[exact], want[exact])
        assert torch.all(y[:, out:] == 7.0)


@pytest.mark.parametrize("rows,inner,out", [(1, 64, 10), (7, 1024, 32), (20, 300, 131), (100, 257, 130),
                                            (200, 784, 1000), (1200, 128, 72), (1030, 1000, 388), (9800, 96, 130), (2433, 300, 1111)])
def test_four_bit_output(agn, torch, rows, inner, out):
    """The 4-bit output is the quantisation of the fp32 one, byte for byte, and nothing else is written."""
    rng = np.random.default_rng(5)
    x, w = operands(agn, torch, rng, rows, inner, out)
    b = torch.tensor(rng.standard_normal(out), dtype=torch.float32, device="cuda")
    for relu in (0, 1):
        y = linear(agn, torch, x, w, rows, inner, out, bias=b, relu=relu)
        c, s = quantize(agn, torch, y)
        c2, s2 = buffers(agn, torch, rows, out)
        agn.agn_mx4_linear(x[0], x[1], w[0], w[1], rows, inner, out, c2, agn.AGN_PREC_MX4, bias=b, relu=relu,
                           y_scales=s2)
        assert torch.equal(c, c2) and torch.equal(s, s2)


def test_random_shapes(agn, torch):
    """Codes at random with scales within a factor of four: every sum is exact in fp32, at any shape, stride,
    start and type of the output."""
    rng = np.random.default_rng(11)
    for i in range(90):
        rows, inner, out = (int(round(np.exp(rng.uniform(0, np.log(hi))))) for hi in (900, 900, 700))
        if i % 6 == 0:
            rows, out = rows + 700, out + 300   # pairs of CTAs, and several tiles
        m = []
        for r in (rows, out):
            nb = R.blocks(inner)
            code = rng.integers(0, 16, (r, nb * 32)).astype(np.uint8)
            code[:, inner:] = 0
            scale = rng.integers(126, 129, (r, nb)).astype(np.uint8)
            c, s = R.mx4_pack(code, scale)
            s = s.copy()
            s[padding(r, inner)[2].ravel()] = 0xFF
            m.append((torch.tensor(c.reshape(-1), device="cuda"), torch.tensor(s, device="cuda"),
                      R.mx4_values(code, scale)[:, :inner]))
        dtype, relu, ldy, start = int(rng.integers(2)), int(rng.integers(2)), out + int(rng.integers(9)), int(rng.integers(9))
        if i % 3 == 0:
            ldy, start = (out + 15) // 8 * 8, 0
        buf = torch.full((start + rows * ldy + 8,), 7.0, device="cuda").to(dt(torch, dtype))
        y = buf[start:start + rows * ldy].view(rows, ldy)
        agn.agn_mx4_linear(*m[0][:2], *m[1][:2], rows, inner, out, y, dtype, relu=relu, ldy=ldy)
        want = m[0][2] @ m[1][2].T
        want = torch.tensor(np.maximum(want, 0) if relu else want, dtype=torch.float32).to(dt(torch, dtype)).double().numpy()
        got = y[:, :out].double().cpu().numpy()
        assert np.array_equal(got, want), (rows, inner, out, dtype, ldy, start)
        y[:, :out] = 7.0
        assert torch.all(buf == 7.0), (rows, inner, out, dtype, ldy, start)


def test_first_calls_in_a_capture(agn, torch):
    """A process whose first calls are captured ones: what a device is asked once is asked then."""
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = """
import torch, paper_1710_02368_gb300 as agn
def mat(r, c): return tuple(torch.zeros(n, dtype=torch.uint8, device="cuda") for n in agn.agn_mx4_bytes(r, c))
x, y, db = torch.randn(600, 300, device="cuda"), torch.empty(600, 300, device="cuda"), torch.empty(300, device="cuda")
q, w = mat(600, 300), mat(200, 300)
z, z1 = torch.empty(600, 200, device="cuda"), torch.empty(5, 200, device="cuda")
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    s = torch.cuda.current_stream().cuda_stream
    agn.agn_dropout(x, y, 0, 600, 300, 0.5, 1, relu=1, stream=s)
    agn.agn_dropout_backward(y, y, 0, 600, 300, 0.5, 1, x=x, relu=1, dbias=db, stream=s)
    agn.agn_mx4_quantize(x, 0, 600, 300, *q, stream=s)
    agn.agn_mx4_quantize(x, 0, 200, 300, *w, stream=s)
    agn.agn_mx4_linear(*q, *w, 600, 300, 200, z, 0, stream=s)
    agn.agn_mx4_linear(*q, *w, 5, 300, 200, z1, 0, stream=s)
g.replay(); torch.cuda.synchronize()
a, b, c = z.clone(), z1.clone(), db.clone()
agn.agn_mx4_linear(*q, *w, 600, 300, 200, z, 0)
agn.agn_mx4_linear(*q, *w, 5, 300, 200, z1, 0)
agn.agn_dropout(x, y, 0, 600, 300, 0.5, 1, relu=1)
agn.agn_dropout_backward(y, y, 0, 600, 300, 0.5, 1, x=x, relu=1, dbias=db)
assert torch.equal(a, z) and torch.equal(b, z1) and torch.equal(c, db) and float(a.abs().sum()) > 0
print("same")
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300, cwd=root)
    assert r.returncode == 0 and "same" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]


def test_two_threads(agn, torch):
    """Calls from two host threads, each on its own stream and buffers."""
    import threading
    rows, dims = 500, (300, 200)
    g = torch.Generator(device="cuda").manual_seed(3)
    xs = [torch.randn(rows, dims[0], generator=g, device="cuda") for _ in range(2)]
    w = quantize(agn, torch, torch.randn(dims[1], dims[0], generator=g, device="cuda"))
    bufs = [(buffers(agn, torch, rows, dims[0]), torch.empty(rows, dims[1], device="cuda")) for _ in range(2)]
    want = []
    for i in range(2):
        q = quantize(agn, torch, xs[i])
        want.append(linear(agn, torch, q, w, rows, *dims))
    torch.cuda.synchronize()
    streams, failed = [torch.cuda.Stream() for _ in range(2)], []

    def work(i):
        try:
            torch.cuda.set_device(0)
            for _ in range(200):
                agn.agn_mx4_quantize(xs[i], 0, rows, dims[0], *bufs[i][0], stream=streams[i].cuda_stream)
                agn.agn_mx4_linear(*bufs[i][0], *w, rows, *dims, bufs[i][1], 0, stream=streams[i].cuda_stream)
                try:
                    agn.agn_mx4_linear(*bufs[i][0], *w, -1 - i, *dims, bufs[i][1], 0)
                except agn.AGNError as e:
                    assert e.code == agn.AGN_E_INVALID
        except Exception as e:  # noqa: BLE001
            failed.append(e)
    ts = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    [t.start() for t in ts]
    [t.join() for t in ts]
    torch.cuda.synchronize()
    assert not failed
    for i in range(2):
        assert torch.equal(bufs[i][1], want[i])


def test_not_finite(agn, torch):
    """A NaN block of a row makes that row NaN and no other; of a feature, that column; through the ReLU
    and into a 4-bit output."""
    rows, inner, out = 40, 300, 70
    g = torch.Generator(device="cuda").manual_seed(1)
    xv = torch.randn(rows, inner, generator=g, device="cuda")
    wv = torch.randn(out, inner, generator=g, device="cuda")
    xv[3, 7], wv[11, 299] = float("inf"), float("nan")
    x, w = quantize(agn, torch, xv), quantize(agn, torch, wv)
    y = linear(agn, torch, x, w, rows, inner, out, relu=1)
    bad = torch.zeros(rows, out, dtype=torch.bool, device="cuda")
    bad[3], bad[:, 11] = True, True
    assert torch.equal(y.isnan(), bad)
    c, s = buffers(agn, torch, rows, out)
    agn.agn_mx4_linear(x[0], x[1], w[0], w[1], rows, inner, out, c, agn.AGN_PREC_MX4, y_scales=s)
    z = torch.empty_like(y)
    agn.agn_mx4_dequantize(c, s, rows, out, z, 0)
    assert torch.all(z[:, :32].isnan()) and not z[4, 32:].isnan().any() and z[3].isnan().all()


def test_layers_in_a_graph_and_on_streams(agn, torch):
    """Quantise, two layers (the first's output in 4 bits), captured twice and replayed on two streams at
    once with an eager call beside; the same bits as one call after another."""
    rows, dims = 300, (200, 260, 90)
    g = torch.Generator(device="cuda").manual_seed(2)
    ws = [quantize(agn, torch, torch.randn(dims[i + 1], dims[i], generator=g, device="cuda")) for i in range(2)]
    xs = [torch.randn(rows, dims[0], generator=g, device="cuda") for _ in range(3)]
    err = torch.zeros(1, dtype=torch.int32, device="cuda")

    def run(x, bufs, stream):
        (c0, s0), (c1, s1), y = bufs
        agn.agn_mx4_quantize(x, 0, rows, dims[0], c0, s0, stream=stream)
        agn.agn_mx4_linear(c0, s0, *ws[0], rows, dims[0], dims[1], c1, agn.AGN_PREC_MX4, relu=1, y_scales=s1,
                           err=err, stream=stream)
        agn.agn_mx4_linear(c1, s1, *ws[1], rows, dims[1], dims[2], y, 0, err=err, stream=stream)

    def fresh():
        return (buffers(agn, torch, rows, dims[0]), buffers(agn, torch, rows, dims[1]),
                torch.empty(rows, dims[2], device="cuda"))
    want = []
    for x in xs:
        b = fresh()
        run(x, b, None)
        want.append(b[2].clone())
    torch.cuda.synchronize()
    bufs, graphs = [fresh() for _ in range(3)], []
    for i in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            run(xs[i], bufs[i], torch.cuda.current_stream().cuda_stream)
        graphs.append(gr)
    streams = [torch.cuda.Stream() for _ in range(3)]
    for _ in range(5):
        for i, gr in enumerate(graphs):
            with torch.cuda.stream(streams[i]):
                gr.replay()
        run(xs[2], bufs[2], streams[2].cuda_stream)
    torch.cuda.synchronize()
    for i in range(3):
        assert torch.equal(bufs[i][2], want[i])
    assert int(err) == 0
    # the first layer's values, from the definitions
    q = R.mx4_values(*R.mx4_quantize(xs[0].double().cpu().numpy()))[:, :dims[0]]
    w0 = R.mx4_unpack(ws[0][0].cpu().numpy()[:dims[1] * R.blocks(dims[0]) * 16], ws[0][1].cpu().numpy(), dims[1], dims[0])
    h = R.mx4_values(*R.mx4_quantize(np.maximum(q @ w0.T, 0).astype(np.float32).astype(np.float64)))[:, :dims[1]]
    got = R.mx4_unpack(bufs[0][1][0].cpu().numpy()[:rows * R.blocks(dims[1]) * 16], bufs[0][1][1].cpu().numpy(), rows, dims[1])
    assert np.mean(got != h) < 1e-3   # (a sum that rounds the other way at a border of the codes)


def test_refuses_other_memory(agn, torch):
    x = torch.randn(4, 64)
    d = torch.randn(4, 64, device="cuda")
    c, s = buffers(agn, torch, 4, 64)
    for bad in (x, x.pin_memory()):
        with pytest.raises(agn.AGNError) as e:
            agn.agn_mx4_quantize(bad, 0, 4, 64, c, s)
        assert e.value.code == agn.AGN_E_INVALID and "current device" in str(e.value)
        with pytest.raises(agn.AGNError):
            agn.agn_dropout(d, bad, 0, 4, 64, 0.5, 1)
