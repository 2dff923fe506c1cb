"""fp32 in the output layer's loss: each of the six products of three bf16 pieces is there, and the sums lose little.

First inputs made of pairs whose leading products cancel, so that what is left lies in the smaller pieces alone: a
product that is missing is 2^-9 of the result or all of it, the allowed error 2^-20 (every value and sum here fits
24 bits, and nothing is added to much larger sums).  Then random inputs, in norms: bounds and where they lie
between what the arithmetic loses and what a missing product would."""

import math

import pytest
import torch

import test_gpu_linear_ce as L
import train_ops_ref as T

pytestmark = pytest.mark.gpu
agn = L.agn
P, Q = 2.0 ** -9, 2.0 ** -18   # the second and third piece of 1 + ... (up to twice them: so no piece is negative)

# plain kernels; few rows; one CTA a tile; w as it is, 64 and 128 rows; pairs with narrow, odd and wide tiles
SIZES = [(40, 64, 30), (8, 1024, 2000), (16, 1600, 301), (100, 1000, 999), (60, 1024, 4000), (120, 1026, 4000), (300, 512, 300),
         (777, 1002, 1500), (2500, 1024, 4000)]


def ints(g, lo, hi, *shape):
    return torch.randint(lo, hi + 1, shape, generator=g, device=g.device).float()


def pairs(kind, n, first, second, g):
    """Two factors along n places, in pairs, whose products' sum is that of small pieces: what varies within a
    pair is the second (kinds 1, 2) or the first factor (3, 4).  first, second: the other dimensions."""
    h = n // 2
    steady, moving = (first, second) if kind <= 2 else (second, first)
    if kind in (1, 3):   # (1 + a P) (1 + s P) - (1 + a P): second pieces times first and second ones
        u = 1 + ints(g, 0, 2, *steady, h) * P
        lo, hi = 1 + ints(g, 1, 2, *moving, h) * P, torch.ones(*moving, h, device=g.device)
    else:                # v + s Q - v: third pieces times first ones
        u = torch.ones(*steady, h, device=g.device)
        hi = torch.full((*moving, h), 1 + P, device=g.device)
        lo = hi + ints(g, 1, 2, *moving, h) * Q
    a = torch.zeros(*steady, n, device=g.device)
    b = torch.zeros(*moving, n, device=g.device)
    a[..., 0:2 * h:2] = a[..., 1:2 * h:2] = u
    b[..., 0:2 * h:2], b[..., 1:2 * h:2] = lo, -hi
    return (a, b) if kind <= 2 else (b, a)


def near(got, want, what):
    err = float(((got.double() - want) / want).abs().max())
    assert err <= 2.0 ** -20, (what, err)


def generator(kind, rows):
    g = torch.Generator(device="cuda")
    g.manual_seed(10 * rows + kind)
    return g


@pytest.mark.parametrize("kind", [1, 2, 3, 4])
@pytest.mark.parametrize("rows,inner,classes", SIZES)
def test_logits(agn, rows, inner, classes, kind):
    """One class that is not masked: lse is its logit."""
    g = generator(kind, rows)
    labels = torch.zeros(rows, dtype=torch.int32, device="cuda")
    x, v = pairs(kind, inner, (rows,), (1,), g)
    for c in (0, classes // 2, classes - 1):
        w = torch.randn(classes, inner, generator=g, device="cuda")
        w[c] = v[0]
        b = torch.full((classes,), -math.inf, device="cuda")
        b[c] = 0.0
        _, lse = L.forward(agn, x, w, b, labels, 0)
        near(lse, x.double() @ v[0].double(), c)


@pytest.mark.parametrize("kind", [1, 2, 3, 4])
@pytest.mark.parametrize("rows,inner,classes", SIZES)
def test_weights_gradient(agn, rows, inner, classes, kind):
    """w and lse are 0, so p is dlse of the row."""
    p, x = pairs(kind, rows, (1,), (inner,), generator(kind, rows))
    p, x = p.expand(inner, rows)[0].contiguous(), x.expand(inner, rows).t().contiguous()
    zeros = torch.zeros(rows, device="cuda")
    out = L.backward(agn, x, torch.zeros(classes, inner, device="cuda"), None, torch.zeros(rows, dtype=torch.int32, device="cuda"),
                     zeros, 0, dloss=zeros, dlse=p)
    near(out["dw"], (p.double() @ x.double()).expand(classes, inner), "dw")
    assert torch.all(out["dx"] == 0)


@pytest.mark.parametrize("kind", [1, 2])
@pytest.mark.parametrize("rows,inner,classes", SIZES)
def test_rows_gradient(agn, rows, inner, classes, kind):
    """x and lse are 0, so p is dlse of the row for all classes; w varies in pairs of classes."""
    g = generator(kind, rows)
    _, w = pairs(kind, classes, (1,), (inner,), g)
    u = 1 + (ints(g, 0, 2, rows) * P if kind == 1 else torch.zeros(rows, device="cuda"))
    zeros = torch.zeros(rows, device="cuda")
    w = w.t().contiguous()
    out = L.backward(agn, torch.zeros(rows, inner, device="cuda"), w, None, torch.zeros(rows, dtype=torch.int32, device="cuda"),
                     zeros, 0, dloss=zeros, dlse=u)
    near(out["dx"], u.double()[:, None] * w.double().sum(0), "dx")
    near(out["dbias"], u.double().sum().expand(classes), "dbias")


@pytest.mark.parametrize("kind", [3, 4])
@pytest.mark.parametrize("rows,inner,classes", SIZES)
def test_rows_gradient_by_pieces_of_p(agn, rows, inner, classes, kind):
    """Two classes that are not masked, with equal weights; p of the one is u, of the other, the label, u - b = -(u + e)."""
    g = generator(kind, rows)
    s = ints(g, 1, 2, rows)
    u, e = (1.0, s * P) if kind == 3 else (1 + P, s * Q)
    v = 1 + ints(g, 0, 2, inner) * P if kind == 3 else torch.ones(inner, device="cuda")
    for c0, c1 in ((0, 1), (classes // 2, classes // 2 - 1), (classes - 1, 0)):
        w = torch.randn(classes, inner, generator=g, device="cuda")
        w[c0] = w[c1] = v
        b = torch.full((classes,), -math.inf, device="cuda")
        b[c0] = b[c1] = 0.0
        labels = torch.full((rows,), c0, dtype=torch.int32, device="cuda")
        out = L.backward(agn, torch.zeros(rows, inner, device="cuda"), w, b, labels, torch.zeros(rows, device="cuda"), 0,
                         dloss=2 * u + e, dlse=-(u + e), without=("dw",))
        near(out["dx"], -e.double()[:, None] * v.double(), (c0, c1))


def norm(t):
    return float(t.double().norm())


@pytest.mark.parametrize("rows,inner,classes", [(777, 1000, 1500), (300, 3000, 200), (128, 2048, 1664), (20, 4096, 640), (60, 5000, 600),
                                                (64, 4096, 1024), (8, 2000, 999), (700, 2100, 15), (257, 601, 900), (2500, 1024, 4000)])
def test_norms(agn, rows, inner, classes):
    """Logits of a spread of 2.  Of a sum over 256 or 512 k each of 16 or 32 additions loses half a unit of 2^-23 or less
    of it, together some 8 units while it grows: 2e-6 of a logit; losses of about 10 are rounded to 2^-21, by half of
    it: 2.5e-6 in the root mean square, 3e-6 allowed.  A product of pieces that is missing makes it 4.7e-6 or more, two pieces for
    three 7e-6 (64-bit arithmetic on the pieces).  dx and dw: 1e-6 by their own sums and 0.6e-6 by p's logits, 2e-6 allowed; two
    pieces for three make 2.8e-6 or more."""
    x, w, b, labels = L.make(rows, inner, classes, 0)
    ref = T.linear_ce(x, w, b, labels, scale=1.0 / rows)
    loss, lse = L.forward(agn, x, w, b, labels, 0)
    assert norm(loss.double() - ref["loss"]) <= 3e-6 * math.sqrt(rows)
    assert norm(lse.double() - ref["lse"]) <= 3e-6 * math.sqrt(rows)
    out = L.backward(agn, x, w, b, labels, lse, 0, scale=1.0 / rows)
    for k in ("dx", "dw", "dbias"):
        assert norm(out[k].double() - ref[k]) <= 2e-6 * norm(ref[k]), k
