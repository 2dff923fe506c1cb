"""The inputs and the bounds of test_gpu_linear_ce_pieces, without a GPU: 64-bit arithmetic on three bf16 pieces of
each operand meets them, and does not where any of the six products of pieces is left out that the inputs are made for."""

import math

import pytest
import torch

import test_gpu_linear_ce_pieces as G
import train_ops_ref as T

SIX = [(0, 0), (0, 1), (1, 0), (1, 1), (0, 2), (2, 0)]


def pieces(t):
    out, rest = [], t.double()
    for _ in range(3):
        out.append(rest.float().bfloat16().double())
        rest = rest - out[-1]
    return out


def product(a, b, which):
    """a [M][K] b [N][K]^T from products of pieces."""
    a, b = pieces(a), pieces(b)
    return sum(a[i] @ b[j].t() for i, j in which)


@pytest.mark.parametrize("kind,left_out", [(1, (0, 1)), (1, (1, 1)), (2, (0, 2)), (3, (1, 0)), (3, (1, 1)), (4, (2, 0))])
def test_pairs_need_each_product(kind, left_out):
    g = torch.Generator()
    g.manual_seed(kind)
    a, b = G.pairs(kind, 600, (40,), (30,), g)
    want = a.double() @ b.double().t()
    off = lambda which: float(((product(a, b, which) - want) / want).abs().min())
    assert float(((product(a, b, SIX) - want) / want).abs().max()) <= 2.0 ** -40
    assert off([p for p in SIX if p != left_out]) >= 2.0 ** -11


@pytest.mark.parametrize("left_out", SIX[1:] + [None, "third pieces"])
def test_norms_need_each_product(left_out):
    rows, inner, classes = 300, 1000, 700
    g = torch.Generator()
    g.manual_seed(1)
    x = torch.randn(rows, inner, generator=g)
    w = torch.randn(classes, inner, generator=g) * 2 / math.sqrt(inner)
    b = 0.5 * torch.randn(classes, generator=g)
    labels = torch.randint(0, classes, (rows,), generator=g)
    ref = T.linear_ce(x, w, b, labels, scale=1.0 / rows)
    which = [p for p in SIX if p != left_out and not (left_out == "third pieces" and 2 in p)]
    z = product(x, w, which) + b.double()
    lse = torch.logsumexp(z, 1)
    loss = lse - z.gather(1, labels[:, None])[:, 0]
    p = torch.exp(z - lse[:, None]) / rows
    p[torch.arange(rows), labels] -= 1 / rows
    p = p.float()
    dx, dw = product(p, w.t(), which), product(p.t(), x.t(), which)
    far = [G.norm(loss - ref["loss"]) / math.sqrt(rows) / 3e-6] + [G.norm(t - ref[k]) / G.norm(ref[k]) / 2e-6
                                                                 for t, k in ((dx, "dx"), (dw, "dw"))]
    if left_out is None:
        assert max(far) <= 0.1
    else:
        assert far[0] > 1.2 and max(far[1:]) > 1.0
