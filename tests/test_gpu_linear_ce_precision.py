"""What the output layer's loss and its gradients keep of their operands, in norms (the bounds of train_ops_ref are
worst cases of every element and every addition)."""

import math

import pytest
import torch

import test_gpu_linear_ce as L
import train_ops_ref as T

pytestmark = pytest.mark.gpu
agn = L.agn


def norm(t):
    return float(t.double().norm())


# pairs of CTAs; rows left out; several pieces of the classes; one CTA a tile; logits by ranges of K in scratch; few rows
@pytest.mark.parametrize("rows,inner,classes,ignored", [
    (777, 1000, 10007, 0.3), (300, 264, 1000, 0.0), (600, 1001, 900, 0.0), (11000, 64, 8003, 0.1), (100, 1000, 999, 0.0),
    (60, 333, 3000, 0.2), (300, 3000, 200, 0.0), (70, 5000, 600, 0.1), (3, 1000, 777, 0.0), (40, 200, 60, 0.0)])
def test_bf16_gradients_are_rounded_once(agn, rows, inner, classes, ignored):
    """dx and dw are as far from the 64-bit ones as those rounded to bf16 are: that is 1.7e-3 of the norm (a half step
    of 2^-8 over mantissas of all sizes), while p in two pieces is off by 2^-17 and logits by some 1e-6: together
    2 % of that at most, and 5 % are allowed.  (p in one bf16 piece makes it 1.4 times, by the rounding of the scale alone.)"""
    x, w, b, labels = L.make(rows, inner, classes, 1, ignored=ignored)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    dlse = 1e-2 * torch.randn(rows, generator=g, device="cuda")
    scale = 1.0 / 777
    ref = T.linear_ce(x, w, b, labels, None, dlse, scale)
    _, lse = L.forward(agn, x, w, b, labels, 1)
    out = L.backward(agn, x, w, b, labels, lse, 1, scale=scale, dlse=dlse)
    for k in ("dx", "dw"):
        once = norm(ref[k].bfloat16().double() - ref[k])
        assert norm(out[k].double() - ref[k]) <= 1.05 * once, k
    assert norm(out["dbias"].double() - ref["dbias"]) <= 2.0 ** -16 * norm(ref["p_size"].sum(0))


@pytest.mark.parametrize("rows,classes", [(2048, 9728), (100, 19456)])
def test_bf16_logits_of_a_long_inner_side(agn, rows, classes):
    """Sums that only grow, over 65536 k.  A sum in the tensor cores loses two units of 2^-23 of itself at most in
    each addition (16 products), so sums of 64 additions, of which 64 are rounded, 2 (64 + 8) 2^-23 + 64 2^-24; over
    all of K it would be some 1e-4.  (All classes have the same logit, so the reference is a product with one vector.)"""
    inner = 65536
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = (0.5 + torch.rand(rows, inner, generator=g, device="cuda")).bfloat16()
    v = ((0.5 + torch.rand(inner, generator=g, device="cuda")) * 2.0 ** -12).bfloat16()
    w = v.expand(classes, inner).contiguous()
    labels = torch.zeros(rows, dtype=torch.int32, device="cuda")
    want = x.double() @ v.double() + math.log(classes)
    loss, lse = L.forward(agn, x, w, None, labels, 1)
    assert float(((lse - want) / want).abs().max()) <= 2 * 72 * 2.0 ** -23 + 66 * 2.0 ** -24
    lse = want.float()   # p is 1 / classes by the same logits
    db = L.backward(agn, x, w, None, labels, lse, 1, dloss=torch.zeros(rows, device="cuda"),
                    dlse=torch.ones(rows, device="cuda"), without=("dx", "dw"))["dbias"]
    # exp of an error of z, 32 or so
    assert float((db * (classes / rows) - 1).abs().max()) <= 1.1 * float(want.max()) * (2 * 72 * 2.0 ** -23 + 66 * 2.0 ** -24)


@pytest.mark.parametrize("dtype", [0, 1])
def test_bias_gradient_of_very_many_rows(agn, dtype):
    """Equal terms, which plain fp32 sums round the same way in every addition (1e-5 here): 32 rows are five
    additions, of a warp's part only the total is rounded, and 32 parts are added."""
    rows, inner, classes = 1 << 22, 8, 33
    x = torch.zeros(rows, inner, device="cuda", dtype=L.DT[dtype])
    w = torch.zeros(classes, inner, device="cuda", dtype=L.DT[dtype])
    zeros = torch.zeros(rows, device="cuda")
    labels = torch.zeros(rows, dtype=torch.int32, device="cuda")
    for term in (2.0 / 3, 0.7, 1.0 + 2.0 ** -20):
        dlse = torch.full((rows,), term, device="cuda")
        out = L.backward(agn, x, w, None, labels, zeros, dtype, dloss=zeros, dlse=dlse, without=("dx", "dw"))
        want = rows * float(dlse[0])   # (z = lse = 0: p is dlse)
        assert float((out["dbias"].double() / want - 1).abs().max()) <= 40 * 2.0 ** -24
