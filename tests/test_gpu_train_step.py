"""The loss, its gradients, their norm and the optimizer's step together, as a program trains a softmax
layer with them: against the same in 64 bits, and two runs bit for bit."""

import math

import numpy as np
import pytest
import torch

import train_ops_ref as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def agn():
    import paper_1710_02368_gb300 as agn
    return agn


def data(rows, inner, classes):
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = torch.randn(rows, inner, generator=g, device="cuda")
    w = torch.randn(classes, inner, generator=g, device="cuda") / math.sqrt(inner)
    labels = torch.randint(-1, classes, (rows,), generator=g, device="cuda", dtype=torch.int32)
    return x, w, labels


def train(agn, rows, inner, classes, steps, bits, dtype):
    x, w, labels = data(rows, inner, classes)
    f = dict(device="cuda")
    z = lambda *s: torch.zeros(*s, **f)
    low = torch.bfloat16 if dtype else torch.float32
    xl, b = x.to(low), z(classes)
    wl = w.to(low).clone()
    dw, db = torch.empty_like(wl), z(classes)
    loss, lse, norm, scale = z(rows), z(rows), z(1), z(1)
    work_bytes = max(agn.agn_linear_ce_bytes(rows, inner, classes, dtype, k) for k in (0, 1))
    work = torch.empty(work_bytes, dtype=torch.uint8, **f)
    tensors = []
    for p, g, gdt, copy, decay in ((w, dw, dtype, wl if dtype else None, 0.01), (b, db, 0, None, 0.0)):
        n = p.numel()
        k = torch.uint8 if bits == 8 else torch.float32
        t = dict(param=p, grad=g, grad_dtype=gdt, copy=copy, n=n, weight_decay=decay,
                 m=torch.zeros(n, dtype=k, **f), v=torch.zeros(n, dtype=k, **f))
        if bits == 8:
            t.update({s: torch.zeros(-(-n // 32), dtype=k, **f) for s in ("m_scale", "v_scale")})
        tensors.append(t)
    plan = agn.AGNOptim(tensors, state_bits=bits)
    wx = wl if dtype else w      # what the loss reads
    losses = []
    for t in range(1, steps + 1):
        agn.agn_linear_ce(xl, wx, labels, dtype, rows, inner, classes, loss, lse, work, work_bytes, bias=b)
        agn.agn_linear_ce_backward(xl, wx, labels, lse, dtype, rows, inner, classes, work, work_bytes, dw=dw, dbias=db,
                                   bias=b, scale=1.0 / rows)
        plan.grad_norm(0.5, norm, scale)
        plan.adamw(1e-2, t, scale=scale, seed=7, offset=(t - 1) * plan.draws)
        losses.append(loss.double().mean().item())
    return w, b, losses


def reference(rows, inner, classes, steps):
    x, w, labels = data(rows, inner, classes)
    w, b = w.double(), torch.zeros(classes, dtype=torch.float64, device="cuda")
    state = [[torch.zeros_like(w), torch.zeros_like(w)], [torch.zeros_like(b), torch.zeros_like(b)]]
    losses = []
    for t in range(1, steps + 1):
        r = T.linear_ce(x, w, b, labels, scale=1.0 / rows)
        losses.append(r["loss"].mean().item())
        g = [r["dw"], r["dbias"]]
        norm = math.sqrt(sum(float((v * v).sum()) for v in g))
        s = min(1.0, 0.5 / norm)
        for p, gr, st, decay in ((w, g[0], state[0], 0.01), (b, g[1], state[1], 0.0)):
            gr = gr * s
            st[0].mul_(0.9).add_(0.1 * gr)
            st[1].mul_(0.999).add_(0.001 * gr * gr)
            p.mul_(1 - 1e-2 * decay).sub_(1e-2 * (st[0] / (1 - 0.9 ** t)) / ((st[1] / (1 - 0.999 ** t)).sqrt() + 1e-8))
    return w, b, losses


@pytest.mark.parametrize("rows,inner,classes", [(40, 20, 12), (12, 64, 700), (700, 96, 1000)])
def test_training(agn, rows, inner, classes):
    """fp32: the first loss as the loss's bound says; Adam's step of an element whose gradient is about its error's
    size may differ by all of its 2 lr a step, the others by little: at most one in a hundred, 6 steps."""
    steps = 6
    w, b, losses = train(agn, rows, inner, classes, steps, 32, 0)
    rw, rb, rl = reference(rows, inner, classes, steps)
    for got, want in zip(losses, rl):
        assert abs(got - want) < 1e-4 * (1 + abs(want))
    for got, want in ((w, rw), (b, rb)):
        d = (got.double() - want).abs()
        assert float(d.max()) <= 2 * steps * 1e-2 and float((d > 1e-4).double().mean()) <= 0.01


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,inner,classes", [(40, 20, 12), (700, 96, 1000)])
def test_two_runs_are_alike(agn, rows, inner, classes, dtype, bits):
    a, b = (train(agn, rows, inner, classes, 4, bits, dtype) for _ in range(2))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and a[2] == b[2]
    assert all(math.isfinite(v) for v in a[2]) and np.isfinite(a[0].cpu().numpy()).all()
