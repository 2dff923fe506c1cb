"""The output layer's loss and the optimizer's step at sizes drawn at random, past 32 bits of elements, on
two threads and beside a training handle."""

import math
import threading

import numpy as np
import pytest
import torch

import agn_inputs as I
import test_gpu_linear_ce as L
import train_ops_ref as T

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def agn():
    import paper_1710_02368_gb300 as agn
    return agn


@pytest.mark.parametrize("seed", range(24))
def test_random_shapes(agn, seed):
    rng = np.random.default_rng(100 + seed)
    rows, inner, classes = (int(np.exp(rng.uniform(0, math.log(m)))) for m in (3000, 900, 6000))
    dtype = seed % 2
    masked = classes // 5 if seed % 3 == 0 else 0
    x, w, b, labels = L.make(rows, inner, classes, dtype, bias=seed % 4 != 1, ignored=(0.0, 0.3)[seed // 2 % 2],
                             masked=masked if seed % 4 != 1 else 0, seed=seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dloss, dlse = (torch.randn(rows, generator=g, device="cuda") for _ in range(2))
    L.check(agn, x, w, b, labels, dtype, scale=0.3, dloss=dloss if seed % 3 else None, dlse=dlse if seed % 5 else None)


def test_weights_past_32_bits(agn):
    """w and dw of 4.9e9 elements (9.8 GB), several pieces of the classes."""
    rows, inner, classes = 130, 8192, 600_000
    assert classes * inner > 1 << 32
    x, w, _, labels = L.make(rows, inner, classes, 1, bias=False)
    labels[:4] = torch.tensor([classes - 1, classes - 300, 524_289, 0], dtype=torch.int32)
    loss, lse = L.forward(agn, x, w, None, labels, 1)
    xd = x.double()
    tops, sums, step = [], 0.0, 20_000
    for c in range(0, classes, step):
        wc = w[c:c + step].double()
        tops.append(torch.logsumexp(xd @ wc.t(), 1))
        sums = max(sums, float((xd.abs() @ wc.abs().t()).max()))
    want = torch.logsumexp(torch.stack(tops), 0)
    e = sums * (2 * T.steps(inner) * 2.0 ** -23 + 2.0 ** -22)
    assert float((lse - want).abs().max()) <= e + 2.0 ** -18 + 2.0 ** -22 * 20
    zl = (xd * w[labels.long()].double()).sum(1)
    assert float((loss - (want - zl)).abs().max()) <= 2 * e + 2.0 ** -18 + 2.0 ** -22 * 20
    out = L.backward(agn, x, w, None, labels, lse, 1, scale=1.0)
    dx = torch.zeros(rows, inner, dtype=torch.float64, device="cuda")
    size = torch.zeros_like(dx)
    rel = 2 * e + 2.0 ** -17 + 2.0 ** -8     # of p: its logits', and its rounding to bf16
    for c in range(0, classes, step):
        wc = w[c:c + step].double()
        p = torch.exp(xd @ wc.t() - want[:, None])
        at = labels.long() - c
        here = (at >= 0) & (at < step)
        q = p.clone()
        q[here, at[here]] += 1.0
        p[here, at[here]] -= 1.0
        dx += p @ wc
        size += q @ wc.abs()
        dw, bound = p.t() @ xd, q.t() @ xd.abs() * (rel + 2.0 ** -19)
        assert torch.all((out["dw"][c:c + step].double() - dw).abs() <= bound + dw.abs() * 2.0 ** -8 + 1e-30)
    err = (out["dx"].double() - dx).abs()
    assert torch.all(err <= size * (rel + 2 * T.steps(classes) * 2.0 ** -23) + dx.abs() * 2.0 ** -8)


def test_states_past_32_bits(agn):
    """8-bit states of 2^32 + 70001 elements in one tensor: its last elements, and some at 2^31 and 2^32."""
    n = (1 << 32) + 70_001
    f, u = dict(device="cuda"), torch.uint8
    nb = -(-n // 32)
    t = dict(param=torch.full((n,), 0.5, **f), grad=torch.zeros(n, dtype=torch.bfloat16, **f),
             m=torch.zeros(n, dtype=u, **f), v=torch.zeros(n, dtype=u, **f), m_scale=torch.full((nb,), 110, dtype=u, **f),
             v_scale=torch.full((nb,), 110, dtype=u, **f), n=n, grad_dtype=1)
    places = [slice((1 << 31) - 64, (1 << 31) + 64), slice((1 << 32) - 64, (1 << 32) + 64), slice(n - 81, n)]
    places[2] = slice((n - 81) // 32 * 32, n)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    for p in places:
        k = p.stop - p.start
        t["grad"][p] = (1e-3 * torch.randn(k, generator=g, device="cuda")).bfloat16()
        t["m"][p] = torch.randint(0, 256, (k,), generator=g, dtype=u, device="cuda")
        t["v"][p] = torch.randint(0, 256, (k,), generator=g, dtype=u, device="cuda")
    old = [{k: t[k][p].clone() for k in ("param", "grad", "m", "v")} for p in places]
    with agn.AGNOptim([t], state_bits=8) as plan:
        plan.adamw(1e-2, 3, seed=4, offset=5)
        norm = torch.zeros(1, **f)
        plan.grad_norm(1.0, norm)
    want = math.sqrt(sum(float((t["grad"][p].double() ** 2).sum()) for p in places))
    assert abs(norm.item() - want) <= 65 * 2.0 ** -24 * want
    for p, o in zip(places, old):
        h = {k: v.cpu() for k, v in o.items()}
        k = p.stop - p.start
        s = np.full(-(-k // 32), 110, np.uint8)
        r = T.r_values(h["v"].numpy(), s)
        new, m, v, r = T.adamw(h["param"].double().numpy(), h["grad"].double().numpy(), T.m_values(h["m"].numpy(), s),
                               T.f32(r * r), 1e-2, 3, 0.9, 0.999, 1e-8, 0.0)
        bm, br = T.random_bits(4, 5 + p.start // 2, k)
        c, ms = T.rounded(np.abs(m), bm, 3)
        assert np.array_equal(t["m"][p].cpu().numpy(), c | (np.signbit(m).astype(np.uint8) << 7))
        c, vs = T.rounded(r, br, 4)
        assert np.array_equal(t["v"][p].cpu().numpy(), np.where(r > 0, np.maximum(c, 1), c))
        b = slice(p.start // 32, -(-p.stop // 32))
        assert np.array_equal(t["m_scale"][b].cpu().numpy(), ms) and np.array_equal(t["v_scale"][b].cpu().numpy(), vs)
        assert np.all(np.abs(t["param"][p].double().cpu().numpy() - new) <= 2.0 ** -22)


def work(agn, steps, stream):
    """Losses, gradients and steps of a few layers, one after the other on a stream."""
    out = []
    with torch.cuda.stream(stream):
        st = stream.cuda_stream
        for rows, inner, classes, dtype in ((32, 128, 10, 0), (8, 512, 3000, 0), (700, 1000, 520, 1), (300, 264, 1000, 0)):
            x, w, b, labels = L.make(rows, inner, classes, dtype, ignored=0.2)
            low = w.clone()
            master = w.float()
            loss, lse, db = (torch.zeros(k, device="cuda") for k in (rows, rows, classes))
            dx, dw = torch.zeros_like(x), torch.zeros_like(w)
            n = max(agn.agn_linear_ce_bytes(rows, inner, classes, dtype, k) for k in (0, 1))
            scratch = torch.zeros(n, dtype=torch.uint8, device="cuda")
            u = dict(dtype=torch.uint8, device="cuda")
            k = master.numel()
            t = dict(param=master, grad=dw, grad_dtype=dtype, copy=low if dtype else None, n=k, m=torch.zeros(k, **u),
                     v=torch.zeros(k, **u), m_scale=torch.zeros(-(-k // 32), **u), v_scale=torch.zeros(-(-k // 32), **u))
            stream.synchronize()
            with agn.AGNOptim([t], state_bits=8) as plan:
                norm, scale = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
                for i in range(1, steps + 1):
                    read = low if dtype else master
                    agn.agn_linear_ce(x, read, labels, dtype, rows, inner, classes, loss, lse, scratch, n, bias=b, stream=st)
                    agn.agn_linear_ce_backward(x, read, labels, lse, dtype, rows, inner, classes, scratch, n, dx=dx,
                                               dw=dw, dbias=db, bias=b, scale=1 / rows, stream=st)
                    plan.grad_norm(0.1, norm, scale, stream=st)
                    plan.adamw(1e-2, i, scale=scale, seed=3, offset=i * plan.draws, stream=st)
                stream.synchronize()
            out += [loss.clone(), dx.clone(), db.clone(), master.clone(), t["m"], t["v"]]
        stream.synchronize()
    return out


def test_two_threads_and_a_training_handle(agn):
    """The same work on two threads' streams while a handle trains on a third: all as alone, bit for bit."""
    dims, n, m, seed, C = (784, 1000, 1000, 10), 4, 128, 5, 24
    w, tau = I.make_schedule(n, C + n, 0, 2, seed)

    def train():
        out = []
        with agn.AGN(dims, n, 4, 0.05, seed, batch=m, n_samples=n * 2 * m) as h:
            for c in range(0, C, 8):
                h.run(8, w[c:], tau[c:])
                out.append(h.loss())
            out.append(h.central())
        return out

    alone, trained = work(agn, 20, torch.cuda.Stream()), train()
    got, errors = {}, []

    def on(name, f):
        try:
            got[name] = f()
        except Exception as e:   # (reported below)
            errors.append(e)
    threads = [threading.Thread(target=on, args=(i, lambda: work(agn, 20, torch.cuda.Stream()))) for i in range(2)]
    threads.append(threading.Thread(target=on, args=("train", train)))
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    for i in range(2):
        assert all(torch.equal(a, b) for a, b in zip(got[i], alone))
    assert all(np.array_equal(a, b) for a, b in zip(got["train"], trained))


def test_two_graphs_share_a_workspace_in_order(agn):
    """Loss and gradients captured apart with one workspace, replayed one after the other."""
    size = (700, 64, 3000)
    x, w, b, labels = L.make(*size, 1, ignored=0.1)
    rows, inner, classes = size
    n = max(agn.agn_linear_ce_bytes(*size, 1, k) for k in (0, 1))
    scratch = torch.zeros(n, dtype=torch.uint8, device="cuda")
    loss, lse, db = (torch.zeros(k, device="cuda") for k in (rows, rows, classes))
    dx, dw = torch.zeros_like(x), torch.zeros_like(w)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    torch.cuda.synchronize()
    with torch.cuda.graph(graphs[0]):
        agn.agn_linear_ce(x, w, labels, 1, *size, loss, lse, scratch, n, bias=b,
                          stream=torch.cuda.current_stream().cuda_stream)
    with torch.cuda.graph(graphs[1]):
        agn.agn_linear_ce_backward(x, w, labels, lse, 1, *size, scratch, n, dx=dx, dw=dw, dbias=db, bias=b,
                                   stream=torch.cuda.current_stream().cuda_stream)
    for _ in range(3):
        graphs[0].replay()
        graphs[1].replay()
    torch.cuda.synchronize()
    want = L.forward(agn, x, w, b, labels, 1)
    grads = L.backward(agn, x, w, b, labels, want[1], 1)
    assert torch.equal(loss, want[0]) and all(torch.equal(t, grads[k]) for t, k in ((dx, "dx"), (dw, "dw"), (db, "dbias")))
