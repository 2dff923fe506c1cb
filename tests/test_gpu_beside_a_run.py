"""The operators' calls on one thread and stream while a handle trains and evaluates on another: the
product's CTAs and the training's share the GPU's SMs and tensor memory.  Both give what they give
alone, bit for bit."""

import threading

import numpy as np
import pytest

import agn_inputs as I

pytestmark = pytest.mark.gpu


def test_products_and_dropout_beside_training_and_evaluation():
    import torch

    import paper_1710_02368_gb300 as agn
    dims, n, m, seed, C = (784, 1000, 1000, 10), 4, 128, 5, 24
    w, tau = I.make_schedule(n, C + n, 0, 2, seed)

    def train():
        out = []
        with agn.AGN(dims, n, 4, 0.05, seed, batch=m, n_samples=n * 2 * m, n_eval=3000, eval_mx4=1, dropout=0.2) as h:
            for c in range(0, C, 8):
                h.run(8, w[c:], tau[c:])
                out += [h.loss(), *h.evaluate(with_pred=True), *h.evaluate_mx4(with_pred=True)]
            out.append(h.central())
        return out

    g = torch.Generator(device="cuda").manual_seed(1)
    shapes = [(3, 784, 1000), (100, 1000, 520), (700, 1000, 1000), (5000, 300, 600)]
    ops = []
    for rows, inner, out in shapes:
        x = torch.randn(rows, inner, generator=g, device="cuda")
        b = [torch.zeros(k, dtype=torch.uint8, device="cuda") for r in (rows, out) for k in agn.agn_mx4_bytes(r, inner)]
        agn.agn_mx4_quantize(torch.randn(out, inner, generator=g, device="cuda"), 0, out, inner, b[2], b[3])
        ops.append((x, *b, torch.empty(rows, out, device="cuda"), torch.empty(rows, out, device="cuda"), torch.empty(out, device="cuda")))
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()

    def layers(stream):
        for (rows, inner, out), (x, q, qs, wq, ws, y, d, db) in zip(shapes, ops):
            agn.agn_mx4_quantize(x, 0, rows, inner, q, qs, stream=stream)
            agn.agn_mx4_linear(q, qs, wq, ws, rows, inner, out, y, 0, err=err, stream=stream)
            agn.agn_dropout(y, d, 0, rows, out, 0.5, 1, relu=1, stream=stream)
            agn.agn_dropout_backward(d, d, 0, rows, out, 0.5, 1, x=y, dbias=db, relu=1, stream=stream)

    layers(None)
    torch.cuda.synchronize()
    want = [[t.clone() for t in o[5:]] for o in ops]
    alone = train()
    stop, failed, rounds = threading.Event(), [], [0]

    def beside():
        try:
            s = torch.cuda.Stream()
            while not stop.is_set():
                for _ in range(20):
                    layers(s.cuda_stream)
                s.synchronize()
                rounds[0] += 1
        except Exception as e:  # noqa: BLE001
            failed.append(e)
    t = threading.Thread(target=beside)
    t.start()
    try:
        both = [train() for _ in range(3)]
    finally:
        stop.set()
        t.join()
    torch.cuda.synchronize()
    assert not failed and rounds[0] > 0 and int(err) == 0
    for got in both:
        assert all(np.array_equal(a, b) for a, b in zip(got, alone))
    for o, v in zip(ops, want):
        assert all(torch.equal(a, b) for a, b in zip(o[5:], v))
