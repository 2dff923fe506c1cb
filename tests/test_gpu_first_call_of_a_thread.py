"""The operators' calls as a host thread's first use of CUDA: the product encodes tensor maps with
the driver, which wants a context that a new thread does not have yet."""

import threading

import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [3, 600, 1200])
def test_operators(rows):
    import torch

    import paper_1710_02368_gb300 as agn
    inner, out = 200, 300
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(rows, inner, generator=g, device="cuda")
    w = torch.randn(out, inner, generator=g, device="cuda")

    def buffers():
        m = [torch.zeros(n, dtype=torch.uint8, device="cuda") for r in (rows, out) for n in agn.agn_mx4_bytes(r, inner)]
        return (*m, torch.zeros(rows, out, device="cuda"), torch.zeros(rows, out, device="cuda"), torch.zeros(out, device="cuda"))
    calls = [
        lambda b: agn.agn_mx4_quantize(x, 0, rows, inner, b[0], b[1]),
        lambda b: agn.agn_mx4_quantize(w, 0, out, inner, b[2], b[3]),
        lambda b: agn.agn_mx4_linear(*b[:4], rows, inner, out, b[4], 0),
        lambda b: agn.agn_dropout(b[4], b[5], 0, rows, out, 0.5, 1, relu=1),
        lambda b: agn.agn_dropout_backward(b[5], b[5], 0, rows, out, 0.5, 1, dbias=b[6]),
    ]
    here, there, failed = buffers(), buffers(), []
    for c in calls:
        c(here)

    def work(c):
        try:
            c(there)
        except Exception as e:  # noqa: BLE001
            failed.append(e)
    for c in calls:   # a new thread each
        t = threading.Thread(target=work, args=(c,))
        t.start()
        t.join()
        torch.cuda.synchronize()
    assert not failed
    assert all(torch.equal(a, b) for a, b in zip(here, there)) and float(here[4].abs().sum()) > 0
