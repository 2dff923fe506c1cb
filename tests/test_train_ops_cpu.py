"""The output layer's loss and the optimizer's step without a GPU: refusals come before any device is
touched, sizes of the scratch, and the plain forms that the GPU tests compare with."""

import math

import numpy as np
import pytest
import torch

import ops_ref as R
import train_ops_ref as T


@pytest.fixture(scope="module")
def agn():
    import __graft_entry__ as g
    g.build()
    import paper_1710_02368_gb300 as agn
    return agn


A = [(i + 1) << 32 for i in range(14)]   # aligned, 4 GB apart, never read
MB = 1 << 20


def refused(agn, call, *words):
    with pytest.raises(agn.AGNError) as e:
        call()
    assert e.value.code == agn.AGN_E_INVALID
    for w in words:
        assert w in str(e.value)


def loss_args(**kw):
    a = dict(x=A[0], w=A[1], labels=A[2], dtype=1, rows=4, inner=8, classes=10, loss=A[3], lse=A[4], work=A[5],
             work_bytes=MB)
    a.update(kw)
    return a


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(dtype=-1), dict(rows=-1), dict(rows=(1 << 28) + 1), dict(inner=0), dict(inner=(1 << 20) + 1),
    dict(classes=0), dict(classes=(1 << 28) + 1), dict(x=None), dict(w=None), dict(labels=None), dict(loss=None),
    dict(lse=None), dict(work=None), dict(work_bytes=0), dict(x=A[0] + 2), dict(w=A[1] + 8), dict(labels=A[2] + 2),
    dict(loss=A[3] + 1), dict(work=A[5] + 128), dict(bias=A[6] + 2), dict(err=A[6] + 2), dict(loss=A[4]),
    dict(loss=A[0]), dict(lse=A[1] + 64), dict(work=A[0]), dict(work=A[3]), dict(err=A[2]), dict(loss=A[2] + 8),
    dict(bias=A[5]), dict(err=A[3]), dict(err=A[5] + 512),
], ids=str)
def test_loss_refuses(agn, bad):
    refused(agn, lambda: agn.agn_linear_ce(**loss_args(**bad)))


def grad_args(**kw):
    a = dict(x=A[0], w=A[1], labels=A[2], lse=A[3], dtype=0, rows=4, inner=8, classes=10, work=A[5], work_bytes=MB,
             dx=A[6], dw=A[7], dbias=A[8])
    a.update(kw)
    return a


@pytest.mark.parametrize("bad", [
    dict(dtype=3), dict(rows=-2), dict(inner=0), dict(classes=0), dict(x=None), dict(w=None), dict(labels=None),
    dict(lse=None), dict(work=None), dict(work_bytes=16), dict(dx=A[6] + 4), dict(dw=A[7] + 8), dict(dbias=A[8] + 2),
    dict(dloss=A[9] + 2), dict(dlse=A[9] + 1), dict(dx=A[0]), dict(dw=A[1]), dict(dx=A[7] + 16), dict(dbias=A[6] + 32),
    dict(dw=A[3]), dict(dbias=A[2]), dict(work=A[6]), dict(dloss=A[8]), dict(dlse=A[7]), dict(err=A[8] + 4),
    dict(bias=A[8] + 16), dict(work=A[1] - 256),
], ids=str)
def test_gradients_refuse(agn, bad):
    refused(agn, lambda: agn.agn_linear_ce_backward(**grad_args(**bad)))


def test_no_rows_touch_nothing(agn):
    agn.agn_linear_ce(None, None, None, 0, 0, 8, 10, None, None, None, 0)
    agn.agn_linear_ce_backward(None, None, None, None, 1, 0, 8, 10, None, 0)


@pytest.mark.parametrize("call", ["agn_linear_ce", "agn_linear_ce_backward"])
def test_host_memory_is_refused(agn, call):
    h = torch.zeros(1 << 16, dtype=torch.uint8)
    at = (h.data_ptr() + 4095) // 4096 * 4096
    a = loss_args(x=at) if call == "agn_linear_ce" else grad_args(x=at)
    with pytest.raises(agn.AGNError) as e:
        getattr(agn, call)(**a)
    assert e.value.code in (agn.AGN_E_INVALID, agn.AGN_E_CUDA)


@pytest.mark.parametrize("dtype", [0, 1])
def test_scratch(agn, dtype):
    """x packed (backward twice: along its rows too), dx's sums, and p's bounded buffer: no logits are kept."""
    for k in (0, 1):
        with pytest.raises(agn.AGNError):
            agn.agn_linear_ce_bytes(-1, 8, 8, dtype, k)
        with pytest.raises(agn.AGNError):
            agn.agn_linear_ce_bytes(8, 8, 8, 5, k)
    for rows, inner, classes in [(8192, 4096, 32768), (8192, 64, 1 << 20), (1 << 20, 64, 1000), (1, 1, 1)]:
        es, x, dx = (4, 6, 4) if dtype == 0 else (2, 2, 4)
        fwd, bwd = (agn.agn_linear_ce_bytes(rows, inner, classes, dtype, k) for k in (0, 1))
        pad = 1 << 20
        packed = x * (rows + 256) * (inner + 64) + (100 * MB if dtype == 0 else 0)
        logits = rows * classes
        assert fwd <= packed + logits / 8 + 16 * rows + pad
        assert bwd <= packed + x * (rows + 256) * (inner + 64) + dx * (rows + 256) * (inner + 64) + max(130 * MB, (rows + 256) * 1024 * es * 1.5) * 1.25 + 65 * MB + pad
    assert agn._lib.load().agn_linear_ce_bytes(1, 1, 1, 0, 0, None) == agn.AGN_E_INVALID


def tensor(i=0, **kw):
    t = dict(param=A[0] + i * MB, grad=A[1] + i * MB, m=A[2] + i * MB, v=A[3] + i * MB, m_scale=A[4] + i * MB,
             v_scale=A[5] + i * MB, copy=A[6] + i * MB, n=1000)
    t.update(kw)
    return t


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [
    dict(n=-1), dict(n=(1 << 40) + 1), dict(grad_dtype=2), dict(weight_decay=-0.1), dict(weight_decay=math.nan),
    dict(grad=None), dict(m=None), dict(v=None), dict(param=A[0] + MB + 2), dict(grad=A[1] + MB + 2),
    dict(copy=A[6] + MB + 1), dict(param=None), dict(param=A[0]), dict(m=A[2] + 500), dict(grad=A[3] + 400),
    dict(v=A[2] + MB), dict(copy=A[0] + 40), dict(grad=A[0] + MB),
], ids=str)
def test_plans_refuse(agn, bad, bits):
    refused(agn, lambda: agn.AGNOptim([tensor(0), tensor(1, **bad)], state_bits=bits), "tensor 1" if "grad" not in bad else "")


def test_plans_refuse_more(agn):
    refused(agn, lambda: agn.AGNOptim([tensor()], state_bits=16))
    refused(agn, lambda: agn.AGNOptim([tensor(m_scale=None)], state_bits=8))
    refused(agn, lambda: agn.AGNOptim([tensor(v_scale=A[4] + 31)], state_bits=8), "overlaps")
    refused(agn, lambda: agn.AGNOptim([tensor(m=A[2] + 2)], state_bits=32), "aligned")
    with pytest.raises(ValueError):
        agn.AGNOptim([tensor(decay=0.1)])
    with pytest.raises(TypeError):
        agn.AGNOptim([tensor(n=10.5)])
    lib = agn._lib.load()
    assert lib.agn_optim_create(None, 0, 32, None) == agn.AGN_E_INVALID
    assert lib.agn_optim_grad_norm(None, 1.0, A[0], None, None) == agn.AGN_E_INVALID
    assert lib.agn_optim_adamw(None, 0.1, 1, 0.9, 0.999, 1e-8, None, 0, 0, None) == agn.AGN_E_INVALID
    lib.agn_optim_destroy(None)


@pytest.mark.parametrize("bad", [dict(lr=math.nan), dict(lr=math.inf), dict(step=0), dict(beta1=1.0), dict(beta2=-0.1),
                                 dict(beta1=math.nan), dict(eps=-1e-8), dict(eps=math.inf), dict(eps=1e-40)], ids=str)
def test_steps_refuse(agn, bad):
    a = dict(plan=None, lr=1e-3, step=1, beta1=0.9, beta2=0.999, eps=1e-8)
    a.update(bad)
    refused(agn, lambda: agn.agn_optim_adamw(**a), "finite lr")


def test_norms_refuse(agn):
    refused(agn, lambda: agn.agn_optim_grad_norm(None, 0.0, A[0], A[1]), "max_norm")
    refused(agn, lambda: agn.agn_optim_grad_norm(None, math.nan, A[0], A[1]), "max_norm")
    refused(agn, lambda: agn.agn_optim_grad_norm(None, 1.0, None, None), "null")
    refused(agn, lambda: agn.agn_optim_grad_norm(None, 1.0, A[0], A[0]), "overlaps")


def test_dequantize_refuses(agn):
    d = agn.agn_adamw_dequantize
    refused(agn, lambda: d(A[0], A[1], A[2], A[3], -1, A[4], A[5], 0))
    refused(agn, lambda: d(A[0], A[1], A[2], A[3], 8, A[4], A[5], 2), "dtype")
    refused(agn, lambda: d(None, A[1], A[2], A[3], 8, A[4], A[5], 0), "null")
    refused(agn, lambda: d(A[0], A[1], A[2], None, 8, A[4], A[5], 0), "null")
    refused(agn, lambda: d(A[0], A[1], A[2], A[3], 8, A[4] + 2, A[5], 0), "aligned")
    refused(agn, lambda: d(A[0], A[1], A[2], A[3], 8, A[4], A[4] + 16, 0), "overlaps")
    refused(agn, lambda: d(A[0], A[1], A[2], A[3], 8, A[0], A[5], 1), "overlaps")
    d(None, None, None, None, 0, A[4], A[5], 0)
    d(None, None, None, None, 8, None, None, 0)


def test_waits_refuse(agn):
    for a in ((-1, 0), (2000000001, 0), (5, 2), (5, -2)):
        refused(agn, lambda: agn.agn_debug_linear_ce_waits(*a))
    agn.agn_debug_linear_ce_waits(0, -1)


@pytest.mark.parametrize("n", [np.int64(5), np.int64(-5), np.uint64(2 ** 64 - 5), np.uint8(5)], ids=repr)
def test_numpy_numbers(agn, n):
    """Seeds and offsets are reduced mod 2^64 like Python's; a fraction is none."""
    got = []

    class Lib:
        def agn_optim_adamw(self, *a):
            got.append(a[-3:-1])
            return 0
    real, agn._lib._LIB = agn._lib.load(), Lib()
    try:
        agn.agn_optim_adamw(None, 1e-3, 1, seed=n, offset=n)
    finally:
        agn._lib._LIB = real
    assert got == [(int(n) % 2 ** 64,) * 2]
    with pytest.raises(TypeError):
        agn.agn_optim_adamw(None, 1e-3, 1, seed=1.5)
    d = np.array([1, 784, 10])
    assert agn.agn_linear_ce_bytes(d[0], d[1], d[2], np.int32(0)) == agn.agn_linear_ce_bytes(1, 784, 10, 0)


# ------------------------------------------------ the plain forms themselves

def test_gradients_of_the_plain_form_are_differences():
    g = torch.Generator().manual_seed(0)
    x, w, b = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((5, 7), (11, 7), (11,)))
    labels = torch.tensor([3, -1, 10, 11, 0], dtype=torch.int32)
    dl, de = (torch.randn(5, generator=g, dtype=torch.float64) for _ in range(2))
    ref = T.linear_ce(x, w, b, labels, dl, de, 0.3)
    assert torch.all(ref["loss"][[1, 3]] == 0) and torch.all(ref["dx"][[1, 3]] == 0)

    def value(x, w, b):
        r = T.linear_ce(x, w, b, labels)
        return float(0.3 * (dl * r["loss"] + de * r["lse"]).sum())
    for name, key in (("x", "dx"), ("w", "dw"), ("b", "dbias")):
        t = dict(x=x, w=w, b=b)
        d = torch.randn(t[name].shape, generator=g, dtype=torch.float64)
        h = 1e-5
        hi, lo = (value(**dict(t, **{name: t[name] + s * h * d})) for s in (1, -1))
        assert abs((hi - lo) / (2 * h) - float((ref[key] * d).sum())) < 1e-8


def test_codes_by_hand():
    """Scale 1 (E = 127): the largest code's value is 2 - 2^-b; codes are a float's exponent and mantissa."""
    one = np.array([127], np.uint8)
    assert T.grid(3)[-1] == 1.875 and T.grid(4)[-1] == 1.9375
    assert list(T.values(np.array([0, 1, 7, 8, 127]), one, 3)) == [0, 2.0 ** -17, 7 * 2.0 ** -17, 2.0 ** -14, 1.875]
    assert list(T.m_values(np.array([127, 255, 128]), one)) == [1.875, -1.875, 0]
    x = np.zeros(32)
    x[:4] = [1.9375, 1.0, 1.03125, 2.0 ** -19]     # 1.03125: half way from 1 to 1.0625
    c, s = T.rounded(x, np.full(32, 32768.0), 4)
    assert s[0] == 127 and list(c[:4]) == [255, 240, 241, 1]
    c, s = T.rounded(x, np.full(32, 0.0), 4)
    assert list(c[:4]) == [255, 240, 240, 0]
    x[0] = 1.94
    assert T.rounded(x, np.zeros(32), 4)[1][0] == 128


def test_random_bits_are_the_generators():
    bm, br = T.random_bits(77, 5, 5)
    for i in range(5):
        d = int(R.draw(R.stream_key(77, 9), np.array([5 + i // 2]))[0]) >> (32 * (i % 2))
        assert (bm[i], br[i]) == (d & 0xFFFF, (d >> 16) & 0xFFFF)
