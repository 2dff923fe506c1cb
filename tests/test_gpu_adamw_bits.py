"""AdamW's parameters bit for bit: every operation of the formula rounded to fp32, as NumPy rounds them."""

import math

import numpy as np
import pytest

import train_ops_ref as T
from test_gpu_adamw import B1, B2, LR, Model, agn   # noqa: F401 (agn: fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [1e-8, 0.0, 2.0 ** -126, 1e30])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gdt", [0, 1])
@pytest.mark.parametrize("step", [1, 7, 100_000])
def test_parameters(agn, bits, gdt, eps, step):
    f = np.float32
    m = Model(agn, [5000, 33, 2048], bits, gdt, False, seed=6)
    m.plan.adamw(LR, step, B1, B2, eps, seed=step)
    rc2, size = f(1 / math.sqrt(1 - B2 ** step)), f(LR / (1 - B1 ** step))
    b1, o1, b2, o2 = f(B1), f(1 - B1), f(B2), f(1 - B2)
    for h, d in zip(m.host, m.dev):
        if bits == 8:
            m0, r0 = f(T.m_values(h["m"], h["m_scale"])), f(T.r_values(h["v"], h["v_scale"]))
            v0 = r0 * r0
        else:
            m0, v0 = h["m"], h["v"]
        g = h["grad"]
        m1 = m0 * b1 + g * o1
        r1 = np.sqrt(v0 * b2 + g * g * o2)
        with np.errstate(all="ignore"):   # (eps 0 where v is 0)
            want = h["param"] * f(1 - LR * h["decay"]) - m1 / (r1 * rc2 + f(eps)) * size
        assert want.dtype == f
        got = d["param"].cpu().numpy()
        assert np.array_equal(got, want, equal_nan=True)
