"""AdamW on gradients that are not finite, or whose squares are not, without a factor that would skip the step: they
touch no other element, in 8-bit states not those of their block either."""

import math

import numpy as np
import pytest
import torch

import train_ops_ref as T
from test_gpu_adamw import B1, B2, EPS, LR, Model, agn   # noqa: F401 (agn: fixture)

pytestmark = pytest.mark.gpu


def bad_places(n):
    """One of a block, several of one, all of one, none of others."""
    at = np.zeros(n, bool)
    at[[i for i in (0, 40, 45, 63, 200, n - 1) if i < n]] = True
    at[96:128] = True
    return at


@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf, 1e30, -3e19])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gdt", [0, 1])
@pytest.mark.parametrize("shift", [0, 1])
def test_they_touch_no_other_element(agn, bits, gdt, value, shift):
    sizes = [5000, 130, 4096]
    m = Model(agn, sizes, bits, gdt, True, shift=shift, seed=2)
    bad = [bad_places(n) for n in sizes]
    bad[2][:] = False
    for d, b in zip(m.dev, bad):
        d["grad"][torch.as_tensor(b).cuda()] = value
    value = float(torch.tensor(value, dtype=m.dev[0]["grad"].dtype))
    for step in (5, 6):
        seed, offset = step, step << 20
        m.plan.adamw(LR, step, B1, B2, EPS, seed=seed, offset=offset)
        for h, d, b, n in zip(m.host, m.dev, bad, sizes):
            g = np.where(b, 0.0, h["grad"].astype(np.float64))
            old = h["param"].astype(np.float64)
            if bits == 8:
                ms, r = T.m_values(h["m"], h["m_scale"]), T.r_values(h["v"], h["v_scale"])
                v = T.f32(r * r)
            else:
                ms, v = h["m"].astype(np.float64), h["v"].astype(np.float64)
            with np.errstate(invalid="ignore"):   # (states that are not finite any more)
                new, ms, v, r = T.adamw(old, g, ms, v, LR, step, B1, B2, EPS, h["decay"])
            good = ~b
            got = d["param"].cpu().numpy()
            bound = 2.0 ** -24 * (4 * np.abs(old) + 16 * np.abs(new - old) + 2 * np.abs(new)) + 1e-38
            assert np.all(np.abs(got - new)[good] <= bound[good])
            if math.isfinite(value):   # m / infinity is 0
                assert np.all(np.abs(got - old * (1 - LR * h["decay"]))[b] <= 2.0 ** -22 * np.abs(old[b]))
            else:
                assert np.all(np.isnan(got[b]))
            h["param"] = got
            if bits == 32:
                h["m"], h["v"] = d["m"].cpu().numpy(), d["v"].cpu().numpy()
                assert np.array_equal(h["m"][good], ms[good].astype(np.float32))
                assert np.array_equal(h["v"][good], v[good].astype(np.float32))
                assert not np.any(np.isfinite(h["v"][b]))
                continue
            bm, br = T.random_bits(seed, offset, n)
            offset += (n + 1) // 2
            ms, r = np.where(b, 0.0, ms), np.where(b, 0.0, r)
            c, h["m_scale"] = T.rounded(np.abs(ms), bm, 3)
            h["m"] = (c | (np.signbit(ms).astype(np.uint8) << 7)).astype(np.uint8)
            c, h["v_scale"] = T.rounded(r, br, 4)
            h["v"] = np.where(b, 255, np.where(r > 0, np.maximum(c, 1), c)).astype(np.uint8)
            for k in ("m", "v", "m_scale", "v_scale"):
                assert np.array_equal(d[k].cpu().numpy(), h[k]), k
    for d, h, b in zip(m.dev, m.host, bad):   # gradients that are finite again
        d["grad"][torch.as_tensor(b).cuda()] = 0.5
        h["grad"] = np.where(b, np.float32(0.5), h["grad"])
    if bits == 8 and math.isfinite(value):
        m.plan.adamw(LR, 7, B1, B2, EPS, seed=1, offset=0)
        m.expect(7, seed=1, offset=0)
        m.compare()
