"""AdamW over many tensors, with 32- and 8-bit states, and the norm of the gradients, against the
64-bit forms of train_ops_ref: states bit for bit, parameters to the roundings of one step."""

import math

import numpy as np
import pytest
import torch

import train_ops_ref as T

pytestmark = pytest.mark.gpu
LR, B1, B2, EPS = 1e-2, 0.9, 0.999, 1e-8
DT = {0: torch.float32, 1: torch.bfloat16}


@pytest.fixture(scope="module")
def agn():
    import paper_1710_02368_gb300 as agn
    return agn


def buffer(values, dtype, shift):
    """A device copy that starts `shift` elements into its allocation, with a border behind it."""
    t = torch.full((len(values) + shift + 40,), 77, dtype=dtype, device="cuda")
    t[shift:shift + len(values)] = torch.as_tensor(values).to("cuda").to(dtype)
    return t, t[shift:shift + len(values)]


class Model:
    def __init__(self, agn, sizes, bits, gdt, copy, shift=0, seed=0, decays=(0.0, 0.01, 0.1)):
        rng = np.random.default_rng(seed)
        self.bits, self.sizes, self.host, self.dev, self.all = bits, sizes, [], [], []
        for i, n in enumerate(sizes):
            f = np.float32
            size = float(np.exp(2 * rng.standard_normal()))
            h = dict(param=rng.standard_normal(n).astype(f), grad=(size * rng.standard_normal(n)).astype(f),
                     decay=decays[i % len(decays)])
            if gdt == 1:
                h["grad"] = torch.as_tensor(h["grad"]).bfloat16().float().numpy()
            h["grad"][rng.random(n) < 0.05] = 0.0
            m, v = 0.3 * size * rng.standard_normal(n), size * size * np.exp(rng.standard_normal(n))
            v[rng.random(n) < 0.1] = 0.0
            if bits == 32:
                h["m"], h["v"] = m.astype(f), v.astype(f)
            else:
                c, h["m_scale"] = T.rounded(np.abs(T.f32(m)), np.full(n, 32768.0), 3)
                h["m"] = (c | (np.signbit(m).astype(np.uint8) << 7)).astype(np.uint8)
                h["v"], h["v_scale"] = T.rounded(T.f32(np.sqrt(v)), np.full(n, 32768.0), 4)
            d = dict(n=n, grad_dtype=gdt, weight_decay=h["decay"])
            kinds = dict(param=torch.float32, grad=DT[gdt], m=torch.float32, v=torch.float32)
            if bits == 8:
                kinds.update(m=torch.uint8, v=torch.uint8, m_scale=torch.uint8, v_scale=torch.uint8)
            for k, dt in kinds.items():
                whole, d[k] = buffer(h[k], dt, shift)
                self.all.append((whole, shift, len(h[k])))
            if copy:
                whole, d["copy"] = buffer(np.zeros(n), torch.bfloat16, shift)
                self.all.append((whole, shift, n))
            self.host.append(h)
            self.dev.append(d)
        self.plan = agn.AGNOptim(self.dev, state_bits=bits)

    def expect(self, step, factor=None, seed=0, offset=0):
        """One step of the host's copy."""
        for h, n in zip(self.host, self.sizes):
            g = h["grad"].astype(np.float64)
            if self.bits == 8:
                m, r = T.m_values(h["m"], h["m_scale"]), T.r_values(h["v"], h["v_scale"])
                v = T.f32(r * r)
            else:
                m, v = h["m"].astype(np.float64), h["v"].astype(np.float64)
            old = h["param"].astype(np.float64)
            new, m, v, r = T.adamw(old, g, m, v, LR, step, B1, B2, EPS, h["decay"], factor)
            h["want"], h["bound"] = new, 2.0 ** -24 * (4 * np.abs(old) + 16 * np.abs(new - old) + 2 * np.abs(new)) + 1e-38
            if self.bits == 8:
                bm, br = T.random_bits(seed, offset, n)
                c, h["m_scale"] = T.rounded(np.abs(m), bm, 3)
                h["m"] = (c | (np.signbit(m).astype(np.uint8) << 7)).astype(np.uint8)
                c, h["v_scale"] = T.rounded(r, br, 4)
                h["v"] = np.where(r > 0, np.maximum(c, 1), c).astype(np.uint8)
                offset += (n + 1) // 2
            else:
                h["m"], h["v"] = m.astype(np.float32), v.astype(np.float32)

    def compare(self):
        for h, d in zip(self.host, self.dev):
            got = d["param"].cpu().numpy()
            assert np.all(np.abs(got.astype(np.float64) - h["want"]) <= h["bound"])
            h["param"] = got
            for k in ("m", "v", "m_scale", "v_scale"):
                if k in h:
                    assert np.array_equal(d[k].cpu().numpy(), h[k]), k
            if "copy" in d:
                assert torch.equal(d["copy"], d["param"].bfloat16())
        for whole, shift, n in self.all:   # what lies around the tensors
            assert torch.all(whole[:shift] == 77) and torch.all(whole[shift + n:] == 77)


SIZES = [[1], [7, 31, 32, 33], [2047, 2048, 2049, 4097], [784 * 10, 10, 0, 3]]


@pytest.mark.parametrize("shift", [0, 1, 8])
@pytest.mark.parametrize("gdt,copy", [(0, False), (0, True), (1, True)])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("sizes", SIZES, ids=str)
def test_steps(agn, sizes, bits, gdt, copy, shift):
    """Three steps; tensors that start anywhere; what lies around them stays."""
    m = Model(agn, sizes, bits, gdt, copy, shift)
    for t in (1, 2, 1000):
        seed, offset = 5 + t, (1 << 64) - 3 if t == 2 else t << 33
        m.plan.adamw(LR, t, B1, B2, EPS, seed=seed, offset=offset)
        m.expect(t, seed=seed, offset=offset)
        m.compare()


@pytest.mark.parametrize("bits", [32, 8])
def test_many_tensors(agn, bits):
    rng = np.random.default_rng(3)
    m = Model(agn, [int(v) for v in np.exp(rng.uniform(0, 9, 60))], bits, 0, True, seed=4)
    m.plan.adamw(LR, 7, B1, B2, EPS, seed=1)
    m.expect(7, seed=1)
    m.compare()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("gdt", [0, 1])
def test_clipping(agn, bits, gdt):
    """The norm, its factor, and the step that reads it; a large limit leaves the gradients alone."""
    m = Model(agn, [5000, 33, 1], bits, gdt, True)
    norm, scale = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    want = math.sqrt(sum(float((h["grad"].astype(np.float64) ** 2).sum()) for h in m.host))
    for limit in (want / 3, want * 2, math.inf):
        m.plan.grad_norm(limit, norm, scale)
        # squares and sums of up to 64 of them in fp32, the total's root rounded
        assert abs(norm.item() - want) <= want * 65 * 2.0 ** -24
        n32 = np.float32(norm.item())
        assert scale.item() == (1.0 if n32 <= np.float32(limit) else np.float32(limit) / n32)
        m.plan.adamw(LR, 3, B1, B2, EPS, scale=scale, seed=2, offset=9)
        m.expect(3, float(scale.item()), seed=2, offset=9)
        m.compare()
    first = norm.item()
    m.plan.grad_norm(1.0, norm, None)
    m.plan.grad_norm(1.0, None, scale)
    assert norm.item() == first


@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_that_is_skipped(agn, bits, bad):
    """A gradient that is not finite: the factor is NaN and nothing changes."""
    m = Model(agn, [300, 40], bits, 0, True)
    m.dev[1]["grad"][7] = bad
    norm, scale = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    m.plan.grad_norm(1.0, norm, scale)
    assert not math.isfinite(norm.item()) and math.isnan(scale.item())
    before = [w.clone() for w, _, _ in m.all]
    m.plan.adamw(LR, 3, B1, B2, EPS, scale=scale)
    scale.fill_(math.inf)
    m.plan.adamw(LR, 3, B1, B2, EPS, scale=scale)
    torch.cuda.synchronize()
    for (w, _, _), b in zip(m.all, before):
        assert torch.equal(w.view(torch.uint8), b.view(torch.uint8))


@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("n,shift", [(1, 0), (33, 0), (5000, 0), (4999, 3)])
def test_dequantize(agn, dtype, n, shift):
    """Every code, in blocks of every kind of scale (exact where the dtype's normal numbers reach)."""
    rng = np.random.default_rng(n)
    m, v = (rng.integers(0, 256, n).astype(np.uint8) for _ in range(2))
    nb = -(-n // 32)
    ms, vs = (rng.integers(40, 220, nb).astype(np.uint8) for _ in range(2))
    ms[0] = vs[-1] = 0
    dev = [buffer(t, torch.uint8, shift)[1] for t in (m, ms, v, vs)]
    whole = [torch.full((n + shift + 9,), 77, dtype=DT[dtype], device="cuda") for _ in range(2)]
    out = [t[shift:shift + n] for t in whole]
    agn.agn_adamw_dequantize(*dev, n, out[0], out[1], dtype)
    for got, want in zip(out, (T.m_values(m, ms), T.r_values(v, vs))):
        assert np.array_equal(got.float().cpu().numpy().astype(np.float64), want)
    assert all(torch.all(t[shift + n:] == 77) and torch.all(t[:shift] == 77) for t in whole)
    one = torch.zeros(n, dtype=DT[dtype], device="cuda")
    agn.agn_adamw_dequantize(None, None, dev[2], dev[3], n, None, one, dtype)
    assert torch.equal(one, out[1])
    agn.agn_adamw_dequantize(dev[0], dev[1], None, None, n, one, None, dtype)
    assert torch.equal(one, out[0])


def test_zeroed_states_are_zeros(agn):
    """A program's first step from zeroed buffers, in both forms."""
    n = 3000
    g = torch.randn(n, device="cuda")
    p = [torch.ones(n, device="cuda") for _ in range(2)]
    a = agn.AGNOptim([dict(param=p[0], grad=g, m=torch.zeros(n, device="cuda"), v=torch.zeros(n, device="cuda"), n=n)])
    z = lambda k: torch.zeros(k, dtype=torch.uint8, device="cuda")
    b = agn.AGNOptim([dict(param=p[1], grad=g, m=z(n), v=z(n), m_scale=z(94), v_scale=z(94), n=n)], state_bits=8)
    a.adamw(LR, 1)
    b.adamw(LR, 1, seed=1)
    assert torch.equal(p[0], p[1]) and not torch.equal(p[0], torch.ones(n, device="cuda"))
    assert b.draws == 1500


def test_rounding_is_right_on_average(agn):
    """v is changed by 1/1000 of it in a step, far below a code: over many elements it moves by that on average."""
    n = 1 << 20
    f = dict(device="cuda")
    g = torch.full((n,), 0.5, **f)
    z = lambda k: torch.zeros(k, dtype=torch.uint8, **f)
    t = dict(param=torch.zeros(n, **f), grad=g, m=z(n), v=z(n), m_scale=z(n // 32), v_scale=z(n // 32), n=n)
    plan = agn.AGNOptim([t], state_bits=8)
    t["v"].fill_(0xF8)        # 1.5 x the scale 2 ^ (126 - 127)
    t["v_scale"].fill_(126)
    r = torch.zeros(n, **f)
    want, draws = 0.75, 0
    for step in range(1, 9):
        plan.adamw(0.0, step, B1, B2, EPS, seed=3, offset=draws)
        draws += plan.draws
        agn.agn_adamw_dequantize(None, None, t["v"], t["v_scale"], n, None, r, 0)
        mean = r.double().mean().item()
        spread = r.double().std().item()
        # (E r' of a rounded r is r' up to the curvature of the root: spread^2 / (2 r) below 1e-3 of a code's 2^-5)
        want = math.sqrt(want * want * B2 + 0.25 * (1 - B2))
        assert abs(mean - want) < 5 * spread / math.sqrt(n) + step * spread * spread
        assert 0 < spread < 2.0 ** -5


def test_same_gradient_twice_and_empty_plans(agn):
    n = 100
    g = torch.randn(n, device="cuda")
    t = [dict(param=torch.zeros(n, device="cuda"), grad=g, m=torch.zeros(n, device="cuda"),
              v=torch.zeros(n, device="cuda"), n=n) for _ in range(2)]
    plan = agn.AGNOptim(t)
    norm = torch.zeros(1, device="cuda")
    plan.grad_norm(1.0, norm)
    assert abs(norm.item() - math.sqrt(2) * g.double().norm().item()) < 1e-5 * norm.item()
    plan.adamw(LR, 1)
    assert torch.equal(t[0]["param"], t[1]["param"])
    for tensors in ([], [dict(n=0)]):
        with agn.AGNOptim(tensors) as empty:
            empty.grad_norm(1.0, norm)
            assert norm.item() == 0
            empty.adamw(LR, 1)
    only = agn.AGNOptim([dict(grad=g, n=n)])
    only.grad_norm(1.0, norm)
    with pytest.raises(agn.AGNError) as e:
        only.adamw(LR, 1)
    assert e.value.code == agn.AGN_E_INVALID


@pytest.mark.parametrize("bits", [32, 8])
def test_in_a_graph_and_on_another_stream(agn, bits):
    """Norm and step captured, replayed on new gradients; the same on a side stream."""
    a, b = (Model(agn, [5000, 33, 2048], bits, 1, True, seed=1) for _ in range(2))
    scale = [torch.zeros(1, device="cuda") for _ in range(2)]

    def calls(m, s):
        st = torch.cuda.current_stream().cuda_stream
        m.plan.grad_norm(1.0, None, s, stream=st)
        m.plan.adamw(LR, 5, B1, B2, EPS, scale=s, seed=1, offset=2, stream=st)

    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        calls(a, scale[0])
    side = torch.cuda.Stream()
    for seed in (1, 2):
        for m in (a, b):
            for i, d in enumerate(m.dev):
                g = torch.Generator(device="cuda")
                g.manual_seed(seed + 10 * i)
                d["grad"].copy_(torch.randn(d["n"], generator=g, device="cuda"))
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            calls(b, scale[1])
        torch.cuda.synchronize()
        for (x, _, _), (y, _, _) in zip(a.all, b.all):
            assert torch.equal(x, y)
