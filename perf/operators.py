"""The hidden layer's operators as a user of the library calls them, as cases that can be timed and compared.

  dropout   `agn_dropout`: bias, ReLU, dropout (and a residual) in one pass.
  backward  `agn_dropout_backward`: its gradient, and the bias's.
  quantize  `agn_mx4_quantize`, and the values that the codes stand for (`agn_mx4_dequantize`).
  linear    `agn_mx4_linear` on rows that are in 4 bits already (an earlier layer's output).
  layer     `agn_mx4_quantize` of the rows, then `agn_mx4_linear`.

The plain form computes the same in 32 bits with elementary torch operations on the
same buffers: the 4-bit weights are decoded from their codes and scales.  `exact`
restates the definitions in 64 bits, apart from the plain form.
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "bf16": 2}
MOST_FLOPS = 2.0 * 16384 * 4096 * 4096
MOST_ELEMENTS = 16384 * 4096


def listed():
    return [
        # The hidden layer of the smallest workload (784-128-10, 32 samples):
        # launches and latency count.
        dict(name="dropout small fp32", kind="dropout", rows=32, cols=128, dtype="fp32", p=0.5,
             relu=True, bias=True, residual=False),
        # A wave of 16 workers with 128 samples each, layers of 1000 (odd in
        # tiles of a power of two).
        dict(name="dropout wave fp32", kind="dropout", rows=2048, cols=1000, dtype="fp32", p=0.5,
             relu=True, bias=True, residual=False),
        # A block's output before its residual, 256 samples of 64 workers.
        dict(name="dropout residual bf16", kind="dropout", rows=16384, cols=4096, dtype="bf16",
             p=0.1, relu=False, bias=True, residual=True),
        # The backward of the same wave, with the bias's gradient.
        dict(name="backward wave fp32", kind="backward", rows=2048, cols=1000, dtype="fp32", p=0.5,
             relu=True, bias=True),
        dict(name="backward large bf16", kind="backward", rows=16384, cols=4096, dtype="bf16",
             p=0.1, relu=True, bias=True),
        # Held-out rows of 784 inputs (the last block of a row is half full).
        dict(name="quantize rows fp32", kind="quantize", rows=10000, cols=784, dtype="fp32"),
        # A layer's weights.
        dict(name="quantize weights bf16", kind="quantize", rows=4096, cols=4096, dtype="bf16"),
        # One row through one layer: bound by the weights and by latency.
        dict(name="linear one row bf16", kind="linear", rows=1, inner=4096, out=4096, dtype="bf16",
             relu=False, bias=False),
        # A ragged few rows through the first layer of a 784-1000-1000-10 net.
        dict(name="linear few rows fp32", kind="linear", rows=37, inner=784, out=1000,
             dtype="fp32", relu=True, bias=True),
        # The held-out set through its second layer.
        dict(name="linear held-out fp32", kind="linear", rows=10000, inner=1000, out=1000,
             dtype="fp32", relu=True, bias=True),
        # The largest: a long batch through a 4096-4096 layer.
        dict(name="linear large bf16", kind="linear", rows=16384, inner=4096, out=4096,
             dtype="bf16", relu=True, bias=True),
        # Rows that arrive in bf16: quantised, then the product.
        dict(name="layer bf16", kind="layer", rows=256, inner=2048, out=2048, dtype="bf16",
             relu=True, bias=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["dropout", "dropout", "backward", "quantize", "linear", "linear", "layer"])
    dtype = rng.choice(["fp32", "bf16"])
    if kind in ("linear", "layer"):
        rows, inner, out = _log(rng, 1, 16384), _log(rng, 32, 8192), _log(rng, 16, 8192)
        while 2.0 * rows * inner * out > MOST_FLOPS:
            rows = max(1, rows // 2)
        return dict(kind=kind, rows=rows, inner=inner, out=out, dtype=dtype,
                    relu=rng.random() < 0.5, bias=rng.random() < 0.7)
    rows, cols = _log(rng, 1, 65536), _log(rng, 8, 8192)
    if rng.random() < 0.5:
        cols = (cols + 7) // 8 * 8
    while rows * cols > MOST_ELEMENTS:
        rows = max(1, rows // 2)
    if kind == "quantize":
        return dict(kind=kind, rows=rows, cols=cols, dtype=dtype)
    case = dict(kind=kind, rows=rows, cols=cols, dtype=dtype, p=rng.choice([0.1, 0.2, 0.5, 0.75]),
                relu=rng.random() < 0.6, bias=rng.random() < 0.6)
    if kind == "dropout":
        case["residual"] = rng.random() < 0.4
    return case


# -------------------------------------------------------------------- inputs

def _blocks(cols):
    return (cols + 31) // 32


def _scale_index(rows, cols):
    """Where the scale of (row, block) is: tiles of 128 rows x 4 blocks, 512 bytes each."""
    r = torch.arange(rows, device=DEV).view(-1, 1)
    k = torch.arange(_blocks(cols), device=DEV).view(1, -1)
    tiles = (_blocks(cols) + 3) // 4
    return ((r // 128) * tiles + k // 4) * 512 + (r % 32) * 16 + (r // 32 % 4) * 4 + k % 4


def _scale_bytes(rows, cols):
    return (rows + 127) // 128 * ((_blocks(cols) + 3) // 4) * 512


def _encode(x):
    """(codes, scales) of the rows of x: what a program keeps of its weights."""
    rows, cols = x.shape
    nb = _blocks(cols)
    v = torch.zeros(rows, nb * 32, device=DEV)
    v[:, :cols] = x.float()
    v = v.view(rows, nb, 32)
    amax = v.abs().amax(2)
    e = (torch.frexp(amax)[1] - 3).clamp(min=-127)
    e = torch.where(amax > 0, e, torch.full_like(e, -127))
    a = torch.ldexp(v, -e.unsqueeze(2)).abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = (torch.round(a / step) * step).clamp(max=6.0)
    grid = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=DEV)
    code = torch.bucketize(q, grid) + 8 * torch.signbit(v)
    code = code.to(torch.uint8).view(rows, nb * 16, 2)
    scales = torch.zeros(_scale_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    scales[_scale_index(rows, cols).view(-1)] = (e + 127).to(torch.uint8).view(-1)
    return (code[:, :, 0] | (code[:, :, 1] << 4)).contiguous(), scales


def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _activations(g, rows, cols):
    """What a hidden layer gives the next one: about half zeros, sizes that differ by feature."""
    h = torch.relu(_randn(g, rows, cols))
    return h * torch.exp(0.5 * _randn(g, 1, cols))


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    kind = case["kind"]
    s = dict(case=case, dt=dt)
    if kind in ("dropout", "backward"):
        rows, cols = case["rows"], case["cols"]
        s["x"] = _randn(g, rows, cols).to(dt)
        s["bias"] = 0.3 * _randn(g, cols) if case["bias"] else None
        s["seed"] = (seed * 0x9E3779B1 + 12345) % (1 << 63)
        s["offset"] = (seed % 1000) << 33   # draws of earlier steps lie before
        s["y"] = torch.empty(rows, cols, dtype=dt, device=DEV)
        if kind == "dropout":
            s["residual"] = _randn(g, rows, cols).to(dt) if case["residual"] else None
        else:
            s["dy"] = (0.01 * _randn(g, rows, cols)).to(dt)
            s["dbias"] = torch.empty(cols, device=DEV)
        return s
    rows = case["rows"]
    if kind == "quantize":
        cols = case["cols"]
        s["x"] = (_randn(g, rows, cols) * torch.exp(_randn(g, rows, 1))).to(dt)
        s["y"] = torch.empty(rows, cols, dtype=dt, device=DEV)
    else:
        cols, out = case["inner"], case["out"]
        limit = math.sqrt(6.0 / (cols + out))
        w = (2 * torch.rand(out, cols, generator=g, device=DEV) - 1) * limit
        s["w_codes"], s["w_scales"] = _encode(w)
        s["bias"] = 0.1 * _randn(g, out) if case["bias"] else None
        x = _activations(g, rows, cols)
        if kind == "linear":
            s["codes"], s["scales"] = _encode(x)
        else:
            s["x"] = x.to(dt)
        s["y"] = torch.empty(rows, out, dtype=dt, device=DEV)
    if kind != "linear":
        s["codes"] = torch.empty(rows, _blocks(cols) * 16, dtype=torch.uint8, device=DEV)
        s["scales"] = torch.empty(_scale_bytes(rows, cols), dtype=torch.uint8, device=DEV)
    return s


# ----------------------------------------------------------------- plain form

G = 0x9E3779B97F4A7C15
C1 = 0xBF58476D1CE4E5B9
C2 = 0x94D049BB133111EB
DROPOUT_STREAM = 8


def _signed(v):
    v %= 1 << 64
    return v - (1 << 64) if v >= 1 << 63 else v


def _mix_int(z):
    z = (z ^ (z >> 30)) * C1 % (1 << 64)
    z = (z ^ (z >> 27)) * C2 % (1 << 64)
    return z ^ (z >> 31)


def _shr(z, n):
    return (z >> n) & ((1 << (64 - n)) - 1)


def _keep(rows, cols, p, seed, offset):
    """Keep mask and scale: 16 bits of splitmix64 an element, against round(65536 p)."""
    t = min(65535, int(round(65536 * p)))
    groups = (cols + 3) // 4
    key = _mix_int((seed ^ (DROPOUT_STREAM * G)) % (1 << 64))
    i = torch.arange(rows * groups, device=DEV)
    z = (i + _signed(offset + 1)) * _signed(G) + _signed(key)
    z = (z ^ _shr(z, 30)) * _signed(C1)
    z = (z ^ _shr(z, 27)) * _signed(C2)
    z = z ^ _shr(z, 31)
    u = torch.stack([z & 0xFFFF, _shr(z, 16) & 0xFFFF, _shr(z, 32) & 0xFFFF, _shr(z, 48)], 1)
    return u.view(rows, groups * 4)[:, :cols] >= t, 65536.0 / (65536 - t)


def _scales_of(scales, rows, cols):
    e = scales[_scale_index(rows, cols).view(-1)].view(rows, -1).int() - 127
    return torch.ldexp(torch.ones_like(e, dtype=torch.float32), e)


E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _decode(codes, scales, rows, cols):
    table = torch.tensor(E2M1 + [-v for v in E2M1], device=DEV)
    q = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], 2).view(rows, -1, 32)
    return (q * _scales_of(scales, rows, cols).unsqueeze(2)).view(rows, -1)[:, :cols]


def _round_mx4(x):
    """The rows of x at the nearest values that 4-bit codes and a scale of each 32 stand for."""
    rows, cols = x.shape
    nb = _blocks(cols)
    v = torch.zeros(rows, nb * 32, device=DEV)
    v[:, :cols] = x.float()
    v = v.view(rows, nb, 32)
    amax = v.abs().amax(2, keepdim=True)
    e = torch.where(amax > 0, torch.frexp(amax)[1] - 3, -127).clamp(min=-127)
    u = torch.ldexp(v, -e)
    a = u.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    q = (torch.round(a / step) * step).clamp(max=6.0) * torch.sign(u)
    return torch.ldexp(q, e).view(rows, -1)[:, :cols]


def _run_plain(s):
    c, kind = s["case"], s["case"]["kind"]
    rows = c["rows"]
    if kind in ("dropout", "backward"):
        keep, scale = _keep(rows, c["cols"], c["p"], s["seed"], s["offset"])
        v = s["x"].float()
        if s["bias"] is not None:
            v = v + s["bias"]
        if kind == "dropout":
            if c["relu"]:
                v = torch.where(v <= 0, 0.0, v)
            v = torch.where(keep, v * scale, 0.0)
            if s["residual"] is not None:
                v = v + s["residual"].float()
            return v.to(s["dt"])
        if c["relu"]:
            keep = keep & ~(v <= 0)
        dx = torch.where(keep, s["dy"].float() * scale, 0.0)
        return dx.to(s["dt"]), dx.sum(0)
    if kind == "quantize":
        return _round_mx4(s["x"]).to(s["dt"])
    x = _decode(s["codes"], s["scales"], rows, c["inner"]) if kind == "linear" else _round_mx4(s["x"])
    y = x @ _decode(s["w_codes"], s["w_scales"], c["out"], c["inner"]).t()
    if s["bias"] is not None:
        y = y + s["bias"]
    if c["relu"]:
        y = torch.where(y <= 0, 0.0, y)
    return y.to(s["dt"])


# ------------------------------------------------------------ the library's calls

def _run_own(s):
    import paper_1710_02368_gb300 as agn

    c, kind, y = s["case"], s["case"]["kind"], s["y"]
    rows = c["rows"]
    prec = agn.AGN_PREC_FP32 if c["dtype"] == "fp32" else agn.AGN_PREC_BF16
    stream = torch.cuda.current_stream().cuda_stream
    if kind == "dropout":
        agn.agn_dropout(s["x"], y, prec, rows, c["cols"], c["p"], s["seed"], s["offset"],
                        bias=s["bias"], residual=s["residual"], relu=c["relu"], stream=stream)
        return y
    if kind == "backward":
        agn.agn_dropout_backward(s["dy"], y, prec, rows, c["cols"], c["p"], s["seed"], s["offset"],
                                 x=s["x"] if c["relu"] else None,
                                 bias=s["bias"] if c["relu"] else None, dbias=s["dbias"],
                                 relu=c["relu"], stream=stream)
        return y, s["dbias"]
    if kind in ("quantize", "layer"):
        cols = c["cols"] if kind == "quantize" else c["inner"]
        agn.agn_mx4_quantize(s["x"], prec, rows, cols, s["codes"], s["scales"], stream=stream)
    if kind == "quantize":
        agn.agn_mx4_dequantize(s["codes"], s["scales"], rows, cols, y, prec, stream=stream)
        return y
    agn.agn_mx4_linear(s["codes"], s["scales"], s["w_codes"], s["w_scales"], rows, c["inner"],
                       c["out"], y, prec, bias=s["bias"], relu=c["relu"], stream=stream)
    return y


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ----------------------------------------------------------------------- work

def work(case):
    es, rows, kind = SIZE[case["dtype"]], case["rows"], case["kind"]
    mx = lambda r, c: r * _blocks(c) * 17.0  # noqa: E731
    if kind in ("dropout", "backward"):
        n = rows * case["cols"]
        arrays = 2 + (case["residual"] if kind == "dropout" else case["relu"])
        vectors = (case["bias"] and (kind == "dropout" or case["relu"])) + (kind == "backward")
        return {"bytes": float(arrays * es * n + 4 * vectors * case["cols"]), "flops": 3.0 * n}
    if kind == "quantize":
        n = rows * case["cols"]
        return {"bytes": 2.0 * es * n + 2 * mx(rows, case["cols"]), "flops": 3.0 * n}
    inner, out = case["inner"], case["out"]
    read = mx(rows, inner) if kind == "linear" else es * rows * inner + 2 * mx(rows, inner)
    return {"bytes": read + mx(out, inner) + es * rows * out + (4 * out if case["bias"] else 0),
            "flops": 2.0 * rows * inner * out}


# ---------------------------------------------------------------------- exact

def _exact_keep(rows, cols, p, seed, offset):
    """The mask from the generator's definition, in unsigned 64-bit numpy."""
    t = min(65535, int(round(65536 * p)))
    groups = -(-cols // 4)
    with np.errstate(over="ignore"):
        def mix(z):
            z = (z ^ (z >> np.uint64(30))) * np.uint64(C1)
            z = (z ^ (z >> np.uint64(27))) * np.uint64(C2)
            return z ^ (z >> np.uint64(31))
        key = mix(np.array([seed], np.uint64) ^ np.array([DROPOUT_STREAM], np.uint64) * np.uint64(G))
        i = np.arange(1, rows * groups + 1, dtype=np.uint64) + np.uint64(offset)
        bits = mix(key + i * np.uint64(G)).astype("<u8").view("<u2").reshape(rows, 4 * groups)
    return torch.from_numpy(bits[:, :cols] >= t).to(DEV), t


def _exact_values(codes, scales, rows, cols):
    sign_less = torch.tensor(E2M1, dtype=torch.float64, device=DEV)
    nibbles = torch.empty(rows, codes.shape[1] * 2, dtype=torch.long, device=DEV)
    nibbles[:, 0::2] = codes.long() % 16
    nibbles[:, 1::2] = codes.long() // 16
    mag = sign_less[nibbles % 8] * (1.0 - 2.0 * (nibbles // 8))
    e = scales.double()[_scale_index(rows, cols)] - 127.0
    return (mag * torch.exp2(e).repeat_interleave(32, 1))[:, :cols]


def _exact_round(x):
    """Nearest of the eight magnitudes by distance, ties to the even code, 64 bits."""
    rows, cols = x.shape
    mags = torch.tensor(E2M1, dtype=torch.float64, device=DEV)
    odd = torch.arange(8, device=DEV) % 2
    v = torch.nn.functional.pad(x.double(), (0, _blocks(cols) * 32 - cols)).view(rows, -1, 32)
    amax = v.abs().amax(2, keepdim=True)
    _, ex = torch.frexp(amax.clamp(min=2.0 ** -149))   # amax = m 2^ex, m in [1/2, 1)
    unit = torch.exp2((ex - 3).clamp(min=-127).double())
    far = ((v.abs() / unit).unsqueeze(3) - mags).abs()
    nearest = far == far.amin(3, keepdim=True)         # two where it is a tie, one of them odd
    code = torch.argmax(nearest * (2 - odd), dim=3)
    return torch.copysign(mags[code] * unit, v).view(rows, -1)[:, :cols]


def exact(case, seed):
    s = prepare(case, seed)
    kind, rows = case["kind"], case["rows"]
    if kind in ("dropout", "backward"):
        keep, t = _exact_keep(rows, case["cols"], case["p"], s["seed"], s["offset"])
        gain = 65536.0 / (65536.0 - t)
        pre = s["x"].double()
        if s["bias"] is not None:
            # the sum as the layer's 32 bits have it: whether it passes zero is decided there
            pre = (s["x"].float() + s["bias"]).double()
        if kind == "dropout":
            if case["relu"]:
                pre = pre.clamp(min=0.0)
            y = pre * keep.double() * gain
            return y if s["residual"] is None else y + s["residual"].double()
        live = keep & (pre > 0) if case["relu"] else keep
        dx = s["dy"].double() * live.double() * gain
        return dx, dx.sum(0)
    if kind == "quantize":
        return _exact_round(s["x"])
    inner, out = case["inner"], case["out"]
    x = _exact_values(s["codes"], s["scales"], rows, inner) if kind == "linear" else _exact_round(s["x"])
    y = torch.matmul(x, _exact_values(s["w_codes"], s["w_scales"], out, inner).transpose(0, 1))
    if s["bias"] is not None:
        y += s["bias"].double()
    return y.clamp(min=0.0) if case["relu"] else y
