"""The output layer's loss over many classes and the optimizer's step, as a user of the library calls them.

  loss   `agn_linear_ce`: the output layer and its softmax cross-entropy, a loss for each row.
  train  `agn_linear_ce`, then `agn_linear_ce_backward`: the loss and the gradients of the rows,
         the weights and the bias.
  norm   `agn_grad_norm`: the norm of all gradients, and the factor that clips it.
  adamw  `agn_adamw`: one step on many tensors (8-bit states are read back with
         `agn_adamw_dequantize`).
  step   `agn_grad_norm`, then `agn_adamw` with its factor.

The plain form computes the same in 32 bits with elementary torch operations on
the same buffers.  `exact` restates the definitions in 64 bits, apart from the
plain form.
"""

import math

import numpy as np
import torch

own = False

DEV = "cuda"
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"fp32": 4, "bf16": 2}
MOST_LOGITS = 8192 * 32768
MOST_PRODUCTS = MOST_LOGITS * 4096
MOST_ELEMENTS = 100_000_000
LR, BETA1, BETA2, EPS, DECAY, STEP = 1e-3, 0.9, 0.999, 1e-8, 0.01, 1000
MAX_NORM = 1.0
BLOCK = 32


def listed():
    return [
        # The output layer of the smallest net (784-128-10) on a minibatch of 32:
        # launches and latency count.
        dict(name="loss small fp32", kind="loss", rows=32, inner=128, classes=10, dtype="fp32",
             bias=True, ignored=0.0, masked=0),
        # One row against many classes: bound by the weights.
        dict(name="loss one row bf16", kind="loss", rows=1, inner=4096, classes=32000,
             dtype="bf16", bias=False, ignored=0.0, masked=0),
        # Held-out rows, an odd number of classes, some rows without a label.
        dict(name="loss held-out bf16", kind="loss", rows=4000, inner=2048, classes=50257,
             dtype="bf16", bias=False, ignored=0.1, masked=0),
        # A wave of 16 workers with 128 samples each, 1000 inputs and classes, fp32.
        dict(name="train wave fp32", kind="train", rows=2048, inner=1000, classes=1000,
             dtype="fp32", bias=True, ignored=0.0, masked=0, z=False),
        # A ragged batch: odd rows, a prime number of classes, rows that only pad it, a few
        # classes masked by a bias of minus infinity, a gradient of lse beside the loss's.
        dict(name="train ragged bf16", kind="train", rows=777, inner=1000, classes=10007,
             dtype="bf16", bias=True, ignored=0.3, masked=5, z=True),
        # The largest: a long batch against a large vocabulary.
        dict(name="train large bf16", kind="train", rows=8192, inner=4096, classes=32768,
             dtype="bf16", bias=False, ignored=0.0, masked=0, z=False),
        # All gradients of the 784-1000-1000-10 net.
        dict(name="norm net fp32", kind="norm", net="784-1000-1000-10", dtype="fp32"),
        # One step of the smallest net (four tensors of very different sizes).
        dict(name="adamw small fp32", kind="adamw", net="784-128-10", dtype="fp32", bits=32,
             copy=False),
        # The wide net: bf16 gradients, fp32 parameters with their bf16 copy.
        dict(name="adamw wide bf16", kind="adamw", net="784-4096-4096-10", dtype="bf16", bits=32,
             copy=True),
        # States in 8 bits on tensors of odd sizes.
        dict(name="adamw 8-bit ragged fp32", kind="adamw", net="", tensors=37, total=3_000_017,
             seed=1, dtype="fp32", bits=8, copy=False),
        # A large model's tensors, states in 8 bits.
        dict(name="adamw 8-bit large bf16", kind="adamw", net="", tensors=300,
             total=100_000_000, seed=2, dtype="bf16", bits=8, copy=True),
        # The whole step of a training program: norm, clipping, update.
        dict(name="step many fp32", kind="step", net="", tensors=150, total=40_000_000, seed=3,
             dtype="fp32", bits=32, copy=True),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["loss", "loss", "train", "train", "train", "norm", "adamw", "adamw", "step"])
    dtype = rng.choice(["fp32", "bf16"])
    if kind in ("loss", "train"):
        rows, inner, classes = _log(rng, 1, 16384), _log(rng, 16, 8192), _log(rng, 2, 131072)
        if rng.random() < 0.5:
            inner = (inner + 7) // 8 * 8
        most = MOST_PRODUCTS // (8 if dtype == "fp32" else 1)
        while rows * inner * classes > most or rows * classes > MOST_LOGITS:
            rows, classes = max(1, rows // 2), max(2, classes * 3 // 4)
        case = dict(kind=kind, rows=rows, inner=inner, classes=classes, dtype=dtype,
                    bias=rng.random() < 0.6, ignored=rng.choice([0.0, 0.0, 0.2, 0.6]),
                    masked=rng.choice([0, 0, classes // 10]))
        case["masked"] = case["masked"] if case["bias"] else 0
        if kind == "train":
            case["z"] = rng.random() < 0.3
        return case
    case = dict(kind=kind, net="", tensors=_log(rng, 1, 400), total=_log(rng, 1000, MOST_ELEMENTS // 2),
                seed=rng.randrange(1 << 20), dtype=dtype)
    if kind != "norm":
        case["bits"] = rng.choice([8, 32])
        case["copy"] = rng.random() < 0.5
    return case


def _sizes(case):
    """(elements, weight decay) of each tensor: matrices decay, biases do not."""
    if case["net"]:
        d = [int(v) for v in case["net"].split("-")]
        return [s for a, b in zip(d, d[1:]) for s in ((a * b, DECAY), (b, 0.0))]
    rng = np.random.default_rng(case["seed"])
    share = np.exp(2.0 * rng.standard_normal(case["tensors"]))
    n = np.maximum(1, (case["total"] * share / share.sum()).astype(np.int64))
    return [(int(v), DECAY if v > 4096 else 0.0) for v in n]


def _places(case):
    """Where each tensor starts in the flat buffers (whole blocks, one after the other), and their length."""
    at, out = 0, []
    for n, _ in _sizes(case):
        out.append(at)
        at += (n + BLOCK - 1) // BLOCK * BLOCK
    return out, at


# -------------------------------------------------------------------- inputs

def _randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def _nearest_codes(x, mantissa):
    """(codes of |x|, block scales) to the nearest: the states that a program has after some steps."""
    shift = 23 - mantissa
    blocks = x.abs().view(-1, BLOCK)
    top = blocks.amax(1).view(torch.int32)
    e = ((top + (1 << shift) - 1) >> 23).clamp(min=1, max=253)
    u = blocks * ((254 - e) << 23).view(torch.float32).unsqueeze(1) * 2.0 ** -112
    code = ((u.view(torch.int32) + (1 << (shift - 1))) >> shift).clamp(max=(16 << mantissa) - 1)
    return code.to(torch.uint8).view(-1), e.to(torch.uint8)


def _prepare_loss(case, s, g):
    rows, inner, classes, dt = case["rows"], case["inner"], case["classes"], s["dt"]
    s["x"] = torch.relu(_randn(g, rows, inner)).to(dt)
    s["w"] = (_randn(g, classes, inner) * (2.0 / math.sqrt(0.5 * inner))).to(dt)
    s["bias"] = None
    if case["bias"]:
        s["bias"] = 0.3 * _randn(g, classes)
        if case["masked"]:
            s["bias"][classes - case["masked"]:] = -math.inf
    labels = torch.randint(0, classes - case["masked"], (rows,), generator=g, device=DEV)
    drop = torch.rand(rows, generator=g, device=DEV) < case["ignored"]
    s["labels"] = torch.where(drop, -1, labels).to(torch.int32)
    s["loss"] = torch.empty(rows, device=DEV)
    s["lse"] = torch.empty(rows, device=DEV)
    train = case["kind"] == "train"
    if train:
        s["scale"] = 1.0 / rows
        s["dlse"] = 1e-2 * _randn(g, rows) if case["z"] else None
        s["dx"] = torch.empty(rows, inner, dtype=dt, device=DEV)
        s["dw"] = torch.empty(classes, inner, dtype=dt, device=DEV)
        s["dbias"] = torch.empty(classes, device=DEV)
    if own:
        import paper_1710_02368_gb300 as agn

        s["bytes"] = max(agn.agn_linear_ce_bytes(rows, inner, classes, s["prec"], b)
                         for b in ([0, 1] if train else [0]))
        s["work"] = torch.empty(s["bytes"], dtype=torch.uint8, device=DEV)


def _prepare_step(case, s, g):
    sizes = _sizes(case)
    at, total = _places(case)
    s["sizes"], s["at"], s["total"] = sizes, at, total
    inside = torch.zeros(total, dtype=torch.bool, device=DEV)
    size = torch.empty(total, device=DEV)   # of a tensor's gradients
    spread = np.exp(np.random.default_rng(len(sizes)).standard_normal(len(sizes)))
    for (n, _), p, f in zip(sizes, at, spread):
        inside[p:p + n] = True
        size[p:p + n] = 1e-3 * float(f)
    s["grad"] = torch.where(inside, _randn(g, total) * size, 0.0).to(s["dt"])
    s["norm"] = torch.empty(1, device=DEV)
    s["factor"] = torch.empty(1, device=DEV)
    if case["kind"] == "norm":
        s["param"] = s["m"] = s["v"] = None
    else:
        s["param"] = torch.where(inside, 0.05 * _randn(g, total), 0.0)
        m = torch.where(inside, 0.3 * size * _randn(g, total), 0.0)
        v = torch.where(inside, size * size * torch.exp(_randn(g, total)), 0.0)
        if case["bits"] == 8:
            code, s["m_scale"] = _nearest_codes(m, 3)
            s["m"] = code | (torch.signbit(m).to(torch.uint8) << 7)
            s["v"], s["v_scale"] = _nearest_codes(torch.sqrt(v), 4)
            s["m_out"] = torch.empty(total, dtype=torch.bfloat16, device=DEV)
            s["r_out"] = torch.empty(total, dtype=torch.bfloat16, device=DEV)
        else:
            s["m"], s["v"] = m, v
        if case["copy"]:
            s["copy"] = torch.zeros(total, dtype=torch.bfloat16, device=DEV)
    if own:
        import paper_1710_02368_gb300 as agn

        def part(name, p, n):
            t = s.get(name)
            return None if t is None else t[p:p + n]

        s["plan"] = agn.AGNOptim(
            [dict(param=part("param", p, n), grad=part("grad", p, n), m=part("m", p, n),
                  v=part("v", p, n), m_scale=part("m_scale", p // BLOCK, (n + BLOCK - 1) // BLOCK),
                  v_scale=part("v_scale", p // BLOCK, (n + BLOCK - 1) // BLOCK),
                  copy=part("copy", p, n), n=n, grad_dtype=s["prec"], weight_decay=decay)
             for (n, decay), p in zip(sizes, at)], state_bits=case.get("bits", 32))


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s = dict(case=case, dt=DTYPES[case["dtype"]], prec=0 if case["dtype"] == "fp32" else 1)
    s["seed"] = (seed * 0x9E3779B1 + 12345) % (1 << 63)
    s["offset"] = (seed % 1000) << 33   # draws of earlier steps lie before
    if case["kind"] in ("loss", "train"):
        _prepare_loss(case, s, g)
    else:
        _prepare_step(case, s, g)
    return s


# ----------------------------------------------------------------- plain form

def _plain_loss(s):
    x, w, labels = s["x"].float(), s["w"].float(), s["labels"].long()
    live = (labels >= 0) & (labels < w.shape[0])
    z = x @ w.t()
    if s["bias"] is not None:
        z += s["bias"]
    top = z.amax(1, keepdim=True)
    lse = (torch.exp(z - top).sum(1, keepdim=True).log() + top).view(-1)
    at = torch.where(live, labels, 0).unsqueeze(1)
    loss = torch.where(live, lse - z.gather(1, at).view(-1), 0.0)
    if s["case"]["kind"] == "loss":
        return loss, torch.where(live, lse, 0.0)
    b = torch.where(live, s["scale"], 0.0)
    a = b if s["dlse"] is None else torch.where(live, s["scale"] + s["scale"] * s["dlse"], 0.0)
    z -= lse.unsqueeze(1)
    p = torch.exp(z) * a.unsqueeze(1)
    p.scatter_add_(1, at, -b.unsqueeze(1))
    dx, dw, dbias = p @ w, p.t() @ x, p.sum(0)
    return loss, torch.where(live, lse, 0.0), dx.to(s["dt"]), dw.to(s["dt"]), dbias


G = 0x9E3779B97F4A7C15
C1 = 0xBF58476D1CE4E5B9
C2 = 0x94D049BB133111EB
STATE_STREAM = 9


def _signed(v):
    v %= 1 << 64
    return v - (1 << 64) if v >= 1 << 63 else v


def _mix_int(z):
    z = (z ^ (z >> 30)) * C1 % (1 << 64)
    z = (z ^ (z >> 27)) * C2 % (1 << 64)
    return z ^ (z >> 31)


def _shr(z, n):
    return (z >> n) & ((1 << (64 - n)) - 1)


def _random_bits(s, first, n):
    """16 bits for m and 16 for sqrt(v) of n elements of a tensor whose draws start at `first`."""
    key = _mix_int((s["seed"] ^ (STATE_STREAM * G)) % (1 << 64))
    i = torch.arange((n + 1) // 2, device=DEV)
    z = (i + _signed(s["offset"] + first + 1)) * _signed(G) + _signed(key)
    z = (z ^ _shr(z, 30)) * _signed(C1)
    z = (z ^ _shr(z, 27)) * _signed(C2)
    z = z ^ _shr(z, 31)
    both = torch.stack([z & 0xFFFFFFFF, _shr(z, 32)], 1).view(-1)[:n]
    return (both & 0xFFFF).to(torch.int32), (both >> 16).to(torch.int32)


def _scale_values(e):
    return (e.to(torch.int32) << 23).view(torch.float32).repeat_interleave(BLOCK)


def _plain_decode(codes, scales, mantissa):
    """The magnitudes that codes of whole blocks stand for."""
    u = (codes.to(torch.int32) << (23 - mantissa)).view(torch.float32) * 2.0 ** 112
    return u * _scale_values(scales)


def _plain_decode_m(codes, scales):
    return _plain_decode(codes & 127, scales, 3) * torch.where(codes > 127, -1.0, 1.0)


def _plain_encode(x, bits, mantissa):
    """Codes of x >= 0, rounded up where the fraction and the 16 random bits pass one."""
    n = x.numel()
    shift = 23 - mantissa
    blocks = torch.zeros((n + BLOCK - 1) // BLOCK * BLOCK, device=DEV)
    blocks[:n] = x
    blocks = blocks.view(-1, BLOCK)
    e = ((blocks.amax(1).view(torch.int32) + ((1 << shift) - 1)) >> 23).clamp(min=1, max=253)
    u = blocks * ((254 - e) << 23).view(torch.float32).unsqueeze(1) * 2.0 ** -112
    add = (bits << (shift - 16)) + (1 << (shift - 17))
    code = (u.view(torch.int32).view(-1)[:n] + add) >> shift
    return code.clamp(max=(16 << mantissa) - 1), e.to(torch.uint8)


def _f32(v):
    return float(np.float32(v))


def _plain_norm(s):
    g = s["grad"].float()
    norm = (g * g).double().sum().sqrt().float().view(1)
    return norm, torch.where(norm > MAX_NORM, MAX_NORM / norm, 1.0)


def _plain_step(s, factor):
    case, first, out = s["case"], 0, []
    c1, c2 = 1.0 - BETA1 ** STEP, 1.0 - BETA2 ** STEP
    b1, ob1, b2, ob2 = _f32(BETA1), _f32(1.0 - BETA1), _f32(BETA2), _f32(1.0 - BETA2)
    for (n, decay), p in zip(s["sizes"], s["at"]):
        here = slice(p, p + n)
        whole = slice(p, p + (n + BLOCK - 1) // BLOCK * BLOCK)
        sc = slice(whole.start // BLOCK, whole.stop // BLOCK)
        g = s["grad"][here].float()
        if factor is not None:
            g = g * factor
        if case["bits"] == 8:
            m = _plain_decode_m(s["m"][whole], s["m_scale"][sc])[:n]
            r = _plain_decode(s["v"][whole], s["v_scale"][sc], 4)[:n]
            v = r * r
        else:
            m, v = s["m"][here], s["v"][here]
        m = m * b1 + g * ob1
        v = v * b2 + (g * g) * ob2
        r = v.sqrt()
        q = m / (r * _f32(1.0 / math.sqrt(c2)) + _f32(EPS))
        w = s["param"][here] * _f32(1.0 - LR * decay) - q * _f32(LR / c1)
        s["param"][here] = w
        if case["copy"]:
            s["copy"][here] = w.bfloat16()
        if case["bits"] == 8:
            bm, bv = _random_bits(s, first, n)
            code, s["m_scale"][sc] = _plain_encode(m.abs(), bm, 3)
            s["m"][here] = (code + 128 * torch.signbit(m)).to(torch.uint8)
            code, s["v_scale"][sc] = _plain_encode(r, bv, 4)
            s["v"][here] = torch.where(r > 0, code.clamp(min=1), code).to(torch.uint8)
        else:
            s["m"][here], s["v"][here] = m, v
        first += (n + 1) // 2
    out = [s["param"]] + ([s["copy"]] if case["copy"] else [])
    if case["bits"] == 8:
        m = _plain_decode_m(s["m"], s["m_scale"])
        return out + [m.bfloat16(), _plain_decode(s["v"], s["v_scale"], 4).bfloat16()]
    return out + [s["m"], s["v"]]


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind in ("loss", "train"):
        return _plain_loss(s)
    if kind == "norm":
        return _plain_norm(s)
    if kind == "adamw":
        return _plain_step(s, None)
    norm, factor = _plain_norm(s)
    return [norm, factor] + _plain_step(s, factor)


# ------------------------------------------------------------ the library's calls

def _run_own(s):
    import paper_1710_02368_gb300 as agn

    c, kind, prec = s["case"], s["case"]["kind"], s["prec"]
    stream = torch.cuda.current_stream().cuda_stream
    if kind in ("loss", "train"):
        agn.agn_linear_ce(s["x"], s["w"], s["labels"], prec, c["rows"], c["inner"], c["classes"],
                          s["loss"], s["lse"], s["work"], s["bytes"], bias=s["bias"],
                          stream=stream)
        if kind == "loss":
            return s["loss"], s["lse"]
        agn.agn_linear_ce_backward(s["x"], s["w"], s["labels"], s["lse"], prec, c["rows"],
                                   c["inner"], c["classes"], s["work"], s["bytes"], dx=s["dx"],
                                   dw=s["dw"], dbias=s["dbias"], bias=s["bias"], dlse=s["dlse"],
                                   scale=s["scale"], stream=stream)
        return s["loss"], s["lse"], s["dx"], s["dw"], s["dbias"]
    plan, out = s["plan"], []
    if kind in ("norm", "step"):
        plan.grad_norm(MAX_NORM, s["norm"], s["factor"], stream=stream)
        out = [s["norm"], s["factor"]]
        if kind == "norm":
            return out
    plan.adamw(LR, STEP, beta1=BETA1, beta2=BETA2, eps=EPS,
               scale=s["factor"] if kind == "step" else None, seed=s["seed"], offset=s["offset"],
               stream=stream)
    out.append(s["param"])
    if c["copy"]:
        out.append(s["copy"])
    if c["bits"] == 32:
        return out + [s["m"], s["v"]]
    agn.agn_adamw_dequantize(s["m"], s["m_scale"], s["v"], s["v_scale"], s["total"], s["m_out"],
                             s["r_out"], agn.AGN_PREC_BF16, stream=stream)
    return out + [s["m_out"], s["r_out"]]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ----------------------------------------------------------------------- work

def work(case):
    es, kind = SIZE[case["dtype"]], case["kind"]
    if kind in ("loss", "train"):
        rows, inner, classes = case["rows"], case["inner"], case["classes"]
        live = rows * (1.0 - case["ignored"])
        matrices = es * (rows * inner + classes * inner)
        small = 12.0 * rows + (4.0 * classes if case["bias"] else 0.0)
        if kind == "loss":
            return {"bytes": matrices + small, "flops": 2.0 * live * inner * classes}
        # the logits, and the two products of their gradient
        return {"bytes": 2.0 * matrices + small + 4.0 * classes,
                "flops": 6.0 * live * inner * classes}
    n = float(sum(k for k, _ in _sizes(case)))
    if kind == "norm":
        return {"bytes": es * n, "flops": 2.0 * n}
    per = 8 + es + 2 * case["copy"]
    # 8-bit states: a byte each and a scale for 32, read and written, and their values in 16 bits
    per += 16 if case["bits"] == 32 else 4 + 4.0 / BLOCK + 2 + 2.0 / BLOCK + 4
    return {"bytes": n * per + (es * n if kind == "step" else 0.0), "flops": 15.0 * n}


# ---------------------------------------------------------------------- exact

def _exact_loss(case, s):
    x, w = s["x"].to(torch.float64), s["w"].to(torch.float64)
    classes, train = case["classes"], case["kind"] == "train"
    loss, lse = [], []
    dw = torch.zeros_like(w) if train else None
    dbias = torch.zeros(classes, dtype=torch.float64, device=DEV)
    dx = []
    piece = max(1, (1 << 28) // classes)
    for r in range(0, case["rows"], piece):
        xr, label = x[r:r + piece], s["labels"][r:r + piece].to(torch.int64)
        known = torch.logical_and(label >= 0, label < classes)
        z = torch.matmul(xr, w.transpose(0, 1))
        if s["bias"] is not None:
            z = z + s["bias"].to(torch.float64)
        total = torch.special.logsumexp(z, dim=1)
        rows = torch.arange(len(label), device=DEV)
        picked = z[rows, label.clamp(min=0)]
        loss.append(torch.where(known, total - picked, torch.zeros_like(total)))
        lse.append(torch.where(known, total, torch.zeros_like(total)))
        if not train:
            continue
        share = torch.exp(z - total[:, None])
        onehot = -known.to(torch.float64) * s["scale"]
        weight = known.to(torch.float64) * s["scale"]
        if s["dlse"] is not None:
            weight = weight * (1.0 + s["dlse"][r:r + piece].to(torch.float64))
        p = share * weight[:, None]
        p[rows, label.clamp(min=0)] += onehot
        dx.append(torch.matmul(p, w))
        dw += torch.matmul(p.transpose(0, 1), xr)
        dbias += p.sum(dim=0)
    out = (torch.cat(loss), torch.cat(lse))
    return out + (torch.cat(dx), dw, dbias) if train else out


def _once(v):
    """Rounded to 32 bits, held in 64."""
    return v.to(torch.float32).to(torch.float64)


def _exact_bits(seed, number, count):
    """The 16-bit halves of draws from the generator's definition, in unsigned 64-bit numpy: [2][count]."""
    with np.errstate(over="ignore"):
        def mix(z):
            z = (z ^ (z >> np.uint64(30))) * np.uint64(C1)
            z = (z ^ (z >> np.uint64(27))) * np.uint64(C2)
            return z ^ (z >> np.uint64(31))
        key = mix(np.array([seed], np.uint64) ^ np.array([STATE_STREAM], np.uint64) * np.uint64(G))
        i = np.arange(1, (count + 1) // 2 + 1, dtype=np.uint64) + np.uint64(number)
        words = mix(key + i * np.uint64(G)).astype("<u8").view("<u2").reshape(-1, 2)[:count]
    return torch.from_numpy(words.T.astype(np.float64)).to(DEV)


def _exact_values(code, e, mantissa):
    """Magnitudes from their fields: (1 + f) 2^(x - 15) with a leading one, f 2^-14 where x is 0."""
    steps = 1 << mantissa
    x, f = torch.div(code, steps, rounding_mode="floor"), torch.remainder(code, steps) / steps
    value = torch.where(x > 0, (1.0 + f) * torch.exp2(x - 15.0), f * 2.0 ** -14)
    return value * torch.exp2(e.to(torch.float64) - 127.0).repeat_interleave(BLOCK)[:code.numel()]


def _exact_rounded(x, random, mantissa):
    """What the state of x >= 0 is after its rounding: the grid's value below, or the one above with
    the probability of the fraction, (16 bits + 1/2) / 65536 deciding."""
    n = x.numel()
    padded = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)
    top = padded.amax(dim=1)
    most = 2.0 - 2.0 ** -mantissa
    _, ex = torch.frexp(top)          # top = f 2^ex, f in [1/2, 1)
    ex = (ex - 1).clamp(min=-126)
    ex = torch.where(top > most * torch.exp2(ex.to(torch.float64)), ex + 1, ex).clamp(max=126)
    unit = torch.exp2(ex.to(torch.float64)).repeat_interleave(BLOCK)[:n]
    u = x / unit
    _, ux = torch.frexp(u)
    step = torch.exp2((ux - 1).clamp(min=-14).to(torch.float64) - mantissa)
    step = torch.where(u > 0, step, torch.ones_like(step))
    whole = torch.floor(u / step)
    up = (u / step - whole) + (random + 0.5) / 65536.0 >= 1.0
    return (whole + up.to(torch.float64)) * step * unit, step, unit


def _exact_step(case, s, factor):
    bits, first = case["bits"], 0
    shape = torch.zeros(s["total"], dtype=torch.float64, device=DEV)
    param, copy, m_out, v_out = (shape.clone() for _ in range(4))
    for (n, decay), p in zip(s["sizes"], s["at"]):
        g = s["grad"][p:p + n].to(torch.float64)
        if factor is not None:
            g = _once(g * factor) if bits == 8 else g * factor
        if bits == 8:
            # the roundings of a state are decided on its 32-bit value, which the definition
            # rounds at each operation
            k, sc = slice(p, p + n), slice(p // BLOCK, (p + n + BLOCK - 1) // BLOCK)
            code = s["m"][k].to(torch.float64)
            sign = 1.0 - 2.0 * (code > 127).to(torch.float64)
            m = sign * _exact_values(torch.remainder(code, 128), s["m_scale"][sc], 3)
            r = _exact_values(s["v"][k].to(torch.float64), s["v_scale"][sc], 4)
            beta1, rest1 = float(np.float32(BETA1)), float(np.float32(1.0 - BETA1))
            beta2, rest2 = float(np.float32(BETA2)), float(np.float32(1.0 - BETA2))
            m = _once(_once(m * beta1) + _once(g * rest1))
            v = _once(_once(_once(r * r) * beta2) + _once(_once(g * g) * rest2))
        else:
            m = s["m"][p:p + n].to(torch.float64) * BETA1 + g * (1.0 - BETA1)
            v = s["v"][p:p + n].to(torch.float64) * BETA2 + g * g * (1.0 - BETA2)
        mean = m / (1.0 - BETA1 ** STEP)
        deviation = torch.sqrt(v / (1.0 - BETA2 ** STEP))
        w = s["param"][p:p + n].to(torch.float64)
        w = w - LR * decay * w - LR * mean / (deviation + EPS)
        param[p:p + n] = w
        if bits == 8:
            random = _exact_bits(s["seed"], s["offset"] + first, n)
            size, _, _ = _exact_rounded(m.abs(), random[0], 3)
            m = torch.copysign(size, m)
            r = _once(torch.sqrt(v))
            size, step, unit = _exact_rounded(r, random[1], 4)
            v = torch.where((r > 0) & (size == 0), step * unit, size)
        m_out[p:p + n] = m
        v_out[p:p + n] = v
        first += (n + 1) // 2
    return [param] + ([param.clone()] if case["copy"] else []) + [m_out, v_out]


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind in ("loss", "train"):
        return _exact_loss(case, s)
    if kind == "adamw":
        return _exact_step(case, s, None)
    total = torch.linalg.vector_norm(s["grad"].to(torch.float64)).view(1)
    clip = (MAX_NORM / total).clamp(max=1.0)
    # (a step's factor is the 32-bit one that the norm's call leaves)
    return [total, clip] + (_exact_step(case, s, _once(clip)) if kind == "step" else [])
