"""Plain 64-bit forms of the output layer's loss and the optimizer's step (test infrastructure;
shares no code with the library), and bounds of what the library's arithmetic may differ by."""

import math

import numpy as np
import torch

import ops_ref as R

HALF = {0: 2.0 ** -24, 1: 2.0 ** -8}   # half a step of fp32, bf16, relative


def linear_ce(x, w, bias, labels, dloss=None, dlse=None, scale=1.0):
    """loss, lse, dx, dw, dbias and the pieces of their bounds, in float64."""
    classes = w.shape[0]
    known = (labels >= 0) & (labels < classes)
    x = torch.where(known[:, None], x.double(), 0.0)   # (rows left out may hold anything)
    w = w.double()
    z = x @ w.t()
    if bias is not None:
        z = z + bias.double()
    lse = torch.logsumexp(z, 1)
    at = torch.where(known, labels, 0).long()[:, None]
    none = lse == -math.inf
    loss = torch.where(none, math.inf, lse - z.gather(1, at)[:, 0])
    one = torch.ones_like(lse)
    dl = one if dloss is None else dloss.double()
    a = scale * (dl + (0 if dlse is None else dlse.double()))
    b = scale * dl
    soft = torch.exp(z - torch.where(none, 0.0, lse)[:, None])
    on = (known & ~none).double()
    p = soft * (a * on)[:, None]
    p.scatter_add_(1, at, -(b * on)[:, None])
    size = (soft * (a * on).abs()[:, None]).scatter_add_(1, at, (b * on).abs()[:, None])   # of p's terms
    zero = torch.zeros_like(lse)
    return dict(loss=torch.where(known, loss, zero), lse=torch.where(known, lse, zero), dx=p @ w, dw=p.t() @ x,
                dbias=p.sum(0), p=p, p_size=size, sums=x.abs() @ w.abs().t(), x=x, w=w, known=known)


def steps(n):
    """Additions of f32 sums over n products, 16 to an MMA (and up to six products of pieces)."""
    return n / 16 + 8


def z_bound(ref, inner, dtype):
    """|error of z|, each row's largest: every addition to a sum may lose two units of 2^-23 of the sum of
    magnitudes (truncation, alignment inside an MMA), pieces lose 2^-22 of it."""
    s = ref["sums"].amax(1)
    return s * (2 * steps(inner) * (6 if dtype == 0 else 1) * 2.0 ** -23 + 2.0 ** -22)


def loss_bounds(ref, inner, dtype):
    e = z_bound(ref, inner, dtype)
    lse = ref["lse"].abs()
    lse = torch.where(torch.isfinite(lse), lse, 0.0)
    # the sums of exponentials (2^-18 covers 2^17 classes in sums of sums), exp2's 2 units, log's, the bias's add
    own = 2.0 ** -18 + 2.0 ** -22 * (1 + lse)
    return 2 * e + own, e + own


def p_bound(ref, inner, dtype):
    """|error of p| before it is rounded."""
    lse = ref["lse"].abs()
    lse = torch.where(torch.isfinite(lse), lse, 0.0)
    rel = 2 * z_bound(ref, inner, dtype) + 2.0 ** -18 + 2.0 ** -22 * (4 + lse)
    return ref["p_size"] * rel[:, None]


def grad_bounds(ref, inner, dtype):
    e = p_bound(ref, inner, dtype)
    # bf16: p itself and the gradients are rounded; three pieces hold p to 2^-24
    r = HALF[dtype]
    ep = e + (ref["p"].abs() + e) * r
    pa = ref["p"].abs() + ep
    rows, classes = ref["p"].shape
    xs, ws = ref["x"].abs(), ref["w"].abs()
    six = 6 if dtype == 0 else 1
    sums = lambda n: 2 * steps(n) * six * 2.0 ** -23 + 2.0 ** -22 + 64 * 2.0 ** -24   # (and ranges along K)
    tiny = 1e-36
    dx = ep @ ws + (pa @ ws) * sums(classes)
    dw = ep.t() @ xs + (pa.t() @ xs) * sums(rows)
    db = e.sum(0) + (ref["p"].abs() + e).sum(0) * (rows * 2.0 ** -24)
    return (dx + (ref["dx"].abs() + dx) * r + tiny, dw + (ref["dw"].abs() + dw) * r + tiny, db + tiny)


# ------------------------------------------------------------------- optimizer

def f32(v):
    return np.asarray(v, np.float64).astype(np.float32).astype(np.float64)


def values(codes, scales, mantissa):
    """Magnitudes of codes (sign removed) with the scales of their blocks of 32."""
    n = len(codes)
    x, f = codes >> mantissa, (codes & ((1 << mantissa) - 1)) / (1 << mantissa)
    v = np.where(x > 0, (1 + f) * 2.0 ** (x - 15.0), f * 2.0 ** -14)
    s = np.where(scales == 0, 0.0, 2.0 ** (scales.astype(float) - 127))
    return v * np.repeat(s, 32)[:n]


def m_values(codes, scales):
    c = codes.astype(np.int64)
    return np.where(c > 127, -1.0, 1.0) * values(c & 127, scales, 3)


def r_values(codes, scales):
    return values(codes.astype(np.int64), scales, 4)


def grid(mantissa):
    """All magnitudes a code can stand for, times the scale 1."""
    c = np.arange(16 << mantissa)
    return values(c, np.full(-(-len(c) // 32), 127, np.uint8), mantissa)


def rounded(x, random, mantissa):
    """(codes, scales) of x >= 0 (float64 holding fp32 values): the grid's value below, or the one above where
    the fraction and (random + 1/2) / 65536 reach one."""
    n = len(x)
    g = grid(mantissa)
    most = g[-1]
    blocks = np.zeros(-(-n // 32) * 32)
    blocks[:n] = x
    blocks = blocks.reshape(-1, 32)
    scales = np.zeros(len(blocks), np.uint8)
    codes = np.zeros(blocks.shape, np.int64)
    rnd = np.zeros(blocks.size)
    rnd[:n] = random
    rnd = rnd.reshape(-1, 32)
    for i, b in enumerate(blocks):
        e = 1
        while b.max() > most * 2.0 ** (e - 127) and e < 253:
            e += 1
        u = b / 2.0 ** (e - 127)
        at = np.clip(np.searchsorted(g, u, side="right") - 1, 0, len(g) - 1)
        up = np.minimum(at + 1, len(g) - 1)
        gap = np.where(up > at, g[up] - g[at], 1.0)
        codes[i] = np.where((u - g[at]) / gap + (rnd[i] + 0.5) / 65536 >= 1, up, at)
        scales[i] = e
    return codes.reshape(-1)[:n].astype(np.uint8), scales


def random_bits(seed, number, n):
    d = R.draw(R.stream_key(seed, 9), (np.arange(-(-n // 2), dtype=np.uint64) + np.uint64(number % 2 ** 64)))
    w = d.astype("<u8").view("<u2").reshape(-1, 2)[:n]
    return w[:, 0].astype(np.float64), w[:, 1].astype(np.float64)


def adamw(param, grad, m, v, lr, step, b1, b2, eps, decay, factor=None):
    """One element-wise step in float64 whose states are rounded to fp32 at each operation (v: r * r for 8
    bits); param is not."""
    g = grad if factor is None else f32(grad * factor)
    B1, O1, B2, O2 = (float(np.float32(t)) for t in (b1, 1 - b1, b2, 1 - b2))
    m = f32(f32(m * B1) + f32(g * O1))
    v = f32(f32(v * B2) + f32(f32(g * g) * O2))
    r = f32(np.sqrt(v))
    q = m / (r * float(np.float32(1 / math.sqrt(1 - b2 ** step))) + float(np.float32(eps)))
    return param * (1 - lr * decay) - lr / (1 - b1 ** step) * q, m, v, r
