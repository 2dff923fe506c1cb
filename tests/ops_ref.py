"""Plain 64-bit forms of the hidden layer's operators (test infrastructure; shares no code with
the library): the dropout mask, microscaled 4-bit quantisation and its layout, the product."""

import numpy as np

G, C1, C2 = (np.uint64(v) for v in (0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB))
M64 = (1 << 64) - 1
E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def mix(z):
    """splitmix64's output function on uint64 arrays."""
    with np.errstate(over="ignore"):
        z = (z ^ (z >> np.uint64(30))) * C1
        z = (z ^ (z >> np.uint64(27))) * C2
        return z ^ (z >> np.uint64(31))


def stream_key(seed, stream):
    with np.errstate(over="ignore"):
        return mix(np.array([seed & M64], np.uint64) ^ (np.array([stream], np.uint64) * G))


def draw(key, i):
    with np.errstate(over="ignore"):
        return mix(key + (np.asarray(i, np.uint64) + np.uint64(1)) * G)


def threshold(p):
    return min(65535, int(np.rint(65536 * p)))


def keep_mask(rows, cols, p, seed, offset=0):
    groups = -(-cols // 4)
    with np.errstate(over="ignore"):
        i = np.arange(rows * groups, dtype=np.uint64) + np.array([offset & M64], np.uint64)
    d = draw(stream_key(seed, 8), i).reshape(rows, groups)
    u = np.stack([(d >> np.uint64(16 * k)) & np.uint64(0xFFFF) for k in range(4)], 2)
    return u.reshape(rows, 4 * groups)[:, :cols] >= threshold(p)


def hidden_seed(seed, worker, layer, layers):
    """The seed of a worker's hidden layer (from 0) in a training run."""
    return int(draw(stream_key(seed, 8), np.array([worker * layers + layer]))[0])


def gain(p):
    return 65536.0 / (65536.0 - threshold(p))


def blocks(cols):
    return -(-cols // 32)


def mx4_quantize(x):
    """(codes as values' indices [rows][32 nb], scale codes [rows][nb]) of float64 rows."""
    rows, cols = x.shape
    nb = blocks(cols)
    v = np.zeros((rows, nb * 32))
    v[:, :cols] = x
    v = v.reshape(rows, nb, 32)
    amax = np.abs(v).max(2)
    bad = ~np.isfinite(amax)
    e = np.full(amax.shape, -127)
    ok = ~bad & (amax > 0)
    e[ok] = np.maximum(np.frexp(amax[ok])[1] - 1 - 2, -127)
    with np.errstate(invalid="ignore"):
        a = np.abs(np.where(bad[:, :, None], 0.0, v)) * 2.0 ** (-e[:, :, None].astype(float))
    d = np.abs(a[..., None] - E2M1)
    near = d == d.min(3, keepdims=True)
    code = np.argmax(near * np.where(np.arange(8) % 2 == 0, 2, 1), 3)   # ties: the even code
    code = code + 8 * (np.signbit(v) & ~bad[:, :, None])
    return code.reshape(rows, nb * 32).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def mx4_pack(code, scale):
    """The library's buffers: codes [rows][16 nb], scales in tiles of 128 rows x 4 blocks."""
    rows, nb = scale.shape
    k = -(-nb // 4)
    tiles = np.zeros((-(-rows // 128), k, 32, 4, 4), np.uint8)   # row tile, k tile, r % 32, r / 32, kb % 4
    for r in range(rows):
        for b in range(nb):
            tiles[r // 128, b // 4, r % 32, r // 32 % 4, b % 4] = scale[r, b]
    return (code[:, 0::2] | (code[:, 1::2] << 4)).astype(np.uint8), tiles.reshape(-1)


def mx4_unpack(codes, scales, rows, cols):
    """Values (float64) of the library's buffers."""
    nb = blocks(cols)
    k = -(-nb // 4)
    t = scales.reshape(-1, k, 32, 4, 4).transpose(0, 3, 2, 1, 4).reshape(-1, 4 * k)[:rows, :nb]
    code = np.empty((rows, nb * 32), np.uint8)
    code[:, 0::2], code[:, 1::2] = codes.reshape(rows, -1) & 15, codes.reshape(rows, -1) >> 4
    return mx4_values(code, t)[:, :cols]


def mx4_values(code, scale):
    s = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(float) - 127))
    sign = np.where(code & 8, -1.0, 1.0)
    return E2M1[code & 7] * sign * np.repeat(s, 32, 1)
