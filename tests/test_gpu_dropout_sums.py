"""agn_dropout_backward's dbias to the last bit.  dy holds whole numbers from 1 to 8, p is 1/2 (scale
2), so every partial sum is a whole number below 2^24 and fp32 holds it exactly in any order: dbias
has to equal the 64-bit sum.  Nothing cancels: a row left out of a column's sum where it is kept,
or counted twice, changes it."""

import numpy as np
import pytest

import ops_ref as R

P, SEED, OFFSET = 0.5, 77, 1 << 33
# few columns and many rows (wide clusters), one unit and several, more columns, sums of a few rows
SHAPES = [(40000, 8), (33001, 4), (20011, 16), (17000, 33), (65536, 2), (65536, 1), (65536, 17), (9000, 3), (5000, 24),
          (2048, 1000), (16384, 200), (3000, 129), (300, 4097), (33, 1000), (1, 8), (7, 31)]


def inputs(rows, cols, relu):
    rng = np.random.default_rng(rows + 7 * cols + relu)
    dy = rng.integers(1, 9, (rows, cols)).astype(np.float64)
    x = rng.integers(-8, 9, (rows, cols)).astype(np.float64) / 4   # (zeros among them)
    b = rng.integers(-2, 3, cols).astype(np.float64) / 4
    live = R.keep_mask(rows, cols, P, SEED, OFFSET)
    if relu:
        live = live & (x + b > 0)
    dx = np.where(live, dy * R.gain(P), 0.0)
    assert R.gain(P) == 2.0 and dx.sum(0).max() < 2 ** 24
    return dy, x, b, dx


@pytest.mark.parametrize("rows,cols", [s for s in SHAPES if s[0] >= 2048])
def test_a_lost_partial_sum_would_show(rows, cols):
    """The values themselves, without a GPU: leaving out the rows of a sixteenth of the matrix, or one
    of 128 interleaved parts of it (a thread's rows of a block), changes some column."""
    _, _, _, dx = inputs(rows, cols, 1)
    full = dx.sum(0)
    per = -(-rows // 16)
    for k in range(0, 16, 3):
        block = dx[k * per:(k + 1) * per]
        assert np.any(full - block.sum(0) != full)
        for t in (0, 1, 63, 127):
            part = block[t::128]
            if part.size >= 16:   # (of fewer elements all may be dropped)
                assert np.any(full - part.sum(0) != full)


def place(torch, dtype, m, ld, start, fill=7.0):
    """A matrix of the values m (None: fill) with row stride ld, `start` elements into its buffer."""
    rows, cols = m.shape if m is not None else (0, 0)
    buf = torch.full((start + rows * ld + 16,), fill, device="cuda").to(torch.bfloat16 if dtype else torch.float32)
    v = buf[start:start + rows * ld].view(rows, ld)
    v[:, :cols] = torch.tensor(m, device="cuda").to(buf.dtype)
    return v


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [0, 1])
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("relu", [0, 1])
def test_sums_are_exact(dtype, rows, cols, relu):
    import torch

    import paper_1710_02368_gb300 as agn
    dy64, x64, b64, dx64 = inputs(rows, cols, relu)
    want = torch.tensor(dx64.sum(0), dtype=torch.float32, device="cuda")
    grad = torch.tensor(dx64, device="cuda").to(torch.bfloat16 if dtype else torch.float32)
    b = torch.tensor(b64, dtype=torch.float32, device="cuda")
    al = 8 if dtype else 4
    up = -(-cols // al) * al
    # row strides of dy, x, dx and where they start: aligned, alike but unaligned, all different
    for ldg, ldx, ldo, sg, sx, so in [(up, up, up, 0, 0, 0), (cols, cols, cols, 0, 0, 0), (up, up, up, 1, 1, 1), (up + 3, up + 3, up + 3, 3, 3, 3),
                                      (cols, up, up + 1, 0, 1, 2)]:
        for place_in in ("", "dy", "x"):
            if place_in == "x" and not relu:
                continue
            dy, x = place(torch, dtype, dy64, ldg, sg), place(torch, dtype, x64, ldx, sx)
            dx, ld = {"": (None, ldo), "dy": (dy, ldg), "x": (x, ldx)}[place_in]
            if dx is None:
                dx = place(torch, dtype, np.full((rows, cols), 7.0), ldo, so)
            db = torch.full((cols + 2,), 7.0, device="cuda")
            agn.agn_dropout_backward(dy, dx, dtype, rows, cols, P, SEED, OFFSET, x=x if relu else None, bias=b if relu else None,
                                     dbias=db[1:], relu=relu, lddy=ldg, ldx=ldx, lddx=ld)
            assert torch.equal(db[1:-1], want), (ldg, ldx, ldo, sg, place_in)
            assert torch.equal(dx[:, :cols], grad) and db[0] == 7 and db[-1] == 7
            assert torch.all(dx[:, cols:] == 7)
