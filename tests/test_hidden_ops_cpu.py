"""The hidden layer's operators without a GPU: refusals come before any device is touched, the
sizes of the 4-bit buffers, and the plain forms that the GPU tests compare with."""

import ctypes as C

import numpy as np
import pytest

import agn_inputs as I
import ops_ref as R


@pytest.fixture(scope="module")
def agn():
    import __graft_entry__ as g
    g.build()
    import paper_1710_02368_gb300 as agn
    return agn


X, Y, Z, W = 1 << 20, 1 << 24, 1 << 28, 1 << 32   # aligned, never read


def refused(agn, call, *words):
    with pytest.raises(agn.AGNError) as e:
        call()
    assert e.value.code == agn.AGN_E_INVALID
    for w in words:
        assert w in str(e.value)


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(dtype=-1), dict(rows=-1), dict(cols=-1), dict(cols=1 << 31), dict(p=1.0),
    dict(p=-0.1), dict(p=float("nan")), dict(ldx=7), dict(ldy=7), dict(x=None), dict(y=None),
    dict(residual=Z, ldr=7), dict(rows=1 << 62, ldx=1 << 20), dict(x=X + 2), dict(y=Y + 2),
    dict(bias=Z + 1), dict(y=X + 4), dict(y=X, ldy=16), dict(bias=Y + 4), dict(residual=Y + 32),
], ids=str)
def test_dropout_refuses(agn, bad):
    a = dict(x=X, y=Y, dtype=0, rows=4, cols=8, p=0.5, seed=1)
    a.update(bad)
    refused(agn, lambda: agn.agn_dropout(**a))


@pytest.mark.parametrize("bad", [
    dict(dtype=3), dict(rows=-2), dict(p=1.5), dict(lddy=7), dict(lddx=7), dict(relu=1),
    dict(relu=1, x=Z, ldx=7), dict(dy=None), dict(dx=None), dict(dbias=Z + 2), dict(dbias=X),
    dict(dbias=Y + 4), dict(dx=X + 8), dict(relu=1, x=Z, dx=Z + 4), dict(relu=1, x=Z, bias=Y),
], ids=str)
def test_dropout_backward_refuses(agn, bad):
    a = dict(dy=X, dx=Y, dtype=0, rows=4, cols=8, p=0.5, seed=1)
    a.update(bad)
    refused(agn, lambda: agn.agn_dropout_backward(**a))


@pytest.mark.parametrize("bad", [
    dict(dtype=2), dict(rows=-1), dict(cols=-1), dict(ldx=39), dict(x=None), dict(codes=None),
    dict(scales=None), dict(codes=Y + 8), dict(scales=Z + 4), dict(x=X + 1), dict(codes=X),
    dict(scales=X + 16), dict(scales=Y + 16),
], ids=str)
def test_quantize_refuses(agn, bad):
    a = dict(x=X, dtype=1, rows=4, cols=40, codes=Y, scales=Z)
    a.update(bad)
    refused(agn, lambda: agn.agn_mx4_quantize(**a))


def test_dequantize_refuses(agn):
    refused(agn, lambda: agn.agn_mx4_dequantize(Y, Z, 4, 40, X, 1, ldy=39))
    refused(agn, lambda: agn.agn_mx4_dequantize(Y, Z, 4, 40, None, 1))
    refused(agn, lambda: agn.agn_mx4_dequantize(Y, Z, 4, 40, Z + 64, 1), "overlaps")
    refused(agn, lambda: agn.agn_mx4_dequantize(Y, Z, 4, 40, X, 2), "dtype")


@pytest.mark.parametrize("bad", [
    dict(rows=-1), dict(inner=0), dict(out=0), dict(inner=(1 << 28) + 1), dict(out=(1 << 31) - 1), dict(rows=(1 << 31) - 1),
    dict(dtype=5), dict(ldy=99), dict(x_codes=None), dict(w_scales=None), dict(y=None),
    dict(dtype=2), dict(x_codes=X + 4), dict(w_scales=W + 4), dict(y=X + 16), dict(err=Z),
    dict(bias=Z + 2), dict(dtype=2, y_scales=Z), dict(dtype=2, y_scales=3 * Z + 4),
    dict(dtype=2, y=Z + 4, y_scales=3 * Z), dict(err=Z + (1 << 26) + 1),
], ids=str)
def test_linear_refuses(agn, bad):
    a = dict(x_codes=X, x_scales=Y, w_codes=W, w_scales=2 * W, rows=4, inner=64, out=100, y=Z,
             dtype=0)
    a.update(bad)
    refused(agn, lambda: agn.agn_mx4_linear(**a))


@pytest.mark.parametrize("kw,code", [(dict(dropout=1.0), "INVALID"), (dict(dropout=-0.1), "INVALID"),
                                     (dict(dropout=float("nan")), "INVALID"), (dict(eval_mx4=1), "INVALID"),
                                     (dict(eval_mx4=1, n_eval=4, dims=(8, 4)), "UNSUPPORTED")], ids=str)
def test_create_refuses(agn, kw, code):
    kw = dict(kw)
    dims = kw.pop("dims", (8, 8, 4))
    with pytest.raises(agn.AGNError) as e:
        agn.AGN(dims, 2, 1, 0.1, 1, **kw)
    assert e.value.name == "AGN_E_" + code


def test_evaluate_mx4_refuses_a_null_handle(agn):
    assert agn._lib.load().agn_evaluate_mx4(None, None, None, None, 0) == agn.AGN_E_INVALID


def test_nothing_to_do_touches_nothing(agn):
    agn.agn_dropout(None, None, 0, 0, 8, 0.5, 1)
    agn.agn_dropout(None, None, 1, 8, 0, 0.5, 1)
    agn.agn_dropout_backward(None, None, 0, 0, 8, 0.5, 1)
    agn.agn_mx4_quantize(None, 0, 0, 8, None, None)
    agn.agn_mx4_dequantize(None, None, 3, 0, None, 0)
    agn.agn_mx4_linear(None, None, None, None, 0, 64, 64, None, 0)


def test_a_host_pointer_is_refused(agn):
    """Whatever is not memory of the current device (or no device at all) is an error, never a launch."""
    x = np.zeros(64, np.float32)
    y = np.zeros(64, np.float32)
    with pytest.raises(agn.AGNError) as e:
        agn.agn_dropout(x.ctypes.data // 16 * 16 + 16, y.ctypes.data // 16 * 16 + 16, 0, 2, 8, 0.5, 1)
    assert e.value.code in (agn.AGN_E_INVALID, agn.AGN_E_CUDA)


@pytest.mark.parametrize("rows,cols", [(0, 0), (1, 1), (1, 32), (127, 33), (128, 128), (129, 129),
                                       (10000, 784), (1 << 33, 4096)])
def test_buffer_sizes(agn, rows, cols):
    nb = -(-cols // 32)
    assert agn.agn_mx4_bytes(rows, cols) == (rows * nb * 16, -(-rows // 128) * -(-nb // 4) * 512)
    lib = agn._lib.load()
    assert lib.agn_mx4_bytes(rows, cols, None, None) == 0
    assert lib.agn_mx4_bytes(-1, cols, None, None) == agn.AGN_E_INVALID


# ------------------------------------------------ the plain forms themselves

def test_mask_is_the_generator_of_the_inputs():
    """The mask's numbers are those of agn_inputs' splitmix64 (pinned there by published outputs)."""
    assert int(R.stream_key(77, 8)[0]) == int(I.stream_key(77, 8))
    keep = R.keep_mask(3, 10, 0.25, 77, offset=5)
    for r, c in [(0, 0), (0, 3), (1, 9), (2, 4)]:
        d = int(R.draw(R.stream_key(77, 8), np.array([5 + r * 3 + c // 4]))[0])
        assert keep[r, c] == (((d >> (16 * (c % 4))) & 0xFFFF) >= 16384)


def test_mask_rate_and_independence():
    """Rates within five standard deviations; rows, columns and neighbours uncorrelated."""
    for p in (0.1, 0.5, 0.75):
        k = R.keep_mask(1000, 1000, p, 3).astype(float)
        q = 1 - R.threshold(p) / 65536
        sd = np.sqrt(q * (1 - q))
        assert abs(k.mean() - q) < 5 * sd / 1000
        z = (k - q) / sd
        for a, b in ((z[:, 1:], z[:, :-1]), (z[1:], z[:-1]), (z[:, 4:], z[:, :-4])):
            assert abs((a * b).mean()) < 5 / np.sqrt(a.size)


def test_quantisation_by_hand():
    x = np.zeros((1, 32))
    x[0, :12] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.9, -0.25, -5.1, 0.2]
    code, scale = R.mx4_quantize(x)     # largest 7.9: the scale is 1
    assert scale[0, 0] == 127
    assert list(R.mx4_values(code, scale)[0, :12]) == [0, 1, 1, 2, 2, 4, 4, 6, 6, 0, -6, 0]
    code, scale = R.mx4_quantize(x / 1024)
    assert scale[0, 0] == 117
    c, s = R.mx4_pack(code, scale)
    assert np.array_equal(R.mx4_unpack(c, s, 1, 32), R.mx4_values(code, scale))


def test_packing_round_trip():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((300, 200)) * np.exp2(rng.integers(-20, 20, (300, 1)))
    code, scale = R.mx4_quantize(x)
    c, s = R.mx4_pack(code, scale)
    assert c.shape == (300, 112) and s.size == 3 * 2 * 512
    v = R.mx4_unpack(c, s, 300, 200)
    assert np.array_equal(v, R.mx4_values(code, scale)[:, :200])
    # E2M1's spacing is at most half a block's power of two times 2 (values 4 .. 6), and saturation
    # takes at most 2 of 8: within 1/4 of the block's largest value
    a = np.abs(np.pad(x, ((0, 0), (0, 24)))).reshape(300, 7, 32).max(2)
    assert np.all(np.abs(v - x) <= 0.25 * np.repeat(a, 32, 1)[:, :200])


def test_ctypes_signatures_take_64_bit_sizes(agn):
    sig = agn._lib.SIGNATURES["agn_dropout"][1]
    assert sig[6:11] == [C.c_int64] * 5 and sig[11] is C.c_double
