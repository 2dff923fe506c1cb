"""The operators take NumPy's numbers where they take Python's: sizes from an array of dimensions,
seeds and offsets from a generator (64-bit numbers, reduced mod 2^64 like Python's)."""

import numpy as np
import pytest


@pytest.fixture(scope="module")
def agn():
    import __graft_entry__ as g
    g.build()
    import paper_1710_02368_gb300 as agn
    return agn


@pytest.mark.parametrize("n", [np.int64(5), np.int64(-5), np.uint64(2 ** 64 - 5), np.int32(-5), np.uint8(5)], ids=repr)
def test_seeds_and_offsets(agn, n):
    got = []

    class Lib:   # what the C call is given
        def agn_dropout(self, *a):
            got.append(a[-3:-1])
            return 0
        agn_dropout_backward = agn_dropout
    real, agn._lib._LIB = agn._lib.load(), Lib()
    try:
        agn.agn_dropout(None, None, 0, 0, 8, 0.5, n, n)
        agn.agn_dropout_backward(None, None, 0, 0, 8, 0.5, n, n)
    finally:
        agn._lib._LIB = real
    want = int(n) % 2 ** 64
    assert got == [(want, want)] * 2
    agn.agn_dropout(None, None, 0, 0, 8, 0.5, n, n)            # and the C call takes them
    agn.agn_dropout_backward(None, None, 0, 0, 8, 0.5, n, n)


def test_sizes_and_probabilities(agn):
    dims = np.array([0, 784, 1000])
    agn.agn_dropout(None, None, np.int32(0), dims[0], dims[1], np.float32(0.5), 1)
    agn.agn_dropout_backward(None, None, 0, dims[0], dims[1], np.float64(0.5), 1, lddy=dims[2], lddx=dims[2])
    agn.agn_mx4_quantize(None, 0, dims[0], dims[1], None, None, ldx=dims[2])
    agn.agn_mx4_dequantize(None, None, dims[0], dims[1], None, 0, ldy=dims[2])
    agn.agn_mx4_linear(None, None, None, None, dims[0], dims[1], dims[2], None, 0)
    assert agn.agn_mx4_bytes(dims[2], dims[1]) == agn.agn_mx4_bytes(1000, 784)


def test_a_fraction_is_no_seed(agn):
    for kw in (dict(seed=1.5), dict(seed=1, offset=np.float64(2))):
        with pytest.raises(TypeError):
            agn.agn_dropout(None, None, 0, 0, 8, 0.5, **kw)
