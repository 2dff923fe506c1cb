"""The norm of gradients whose squares, or sums of squares, are past fp32's range while the norm is not."""

import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
MOST = float(np.finfo(np.float32).max)


@pytest.fixture(scope="module")
def agn():
    import paper_1710_02368_gb300 as agn
    return agn


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("shift", [0, 3])
@pytest.mark.parametrize("size", [1e16, 1e18, 1e19, 3e19, 1e25, 1e34, 1e37])
@pytest.mark.parametrize("sizes", [[3], [5000, 33], [700_001], [100, 3_000_000]], ids=str)
def test_large_gradients(agn, sizes, size, shift, dtype):
    """All of a size, one among ordinary ones, and the factor: as far off as for ordinary ones (sums of up to 64 in fp32,
    the root rounded)."""
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    whole = [torch.randn(n + shift, generator=g, device="cuda") for n in sizes]
    f = dict(device="cuda")
    norm, scale = torch.zeros(1, **f), torch.zeros(1, **f)
    for one in (False, True):
        grads = [(t if one else t * size).to(dtype)[shift:] for t in whole]
        if one:
            grads[-1][len(grads[-1]) // 2] = -size
        with agn.AGNOptim([dict(grad=t, n=t.numel(), grad_dtype=int(dtype is torch.bfloat16)) for t in grads]) as plan:
            plan.grad_norm(1e-3, norm, scale)
        want = math.sqrt(sum(float((t.double() ** 2).sum()) for t in grads))
        if want > MOST * (1 + 2.0 ** -10):
            assert norm.item() == math.inf and math.isnan(scale.item())
        elif want < MOST * (1 - 2.0 ** -10):
            assert abs(norm.item() - want) <= 65 * 2.0 ** -24 * want
            assert scale.item() == float(np.float32(1e-3) / np.float32(norm.item()))


@pytest.mark.parametrize("bad", [math.nan, math.inf])
def test_one_that_is_not_finite_among_large_ones(agn, bad):
    t = torch.full((100_000,), 1e19, device="cuda")
    t[77_777] = bad
    norm, scale = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    with agn.AGNOptim([dict(grad=t, n=t.numel())]) as plan:
        plan.grad_norm(1.0, norm, scale)
    assert not math.isfinite(norm.item()) and math.isnan(scale.item())
