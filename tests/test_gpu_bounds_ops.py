"""The hidden layer's operators in the bounds-checked build: their own tests in a child process
that loads it (every global access checked against the call's buffers, tensor maps against their
extents), but for captured calls and calls of two threads, which that build's uploads do not allow, and the 4 GB
matrix."""

import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("name", ["test_gpu_dropout.py", "test_gpu_mx4.py", "test_gpu_dropout_run.py"])
def test_in_the_checked_build(name):
    env = dict(os.environ, AGN_LIB_VARIANT="check")
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.join(ROOT, "tests", name), "-x", "-q", "-p",
                        "no:cacheprovider", "-k", "not graph and not capture and not threads and not past_32_bits"],
                       env=env, capture_output=True, text=True, timeout=900, cwd=ROOT)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-2000:]
    assert " passed" in r.stdout and "skipped" not in r.stdout


def test_it_detects():
    """Buffers registered 64 bytes short: the accesses to their ends are refused and reported."""
    code = """
import torch, paper_1710_02368_gb300 as agn
assert agn.library_path().endswith("libagn_gb300_check.so")
x = torch.randn(64, 64, device="cuda"); y = torch.zeros_like(x)
c, s = (torch.zeros(n, dtype=torch.uint8, device="cuda") for n in agn.agn_mx4_bytes(64, 64))
for f in (lambda: agn.agn_dropout(x, y, 0, 64, 64, 0.0, 1), lambda: agn.agn_dropout_backward(x, y, 0, 64, 64, 0.0, 1),
          lambda: agn.agn_mx4_quantize(x, 0, 64, 64, c, s), lambda: agn.agn_mx4_dequantize(c, s, 64, 64, y, 0),
          lambda: agn.agn_mx4_linear(c, s, c, s, 64, 64, 64, y, 0)):
    try:
        f()
    except agn.AGNError as e:
        assert e.code == agn.AGN_E_BOUNDS, e
    else:
        raise SystemExit("not detected")
assert torch.all(y.view(-1)[-16:] == 0)
print("detected")
"""
    env = dict(os.environ, AGN_LIB_VARIANT="check", AGN_BOUNDS_TEST_SHRINK="64")
    r = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True, timeout=300, cwd=ROOT)
    assert r.returncode == 0 and "detected" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]
