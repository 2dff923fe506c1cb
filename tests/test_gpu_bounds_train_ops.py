"""The output layer's loss and the optimizer's step in the bounds-checked build: their own tests in a
child process that loads it, but for captured calls (that build's uploads do not allow them), plans
of more tensors than its table has room for and calls of several threads."""

import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("name", ["test_gpu_linear_ce.py", "test_gpu_adamw.py", "test_gpu_train_step.py"])
def test_in_the_checked_build(name):
    env = dict(os.environ, AGN_LIB_VARIANT="check")
    r = subprocess.run([sys.executable, "-m", "pytest", os.path.join(ROOT, "tests", name), "-x", "-q", "-p",
                        "no:cacheprovider", "-k", "not graph and not many and not threads and not pieces"],
                       env=env, capture_output=True, text=True, timeout=900, cwd=ROOT)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-2000:]
    assert " passed" in r.stdout and "skipped" not in r.stdout


def test_it_detects():
    """Buffers registered 64 bytes short: the accesses to their ends are refused and reported."""
    code = """
import torch, paper_1710_02368_gb300 as agn
assert agn.library_path().endswith("libagn_gb300_check.so")
z = lambda n, k=torch.float32: torch.zeros(n, dtype=k, device="cuda")
def loss(rows, inner, classes, dtype):
    t = torch.bfloat16 if dtype else torch.float32
    x, w, labels = z(rows * inner, t), z(classes * inner, t), z(rows, torch.int32)
    out, lse, work = z(rows), z(rows), z(1 << 24, torch.uint8)
    agn.agn_linear_ce(x, w, labels, dtype, rows, inner, classes, out, lse, work, 1 << 24)
def grads(rows, inner, classes, dtype):
    t = torch.bfloat16 if dtype else torch.float32
    x, w, labels = z(rows * inner, t), z(classes * inner, t), z(rows, torch.int32)
    lse, work = z(rows), z(1 << 24, torch.uint8)
    agn.agn_linear_ce_backward(x, w, labels, lse, dtype, rows, inner, classes, work, 1 << 24, dx=z(rows * inner, t), dw=z(classes * inner, t))
def plan():
    u = torch.uint8
    return agn.AGNOptim([dict(param=z(4000), grad=z(4000), m=z(4000, u), v=z(4000, u), m_scale=z(125, u), v_scale=z(125, u), n=4000)], state_bits=8)
u = torch.uint8
for f in (lambda: loss(40, 32, 30, 0), lambda: loss(8, 32, 3000, 0), lambda: loss(600, 64, 300, 1), lambda: loss(600, 64, 300, 0),
          lambda: grads(40, 32, 30, 1), lambda: grads(4, 32, 3000, 1), lambda: grads(600, 64, 300, 1),
          lambda: plan().adamw(0.1, 1), lambda: plan().grad_norm(1.0, z(1)),
          lambda: agn.agn_adamw_dequantize(z(999, u), z(32, u), z(999, u), z(32, u), 999, z(999), z(999), 0)):
    try:
        f()
    except agn.AGNError as e:
        assert e.code == agn.AGN_E_BOUNDS, e
    else:
        raise SystemExit("not detected")
print("detected")
"""
    env = dict(os.environ, AGN_LIB_VARIANT="check", AGN_BOUNDS_TEST_SHRINK="64")
    r = subprocess.run([sys.executable, "-c", code], env=env, capture_output=True, text=True, timeout=300, cwd=ROOT)
    assert r.returncode == 0 and "detected" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]
