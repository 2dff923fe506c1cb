"""The products that read w as it is in the bounds-checked build: their tests in a child process that loads it (but for
captured calls), and accesses past a buffer's end, which are refused and reported."""

import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def child(*args, **env):
    return subprocess.run([sys.executable, *args], env=dict(os.environ, AGN_LIB_VARIANT="check", **env),
                          capture_output=True, text=True, timeout=900, cwd=ROOT)


def test_in_the_checked_build():
    r = child("-m", "pytest", os.path.join(ROOT, "tests", "test_gpu_linear_ce_raw.py"), "-x", "-q", "-p",
              "no:cacheprovider", "-k", "not captured")
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-2000:]
    assert " passed" in r.stdout and "skipped" not in r.stdout


@pytest.mark.parametrize("rows,inner,classes", [(60, 1024, 3200), (100, 1023, 3201)])
def test_it_detects(rows, inner, classes):
    code = f"""
import torch, paper_1710_02368_gb300 as agn
assert agn.library_path().endswith("libagn_gb300_check.so")
rows, inner, classes = {rows}, {inner}, {classes}
z = lambda *n, k=torch.float32: torch.zeros(*n, dtype=k, device="cuda")
x, w, labels, lse = z(rows, inner), z(classes, inner), z(rows, k=torch.int32), z(rows)
n = max(agn.agn_linear_ce_bytes(rows, inner, classes, 0, k) for k in (0, 1))
work = z(n, k=torch.uint8)
for f in (lambda: agn.agn_linear_ce(x, w, labels, 0, rows, inner, classes, z(rows), lse, work, n),
          lambda: agn.agn_linear_ce_backward(x, w, labels, lse, 0, rows, inner, classes, work, n, dx=z(rows, inner))):
    try:
        f()
    except agn.AGNError as e:
        assert e.code == agn.AGN_E_BOUNDS, e
    else:
        raise SystemExit("not detected")
print("detected")
"""
    r = child("-c", code, AGN_BOUNDS_TEST_SHRINK="64")
    assert r.returncode == 0 and "detected" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]
