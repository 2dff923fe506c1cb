"""What decides how the output layer's products are cut (csrc/linear_ce.cu): the time of the CTA that ends last, its own
source compiled here and compared with the units given out one by one; sizes of the scratch up to the largest."""

import os
import re
import shutil
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1710_02368_gb300", "csrc")

PROGRAM = r"""
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <queue>
#include <vector>
@SOURCE@
// The longer units in turn, then each of the others to the CTA that is free first.
double in_turn(int64_t at_once, const int64_t (&n)[2], const double (&cost)[2]) {
  const int longer = cost[1] > cost[0] ? 1 : 0;
  std::vector<double> busy(at_once, 0.0);
  for (int64_t i = 0; i < n[longer]; ++i) busy[i % at_once] += cost[longer];
  std::priority_queue<double, std::vector<double>, std::greater<double>> q(busy.begin(), busy.end());
  double last = *std::max_element(busy.begin(), busy.end());
  for (int64_t i = 0; i < n[1 - longer]; ++i) {
    const double t = q.top() + cost[1 - longer];
    q.pop();
    q.push(t);
    last = std::max(last, t);
  }
  return last;
}
int main(int argc, char** argv) {
  if (argc > 1) {   // far apart: it has to end
    const int64_t n[2] = {std::atoll(argv[1]), std::atoll(argv[2])};
    const double cost[2] = {std::atof(argv[3]), std::atof(argv[4])};
    const double t = makespan(76, n, cost), work = (n[0] * cost[0] + n[1] * cost[1]) / 76;
    return t >= work * (1 - 1e-9) && t <= work + 2 * (cost[0] + cost[1]) ? 0 : 1;
  }
  uint64_t s = 1;
  auto below = [&](int64_t m) { return (int64_t)((s = s * 6364136223846793005ull + 1442695040888963407ull) >> 33) % m; };
  for (int i = 0; i < 20000; ++i) {
    const int64_t at_once = 1 + below(i % 2 ? 160 : 9), n[2] = {below(400), below(400)};
    // (halves and quarters: their sums are exact)
    const double cost[2] = {0.5 + 0.25 * below(i % 3 ? 200 : 8), 0.5 + 0.25 * below(i % 5 ? 200 : 8)};
    const double a = makespan(at_once, n, cost), b = in_turn(at_once, n, cost);
    if (!(std::fabs(a - b) <= 1e-9 * b)) {
      std::printf("%ld: %ld %ld of %g %g: %g, in turn %g\n", (long)at_once, (long)n[0], (long)n[1], cost[0], cost[1], a, b);
      return 1;
    }
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if not shutil.which("g++"):
        pytest.skip("no g++")
    text = open(os.path.join(CSRC, "linear_ce.cu")).read()
    where = tmp_path_factory.mktemp("cuts")
    src, exe = where / "cuts.cpp", where / "cuts"
    src.write_text(PROGRAM.replace("@SOURCE@", re.search(r"^double makespan\(.*?^}\n", text, re.S | re.M).group(0)))
    subprocess.run(["g++", "-std=c++17", "-O2", str(src), "-o", str(exe)], check=True)
    return str(exe)


def test_against_units_given_out_one_by_one(program):
    r = subprocess.run([program], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout


@pytest.mark.parametrize("args", ["18 2154184651 50259.5 30.757178422302548", "11915 3193106021 673176.5 2.6784736875190522",
                                  "29900 387386898 698771.5 15.491512323916925", "2044 1693981708 3315025.5 6.4"])
def test_very_many_units(program, args):
    """Times that differ by a unit's in the last place of a double."""
    assert subprocess.run([program, *args.split()], timeout=20).returncode == 0


@pytest.mark.parametrize("size", [(212161569, 523138, 251, 1), (1 << 28, 1 << 20, 1 << 28, 0), (1 << 28, 1 << 20, 1000, 1),
                                  (207515811, 848547, 131, 0), ((1 << 28) - 1, 1 << 20, 253, 1)])
def test_scratch_of_the_largest_sizes(size):
    """They are answered, and at once (no buffers of such sizes exist; the products' cuts are still worked out)."""
    code = ("import time, __graft_entry__ as g; g.build(); import paper_1710_02368_gb300 as a; a._lib.load(); t = time.monotonic(); "
            f"print([a.agn_linear_ce_bytes(*{size}, k) for k in (0, 1)]); assert time.monotonic() - t < 1.0")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=120, cwd=ROOT)
    assert r.returncode == 0, r.stderr[-500:]
