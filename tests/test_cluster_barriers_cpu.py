"""The aligned form of the cluster barrier asks for a converged warp; the loops before it are left by
the lanes of a warp on different trips (columns past the tile's last, rows past the matrix).  So each
use in csrc/ has a __syncwarp() directly before it."""

import os
import re

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1710_02368_gb300", "csrc")


def test_warps_converge_before_aligned_cluster_barriers():
    uses, bare = 0, []
    for name in sorted(os.listdir(CSRC)):
        text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
        for m in re.finditer(r"asm volatile\(\s*\"barrier\.cluster\.arrive[^\"]*\.aligned", text):
            uses += 1
            if not re.search(r"__syncwarp\(\);\s*$", text[:m.start()]):
                bare.append((name, text[:m.start()].count("\n") + 1))
    assert uses > 0 and not bare, bare
