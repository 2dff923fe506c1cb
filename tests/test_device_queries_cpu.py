"""What csrc/ops.cuh asks of a device once (multiprocessors, resident clusters), compiled here with
fakes of the runtime's queries: an answer that is an error ends the call that got it and is not
kept, so the next call decides on the device's own answer; a right answer is asked for once."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1710_02368_gb300", "csrc")

PROGRAM = r"""
#include <cuda_runtime.h>
static int g_fail = 0, g_asked = 0;   // query number g_fail from here (1: the next) fails
static cudaError_t answer(int* n, int v) {
  ++g_asked;
  if (g_fail > 0 && --g_fail == 0) return cudaErrorUnknown;
  if (n) *n = v;
  return cudaSuccess;
}
template <typename K> static cudaError_t fake_clusters(int* n, K, const cudaLaunchConfig_t*) { return answer(n, 36); }
template <typename K> static cudaError_t fake_attribute(K, cudaFuncAttribute, int) { return answer(nullptr, 0); }
static cudaError_t fake_device_attribute(int* n, cudaDeviceAttr, int) { return answer(n, 152); }
#define cudaOccupancyMaxActiveClusters fake_clusters
#define cudaFuncSetAttribute fake_attribute
#define cudaDeviceGetAttribute fake_device_attribute
#include "ops.cuh"
#define CHECK(x) do { if (!(x)) return __LINE__; } while (0)
template <int> struct Tag {};
static void kern(int) {}
int main() {
  using namespace agn;
  int n = -7;
  for (int dev : {0, kMaxDevices - 1}) {
    g_fail = 1;
    CHECK(device_sms(dev, &n).code == AGN_E_CUDA);
    CHECK(device_sms(dev, &n).ok() && n == 152);
    g_asked = 0;
    CHECK(device_sms(dev, &n).ok() && n == 152 && g_asked == 0);
    // each of the queries behind the clusters fails once
    for (int c : {4, 8, 16}) {
      const int queries = 1 + 1 + (c > 8);
      for (int at = 0; at < queries; ++at) {
        g_fail = at + 1;
        CHECK(max_clusters<Tag<0>>(kern, 256, 1024, c, dev, &n).code == AGN_E_CUDA);
      }
      CHECK(max_clusters<Tag<0>>(kern, 256, 1024, c, dev, &n).ok() && n == 36);
      g_asked = 0;
      CHECK(max_clusters<Tag<0>>(kern, 256, 1024, c, dev, &n).ok() && n == 36 && g_asked == 0);
    }
    CHECK(max_clusters<Tag<1>>(kern, 256, 0, 4, dev, &n).ok() && g_asked == 1);   // another kernel
  }
  g_asked = 0;   // ordinals that are not kept
  for (int i = 0; i < 2; ++i) CHECK(device_sms(kMaxDevices, &n).ok() && max_clusters<Tag<0>>(kern, 256, 0, 4, kMaxDevices, &n).ok());
  CHECK(g_asked == 4);
  CHECK(!max_clusters<Tag<0>>(kern, 256, 0, 17, 0, &n).ok() && !max_clusters<Tag<0>>(kern, 256, 0, 1, 0, &n).ok());
  return 0;
}
"""


def test_failed_queries_are_returned_and_not_kept(tmp_path):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        pytest.skip("no nvcc")
    src, exe = tmp_path / "queries.cu", tmp_path / "queries"
    src.write_text(PROGRAM)
    subprocess.run([nvcc, "-std=c++17", "-O1", "--expt-relaxed-constexpr", "-gencode", "arch=compute_103a,code=sm_103a",
                    "-I", CSRC, "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)]).returncode == 0
