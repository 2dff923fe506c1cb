"""A finishing warp's staged tile of the output layer's products (csrc/linear_ce_gemm.cu, Writer): bulk stores read
it after the warp has gone on, so whatever overwrites it has to wait for those that still do.  The struct's own
source is compiled here for the host with a stand-in for the copy engine that reads as late as the waits allow and
reports a tile that changed in between.  What a tile goes through: the ways out of a launch's products, one
after the other (of one product in a launch of its own, of two in dw's and dx's joint launch)."""

import itertools
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1710_02368_gb300", "csrc")

PROGRAM = r"""
#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <deque>
#include <algorithm>
using std::min;
typedef __nv_bfloat16 bf16;
#define AGN_ST(p, v) (void)(*(p) = (v))
#define __syncwarp() ((void)0)
#define __all_sync(m, p) (p)
#define __shfl_sync(m, v, l) (v)
#undef __device__
#define __device__
#undef __forceinline__
#define __forceinline__ inline

// The bulk stores that have not read their source yet, oldest first: what it was when they were issued.
struct Store { const uint8_t* src; int bytes; uint8_t was[4096]; };
static std::deque<Store> g_under_way, g_open;
static int g_bytes = 0, g_changed = 0;
static void read_all_but(size_t left) {
  for (; g_under_way.size() > left; g_under_way.pop_front()) {
    const Store& s = g_under_way.front();
    if (std::memcmp(s.src, s.was, s.bytes)) ++g_changed;
  }
}
namespace tc {
static void fence_proxy_async_smem() {}
static void store(const void* src) {
  Store s;
  s.src = (const uint8_t*)src;
  s.bytes = g_bytes;
  std::memcpy(s.was, src, g_bytes);
  g_open.push_back(s);
}
static void tma_store_2d(const CUtensorMap*, const void* src, int, int) { store(src); }
static void tma_add_2d(const CUtensorMap*, const void* src, int, int) { store(src); }
static void bulk_commit() { g_under_way.insert(g_under_way.end(), g_open.begin(), g_open.end()); g_open.clear(); }
static void bulk_wait_read() { read_all_but(0); }
static void bulk_wait_read_1() { read_all_but(1); }
}
@SOURCE@
int main(int argc, char** argv) {   // ways: b bf16, f fp32, B and F the same transposed, r and R rows of bf16 and fp32
  alignas(1024) static uint8_t tile[4096];
  alignas(16) static float out[64 * 64];
  Writer w{};
  w.tile = tile;
  float value = 1.f;
  for (const char* c = argv[1]; *c; ++c) {
    float v[32];
    uint32_t words[16];
    for (int i = 0; i < 32; ++i) v[i] = value;
    for (int i = 0; i < 16; ++i) words[i] = (uint32_t)value * 0x10001u;
    value += 1.f;
    g_bytes = *c == 'b' || *c == 'B' ? 2048 : 4096;
    if (*c == 'b') w.put_bf16(words, 0, 0);
    else if (*c == 'f') w.put_fp32(v, 0, 0, false);
    else if (*c == 'B') w.put_transposed<bf16>(v, 0, 0, false);
    else if (*c == 'F') w.put_transposed<float>(v, 0, 0, true);
    else if (*c == 'r') w.put_rows<bf16>(v, (bf16*)out, 0, 1, 32, false);
    else if (*c == 'R') w.put_rows<float>(v, out, 0, 1, 32, true);
    else return 99;
  }
  read_all_but(0);
  return g_changed ? 1 : 0;
}
"""


@pytest.fixture(scope="module")
def model(tmp_path_factory):
    nvcc = shutil.which("nvcc") or "/usr/local/cuda/bin/nvcc"
    if not os.path.exists(nvcc):
        pytest.skip("no nvcc")
    text = open(os.path.join(CSRC, "linear_ce_gemm.cu")).read()
    parts = [re.search(pattern, text, re.S | re.M).group(0) for pattern in (
        r"^template <int kRow>\n__device__[^\n]*staged_at.*?^}\n", r"^__device__[^\n]* pack2\(.*?^}\n", r"^struct Writer {.*?^};\n")]
    where = tmp_path_factory.mktemp("writer")
    src, exe = where / "writer.cu", where / "writer"
    src.write_text(PROGRAM.replace("@SOURCE@", "".join(parts)))
    subprocess.run([nvcc, "-std=c++17", "-O1", "-w", "-gencode", "arch=compute_103a,code=sm_103a", str(src), "-o", str(exe)],
                   check=True)
    return str(exe)


def overwritten(model, ways):
    rc = subprocess.run([model, ways]).returncode
    assert rc in (0, 1)
    return rc == 1


def test_one_way_alone(model):
    for way in "bfBFrR":
        assert not overwritten(model, way * 9), way


@pytest.mark.parametrize("rows", "rR")
@pytest.mark.parametrize("way", "bfBF")
def test_rows_after_bulk_stores(model, way, rows):
    """Rows one by one through a tile that the stores of the product before may still read."""
    for n in (1, 2, 3):
        assert not overwritten(model, way * n + rows + way * n + rows + way)


def test_stores_of_all_kinds_in_turn(model):
    """Half a tile of bf16 after a whole one of fp32 and the other way round, also after rows."""
    for n in (2, 3, 4):
        for ways in itertools.product("bfBF", repeat=n):
            assert not overwritten(model, "".join(ways)), ways
            assert not overwritten(model, "".join(ways) + "r" + "".join(ways)), ways
