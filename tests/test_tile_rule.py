"""The rule that picks a tile shape (csrc/gemm_launch.hpp), compiled for the host of a chip with 256 compute units and 160 KB of LDS and
asked for many shapes: what it picks has to be what then runs, and not a shape that its launcher turns down for another one."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

DRIVER = r"""
#include <cstdio>
#include "gemm_launch.hpp"

namespace semmoe {
int32_t device_info(DeviceInfo* out) { *out = DeviceInfo{256, 163840}; return SEMMOE_OK; }
int32_t allow_max_dynamic_lds(std::atomic<uint64_t>*, const void*) { return SEMMOE_OK; }
int tuning_value(int) { return -1; }
}  // namespace semmoe
using namespace semmoe;

// LDS of the launch that a tile id stands for, 0 for those that do not follow the number of groups or fit any
template <int MODE>
static size_t lds_of(int id, int nq) {
  switch (id) {
    case 22: return W4Cfg<MODE, 64, 2, 2>::kLdsBytes;
    case 33: return W4Cfg<MODE, 64, 3, 2, 2>::lds_bytes(nq);
    case 30: case 34: return StreamCfg<MODE, 2, 4>::lds_bytes(nq);
    case 32: case 35: return StreamCfg<MODE, 4, 4>::lds_bytes(nq);
    default: return 0;
  }
}

template <int MODE>
static int ask() {
  int bad = 0, picked = 0, offsets = 0;
  for (int nq : {1, 8, 64, 128, 256, 285, 286, 287, 288, 300, 382, 383, 384, 400, 512})
    for (int est : {1, 8, 16, 24, 36, 40, 95, 96, 160, 191, 192, 200, 300, 383, 384, 1000})
      for (int K : {200, 400, 512, 720, 1024, 1440, 2048, 2880, 4096})
        for (int N : {256, 512, 2880})
          for (int all : {0, 1}) {
            GemmArgs a{};
            a.offsets = &offsets; a.nq = nq; a.K = K; a.N = N;
            const int id = default_tile(a, nq * est * (all ? 1 : 16), est, kPaired<MODE> ? 2 * N : N, kI8<MODE>);
            picked += id == 33;
            if (lds_of<MODE>(id, nq) > 163840) {
              if (bad++ < 20) std::printf("mode %d: %d groups of %d rows, K %d, N %d, all %d: tile %d needs %zu bytes\n", MODE, nq, est, K, N, all, id, lds_of<MODE>(id, nq));
            }
          }
  std::printf("mode %d: %d of 256 x 128\n", MODE, picked);
  return bad;
}

int main() {
  const int bad = ask<kModeSwiglu>() + ask<kModeStore>() + ask<kModeSwigluI8>() + ask<kModeStoreI8>();
  return bad != 0;
}
"""


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    d = tmp_path_factory.mktemp("tile_rule")
    (d / "rule.hip").write_text(DRIVER)
    subprocess.run([HIPCC, "-O1", "-std=c++17", "-w", "--offload-host-only", "-I" + os.path.join(ROOT, "include"),
                    "-I" + os.path.join(ROOT, "paper_2503_04398_amd", "csrc"), str(d / "rule.hip"), "-o", str(d / "rule")], check=True)
    return str(d / "rule")


def test_the_rule_picks_what_fits(driver):
    r = subprocess.run([driver], stdout=subprocess.PIPE, text=True, timeout=120)
    assert r.returncode == 0, r.stdout[:3000]
