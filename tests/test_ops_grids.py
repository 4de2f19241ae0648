"""The grids of the operators' launches, on the host: no dimension of a launch reaches 2^32
threads, whatever the size of its workgroups, and every workgroup has a place."""
import os
import subprocess

from paper_2607_11262_amd import build

SOURCE = r"""
#include <hip/hip_runtime.h>

#include <cstdio>
#include <initializer_list>

#include "gts_ops.h"

template <uint32_t THREADS>
int check() {
  const uint64_t row = gts::kGridRow<THREADS>;
  int bad = 0;
  for (const uint64_t base : std::initializer_list<uint64_t>{1, row / 2, row, 2 * row, 7 * row, 1 << 22, 1 << 23, 1ull << 31})
    for (int64_t d = -2; d <= 2; ++d) {
      const uint64_t blocks = base + d;
      if ((int64_t)blocks < 1 || blocks > 1ull << 31) continue;
      const dim3 g = gts::grid_of<THREADS>(blocks);
      const bool ok = (uint64_t)g.x * THREADS < 1ull << 32 && g.y >= 1 && g.y <= 65535 && g.z == 1 &&
                      (uint64_t)g.x * g.y >= blocks && (uint64_t)g.x * (g.y - 1) < blocks && (g.y == 1 || g.x == row);
      if (!ok) {
        printf("%u threads, %llu workgroups: %u x %u\n", THREADS, (unsigned long long)blocks, g.x, g.y);
        ++bad;
      }
    }
  return bad;
}

int main() { return check<256>() + check<512>() + check<1024>() ? 1 : 0; }
"""


def test_no_launch_reaches_2_to_the_32_threads(tmp_path):
    src, exe = tmp_path / "grids.hip", str(tmp_path / "grids")
    src.write_text(SOURCE)
    subprocess.check_call([build.HIPCC, "-O1", "-std=c++17", f"--offload-arch={build.ARCH}", "-I", build.CSRC, str(src), "-o", exe])
    r = subprocess.run([exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
