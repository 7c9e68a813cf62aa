"""The grid of the slot map's own launch, on the host."""
import os
import shutil
import subprocess

import pytest

from paper_2606_05742_amd import build

GRID = r"""
#include <hip/hip_runtime.h>
#include <climits>
#include <cstdio>
#include "kv4.h"
using namespace adapld;
int main() {
  constexpr long long per = kKv4SlotsPerBlock;
  static_assert(kv4_slot_blocks(INT_MAX) == (INT_MAX + per - 1) / per, "the largest slot map");
  for (long long n : {1ll, per - 1, per, per + 1, 5 * per, INT_MAX - per, INT_MAX - per + 1, INT_MAX - 1ll, (long long)INT_MAX}) {
    const long long blocks = kv4_slot_blocks((int)n);
    if (blocks * per < n || (blocks - 1) * per >= n) return 1;
    if (blocks * per - 1 > INT_MAX) return 2;      // the kernel's index of a slot is an int
    if (blocks * (per / 4) >= 1ll << 32) return 3; // threads of a launch
  }
  puts("ok");
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_blocks_cover_the_longest_slot_map(tmp_path):
    """Blocks for N slots of a sequence, up to the largest N that the entry
    point takes, where N plus a block no longer fits 31 bits."""
    src, exe = tmp_path / "grid.cpp", tmp_path / "grid"
    src.write_text(GRID)
    rocm = os.path.dirname(os.path.dirname(os.path.realpath(build.hipcc())))
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(rocm, "include"), "-I",
                    build.INCLUDE, "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and r.stdout == "ok\n", r.returncode
