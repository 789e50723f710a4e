"""The launch grid of the cache's prefill (csrc/gmc_cache_grid.h), on the CPU:
every row block of every head is taken once, few blocks have no work, and what
the argument checks admit fits a launch."""
import os
import shutil
import subprocess

import pytest

from paper_2608_02134_amd import binding as B

PROGRAM = r"""
#include <stdio.h>
#include <algorithm>
#include <vector>
#include "gmc_cache_grid.h"
using namespace gmc;

static int fail(const char* what, long long items, long long heads, long long x) {
  printf("%s: %lld items, %lld heads: %lld\n", what, items, heads, x);
  return 1;
}

int main() {
  // every item of every head once; the header's own bounds on blocks without work
  const int few[] = {1, 2, 3, 5, 7, 8, 9, 31, 32, 33, 34, 63, 64, 65, 66, 95, 100, 511, 512, 900};
  const int many[] = {1, 2, 3, 4, 8, 12, 28, 63, 64, 65, 200, 512, 2048};
  for (int items : few)
    for (int heads : many) {
      const PreGrid g = pre_grid(items, heads);
      if (g.run < 1 || g.run > 32) return fail("run", items, heads, g.run);
      std::vector<int> taken(static_cast<size_t>(items) * heads);
      long long worked = 0;
      for (long long x = 0; x < g.blocks; ++x) {
        int head = -1, item = -1;
        if (!pre_place(g, static_cast<unsigned>(x), heads, &head, &item)) continue;
        if (head < 0 || head >= heads || item < 0 || item >= items) return fail("out of range", items, heads, x);
        ++taken[static_cast<size_t>(head) * items + item];
        ++worked;
      }
      for (int n : taken)
        if (n != 1) return fail("taken", items, heads, n);
      if (worked != static_cast<long long>(items) * heads) return fail("worked", items, heads, worked);
      if (3 * (g.blocks - 7 * g.run) > 4 * worked) return fail("without work", items, heads, g.blocks - worked);
    }
  // as many blocks as a call may have: fewer than 2^32 threads of 256 a block, at most 65535 sequences of 256 heads
  for (long long items = 1; items <= kPreMaxBlocks; items = items < 3000 ? items + 1 : items * 5 / 4) {
    const long long heads = std::min(kPreMaxBlocks / items, 65535ll * 256);
    for (long long h = heads; h >= 1 && h > heads - 70; --h) {
      const PreGrid g = pre_grid(static_cast<int>(items), h);
      if (g.blocks * 256 >= 1ll << 32) return fail("threads", items, h, g.blocks);
      if (g.blocks < items * h) return fail("too few", items, h, g.blocks);
    }
  }
  printf("ok\n");
  return 0;
}
"""


def test_every_row_block_once_and_no_launch_too_large(tmp_path):
    cxx = shutil.which("g++") or shutil.which("clang++")
    if not cxx:
        pytest.skip("no C++ compiler")
    src, exe = tmp_path / "grid.cpp", tmp_path / "grid"
    src.write_text(PROGRAM)
    csrc = os.path.join(os.path.dirname(B.LIB_PATH), "csrc")
    subprocess.run([cxx, "-std=c++17", "-O2", "-Wall", "-Werror", "-I", csrc, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
