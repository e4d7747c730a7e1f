"""The search for an id's first sorted token, up to the most tokens that a plan takes: compiled for the host, over keys
that are a function of their place (CPU only)."""
import os
import shutil
import subprocess

import pytest

from test_kernel_source import CSRC, source

PROGRAM = r"""
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include "search.cuh"
int main() {
  const int sizes[] = {0, 1, 2, 4096, 1 << 30, (1 << 30) + 1, 0x7fffffff - 4096, 0x7fffffff};
  for (int n : sizes)
    for (uint32_t per : {1u, 127u, 1u << 20}) {  // neighbours with the same key
      auto key = [&](int i) {
        if (i < 0 || i >= n) {
          std::printf("read at %d of %d\n", i, n);
          std::exit(1);
        }
        return (uint32_t)i / per;
      };
      const uint32_t last = n ? (uint32_t)(n - 1) / per : 0;
      for (uint32_t v : {0u, 1u, last / 2, last - (last > 0), last, last + 1}) {
        const uint64_t first = (uint64_t)v * per, want = first < (uint64_t)n ? first : (uint64_t)n;
        const int got = dpc::lower_bound(key, n, v);
        if ((uint64_t)got != want) {
          std::printf("%d of %d for %u\n", got, n, v);
          return 1;
        }
      }
    }
  return 0;
}
"""


def test_search_near_the_largest_int(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "search.cpp", tmp_path / "search"
    src.write_text(PROGRAM)
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout


def test_the_plan_uses_it():
    src = source("embed.cu")
    assert "dpc::lower_bound(" in src and "(lo + hi) >> 1" not in src
    assert os.path.exists(os.path.join(CSRC, "search.cuh"))
