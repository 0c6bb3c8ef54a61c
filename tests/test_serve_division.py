"""fast_div and fdiv of the serving kernels as they are compiled, on the host: exact for every divisor of 31 bits and
0 <= n < 2^31, tried at the multiples' neighbours, where a reciprocal too small or large would show."""
from __future__ import annotations

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")
PROGRAM = r"""
#include "launch.hpp"
#include <cstdio>
static long tried;
static bool exact(uint32_t d) {
  const lsa::FastDiv f = lsa::fast_div(d);
  const int64_t top = INT32_MAX;
  if (f.d != d || (unsigned __int128)top * f.mul >> 64) return false;
  auto ok = [&](int64_t n) { return n < 0 || n > top || (++tried, lsa::fdiv(f, (int)n) == (int)(n / d)); };
  for (int64_t k = 0; k < 70; ++k)          // multiples from all over the range
    for (int64_t n : {top / d * k / 69 * d, (top / d - k) * d, k * d})
      for (int64_t i = -2; i <= 2; ++i)
        if (!ok(n + i)) return false;
  return ok(top) && ok(0);
}
int main() {
  for (uint32_t d = 1; d < 5000; ++d)
    if (!exact(d)) return std::printf("%u\n", d), 1;
  uint32_t x = 1;
  for (int i = 0; i < 20000; ++i) {
    x = x * 1664525u + 1013904223u;
    const uint32_t d = (x >> 1) >> (i % 31);
    if (d && !exact(d)) return std::printf("%u\n", d), 1;
  }
  for (uint32_t p = 1; p < 31; ++p)
    for (int i = -1; i <= 1; ++i)
      if (!exact((1u << p) + i)) return std::printf("2^%u %+d\n", p, i), 1;
  if (!exact(INT32_MAX) || !exact(INT32_MAX - 1)) return std::printf("the largest\n"), 1;
  std::printf("%ld\n", tried);
}
"""


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.exists(os.path.join(ROCM, "include", "hip")), reason="needs g++ and HIP's headers")
def test_division_by_what_the_host_knows(tmp_path):
    (tmp_path / "t.cpp").write_text(PROGRAM)
    subprocess.run(["g++", "-O2", "-std=c++17", "-w", "-D__HIP_PLATFORM_AMD__", f"-I{os.path.join(ROCM, 'include')}",
                    f"-I{os.path.join(ROOT, 'paper_2608_01662_amd', 'csrc')}", str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t"),
                    f"-L{os.path.join(ROCM, 'lib')}", "-lamdhip64", f"-Wl,-rpath,{os.path.join(ROCM, 'lib')}"], check=True, timeout=120)
    r = subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and int(r.stdout) > 1_000_000, r.stdout
