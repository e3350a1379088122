"""The search of a workgroup's request (csrc/laq_find.h) with 64 lanes played on the host (no GPU needed)."""
import os
import subprocess

import pytest

MAIN = r"""
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>
#include "laq_find.h"
using namespace laq;

// As the kernels do it: the count of the lanes whose place lies before, unsigned as a device counts lanes.
template <typename Before>
static int find(int n, const Before& before) {
  Find f{0, n};
  for (int times = 0; f.n > 1; ++times) {
    unsigned count = 0;
    for (int lane = 0; lane < 64; ++lane) {
      if (!f.looks(lane)) continue;
      const long long i = f.lo + (long long)lane * f.step();
      if (i < 0 || i >= n) { printf("place %lld of %d\n", i, n); exit(2); }
      count += before(lane, (int)i);
    }
    const Find was = f;
    f.narrow((int)count);
    if (f.n < 1 || f.lo < was.lo || f.lo + (long long)f.n > was.lo + (long long)was.n || times > 6) { printf("left %d + %d of %d + %d\n", f.lo, f.n, was.lo, was.n); exit(3); }
  }
  if (f.lo < 0 || f.lo >= n) { printf("found %d of %d\n", f.lo, n); exit(4); }
  return f.lo;
}

int main() {
  std::mt19937 rng(7);
  std::vector<int> sizes{1, 2, 3, 63, 64, 65, 80, 127, 128, 129, 4095, 4096, 4097, 70000, 2147483647, 2147483646, 2147483584};
  for (int i = 0; i < 300; ++i) sizes.push_back(1 + (int)(rng() % (i % 2 ? 300 : 100000)));
  for (int n : sizes) {
    // places in order: the last one that lies before
    for (int i = 0; i < 40; ++i) {
      const int at = i == 0 ? 0 : i == 1 ? n - 1 : (int)(rng() % (unsigned)n);
      if (find(n, [&](int, int place) { return place <= at; }) != at) { printf("%d of %d\n", at, n); return 1; }
    }
    // none, all, and places in no order at all
    if (find(n, [](int, int) { return false; }) != 0 || find(n, [](int, int) { return true; }) != n - 1) return 5;
    for (int i = 0; i < 200; ++i) {
      const unsigned share = rng() % 5;
      find(n, [&](int, int) { return rng() % 4 < share; });
    }
    // many before at first, none of what is left
    int look = 0;
    find(n, [&](int lane, int) { look += lane == 0; return look < 2; });
  }
  return 0;
}
"""


def test_what_is_found_and_looked_at_lies_among_the_places(repo_root, tmp_path):
    src, exe = tmp_path / "find.cpp", tmp_path / "find"
    src.write_text(MAIN)
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-Wall", "-ftrapv", "-I",
                    os.path.join(repo_root, "paper_2505_20334_amd", "csrc"), "-o", str(exe), str(src)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=100)
    assert r.returncode == 0, r.stdout + r.stderr


@pytest.mark.parametrize("n,before,lo,left", [(80, 0, 0, 2), (80, 1, 0, 2), (80, 40, 78, 2), (2, 0, 0, 1), (2, 2, 1, 1), (129, 43, 126, 3), (130, 44, 129, 1)])
def test_one_look(repo_root, tmp_path, n, before, lo, left):
    src, exe = tmp_path / "look.cpp", tmp_path / "look"
    src.write_text('#include <cstdio>\n#include "laq_find.h"\nint main() { laq::Find f{0, %d}; f.narrow(%d); printf("%%d %%d", f.lo, f.n); }\n' % (n, before))
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-I", os.path.join(repo_root, "paper_2505_20334_amd", "csrc"), "-o", str(exe), str(src)], check=True)
    assert subprocess.run([str(exe)], capture_output=True, text=True, timeout=20).stdout == "%d %d" % (lo, left)
