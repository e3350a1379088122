"""The numbers that launches mark their finished work with in an unwritten workspace (csrc/laq_marks.h; no GPU needed)."""
import os
import subprocess

import pytest

MAIN = r"""
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <thread>
#include "laq_marks.h"
using namespace laq;
int main(int argc, char** argv) {
  if (!strcmp(argv[1], "from")) {                      // start, how many
    MarkNumbers m(strtoull(argv[2], nullptr, 0));
    for (int i = 0; i < atoi(argv[3]); ++i) printf("%016llx\n", (unsigned long long)m.next());
    return 0;
  }
  static MarkNumbers m;                                // as the library has it, from two threads
  unsigned long long got[2][2000];
  const auto take = [&](int t) { for (unsigned long long& x : got[t]) x = m.next(); };
  std::thread a(take, 0), b(take, 1);
  a.join(), b.join();
  for (const auto& g : got) for (unsigned long long x : g) printf("%016llx\n", x);
  return 0;
}
"""


@pytest.fixture(scope="module")
def numbers(repo_root, tmp_path_factory):
    d = tmp_path_factory.mktemp("marks")
    src, exe = d / "marks.cpp", d / "marks"
    src.write_text(MAIN)
    subprocess.run([os.environ.get("CXX", "g++"), "-std=c++17", "-O1", "-Wall", "-pthread", "-I", os.path.join(repo_root, "paper_2505_20334_amd", "csrc"),
                    "-o", str(exe), str(src)], check=True)

    def run(*args):
        r = subprocess.run([str(exe)] + [str(a) for a in args], capture_output=True, text=True, timeout=60)
        assert r.returncode == 0
        return [int(x, 16) for x in r.stdout.split()]
    return run


# around 0, around the wrap of 32 and of 64 bits, and from anywhere
@pytest.mark.parametrize("start", [0, 1, 2 ** 32 - 5000, 2 ** 63 - 5000, 2 ** 64 - 5000, 0x243F6A8885A308D3])
def test_no_small_integer_and_no_number_beside_a_zero_is_a_mark(numbers, start):
    got = numbers("from", start, 200000)
    assert len(set(got)) == 200000                     # no launch has another's
    assert min(got) >= 1 << 32                         # (0, which clears a mark, among those that are none)
    # all 64 bits are used: each is set in half of the numbers, to within 6 standard deviations
    for bit in range(64):
        assert abs(sum(x >> bit & 1 for x in got) - 100000) < 6 * 200000 ** 0.5 / 2


def test_processes_and_threads_have_their_own(numbers):
    first, second = numbers("own"), numbers("own")
    assert len(set(first + second)) == 8000
