"""The range that a search over histograms narrows, compiled for the host: it ends
whatever the search before it gave, a search that found nothing among them."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_19889_amd", "csrc")

PROGRAM = r"""
#include <cstdio>
#include <random>
#include "search_range.h"
using axon::BINS;
using axon::KeyRange;

#define CHECK(x) if (!(x)) { printf("%s: %u .. %u entry %d\n", #x, r.lo, r.hi, at); return 1; }

int main() {
  std::mt19937_64 g(1);
  const uint32_t edges[] = {0, 1, 2047, 2048, 2049, 4095, 4096, 1u << 21, (1u << 31) - 1, 1u << 31, 0xfffffffeu, 0xffffffffu};
  for (int i = 0; i < 200000; ++i) {
    uint32_t a = i % 3 ? (uint32_t)g() : edges[g() % 12], b = i % 5 ? (uint32_t)g() >> (g() % 32) : edges[g() % 12];
    KeyRange r{a < b ? a : b, a < b ? b : a};
    for (int round = 0;; ++round) {
      const KeyRange was = r;
      const int s = r.shift();
      int at = -1;
      CHECK((r.hi - r.lo) >> s < (uint32_t)BINS && (s == 0 || (r.hi - r.lo) >> (s - 1) >= (uint32_t)BINS));
      for (int wrong : {-1, -2147483647 - 1, (int)BINS, 2147483647, BINS - 2 - (int)((r.hi - r.lo) >> s)}) {
        at = wrong;  // (the last one: the bin behind the range's)
        CHECK(!r.narrow(wrong) && r.lo == was.lo && r.hi == was.hi);
      }
      // the keys of an entry are those of its bin
      const uint32_t key = was.lo + (was.hi - was.lo ? (uint32_t)(g() % ((uint64_t)(was.hi - was.lo) + 1)) : 0);
      at = BINS - 1 - (int)((key - was.lo) >> s);
      CHECK(r.narrow(at));
      CHECK(r.lo >= was.lo && r.hi <= was.hi && r.lo <= key && key <= r.hi && ((r.lo - was.lo) >> s) == ((r.hi - was.lo) >> s));
      CHECK(r.lo == was.lo || ((r.lo - 1 - was.lo) >> s) < ((key - was.lo) >> s));
      CHECK(r.hi == was.hi || ((r.hi + 1 - was.lo) >> s) > ((key - was.lo) >> s));
      if (r.lo == r.hi) break;
      CHECK(r.hi - r.lo < was.hi - was.lo && round < 3);
    }
  }
  return 0;
}
"""


def test_a_search_ends_whatever_it_finds(tmp_path):
    src, exe = tmp_path / "range.cpp", tmp_path / "range"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    done = subprocess.run([str(exe)], capture_output=True, text=True)
    assert done.returncode == 0, done.stdout
