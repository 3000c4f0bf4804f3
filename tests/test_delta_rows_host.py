"""Rows of the gated delta rule's chunks up to the 2^31 - 1 that a call may have, without a GPU: the kernels' own expressions,
evaluated as constants by the host's compiler, which refuses a sum that passes 32 bits."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_15437_amd", "csrc")

CHECKS = r"""
#include "delta_rows.hpp"
using namespace mmbev;
constexpr int32_t kMost = INT32_MAX;
// every chunk's rows from lo to hi, each once: those that are there, and the row that a thread without one reads instead
constexpr bool whole(int32_t lo, int32_t hi) {
  const int32_t n = delta_chunks(lo, hi);
  int64_t rows = 0;
  for (int32_t c = n > 2 ? n - 2 : 0; c < n; ++c) {
    const int32_t s0 = delta_chunk(lo, c);
    if (s0 < lo || s0 >= hi) return false;
    for (int i = 0; i < kDeltaRows; ++i) {
      const bool there = delta_row_there(s0, i, hi);
      const int32_t row = delta_row(s0, i, hi);
      if (there != ((int64_t)s0 + i < hi) || row < lo || row >= hi || (there && row != s0 + i)) return false;
      rows += there;
    }
  }
  const int64_t before = n > 2 ? (int64_t)(n - 2) * kDeltaRows : 0;
  return before + rows == (int64_t)hi - lo;
}
static_assert(delta_chunks(7, 7) == 0 && delta_chunks(0, 1) == 1 && delta_chunks(0, 32) == 1 && delta_chunks(0, 33) == 2, "");
static_assert(delta_chunks(0, kMost) == 1 << 26, "one run of all rows");
static_assert(whole(0, 1) && whole(5, 36) && whole(5, 37) && whole(5, 38) && whole(0, 100), "");
static_assert(whole(0, kMost) && whole(1, kMost) && whole(31, kMost), "runs of nearly all rows");
static_assert(whole(kMost - 1, kMost) && whole(kMost - 5, kMost) && whole(kMost - 32, kMost) && whole(kMost - 33, kMost), "the last rows");
static_assert(whole(kMost - 40, kMost - 3), "");
int main() {}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")
def test_rows_up_to_the_last(tmp_path):
    src = tmp_path / "rows.cpp"
    src.write_text(CHECKS)
    r = subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-fsyntax-only", "-I" + CSRC, str(src)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    # the same with a sum of rows in the place of a comparison of what is left does not pass
    bad = (tmp_path / "delta_rows.hpp")
    text = open(os.path.join(CSRC, "delta_rows.hpp")).read()
    for right, wrong in (("(hi - lo) / kDeltaRows + ((hi - lo) % kDeltaRows != 0)", "(hi - lo + kDeltaRows - 1) / kDeltaRows"),
                         ("i < hi - s0;", "s0 + i < hi;"), ("s0 + (i < hi - s0 - 1 ? i : hi - s0 - 1)", "s0 + i < hi - 1 ? s0 + i : hi - 1")):
        assert right in text
        bad.write_text(text.replace(right, wrong))
        r = subprocess.run(["g++", "-std=c++17", "-fsyntax-only", "-I" + str(tmp_path), str(src)], capture_output=True, text=True)
        assert r.returncode != 0 and "overflow" in r.stderr, right
