"""Which sequence a packed row belongs to, whatever the offsets hold: the kernels' rule compiled for the host, behind a model of
the search over 64 lanes.  No GPU needed."""
import os
import subprocess

import pytest

from paper_2606_27748_amd import build as B

DRIVER = r"""
#include <algorithm>
#include <cstdio>
#include <random>
#include <vector>
#include "flex_rows.hpp"

// the search of the kernels: 64 probes a round
static int leading(const std::vector<int>& off, int B, int t) {
  int lo = 0, n = B;
  while (n > 0) {
    const int step = (n + 63) / 64;
    int c = 0;
    for (int l = 0; l < 64; ++l) {
      const int at = (l + 1) * step - 1;
      c += at < n && off[lo + std::min(at, n - 1)] <= t;
    }
    lo += c * step;
    n = step == 1 ? 0 : std::min(step, n - c * step);
  }
  return lo;
}

// rows that are answered wrongly: a sequence without the row, no way on, or, of offsets in order, another sequence
static long wrong(const std::vector<int>& off, int T, bool in_order) {
  const int B = (int)off.size() - 1;
  long bad = 0;
  for (int t = 0; t < T; ++t) {
    const int cnt = leading(off, B, t);
    if (cnt < 0 || cnt > B) { ++bad; continue; }
    const flex::RowSeq q = flex::row_seq(cnt, off[std::max(cnt - 1, 0)], off[cnt], B, T, t);
    bad += q.end <= t || q.end > T || q.b >= B;
    if (q.b >= 0) bad += q.first > t || q.first != off[q.b] || q.end != off[q.b + 1];
    if (!in_order) continue;
    int want = -1;
    for (int b = 0; b < B; ++b)
      if (off[b] <= t && t < off[b + 1]) want = b;
    bad += q.b != want;
    if (want < 0)
      for (int s = t; s < q.end; ++s)
        for (int b = 0; b < B; ++b) bad += off[b] <= s && s < off[b + 1];
  }
  return bad;
}

int main() {
  std::mt19937 rng(1);
  long bad = wrong({0, 200, 220, 60, 230}, 230, false);
  std::printf("%ld\n", bad);
  for (int k = 0; k < 6000; ++k) {
    const int sizes[] = {1, 2, 3, 4, 5, 8, 63, 64, 65, 70, 130, 300}, B = sizes[rng() % 12], T = 1 + rng() % (k % 2 ? 12 : 300);
    std::vector<int> off(B + 1);
    for (int& x : off) x = std::min(std::max((int)(rng() % (T + 40)) - 20, 0), T);   // as the kernels clamp them
    const bool in_order = k % 3 == 0;
    if (in_order) std::sort(off.begin(), off.end());
    const long w = wrong(off, T, in_order);
    if (w && !bad) std::printf("B %d, T %d, in order %d: %ld\n", B, T, in_order, w);
    bad += w;
  }
  std::printf("%ld\n", bad);
  return bad != 0;
}
"""


@pytest.mark.skipif(not os.path.exists(B.HIPCC), reason="needs hipcc")
def test_a_row_is_one_of_the_sequence_that_is_found(tmp_path):
    src, exe = tmp_path / "driver.hip", str(tmp_path / "driver")
    src.write_text(DRIVER)
    subprocess.run([B.HIPCC, "--offload-arch=gfx950", "--offload-host-only", "-O2", "-std=c++17", "-I", B.CSRC, str(src), "-o", exe],
                   check=True, capture_output=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout
