"""Overlapping outputs of the rotation: the check (csrc/strides.hpp, compiled for the CPU)
against all pairs of rows, and the refusal of the C ABI and the Python form."""
import os
import shutil
import subprocess

import pytest

import paper_2609_33916_amd as pkg
from test_paged_host import FAKE, _ll, _rope

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_33916_amd", "csrc")

MAIN = r"""
#include <cstdio>
#include <cstdlib>
#include <random>
#include "strides.hpp"
using attn::Strides;
int main() {
  std::mt19937 g(7);
  auto pick = [&](int lo, int hi) { return lo + (int)(g() % (unsigned)(hi - lo + 1)); };
  int met = 0, apart = 0, refused = 0;
  for (int it = 0; it < 300000; ++it) {
    const int d = 4, B = pick(1, 3), n = pick(1, 4), Hx = pick(1, 4), Hy = pick(1, 4), H = Hx > Hy ? Hx : Hy;
    // the axes in a random order, each stepping over the smaller ones and a random gap
    int order[3] = {0, 1, 2}, size[3] = {B, H + pick(0, 4), n};
    for (int i = 2; i > 0; --i) std::swap(order[i], order[pick(0, i)]);
    long long step[3], span = d;
    for (int i : order) {
      step[i] = span + 4 * pick(0, 1);
      span = step[i] * size[i];
    }
    auto strides = [&](int h) { return Strides{B > 1 ? step[0] : 0, h > 1 ? step[1] : 0, n > 1 ? step[2] : 0}; };
    const Strides x = strides(Hx), y = strides(Hy);
    if (!attn::writable(x, B, Hx, n, d) || !attn::writable(y, B, Hy, n, d)) { ++refused; continue; }
    const long long delta = 4 * pick(-(int)span / 4 - 2, (int)span / 4 + 2) + (it % 8 == 0 ? pick(-3, 3) : 0);
    bool want = false;
    for (int b = 0; b < B; ++b) for (int i = 0; i < Hx; ++i) for (int t = 0; t < n; ++t)
      for (int c = 0; c < B; ++c) for (int j = 0; j < Hy; ++j) for (int u = 0; u < n; ++u)
        want = want || std::llabs(delta + c * y.b + j * y.h + u * y.t - b * x.b - i * x.h - t * x.t) < d;
    if (attn::rows_meet(x, Hx, y, Hy, B, n, d, delta) != want) {
      std::printf("B %d n %d H %d %d steps %lld %lld %lld delta %lld: %d\n", B, n, Hx, Hy, step[0], step[1], step[2], delta, want);
      return 1;
    }
    ++(want ? met : apart);
  }
  // far apart, and sizes whose products pass 64 bits: no endless search
  const Strides far{1LL << 50, 128, 1LL << 20};
  if (!attn::rows_meet(far, 64, far, 64, 1 << 9, 1 << 20, 128, 128) || attn::rows_meet(far, 64, far, 64, 1 << 9, 1 << 20, 128, 64 * 128))
    return 1;
  // other strides, two without gaps (all are told), then one with (none is called apart or met wrongly
  // where its first or last row decides)
  for (int it = 0; it < 100000; ++it) {
    const int d = 4, B = pick(1, 3), n = pick(1, 4), Hx = pick(1, 4), Hy = pick(1, 4), gap = it % 2 ? 4 * pick(0, 3) : 0;
    const Strides x{B > 1 ? Hx * n * d : 0, Hx > 1 ? n * d : 0, n > 1 ? d : 0};
    const long long row = Hy * d + gap;
    const Strides y{B > 1 ? n * row : 0, Hy > 1 ? d : 0, n > 1 ? row : 0};
    const long long delta = pick(-200, 200);
    bool want = false, edge = std::llabs(delta) < d;
    const long long end = delta + (B * n - 1) * row + Hy * d;   // of y's last row
    for (int k = 0; k < B * Hx * n; ++k) {
      for (int c = 0; c < B * n; ++c) for (int j = 0; j < Hy; ++j) want = want || std::llabs(delta + c * row + j * d - k * d) < d;
      edge = edge || std::llabs(delta - k * d) < d || std::llabs(end - d - k * d) < d;
    }
    for (int swap = 0; swap < 2; ++swap) {
      const bool got = swap ? attn::rows_meet(y, Hy, x, Hx, B, n, d, -delta) : attn::rows_meet(x, Hx, y, Hy, B, n, d, delta);
      if ((got && !want) || (!got && (gap == 0 ? want : edge))) {
        std::printf("B %d n %d H %d %d gap %d delta %lld: %d, not %d\n", B, n, Hx, Hy, gap, delta, got, want);
        return 1;
      }
    }
  }
  if (refused || met < 1000 || apart < 1000) return 1;
  std::printf("ok\n");
  return 0;
}
"""


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_rows_meet(tmp_path):
    src, exe = tmp_path / "strides.cpp", tmp_path / "strides"
    src.write_text(MAIN)
    subprocess.run(["g++", "-std=c++17", "-O2", "-Wall", "-Werror", "-fsanitize=undefined", "-I", CSRC, str(src), "-o", str(exe)],
                   check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=100)
    assert out.returncode == 0 and out.stdout.strip() == "ok" and not out.stderr, out.stdout + out.stderr


@pytest.mark.parametrize("fn", ["attn_rope", "attn_rope_bwd"])
def test_outputs_that_overlap_are_refused(fn):
    """q's output on k's: the same place, a head in common, one inside the other's rows."""
    L = pkg.lib()
    B, Hq, Hk, n, d = 2, 4, 2, 8, 64
    assert _rope(L, fn) == -7                                       # dense, both at one address
    assert _rope(L, fn, ko=FAKE + 2 * B * Hq * n * d - 16) == -7    # k's first row begins in q's last
    row = (Hq + 2 * Hk) * d
    packed = _ll(*[n * row, d, row] * 4)
    for head in range(1 - Hk, Hq):
        assert _rope(L, fn, qo=FAKE, ko=FAKE + 2 * head * d, strides=packed) == -7, head
    assert _rope(L, fn, qo=FAKE, ko=FAKE + 2 * (3 * row + d), strides=packed) == -7
    assert "overlap" in pkg.attn_strerror(-7)
