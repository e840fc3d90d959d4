// Rows of strided tensors [B, H, n, d] whose last axis is dense, on the host (no HIP
// headers needed, so that the checks can be tested on the CPU).
#pragma once

#include <algorithm>
#include <array>

namespace attn {

struct Strides {
  long long b, h, t;   // elements between sequences, heads, tokens; not negative, 0 along an axis of one entry
};

// Rows of a written tensor must not overlap: from the smallest stride on, each
// has to step over all that the smaller ones span.
inline bool writable(const Strides& s, int B, int H, int n, int d) {
  struct { long long step; int size; } dim[3] = {{s.b, B}, {s.h, H}, {s.t, n}};
  std::sort(dim, dim + 3, [](const auto& x, const auto& y) { return x.step < y.step; });
  __int128 span = d;
  for (const auto& x : dim) {
    if (x.size == 1) continue;
    if (x.step < span) return false;
    span += (__int128)x.step * (x.size - 1);
  }
  return true;
}

// Whether a row of x [B, Hx, n, d] and one of y [B, Hy, n, d], both writable, have an element in
// common; y starts `delta` elements behind x. Tensors that step alike (views of one buffer)
// are told exactly: along an axis rows differ by a number i of steps, and from the largest
// step on only those i matter that the smaller steps can still make up for. Of others the
// first rows are compared, and the first and last of one with all of the other if that has no
// gaps: any two tensors without gaps that reach into each other are found.
inline bool rows_meet(const Strides& x, int Hx, const Strides& y, int Hy, int B, int n, int d, __int128 delta) {
  struct Axis { __int128 step, lo, hi; };
  Axis axis[3] = {{x.b, 1 - B, B - 1}, {std::max(x.h, y.h), 1 - Hx, Hy - 1}, {x.t, 1 - n, n - 1}};
  __int128 ends_x = d, ends_y = d;
  for (const auto& [sx, sy, nx, ny] : {std::array<long long, 4>{x.b, y.b, B, B}, {x.h, y.h, Hx, Hy}, {x.t, y.t, n, n}}) {
    ends_x += (__int128)sx * (nx - 1);
    ends_y += (__int128)sy * (ny - 1);
  }
  if (delta >= ends_x || -delta >= ends_y) return false;
  if (x.b != y.b || x.t != y.t || (x.h != y.h && Hx > 1 && Hy > 1)) {
    if (delta < d && -delta < d) return true;
    const bool dense_x = ends_x == (__int128)B * Hx * n * d, dense_y = ends_y == (__int128)B * Hy * n * d;
    return (dense_x && (delta > -d || delta + ends_y < ends_x + d)) || (dense_y && (delta < d || delta + ends_y > ends_x - d));
  }
  std::sort(axis, axis + 3, [](const Axis& p, const Axis& q) { return p.step > q.step; });
  const auto meet = [&](const auto& self, int k, __int128 at) -> bool {
    if (k == 3) return at < d && -at < d;
    const Axis& a = axis[k];
    if (a.step == 0) return self(self, k + 1, at);
    __int128 reach = d - 1;
    for (int j = k + 1; j < 3; ++j) reach += axis[j].step * std::max(-axis[j].lo, axis[j].hi);
    // from the first i with at + i step >= -reach
    const __int128 gap = -reach - at;
    __int128 i = gap >= 0 ? (gap + a.step - 1) / a.step : -(-gap / a.step);
    for (i = std::max(i, a.lo); i <= a.hi && at + i * a.step <= reach; ++i)
      if (self(self, k + 1, at + i * a.step)) return true;
    return false;
  };
  return meet(meet, 0, delta);
}

}  // namespace attn
