// Rows of strided tensors [B, H, n, d] whose last axis is dense, on the host (no HIP
// headers needed, so that the checks can be tested on the CPU).
#pragma once

#include <algorithm>
#include <array>
#include <utility>

namespace attn {

struct Strides {
  long long b, h, t;   // elements between sequences, heads, tokens; not negative, 0 along an axis of one entry
};

// The caller's strides (sequence, head, token), or those of a dense [B, H, n, d].
// That of an axis of one entry says nothing.
inline Strides strides_of(const long long* s, int B, int H, int n, int d) {
  Strides r = {(long long)H * n * d, (long long)n * d, d};
  if (s) r = {s[0], s[1], s[2]};
  if (B == 1) r.b = 0;
  if (H == 1) r.h = 0;
  if (n == 1) r.t = 0;
  return r;
}
// Rows start at multiples of 16 bytes.
inline bool aligned(const Strides& s, int elem) {
  const int m = 16 / elem;
  return s.b % m == 0 && s.h % m == 0 && s.t % m == 0;
}
inline bool fits(const Strides& s, int B, int H, int n) {   // offsets in 62 bits
  __int128 far = 0;
  for (const auto& [step, size] : {std::pair<long long, int>{s.b, B}, {s.h, H}, {s.t, n}}) {
    if (step < 0) return false;
    far += (__int128)step * (size - 1);
  }
  return far < ((__int128)1 << 60);
}

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

// Whether a row of a tensor [B, H, n, d] has an element among [lo, lo + size), counted from its start. As in rows_meet, from
// the largest step on only those rows matter that the smaller steps can still bring there.
inline bool rows_reach(const Strides& x, int B, int H, int n, int d, __int128 lo, __int128 size) {
  struct { __int128 step, last; } axis[3] = {{x.b, B - 1}, {x.h, H - 1}, {x.t, n - 1}};
  std::sort(axis, axis + 3, [](const auto& p, const auto& q) { return p.step > q.step; });
  const auto meet = [&](const auto& self, int k, __int128 at) -> bool {   // rows from `at` on
    if (k == 3) return at > lo - d && at < lo + size;
    const auto& a = axis[k];
    if (a.step == 0) return self(self, k + 1, at);
    __int128 reach = d - 1;
    for (int j = k + 1; j < 3; ++j) reach += axis[j].step * axis[j].last;
    const __int128 gap = lo - reach - at;   // from the first i with at + i step + reach >= lo
    for (__int128 i = gap > 0 ? (gap + a.step - 1) / a.step : 0; i <= a.last && at + i * a.step < lo + size; ++i)
      if (self(self, k + 1, at + i * a.step)) return true;
    return false;
  };
  return meet(meet, 0, 0);
}
// Whether tensors x [B, Hx, nx, d] and y [B, Hy, ny, d] of any lengths certainly meet: their first rows do, or one of them
// has no gaps and a row of the other reaches into it. y starts `delta` elements behind x.
inline bool ranges_meet(const Strides& x, int Hx, int nx, const Strides& y, int Hy, int ny, int B, int d, __int128 delta) {
  const auto dense = [&](const Strides& s, int H, int n) {
    const __int128 size = (__int128)B * H * n * d;
    const __int128 end = (__int128)s.b * (B - 1) + (__int128)s.h * (H - 1) + (__int128)s.t * (n - 1) + d;
    return end == size && writable(s, B, H, n, d) ? size : 0;   // (an input's rows may lie on each other)
  };
  if (delta < d && -delta < d) return true;
  const __int128 size_x = dense(x, Hx, nx), size_y = dense(y, Hy, ny);
  return (size_x > 0 && rows_reach(y, B, Hy, ny, d, -delta, size_x)) || (size_y > 0 && rows_reach(x, B, Hx, nx, d, delta, size_y));
}

}  // namespace attn
