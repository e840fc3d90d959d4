// Rotary positions: a head's columns are taken in pairs, and pair i of the token
// at position p is turned by the angle p f_i and stretched by an amplitude a:
//   u' = a (u cos t - w sin t),  w' = a (w cos t + u sin t),  t = p f_i.
// The first r columns are paired, (x_i, x_{i + r/2}) or interleaved
// (x_{2i}, x_{2i+1}); columns from r on stay as they are. The transpose of a
// turn is the turn back, so the gradient is the same with sin t negated. A
// scaling for long contexts is a choice of the f_i and of a, made by the caller.
//
// The f_i are float64 and the angle is reduced to a fraction of a circle in 64
// bits: in 32 bits the angle of position 10^6 would be off by 0.03 radian. The
// sine and cosine of the remaining fraction are float32 (far below the rounding of a
// bfloat16 result and at that of a float32 one); where the result is rounded to 4 bits
// they are float64 (see Quant4).
#pragma once

#include "common.hpp"
#include "pages.hpp"
#include "strides.hpp"

namespace attn {

struct Rotation {
  const double* freqs;   // [r / 2] radians per position
  int r;                 // columns that turn (a multiple of 16), 0: none
  float amplitude;
};

// Every operation here is rounded as written (no contraction of the compiler's choice),
// so that all kernels turn a row to the same bits.

// p f, as a fraction of a circle in [-1/2, 1/2]
__device__ __forceinline__ double turn(int p, double f) {
#pragma clang fp contract(off)
  const double x = (double)p * f * 0.15915494309189535;   // 1 / (2 pi)
  return x - rint(x);
}
// a cos(p f), a sin(p f): with q the nearest quarter turn and z the rest, |z| <= pi / 4,
// cos z = 1 + (cos z - 1) and sin z = z + (sin z - z), the parentheses, small, by their
// Taylor series (to z^10 and z^9: the next terms are below 2^-33 and 2^-28). a and a z,
// which is rounded from 64 bits, come in with the last addition. Off by 7.9e-8 at most
// (a = 1), the device library's sine and cosine of a fraction in 32 bits by 1.1e-7; a
// turned float32 row's error is 3.9e-8 of its length, with those 5.2e-8.
__device__ __forceinline__ void turn_cs(int p, double f, float a, float& c, float& s) {
#pragma clang fp contract(off)
  const double y = 4.0 * turn(p, f), q = rint(y), r = y - q;
  const float z = (float)(r * 1.5707963267948966), az = (float)(r * (1.5707963267948966 * (double)a)), z2 = z * z;
  const float e = fmaf(z2, fmaf(z2, fmaf(z2, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6) * z2;
  const float g = fmaf(z2, fmaf(z2, fmaf(z2, fmaf(z2, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -.5f) * z2;
  const float sz = fmaf(az, e, az), cz = fmaf(a, g, a);
  const int k = (int)q;   // -2 .. 2
  c = k & 1 ? sz : cz;
  s = k & 1 ? cz : sz;
  c = (k + 1) & 2 ? -c : c;
  s = k & 2 ? -s : s;
}
__device__ __forceinline__ void turn_cs(int p, double f, float a, double& c, double& s) {
#pragma clang fp contract(off)
  double c0, s0;
  sincospi(2.0 * turn(p, f), &s0, &c0);
  c = c0 * (double)a;
  s = s0 * (double)a;
}

// (u, w) turned by the angle of (c, s)
template <typename R> __device__ __forceinline__ void turn_pair(R& u, R& w, R c, R s) {
#pragma clang fp contract(off)
  const R x = u, y = w, ys = y * s, xs = x * s;
  u = __builtin_elementwise_fma(x, c, -ys);
  w = __builtin_elementwise_fma(y, c, xs);
}

// 16 bytes of a row and its values
template <typename T> struct Chunk;
template <> struct Chunk<bf16> {
  static constexpr int N = 8;
  __device__ __forceinline__ static void get(u32x4 x, float (&v)[8]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      v[2 * e] = __uint_as_float(x[e] << 16);
      v[2 * e + 1] = __uint_as_float(x[e] & 0xffff0000u);
    }
  }
  __device__ __forceinline__ static u32x4 put(const float (&v)[8]) {
    u32x4 x;
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = pack_bf16x2(v[2 * e], v[2 * e + 1]);
    return x;
  }
};
template <> struct Chunk<float> {
  static constexpr int N = 4;
  __device__ __forceinline__ static void get(u32x4 x, float (&v)[4]) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __uint_as_float(x[e]);
  }
  __device__ __forceinline__ static u32x4 put(const float (&v)[4]) {
    return (u32x4){__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  }
};

// A thread's two 16-byte chunks of a row and their N pairs. Thread j of the d / 2N
// that share a row takes chunk j of each half of the rotated columns; past them, two
// neighbouring chunks to copy. A pair of halves (i, i + r/2), or a neighbouring pair
// inside a chunk, never leaves its thread, so a row may be turned in place, and
// each load of a wave covers whole 64-byte pieces.
template <typename T, bool INTER> struct PairChunks {
  static constexpr int N = Chunk<T>::N;
  int col[2];
  bool turns;
  float c[N], s[N];
  __device__ __forceinline__ PairChunks(const Rotation& rot, int j) {
    turns = j < rot.r / (2 * N);
    col[0] = turns ? N * j : 2 * N * j;
    col[1] = turns ? rot.r / 2 + N * j : 2 * N * j + N;
  }
  // position p; `sign` of the sine
  __device__ __forceinline__ void angles(const Rotation& rot, int j, int p, float sign) {
#pragma unroll
    for (int e = 0; e < N; ++e) c[e] = 1.f, s[e] = 0.f;
    if (turns) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int i = !INTER ? N * j + e : (e < N / 2 ? N * j / 2 : rot.r / 4 + N * j / 2 - N / 2) + e;
        turn_cs(p, rot.freqs[i], rot.amplitude, c[e], s[e]);
        s[e] *= sign;
      }
    }
  }
  __device__ __forceinline__ void apply(u32x4& xa, u32x4& xb) const {
    if (!turns) return;   // the copied columns keep their bits
    float a[N], b[N];
    Chunk<T>::get(xa, a);
    Chunk<T>::get(xb, b);
    if (INTER) {
#pragma unroll
      for (int e = 0; e < N / 2; ++e) {
        turn_pair(a[2 * e], a[2 * e + 1], c[e], s[e]);
        turn_pair(b[2 * e], b[2 * e + 1], c[N / 2 + e], s[N / 2 + e]);
      }
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) turn_pair(a[e], b[e], c[e], s[e]);
    }
    xa = Chunk<T>::put(a);
    xb = Chunk<T>::put(b);
  }
};

// ---------------------------------------------------------------- attn_rope --
struct RopeArgs {
  const void *q, *k;
  void *qo, *ko;
  Strides qs, ks, qos, kos;
  const int* pos;          // positions, or null: start + token
  long long pos_stride;    // entries between sequences (0: shared)
  int start;
  Rotation rot;
  int Hq, Hk, n, d;
  int tokens;              // B n
  int hgroup;              // heads (q's, then k's) per workgroup
  float sign;              // of the sine: -1 for the gradient
};

// Bound by memory: every element is read and written once. The angles belong to a
// token, not to a head, so a thread keeps its pairs' sines and cosines in registers
// and walks over the heads, U at a time with all their loads in flight. 2 sequences
// of 16384 tokens, 64 heads, d = 128, bfloat16: 195 us, 5.5 TB/s (a large copy on the
// same card 4.9); a short call is one launch (333 tokens, 10 heads: 3.9 us). Loads before
// the angles, and non-temporal loads or stores, were no faster.
template <typename T, bool INTER>
__global__ void __launch_bounds__(256) rope_kernel(const RopeArgs a) {
  constexpr int N = Chunk<T>::N, U = 4;
  const int tpt = a.d / (2 * N);   // threads per token
  const int j = threadIdx.x % tpt;
  const int tok = blockIdx.x * (256 / tpt) + threadIdx.x / tpt;
  if (tok >= a.tokens) return;
  const int b = tok / a.n, i = tok - b * a.n;
  const int p = a.pos ? a.pos[b * a.pos_stride + i] : a.start + i;
  PairChunks<T, INTER> pc(a.rot, j);
  pc.angles(a.rot, j, p, a.sign);
  const int h1 = min((int)(blockIdx.y + 1) * a.hgroup, a.Hq + a.Hk);
  for (int h0 = blockIdx.y * a.hgroup; h0 < h1; h0 += U) {
    u32x4 xa[U], xb[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (h0 + u < h1) {
        const bool isk = h0 + u >= a.Hq;
        const Strides& st = isk ? a.ks : a.qs;
        const T* src = (const T*)(isk ? a.k : a.q) + b * st.b + (h0 + u - (isk ? a.Hq : 0)) * st.h + i * st.t;
        xa[u] = *(const u32x4*)(src + pc.col[0]);
        xb[u] = *(const u32x4*)(src + pc.col[1]);
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (h0 + u < h1) {
        const bool isk = h0 + u >= a.Hq;
        const Strides& st = isk ? a.kos : a.qos;
        T* dst = (T*)(isk ? a.ko : a.qo) + b * st.b + (h0 + u - (isk ? a.Hq : 0)) * st.h + i * st.t;
        pc.apply(xa[u], xb[u]);
        *(u32x4*)(dst + pc.col[0]) = xa[u];
        *(u32x4*)(dst + pc.col[1]) = xb[u];
      }
  }
}

}  // namespace attn
