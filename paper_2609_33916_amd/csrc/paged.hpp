// The paged key/value cache: append (with the rotation of rope.hpp on the way),
// read back, and one decode step's attention, over bf16 pages and over pages of
// 4-bit codes.
//
// 4-bit pages. A row of d columns is d / 2 bytes of codes (column 2i in the low
// half of byte i) and d / 32 bytes of scales. A code is a sign and one of the
// magnitudes 0, 1/2, 1, 3/2, 2, 3, 4, 6; byte x as a scale of 32 columns stands
// for 2^(x - 127), and 255 for "not a number" (the OCP microscaling format with
// E2M1 elements, which gfx950 converts to bfloat16, scale included, two at a time;
// every value but the ends of the range is exact there). Writing takes the
// smallest power of two 2^e with all magnitudes of the block below 7 2^e (values
// between 6 and 7 round down to 6 by at most half a step, those from 7 on would be
// further off than under the next power), then the nearest code, ties to the
// even one, of those that bfloat16 holds. 2^e is at least 2^-125; a block holding
// a value that is not finite reads as NaN.
#pragma once

#include <climits>
#include <type_traits>

#include "common.hpp"
#include "pages.hpp"
#include "rope.hpp"

namespace attn {

// ------------------------------------------------------------ 4-bit values --
struct Quant4 {
  // A float that rounds to the codes as y does: y cut to 20 bits behind its first, the last
  // of them set if anything was lost. (A plain conversion could carry a value next to a
  // border of the codes onto it. The rotation before it is in 64 bits for the same reason:
  // a row's codes then do not depend on how 32-bit sums are ordered.) From 2^128 on it is
  // infinite, as is NaN; up to 2^-127 it is 0; between 2^-127 and 2^-126, where a float's bits
  // have no room for the first, they are those behind it, which put() sets right.
  __device__ __forceinline__ static float odd(double y) {
    const uint64_t bits = __builtin_bit_cast(uint64_t, y);
    const uint32_t hi = (uint32_t)(bits >> 32), lo = (uint32_t)bits;
    const uint32_t mag = (hi & 0x7fffffffu) | min(lo, 1u);
    const uint32_t m = min(max(mag, 896u << 20), 1151u << 20);   // exponents 0 and 255 of a float
    return __uint_as_float(((m << 3) - (896u << 23)) | (hi & 0x80000000u));
  }
  // largest magnitude, as bits, of the four lanes of a quad
  __device__ __forceinline__ static uint32_t quad_max(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xf, 0xf, true));   // lanes 1 0 3 2
    return max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xf, 0xf, true));   // lanes 2 3 0 1
  }
  // Eight values of each lane of a quad (a block of 32): the lane's four bytes
  // of codes and the block's scale. All four lanes have to be active. ODD: the values may
  // come from odd() (`from_odd`: they do).
  template <bool ODD> __device__ __forceinline__ static uint32_t put(float (&v)[8], uint32_t& scale, bool from_odd = false) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(v[e]) & 0x7fffffffu);
    m = quad_max(m);
    if (m >= 0x7f800000u) {   // codes 0: 0 times "infinity" (the scale's bits) is NaN for every reader
      scale = 255;
      return 0;
    }
    scale = (uint32_t)max((int)((m + 0x200000u) >> 23) - 2, 2);   // 1.75 2^k carries into the next exponent
    const float unit = __uint_as_float(scale << 23);
    if (ODD && scale == 2 && from_odd) {   // above 2^-127, a quarter of the unit and a border of the codes, not yet above 2^-126
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t y = __float_as_uint(v[e]) & 0x7fffffffu;
        if (y) v[e] = copysignf(__uint_as_float(max(y, 0x600000u)), v[e]);
      }
    }
    if (scale == 253) {   // 4 2^126 would be infinite in bfloat16
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = fminf(fmaxf(v[e], -3.f * unit), 3.f * unit);
    }
    uint32_t x = 0;
    x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(x, v[0], v[1], unit, 0);
    x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(x, v[2], v[3], unit, 1);
    x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(x, v[4], v[5], unit, 2);
    x = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(x, v[6], v[7], unit, 3);
    return x;
  }
  // eight codes times the scale with float bits `unit` << 23
  __device__ __forceinline__ static bf16x8 get(uint32_t x, float unit) {
    typedef bf16 bf16x2 __attribute__((ext_vector_type(2)));
    u32x4 r;
    r[0] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, unit, 0));
    r[1] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, unit, 1));
    r[2] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, unit, 2));
    r[3] = __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(x, unit, 3));
    return __builtin_bit_cast(bf16x8, r);
  }
};

// ------------------------------------------------------------------- append --
struct AppendArgs {
  const void *k_new, *v_new;   // bf16 [B, Hkv, T, d], strided
  Strides ks, vs;
  void *kp, *vp;               // pools
  uint8_t *ksc, *vsc;          // 4 bits: their scales
  Pages pg;
  const int *lens, *new_lens;  // tokens cached before, tokens to append (null: T)
  const int* pos;              // positions [B, T], or null: the token's place in the sequence
  Rotation rot;
  int T, d, tokens;            // tokens: B T
  int hgroup;                  // heads per workgroup
};

// Where a thread's token goes: the pool's row, -1 where it has none (past the
// sequence's count, behind its table, no page), and its position.
__device__ __forceinline__ long long append_row(const AppendArgs& a, int b, int t, int& p) {
  const int len = a.lens[b];
  if (t >= (a.new_lens ? a.new_lens[b] : a.T) || len < 0 || len > INT_MAX - t) return -1;
  p = a.pos ? a.pos[(long long)b * a.T + t] : len + t;
  return page_row(a.pg, a.pg.table + (long long)b * a.pg.width, len + t);
}

// bf16 pages: as rope_kernel, the values copied beside the keys. 8 x 1024 tokens of 8
// heads, d = 128: 12.9 us (67 MB, 5.2 TB/s). The first rows are read before the counts are
// known: where sequences bring 512 to 1024 of the 1024 tokens 33.7 MB for 26.2, 14.9 us.
template <bool INTER>
__global__ void __launch_bounds__(256) append_kernel(const AppendArgs a) {
  constexpr int U = 4;
  const int tpt = a.d / 16;
  const int j = threadIdx.x % tpt;
  const int tok = blockIdx.x * (256 / tpt) + threadIdx.x / tpt;
  if (tok >= a.tokens) return;
  const int b = tok / a.T, t = tok - b * a.T;
  PairChunks<bf16, INTER> pc(a.rot, j);
  const bf16* ks = (const bf16*)a.k_new + b * a.ks.b + t * a.ks.t;
  const bf16* vs = (const bf16*)a.v_new + b * a.vs.b + t * a.vs.t;
  const int h1 = min((int)(blockIdx.y + 1) * a.hgroup, a.pg.Hkv);
  u32x4 ka[U], kb[U], va[U], vb[U];
  auto load = [&](int h0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (h0 + u < h1) {
        const bf16 *k = ks + (h0 + u) * a.ks.h, *v = vs + (h0 + u) * a.vs.h;
        ka[u] = *(const u32x4*)(k + pc.col[0]);
        kb[u] = *(const u32x4*)(k + pc.col[1]);
        va[u] = *(const u32x4*)(v + pc.col[0]);
        vb[u] = *(const u32x4*)(v + pc.col[1]);
      }
  };
  load(blockIdx.y * a.hgroup);   // in flight while the place and the angles are found
  int p = 0;
  const long long row = append_row(a, b, t, p);
  if (row < 0) return;
  pc.angles(a.rot, j, p, 1.f);
  bf16* kd = (bf16*)a.kp + row * a.d;
  bf16* vd = (bf16*)a.vp + row * a.d;
  const long long hs = (long long)a.d << a.pg.shift;
  for (int h0 = blockIdx.y * a.hgroup; h0 < h1; h0 += U) {
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (h0 + u < h1) {
        pc.apply(ka[u], kb[u]);
        bf16 *k = kd + (h0 + u) * hs, *v = vd + (h0 + u) * hs;
        *(u32x4*)(k + pc.col[0]) = ka[u];
        *(u32x4*)(k + pc.col[1]) = kb[u];
        *(u32x4*)(v + pc.col[0]) = va[u];
        *(u32x4*)(v + pc.col[1]) = vb[u];
      }
    load(h0 + U);
  }
}

// 4-bit pages: a thread takes 8 consecutive columns, a quad a block of 32. The
// other halves of its pairs are read too (by another thread as well: from
// cache), so that the result is in the order it is stored in. The 64-bit sines and
// cosines, a hundred instructions each, are made once per token and pair, in LDS.
// 4 x 4000 tokens of 8 heads, d = 128: 23.8 us (83 MB, 3.5 TB/s), 17.5 with 64
// interleaved columns turned; with the rotation in 32 bits a fifth less.
template <int D, bool INTER>
__global__ void __launch_bounds__(256) append4_kernel(const AppendArgs a) {
  constexpr int TPT = D / 8, TOK = 256 / TPT;   // threads per token, tokens
  __shared__ double tab[2][TOK][D / 2];
  const int ch = threadIdx.x % TPT, col = 8 * ch, lt = threadIdx.x / TPT;
  const int tok = blockIdx.x * TOK + lt;
  int b = 0, t = 0, p = 0;
  long long row = -1;
  if (tok < a.tokens) {
    b = tok / a.T;
    t = tok - b * a.T;
    row = append_row(a, b, t, p);
  }
  if (row >= 0)
    for (int i = ch; i < a.rot.r / 2; i += TPT) turn_cs(p, a.rot.freqs[i], a.rot.amplitude, tab[0][lt][i], tab[1][lt][i]);
  __syncthreads();
  if (row < 0) return;   // the same for the whole quad
  const bool turns = col < a.rot.r, second = col >= a.rot.r / 2;
  const int mate = INTER ? col : second ? col - a.rot.r / 2 : col + a.rot.r / 2;
  double c[8], s[8];
  if (turns) {
    const int i0 = INTER ? col / 2 : second ? mate : col;
#pragma unroll
    for (int e = 0; e < (INTER ? 4 : 8); ++e) {
      c[e] = tab[0][lt][i0 + e];
      s[e] = second && !INTER ? -tab[1][lt][i0 + e] : tab[1][lt][i0 + e];   // w' = w c + u s, u' = u c - w s
    }
  }
  const bf16* ks = (const bf16*)a.k_new + b * a.ks.b + t * a.ks.t;
  const bf16* vs = (const bf16*)a.v_new + b * a.vs.b + t * a.vs.t;
  const int h1 = min((int)(blockIdx.y + 1) * a.hgroup, a.pg.Hkv);
  // a row's scale bytes, one store
  auto put_scales = [&](uint8_t* dst, uint32_t sc) __attribute__((always_inline)) {
    if constexpr (D == 128) {   // the row's 16 lanes: a quad's byte to all of them
      uint32_t y = sc << (8 * (ch / 4));
      y |= (uint32_t)__builtin_amdgcn_mov_dpp((int)y, 0x124, 0xf, 0xf, true);
      y |= (uint32_t)__builtin_amdgcn_mov_dpp((int)y, 0x128, 0xf, 0xf, true);
      if (ch == 0) *(uint32_t*)dst = y;
    } else {
      if (ch % 4 == 0) dst[ch / 4] = (uint8_t)sc;
    }
  };
  constexpr int U = 2;
  for (int h0 = blockIdx.y * a.hgroup; h0 < h1; h0 += U) {
    u32x4 xk[U], xm[U], xv[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (h0 + u < h1) {
        xk[u] = *(const u32x4*)(ks + (h0 + u) * a.ks.h + col);
        if (!INTER && turns) xm[u] = *(const u32x4*)(ks + (h0 + u) * a.ks.h + mate);
        xv[u] = *(const u32x4*)(vs + (h0 + u) * a.vs.h + col);
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (h0 + u < h1) {
        float k[8], v[8];
        Chunk<bf16>::get(xk[u], k);
        Chunk<bf16>::get(xv[u], v);
        if (turns) {
          if (INTER) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              double y = k[2 * e], z = k[2 * e + 1];
              turn_pair(y, z, c[e], s[e]);
              k[2 * e] = Quant4::odd(y);
              k[2 * e + 1] = Quant4::odd(z);
            }
          } else {
            float m[8];
            Chunk<bf16>::get(xm[u], m);
#pragma unroll
            for (int e = 0; e < 8; ++e) {   // s is negated in the second half
              double y = k[e], z = m[e];
              turn_pair(y, z, c[e], s[e]);
              k[e] = Quant4::odd(y);
            }
          }
        }
        const long long r = row + ((long long)(h0 + u) << a.pg.shift);
        uint32_t sc;
        ((uint32_t*)a.kp)[r * TPT + ch] = Quant4::put<true>(k, sc, turns);
        put_scales(a.ksc + r * (D / 32), sc);
        ((uint32_t*)a.vp)[r * TPT + ch] = Quant4::put<false>(v, sc);
        put_scales(a.vsc + r * (D / 32), sc);
      }
  }
}

// ------------------------------------------------------------------- gather --
struct GatherArgs {
  const void *kp, *vp;
  const uint8_t *ksc, *vsc;   // null: bf16 pages
  Pages pg;
  const int *lens, *starts;   // tokens in each sequence; first row wanted, or null: 0
  void *k, *v;                // dense bf16 [B, Hkv, n, d]
  int n, d;
};

// Rows starts[b] + [0, n) of every cache head, zeros where the sequence has no
// such token (or no page for it). A thread moves 16 bytes of K and of V: 8 sequences of
// 2300 tokens, 8 heads, d = 128 23.9 us (151 MB, 6.3 TB/s), one row 2.9 to 4.5.
template <bool Q4>
__global__ void __launch_bounds__(256) gather_kernel(const GatherArgs a) {
  const int tpr = a.d / 8;
  const int ch = threadIdx.x % tpr, h = blockIdx.y, b = blockIdx.z;
  const int j = blockIdx.x * (256 / tpr) + threadIdx.x / tpr;
  if (j >= a.n) return;
  const long long p = (a.starts ? a.starts[b] : 0) + (long long)j;
  long long row = p < a.lens[b] ? page_row(a.pg, a.pg.table + (long long)b * a.pg.width, (int)p) : -1;
  u32x4 k = {0u, 0u, 0u, 0u}, v = {0u, 0u, 0u, 0u};
  if (row >= 0) {
    row += (long long)h << a.pg.shift;
    if (Q4) {
      const long long s = row * (a.d / 32) + ch / 4;
      k = __builtin_bit_cast(u32x4, Quant4::get(((const uint32_t*)a.kp)[row * tpr + ch],
                                                __uint_as_float((uint32_t)a.ksc[s] << 23)));
      v = __builtin_bit_cast(u32x4, Quant4::get(((const uint32_t*)a.vp)[row * tpr + ch],
                                                __uint_as_float((uint32_t)a.vsc[s] << 23)));
    } else {
      k = ((const u32x4*)a.kp)[row * tpr + ch];
      v = ((const u32x4*)a.vp)[row * tpr + ch];
    }
  }
  const long long o = (((long long)b * a.pg.Hkv + h) * a.n + j) * tpr + ch;
  ((u32x4*)a.k)[o] = k;
  ((u32x4*)a.v)[o] = v;
}

// ------------------------------------------------------------------- decode --
// One new query token per head against the pages. As in decode_kernel a
// workgroup owns one cache head, one split of its keys and up to 16 NQ of the
// query heads that share it (the columns of S^T = K Q^T), so a cached row is read
// once for all of these. Its four waves take blocks of BK keys in turn, each with
// its own running (maximum, sum, O) and its own part of LDS: there is no barrier
// in the loop, and a block's loads are in flight while the previous one is worked
// on. Products are 16x16x32 (a lane of group g = lane / 16, column c = lane % 16):
//   S^T: A = 16 keys (lane c's key, 8 columns of d per lane and step), B = Q^T;
//        the lane then holds keys 16 kb + 4g + [0, 4) of query c.
//   O^T += V^T P^T: the lane's keys of two (bf16) or four (4 bits) key rows of
//        16 are its k slots; V goes through LDS to be read transposed.
// 4 bits: the K operand is converted in registers, scale included (a lane's 8
// columns lie in one block of 32). V's codes are transposed as they are (a
// 64-bit read gives a lane 16 keys of its column) and converted without a scale,
// since the scales run along the keys; they multiply P, one product per
// 32 columns.
//
// Bound by the pages' bytes where there are many: 16 sequences of 8192 tokens, 64
// heads on 8, d = 128 84.8 us (537 MB, 6.3 TB/s); a sequence of 131072 in 4 bits 30.0
// (143 MB, 4.8 TB/s), of which some 7 us are the way to the first key (lengths, page
// numbers, the frequencies' turn, cold loads behind each other) and the end of the last
// wave. In 4 bits the conversions and the softmax would bound it, with two waves per SIMD 5
// clocks an instruction: hence the transposed reads of codes, the replicas below, and
// the maximum that rarely moves; from 9 query heads per cache head on they do. Short caches
// are that fixed part: 1000 tokens 7.2 us. (These are the kernel's times alone.)
// Not faster, by the ratio of two runs in turn: three waves per SIMD (registers spill, 1.7
// times as long), eight waves in a workgroup (1000 tokens 1.3 times), two blocks loaded
// ahead (below).
struct PagedArgs {
  const void* q;               // bf16 [B, Hq, d], sequences q_b elements apart
  const void *k_new, *v_new;   // bf16 [B, Hkv, d], or null
  long long q_b, k_b, v_b;
  void *kp, *vp;
  uint8_t *ksc, *vsc;
  Pages pg;
  const int* lens;
  const int* pos;              // [B] positions of the queries (and new keys), or null: T_b - 1
  Rotation rot;
  float* part;                 // nsplit > 1: [rows][nsplit][d] unnormalised O, then [rows][nsplit] (max2, sum)
  void* o;
  float* lse;
  int Hq, G, n, append, rows;
  int nsplit, qchunks;
  float sl2;
  int interleaved;
  int negate;                  // the scale is negative
};

constexpr int kShort = 64;   // keys of a short sequence: L is off by 1e-6 with two parts and one key, by 2e-7 with ten

typedef const __attribute__((address_space(4))) int* ConstInt;   // uniform reads by the scalar unit

// A barrier that orders LDS only: loads stay in flight across it.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// A buffer of `bytes` bytes; W words of each lane at byte offset `off` + `at` (the
// same for all lanes), zeros behind its end.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_rsrc(const void* base, int bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), (short)0, bytes, 0x00020000);
}
// The pages are read once per step, and between two steps a model reads far more
// than the caches hold: 16 sequences of 8192 tokens, 64 heads, d = 128 82.4 us a
// step, 93.5 with ordinary loads; one of 131072 in 4 bits 31.6, 33.7; small calls the
// same to 1 %.
constexpr int kNonTemporal = 2;
template <int W> struct Words;
template <> struct Words<1> {
  typedef uint32_t type;
  __device__ __forceinline__ static type load(__amdgpu_buffer_rsrc_t r, unsigned off, int at) {
    return __builtin_amdgcn_raw_buffer_load_b32(r, off, at, kNonTemporal);
  }
};
template <> struct Words<2> {
  typedef u32x2 type;
  __device__ __forceinline__ static type load(__amdgpu_buffer_rsrc_t r, unsigned off, int at) {
    return __builtin_amdgcn_raw_buffer_load_b64(r, off, at, kNonTemporal);
  }
};
template <> struct Words<4> {
  typedef u32x4 type;
  __device__ __forceinline__ static type load(__amdgpu_buffer_rsrc_t r, unsigned off, int at) {
    return __builtin_amdgcn_raw_buffer_load_b128(r, off, at, kNonTemporal);
  }
};
__device__ __forceinline__ uint32_t word(uint32_t x, int) { return x; }
template <typename V> __device__ __forceinline__ uint32_t word(V x, int i) { return x[i]; }
// f(word, its index) of every word
template <typename F> __device__ __forceinline__ uint32_t map_words(uint32_t x, F f) { return f(x, 0); }
template <typename F> __device__ __forceinline__ u32x2 map_words(u32x2 x, F f) { return (u32x2){f(x[0], 0), f(x[1], 1)}; }
template <typename F> __device__ __forceinline__ u32x4 map_words(u32x4 x, F f) {
  return (u32x4){f(x[0], 0), f(x[1], 1), f(x[2], 2), f(x[3], 3)};
}

// 2^(byte B of w - 127), the scale that the byte means, in one instruction: but 0 for
// byte 0 (2^-127; no writer here stores it) and infinite for 255, of which two_parts makes
// not a number whatever the code and the probability
template <int B> __device__ __forceinline__ float byte_power(uint32_t w) {
  float r;
  if constexpr (B == 0)
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_0" : "=v"(r) : "v"(23), "v"(w));
  else if constexpr (B == 1)
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_1" : "=v"(r) : "v"(23), "v"(w));
  else if constexpr (B == 2)
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_2" : "=v"(r) : "v"(23), "v"(w));
  else
    asm("v_lshlrev_b32_sdwa %0, %1, %2 dst_sel:DWORD dst_unused:UNUSED_PAD src0_sel:DWORD src1_sel:BYTE_3" : "=v"(r) : "v"(23), "v"(w));
  return r;
}

// P in two bfloat16: the float cut to its first 16 bits, and the rest rounded, so that 15
// bits of the factor stay. (With P in one, O was off by 2.0e-3 to 2.4e-3 of its length,
// with two by the 1.6e-3 of its own last rounding. A step takes no longer in bf16; in 4
// bits 3 % longer (32 ragged sequences up to 4096, 4 heads per cache head), 5 % (one of
// 131072, 8 heads), 24 % where instructions bound it (220 of 8000, d = 64, 32 heads).)
// Infinite values of V need a rest above 0, for 0 times infinity is not a number; in 4 bits
// the rest of a product with a scale of 255 has to be not a number, as infinity less infinity
// is.
constexpr float kLeastRest = 0x1p-100f;
template <bool Q4> __device__ __forceinline__ void two_parts(const f32x4& a, const f32x4& b, bf16x8& first, bf16x8& rest) {
  f32x4 ra, rb;
  u32x4 f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const f32x4& x = i < 2 ? a : b;
    f[i] = __builtin_amdgcn_perm(__float_as_uint(x[2 * i % 4 + 1]), __float_as_uint(x[2 * i % 4]), 0x07060302u);
    ra[i] = a[i] - __uint_as_float(__float_as_uint(a[i]) & 0xffff0000u);
    rb[i] = b[i] - __uint_as_float(__float_as_uint(b[i]) & 0xffff0000u);
    if constexpr (!Q4) ra[i] = fmaxf(ra[i], kLeastRest), rb[i] = fmaxf(rb[i], kLeastRest);
  }
  first = __builtin_bit_cast(bf16x8, f);
  rest = frag16(ra, rb);
}

// REP: the query heads (at most 16 / REP of them) stand REP times in the 16 columns, and a
// lane scales P for only 1 / REP of the 32-column blocks of d; the two parts of the
// query are then columns, not products of their own (131072 tokens, 8 heads per cache
// head: REP = 2 33.6 us a step, without 37; 32 ragged sequences, 4 heads: REP = 4 28.3, without
// 36.7). PAGE: the least number of keys that lie in one page, 16 or a whole block, which
// then has one page number and one buffer (part of the same figures).
template <int D, int NQ, int REP, bool Q4, int PAGE>
__global__ void __launch_bounds__(256, 2) paged_decode_kernel(const PagedArgs a) {
  constexpr int BK = Q4 ? 64 : 32, KB = BK / kGranule;   // keys of a block, in rows of 16
  constexpr int NG = BK / PAGE, GB = PAGE / kGranule;    // its pieces of pages, rows of 16 in one
  constexpr int HR = 16 / REP;                           // heads side by side
  static_assert(REP == 1 || (Q4 && NQ == 1 && D / 32 % REP == 0), "replicas share the blocks of d");
  constexpr int TD = D / 32, DB = D / 16;                // steps over d, output rows of 16
  constexpr int C = 16 * NQ;                             // query columns
  constexpr int RB = Q4 ? D / 2 : 2 * D;                 // bytes of a row
  constexpr int QS = D + 8;                              // row stride of the queries in LDS (elements)
  constexpr int VBYTES = 4 * BK * RB, OS = D + 4, OBYTES = 4 * C * OS * 4;
  constexpr int BYTES = VBYTES + (REP == 1 ? 3 : 2) * C * QS * 2;
  // the waves' stages of V and the queries; at the end the waves' O
  __shared__ __attribute__((aligned(16))) unsigned char smem[BYTES > OBYTES ? BYTES : OBYTES];
  __shared__ float ml[2][4][C];
  // the new key and value as they are stored; 4 bits: their scales, and before that their values
  __shared__ __attribute__((aligned(16))) uint32_t nrow[2][RB / 4];
  __shared__ uint32_t nscale[2];
  __shared__ float nval[2][Q4 ? D : 1];

  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int split = (int)gridDim.x - 1 - (int)blockIdx.x;   // the one with the new row starts first
  const int qc = blockIdx.y % a.qchunks, bh = blockIdx.y / a.qchunks;
  const int b = bh / a.pg.Hkv, hk = bh - b * a.pg.Hkv;
  const int h0 = hk * a.G + qc * C, nq = min(C, a.G - qc * C);
  // The queries and their frequencies first: loads come back in order, and behind
  // the keys' and values' they would wait for those.
  constexpr int P = D / 2;                    // pairs of a row, or neighbours that do not turn
  const int pr = tid % P, nrot = a.rot.r / 2;
  const bool turns = pr < nrot, halves = turns && !a.interleaved;
  const int c0 = halves ? pr : 2 * pr, c1 = halves ? pr + nrot : 2 * pr + 1;
  float u[C * P / 256], x[C * P / 256];
#pragma unroll
  for (int i = 0; i < C * P / 256; ++i) {
    const int r = tid / P + 256 / P * i;
    const bf16* src = (const bf16*)a.q + b * a.q_b + (size_t)(h0 + min(REP == 1 ? r : r % HR, nq - 1)) * D;
    u[i] = (float)src[c0];
    x[i] = (float)src[c1];
  }
  double freq = 0.0;
  if (turns) freq = a.rot.freqs[pr];
  __builtin_amdgcn_sched_barrier(0);

  const int len = min(max(((ConstInt)(uintptr_t)a.lens)[b], 0), a.n);
  const int T_b = len + a.append;
  // the sequence's own blocks, evenly over the splits
  const unsigned blocks = (unsigned)(T_b + BK - 1) / BK, ns = (unsigned)a.nsplit;
  const unsigned per = blocks / ns, more = blocks - per * ns, us = (unsigned)split;
  const int k_lo = BK * (int)(us * per + min(us, more));
  const int k_hi = min(T_b, k_lo + BK * (int)(per + (us < more ? 1u : 0u)));
  const int* table = a.pg.table + (size_t)b * a.pg.width;
  const int pos = a.pos ? ((ConstInt)(uintptr_t)a.pos)[b] : T_b - 1;

  // 4 bits: the byte, of the scales of 16 keys, of this lane's columns of its key
  const int ksb = c * TD + g * TD / 4;
  typedef Words<Q4 ? TD : 4> Part;   // of a row: a lane's loads
  typedef typename Part::type part_t;
  constexpr int NP = Q4 ? 1 : TD;
  struct Block {
    part_t k[KB][NP], v[KB][NP];
    uint32_t ks[Q4 ? KB : 1];
    part_t vs[Q4 ? KB : 1];
    int lim[NG];   // keys of each piece that take part
  };
  auto limit = [](const Block& x, int kb) __attribute__((always_inline)) {   // of a row of 16
    return GB == 1 ? x.lim[kb] : max(0, min(x.lim[kb / GB] - kb % GB * kGranule, kGranule));
  };
  // page numbers of the block at key kv0 (a multiple of 16); behind the split, of its last key
  struct Ids {
    int page[NG];
  };
  auto fetch = [&](Ids& ids, int kv0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NG; ++i)
      ids.page[i] = ((ConstInt)(uintptr_t)table)[min(kv0 + PAGE * i, k_hi - 1) >> a.pg.shift];
  };
  // The block's loads. Each piece has a buffer of its own that ends behind its last
  // key, so what takes no part (keys behind the end, pages that are none, blocks
  // behind the split) reads as zeros, without an access.
  const unsigned koff = c * RB + (Q4 ? RB / 4 * g : 16 * g), voff = Q4 ? RB / 4 * lane : 16 * lane;
  auto load = [&](Block& x, const Ids& ids, int kv0) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < NG; ++i) {
      const int p = kv0 + PAGE * i;
      const bool ok = p < k_hi && page_ok(a.pg, ids.page[i]);
      x.lim[i] = ok ? min(k_hi - p, PAGE) : 0;
      const long long row = ok ? (((long long)ids.page[i] * a.pg.Hkv + hk) << a.pg.shift) + (p & ((1 << a.pg.shift) - 1)) : 0;
      const auto kr = rows_rsrc((const unsigned char*)a.kp + row * RB, x.lim[i] * RB);
      const auto vr = rows_rsrc((const unsigned char*)a.vp + row * RB, x.lim[i] * RB);
      const int scales = Q4 && ok ? PAGE * TD : 0;
      const auto ksr = rows_rsrc(a.ksc + row * TD, scales), vsr = rows_rsrc(a.vsc + row * TD, scales);
#pragma unroll
      for (int j = 0; j < GB; ++j) {
        const int kb = GB * i + j, at = kGranule * RB * j;
        if constexpr (!Q4) {
#pragma unroll
          for (int t = 0; t < TD; ++t) x.k[kb][t] = Part::load(kr, koff + 64 * t, at);
#pragma unroll
          for (int t = 0; t < TD; ++t) x.v[kb][t] = Part::load(vr, voff + 1024 * t, at);
        } else {
          x.ks[kb] = Words<1>::load(ksr, ksb & ~3, kGranule * TD * j);
          x.k[kb][0] = Part::load(kr, koff, at);
          x.v[kb][0] = Part::load(vr, voff, at);
          x.vs[kb] = Part::load(vsr, 4 * TD * g, kGranule * TD * j);
        }
      }
    }
  };
  Block A, B2;
  Ids ids;
  int kv = k_lo + BK * w;
  if (kv < k_hi) {   // in flight while the queries are made
    fetch(ids, kv);
    load(A, ids, kv);
    fetch(ids, kv + 4 * BK);
  }
  // This split holds the new row: it takes it from LDS, and the first of the query
  // chunks writes it.
  const bool fresh = a.append && T_b - 1 >= k_lo && T_b - 1 < k_hi;

  // ---- the queries, turned, as two bfloat16 each (their sum is 16 bits of the
  // result; one alone would cost L its last digits), in short sequences, where a
  // score's error does not average out, as three (24 bits); and the new row
  bf16 *const qh = (bf16*)(smem + VBYTES), *const ql = qh + C * QS, *const qm = REP == 1 ? ql + C * QS : ql;
  {
    float cs = 1.f, sn = 0.f;
    if (turns) turn_cs(pos, freq, a.rot.amplitude, cs, sn);
#pragma unroll
    for (int i = 0; i < C * P / 256; ++i) {
      const int r = tid / P + 256 / P * i;
      if ((REP == 1 ? r : r % HR) >= nq) continue;   // columns without a head repeat the last one's query
      float y = u[i], z = x[i];
      if (turns) turn_pair(y, z, cs, sn);
      if (a.negate) y = -y, z = -z;
      const bf16 yh = (bf16)y, zh = (bf16)z;
      const float yr = turns ? y - (float)yh : 0.f, zr = turns ? z - (float)zh : 0.f;
      const bf16 yl = (bf16)yr, zl = (bf16)zr;
      const bool third = REP == 1 || r / HR % 2 == 0;
      qm[r * QS + c0] = (bf16)(third ? yr - (float)yl : 0.f);
      qm[r * QS + c1] = (bf16)(third ? zr - (float)zl : 0.f);
      if constexpr (REP == 1) {
        qh[r * QS + c0] = yh;
        qh[r * QS + c1] = zh;
        ql[r * QS + c0] = yl;
        ql[r * QS + c1] = zl;
      } else {   // the two parts in replicas side by side
        const bool low = r / HR & 1;
        qh[r * QS + c0] = low ? yl : yh;
        qh[r * QS + c1] = low ? zl : zh;
      }
    }
    if (fresh) {
      const long long at = qc == 0 ? page_row(a.pg, table, T_b - 1) : -1;
      const long long r = at + ((long long)hk << a.pg.shift);
      if (tid < P) {
        typedef typename std::conditional<Q4, double, float>::type R;
        const bf16* kn = (const bf16*)a.k_new + b * a.k_b + (size_t)hk * D;
        const bf16* vn = (const bf16*)a.v_new + b * a.v_b + (size_t)hk * D;
        const bf16 v0 = vn[c0], v1 = vn[c1];
        bf16 k0 = kn[c0], k1 = kn[c1];
        R y = (R)(float)k0, z = (R)(float)k1;
        if (turns) {
          R rc, rs;
          turn_cs(pos, freq, a.rot.amplitude, rc, rs);
          turn_pair(y, z, rc, rs);
          k0 = (bf16)y;
          k1 = (bf16)z;
        }
        if constexpr (Q4) {
          nval[0][c0] = Quant4::odd(y);
          nval[0][c1] = Quant4::odd(z);
          nval[1][c0] = (float)v0;
          nval[1][c1] = (float)v1;
        } else {
          bf16 *kd = (bf16*)nrow[0], *vd = (bf16*)nrow[1];
          kd[c0] = k0, kd[c1] = k1;
          vd[c0] = v0, vd[c1] = v1;
          if (at >= 0) {
            kd = (bf16*)a.kp + r * D, vd = (bf16*)a.vp + r * D;
            kd[c0] = k0, kd[c1] = k1;
            vd[c0] = v0, vd[c1] = v1;
          }
        }
      }
      if constexpr (Q4) {
        lds_barrier();   // the same for the whole workgroup
        if (tid < D / 4) {
          const int which = tid / (D / 8), ch = tid % (D / 8);
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = nval[which][8 * ch + e];
          uint32_t sc;
          const uint32_t y = Quant4::put<true>(v, sc, which == 0);
          nrow[which][ch] = y;
          if (ch % 4 == 0) ((uint8_t*)&nscale[which])[ch / 4] = (uint8_t)sc;
          if (at >= 0) {
            ((uint32_t*)(which ? a.vp : a.kp))[r * (D / 8) + ch] = y;
            if (ch % 4 == 0) (which ? a.vsc : a.ksc)[r * (D / 32) + ch / 4] = (uint8_t)sc;
          }
        }
      }
    }
  }
  lds_barrier();
  // With two columns of queries at d = 128 their operands stay in LDS (64 registers).
  constexpr bool QLDS = NQ == 2 && D == 128;
  const int qrow = REP == 1 ? 0 : c / HR * HR + min(c % HR, nq - 1);
  auto query = [&](const bf16* part, int x, int t) __attribute__((always_inline)) {
    return *(const bf16x8*)(part + (REP == 1 ? min(16 * x + c, nq - 1) : qrow) * QS + (Q4 ? D / 4 * g + 8 * t : 32 * t + 8 * g));
  };
  bf16x8 qf[NQ][TD], qr[NQ][TD];
  if constexpr (!QLDS) {
#pragma unroll
    for (int x = 0; x < NQ; ++x)
#pragma unroll
      for (int t = 0; t < TD; ++t) {
        qf[x][t] = query(qh, x, t);
        if constexpr (REP == 1) qr[x][t] = query(ql, x, t);
      }
  }

  f32x4 oacc[NQ][DB];
  float m_use[NQ], lsum[NQ];
#pragma unroll
  for (int x = 0; x < NQ; ++x) {
    m_use[x] = -INFINITY;
    lsum[x] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[x][db] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }

  unsigned char* vst = smem + w * (BK * RB);
  const unsigned kshift = 8 * (ksb & 3);
  const float sl2 = a.sl2;
  // the new row in place of what its page held: lane (g, c) has a part of key c and,
  // of V, 16 (bf16) or RB / 4 bytes at its place in the 16 rows. Without a page it takes
  // no part: its values stay out, for 0 times one that is not finite is not 0.
  auto patch = [&](Block& x, int at) __attribute__((always_inline)) {
    const int row = at & 15;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const bool here = at >> 4 == kb && limit(x, kb) > 0;
      const bool k_mine = here && c == row;
      if constexpr (!Q4) {
#pragma unroll
        for (int t = 0; t < TD; ++t) {
          if (k_mine) x.k[kb][t] = *(const u32x4*)&nrow[0][16 * t + 4 * g];
          if (here && (1024 * t + voff) / RB == row) x.v[kb][t] = *(const u32x4*)&nrow[1][(1024 * t + voff) % RB / 4];
        }
      } else {
        if (k_mine) {
          x.k[kb][0] = *(const part_t*)&nrow[0][TD * g];
          x.ks[kb] = nscale[0] >> (8 * (g * TD / 4)) << kshift;
        }
        if (here && voff / RB == row) x.v[kb][0] = *(const part_t*)&nrow[1][voff % RB / 4];
        // the row's TD bytes are bytes (row % 4) TD on of the 4 TD that lanes of its group hold
        const unsigned first = (row & 3) * TD, shift = 8 * (first & 3);
        const uint32_t mask = here && g == row >> 2 ? (TD == 4 ? ~0u : (1u << (8 * TD % 32)) - 1) << shift : 0u;
        const uint32_t fresh = nscale[1] << shift;
        x.vs[kb] = map_words(x.vs[kb], [=](uint32_t y, unsigned t) {
          return first / 4 == t ? (y & ~mask) | (fresh & mask) : y;
        });
      }
    }
  };
  auto step = [&](Block& x, int kv0) __attribute__((always_inline)) {
    if (fresh && T_b - 1 - kv0 < BK) patch(x, T_b - 1 - kv0);
    bool whole = true;
#pragma unroll
    for (int i = 0; i < NG; ++i) whole = whole && x.lim[i] == PAGE;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      if constexpr (!Q4) {
#pragma unroll
        for (int t = 0; t < TD; ++t) {
          constexpr int RPL = 1024 / RB, CPR = 64 / RPL;
          const int r = kGranule * kb + RPL * t + lane / CPR, ch = lane % CPR;
          *(part_t*)(vst + r * RB + 16 * (ch ^ swz16<D>(r))) = x.v[kb][t];
        }
      } else {
        // 8-byte pieces; the eight rows that a half-wave's transposed read takes at one
        // place of a 256-byte line get different pieces of it
        const int r = kGranule * kb + lane / 4;
        if constexpr (TD == 4) {
          const int p = 2 * (lane & 3), f = 2 * kb + ((r >> 2) & 1);
          const part_t y = x.v[kb][0];
          *(u32x2*)(vst + r * RB + 8 * (p ^ f)) = (u32x2){y[0], y[1]};
          *(u32x2*)(vst + r * RB + 8 * ((p + 1) ^ f)) = (u32x2){y[2], y[3]};
        } else if constexpr (TD == 2) {
          *(part_t*)(vst + r * RB + 8 * ((lane & 3) ^ kb)) = x.v[kb][0];
        } else {
          *(part_t*)(vst + r * RB + 8 * ((lane >> 1 & 1) ^ (kb & 1)) + 4 * (lane & 1)) = x.v[kb][0];
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    f32x4 s[NQ][KB];
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) s[q][kb] = (f32x4){0.f, 0.f, 0.f, 0.f};
    float unit[KB];
    if constexpr (Q4) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) unit[kb] = __uint_as_float(((x.ks[kb] >> kshift) & 255u) << 23);
    }
#pragma unroll
    for (int t = 0; t < TD; ++t) {   // the chains of the KB sums side by side
      if constexpr (QLDS) {
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          qf[q][t] = query(qh, q, t);
          qr[q][t] = query(ql, q, t);
        }
      }
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        bf16x8 kf;
        if constexpr (Q4) kf = Quant4::get(word(x.k[kb][0], t), unit[kb]);
        else kf = __builtin_bit_cast(bf16x8, x.k[kb][t]);
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          mma16(s[q][kb], kf, qf[q][t]);
          if constexpr (REP == 1) mma16(s[q][kb], kf, qr[q][t]);
        }
      }
    }
    if (T_b <= kShort) {
#pragma unroll
      for (int q = 0; q < NQ; ++q)
#pragma unroll
        for (int t = 0; t < TD; ++t) {
          const bf16x8 qf3 = query(qm, q, t);
#pragma unroll
          for (int kb = 0; kb < KB; ++kb) {
            if constexpr (Q4) {
              float u = unit[kb];
              asm("" : "+v"(u));   // converted again: kept from above, the operands would take 64 registers
              mma16(s[q][kb], Quant4::get(word(x.k[kb][0], t), u), qf3);
            } else mma16(s[q][kb], __builtin_bit_cast(bf16x8, x.k[kb][t]), qf3);
          }
        }
    }
    if constexpr (REP > 1) {   // the sum of the two parts, in both
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          s[0][kb][i] += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(s[0][kb][i]), 0x120 + HR, 0xf, 0xf, true));
    }
    if (!whole) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
          for (int q = 0; q < NQ; ++q) s[q][kb][i] = 4 * g + i < limit(x, kb) ? s[q][kb][i] : -INFINITY;
        }
    }
#pragma unroll
    for (int q = 0; q < NQ; ++q) {
      float mx = -INFINITY;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[q][kb][i]);
      // the maximum moves only by more than a factor of 2^kRescaleThresh, so most
      // blocks need neither the other lanes' maxima nor a rescaling
      if (__builtin_amdgcn_ballot_w64(mx * sl2 > m_use[q] + kRescaleThresh)) {
        auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
        const float mt = halves_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]))) * sl2;
        const bool up = mt > m_use[q] + kRescaleThresh;
        const float alpha = up ? exp2_fast(m_use[q] - mt) : 1.f;
        if (up) m_use[q] = mt;
        lsum[q] *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) oacc[q][db] *= alpha;
      }
      const float mb = m_use[q] == -INFINITY ? 0.f : -m_use[q];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = exp2_fast(fmaf(s[q][kb][i], sl2, mb));
          lsum[q] += p;
          s[q][kb][i] = p;
        }
    }
    if constexpr (!Q4) {
      bf16x8 pf[NQ], pr[NQ];
#pragma unroll
      for (int q = 0; q < NQ; ++q) two_parts<false>(s[q][0], s[q][1], pf[q], pr[q]);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const bf16x8 vf = tr_read16<D, BK>((const bf16*)vst, 0, db, g, c);
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          mma16(oacc[q][db], vf, pf[q]);
          mma16(oacc[q][db], vf, pr[q]);
        }
      }
    } else {
      if (!whole) {   // scales of rows that take no part
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          const int bytes = max(0, min(limit(x, kb) - 4 * g, 4)) * TD;
          x.vs[kb] = map_words(x.vs[kb], [&](uint32_t y, int t) {
            const int keep = bytes - 4 * t;
            return y & (keep >= 4 ? ~0u : keep <= 0 ? 0u : (1u << (8 * keep)) - 1);
          });
        }
      }
      const int rr = 16 * (c >> 2) + 4 * g + (c & 3);   // the row whose columns this lane fetches
      const int f = D == 128 ? ((rr >> 4) & 3) * 2 + ((rr >> 2) & 1) : D == 64 ? (rr >> 4) & 3 : (rr >> 4) & 1;
      // P for this lane's blocks of d, those from DL c / HR on; of the products below a
      // block's are right in the columns whose lanes scaled P for it
      constexpr int DL = TD / REP;
      bf16x8 pf[NQ][2], pr[NQ][2];
      part_t vs[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
        vs[kb] = map_words(x.vs[kb], [&](uint32_t y, int) { return REP == 1 ? y : y >> (8 * DL * (c / HR)); });
      auto scaled = [&](auto dl) __attribute__((always_inline)) {
        constexpr int B = decltype(dl)::value;
        f32x4 sc[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
          sc[kb] = (f32x4){byte_power<B>(word(vs[kb], 0)), byte_power<(TD + B) % 4>(word(vs[kb], TD / 4)),
                           byte_power<(2 * TD + B) % 4>(word(vs[kb], 2 * TD / 4)),
                           byte_power<(3 * TD + B) % 4>(word(vs[kb], 3 * TD / 4))};
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          two_parts<true>(s[q][0] * sc[0], s[q][1] * sc[1], pf[q][0], pr[q][0]);
          two_parts<true>(s[q][2] * sc[2], s[q][3] * sc[3], pf[q][1], pr[q][1]);
        }
      };
      auto products = [&](int dg) __attribute__((always_inline)) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int db = 2 * dg + e;
          typedef int i32x2 __attribute__((ext_vector_type(2)));
          const i32x2 y = __builtin_amdgcn_ds_read_tr4_b64_v2i32((ATTN_LDS i32x2*)(vst + rr * RB + 8 * (db ^ f)));
          const bf16x8 v0 = Quant4::get((uint32_t)y[0], 1.f), v1 = Quant4::get((uint32_t)y[1], 1.f);
#pragma unroll
          for (int q = 0; q < NQ; ++q) {
            mma16(oacc[q][db], v0, pf[q][0]);
            mma16(oacc[q][db], v1, pf[q][1]);
            mma16(oacc[q][db], v0, pr[q][0]);
            mma16(oacc[q][db], v1, pr[q][1]);
          }
        }
      };
      auto block = [&](auto dl) __attribute__((always_inline)) {
        scaled(dl);
#pragma unroll
        for (int r = 0; r < REP; ++r) products(r * DL + decltype(dl)::value);
      };
      block(std::integral_constant<int, 0>{});
      if constexpr (DL > 1) block(std::integral_constant<int, 1>{});
      if constexpr (DL > 2) {
        block(std::integral_constant<int, 2>{});
        block(std::integral_constant<int, 3>{});
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };

  // The next block's loads are issued whether there is one or not (they then end before
  // memory): behind a branch the compiler, counting the loads that are certainly in
  // flight, would wait for them before it uses this block's. (Two blocks ahead, both
  // from the start, short caches were slower: 256 groups, 512 tokens by an eighth.)
  for (; kv < k_hi; kv += 8 * BK) {
    load(B2, ids, kv + 4 * BK);
    fetch(ids, kv + 8 * BK);
    step(A, kv);
    load(A, ids, kv + 8 * BK);
    fetch(ids, kv + 12 * BK);
    if (kv + 4 * BK < k_hi) step(B2, kv + 4 * BK);
  }

  // ---- merge the waves through LDS: O parts [4][C][D] (rows padded by 16 bytes), maxima
  // and sums [4][C]
  lds_barrier();
  float* ow = (float*)smem;
#pragma unroll
  for (int q = 0; q < NQ; ++q) {
    auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(lsum[q]), __float_as_uint(lsum[q]), false, false);
    const float l = halves_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
    if (g == 0) {
      ml[0][w][16 * q + c] = m_use[q];
      ml[1][w][16 * q + c] = l;
    }
#pragma unroll
    for (int db = 0; db < DB; ++db) *(f32x4*)(ow + (w * C + 16 * q + c) * OS + 16 * db + 4 * g) = oacc[q][db];
  }
  lds_barrier();
  for (int it = tid; it < nq * (D / 4); it += 256) {
    const int col = it / (D / 4), d4 = it % (D / 4);
    float M = -INFINITY, l = 0.f;
#pragma unroll
    for (int v = 0; v < 4; ++v) M = fmaxf(M, ml[0][v][col]);
    f32x4 acc = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float f = M == -INFINITY ? 0.f : exp2_fast(ml[0][v][col] - M);
      l += f * ml[1][v][col];
      acc += f * *(const f32x4*)(ow + (v * C + col + HR * (4 * d4 / (D / REP))) * OS + 4 * d4);
    }
    const size_t row = (size_t)b * a.Hq + h0 + col;
    if (a.nsplit == 1) {
      const float inv = l == 0.f ? 0.f : 1.f / l;   // NaN stays
      Quad<bf16>::store((bf16*)a.o + row * D + 4 * d4, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
      if (a.lse && d4 == 0) a.lse[row] = l == 0.f ? -INFINITY : (M + log2f(l)) * kLn2;
    } else {
      *(f32x4*)(a.part + (row * a.nsplit + split) * D + 4 * d4) = acc;
      if (d4 == 0) {
        float* pml = a.part + (size_t)a.rows * a.nsplit * D + (row * a.nsplit + split) * 2;
        pml[0] = M;
        pml[1] = l;
      }
    }
  }
}

// O = sum_s 2^(m_s - M) O_s / l and L = (M + log2 l) ln 2 with M = max_s m_s, l =
// sum_s 2^(m_s - M) l_s over the splits of a query row: W waves per row, 64 / (D / 4)
// splits of a wave side by side, U loads of each in flight.
template <int D, int W>
__global__ void __launch_bounds__(64 * W) paged_combine_kernel(const float* part, void* o, float* lse, int rows, int nsplit) {
  constexpr int DL = D / 4, SL = 64 / DL, U = 8;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, dl = lane % DL, row = blockIdx.x;
  const float* po = part + (size_t)row * nsplit * D + 4 * dl;
  const f32x2* pml = (const f32x2*)(part + (size_t)rows * nsplit * D + (size_t)row * nsplit * 2);
  float m = -INFINITY, l = 0.f;
  f32x4 acc = (f32x4){0.f, 0.f, 0.f, 0.f};
  // to the maximum `to`; an empty part (maximum -inf) counts 0 times, so that a NaN in it stays
  auto weight = [](float from, float to) __attribute__((always_inline)) { return from == -INFINITY ? 0.f : exp2_fast(from - to); };
  for (int s0 = w * SL + lane / DL; s0 < nsplit; s0 += W * SL * U) {
    f32x2 ml[U];
    f32x4 v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int s = s0 + W * SL * u;
      ml[u] = (f32x2){-INFINITY, 0.f};
      v[u] = (f32x4){0.f, 0.f, 0.f, 0.f};
      if (s < nsplit) {
        ml[u] = pml[s];
        v[u] = *(const f32x4*)(po + (size_t)s * D);
      }
    }
    float M = m;
#pragma unroll
    for (int u = 0; u < U; ++u) M = fmaxf(M, ml[u][0]);
    const float f = weight(m, M);
    l *= f;
    acc *= f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float fu = weight(ml[u][0], M);
      l += fu * ml[u][1];
      acc += fu * v[u];
    }
    m = M;
  }
  auto join = [&](float m2, float l2, f32x4 a2) __attribute__((always_inline)) {
    const float M = fmaxf(m, m2), f = weight(m, M), f2 = weight(m2, M);
    l = f * l + f2 * l2;
    acc = f * acc + f2 * a2;
    m = M;
  };
#pragma unroll
  for (int k = DL; k < 64; k *= 2)
    join(__shfl_xor(m, k), __shfl_xor(l, k),
         (f32x4){__shfl_xor(acc[0], k), __shfl_xor(acc[1], k), __shfl_xor(acc[2], k), __shfl_xor(acc[3], k)});
  if constexpr (W > 1) {
    __shared__ float sm[W - 1], sl[W - 1];
    __shared__ __attribute__((aligned(16))) f32x4 sa[W - 1][DL];
    if (w && lane < DL) {
      if (lane == 0) sm[w - 1] = m, sl[w - 1] = l;
      sa[w - 1][lane] = acc;
    }
    __syncthreads();
    if (w) return;
#pragma unroll
    for (int k = 0; k < W - 1; ++k) join(sm[k], sl[k], sa[k][dl]);
  }
  if (lane < DL) {
    const float inv = l == 0.f ? 0.f : 1.f / l;   // NaN stays
    Quad<bf16>::store((bf16*)o + (size_t)row * D + 4 * lane, acc[0] * inv, acc[1] * inv, acc[2] * inv, acc[3] * inv);
    if (lse && lane == 0) lse[row] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
  }
}

}  // namespace attn
