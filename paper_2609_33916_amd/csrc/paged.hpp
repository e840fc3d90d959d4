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
  // A float that rounds to every shorter format as y does: y cut to 24 bits, the
  // last one set if anything was lost. (A plain conversion could carry a value
  // next to a border of the codes onto it. The rotation before it is in 64 bits
  // for the same reason: a row's codes then do not depend on how 32-bit sums are
  // ordered, and the pass is bound by memory either way.)
  __device__ __forceinline__ static float odd(double y) {
    const float f = (float)y;
    const double d = (double)f;
    if (d == y) return f;
    uint32_t bits = __float_as_uint(f);
    if (fabs(d) > fabs(y)) bits -= 1;
    return __uint_as_float(bits | 1u);
  }
  // largest magnitude, as bits, of the four lanes of a quad
  __device__ __forceinline__ static uint32_t quad_max(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xf, 0xf, true));   // lanes 1 0 3 2
    return max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xf, 0xf, true));   // lanes 2 3 0 1
  }
  // Eight values of each lane of a quad (a block of 32): the lane's four bytes
  // of codes and the block's scale. All four lanes have to be active.
  __device__ __forceinline__ static uint32_t put(float (&v)[8], uint32_t& scale) {
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
  int limit;                   // lengths are clamped to [0, limit], as in the decode step; -1: not
  int hgroup;                  // heads per workgroup
};

// Where a thread's token goes: the pool's row, -1 where it has none (past the
// sequence's count, behind its table, no page), and its position.
__device__ __forceinline__ long long append_row(const AppendArgs& a, int b, int t, int& p) {
  const int len = a.limit >= 0 ? min(max(a.lens[b], 0), a.limit) : a.lens[b];
  if (t >= (a.new_lens ? a.new_lens[b] : a.T) || len < 0 || len > INT_MAX - t) return -1;
  p = a.pos ? a.pos[(long long)b * a.T + t] : len + t;
  return page_row(a.pg, a.pg.table + (long long)b * a.pg.width, len + t);
}

// bf16 pages: as rope_kernel, the values copied beside the keys.
template <bool INTER>
__global__ void __launch_bounds__(256) append_kernel(const AppendArgs a) {
  constexpr int U = 4;
  const int tpt = a.d / 16;
  const int j = threadIdx.x % tpt;
  const int tok = blockIdx.x * (256 / tpt) + threadIdx.x / tpt;
  if (tok >= a.tokens) return;
  const int b = tok / a.T, t = tok - b * a.T;
  int p = 0;
  const long long row = append_row(a, b, t, p);
  if (row < 0) return;
  const PairChunks<bf16, INTER> pc(a.rot, j, p, 1.f);
  const bf16* ks = (const bf16*)a.k_new + b * a.ks.b + t * a.ks.t;
  const bf16* vs = (const bf16*)a.v_new + b * a.vs.b + t * a.vs.t;
  bf16* kd = (bf16*)a.kp + row * a.d;
  bf16* vd = (bf16*)a.vp + row * a.d;
  const long long hs = (long long)a.d << a.pg.shift;
  const int h1 = min((int)(blockIdx.y + 1) * a.hgroup, a.pg.Hkv);
  for (int h0 = blockIdx.y * a.hgroup; h0 < h1; h0 += U) {
    u32x4 ka[U], kb[U], va[U], vb[U];
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (h0 + u < h1) {
        const bf16 *k = ks + (h0 + u) * a.ks.h, *v = vs + (h0 + u) * a.vs.h;
        ka[u] = *(const u32x4*)(k + pc.col[0]);
        kb[u] = *(const u32x4*)(k + pc.col[1]);
        va[u] = *(const u32x4*)(v + pc.col[0]);
        vb[u] = *(const u32x4*)(v + pc.col[1]);
      }
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
  }
}

// 4-bit pages: a thread takes 8 consecutive columns, a quad a block of 32. The
// other halves of its pairs are read too (by another thread as well: from
// cache), so that the result is in the order it is stored in.
template <bool INTER>
__global__ void __launch_bounds__(256) append4_kernel(const AppendArgs a) {
  const int tpt = a.d / 8;
  const int ch = threadIdx.x % tpt, col = 8 * ch;
  const int tok = blockIdx.x * (256 / tpt) + threadIdx.x / tpt;
  if (tok >= a.tokens) return;
  const int b = tok / a.T, t = tok - b * a.T;
  int p = 0;
  const long long row = append_row(a, b, t, p);
  if (row < 0) return;   // the same for the whole quad
  const bool turns = col < a.rot.r, second = col >= a.rot.r / 2;
  const int mate = INTER ? col : second ? col - a.rot.r / 2 : col + a.rot.r / 2;
  double c[8], s[8];
  if (turns) {
    if (INTER) {
#pragma unroll
      for (int e = 0; e < 4; ++e) turn_cs(p, a.rot, col / 2 + e, c[e], s[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        turn_cs(p, a.rot, (second ? mate : col) + e, c[e], s[e]);
        if (second) s[e] = -s[e];   // w' = w c + u s, u' = u c - w s
      }
    }
  }
  const bf16* ks = (const bf16*)a.k_new + b * a.ks.b + t * a.ks.t;
  const bf16* vs = (const bf16*)a.v_new + b * a.vs.b + t * a.vs.t;
  const int h1 = min((int)(blockIdx.y + 1) * a.hgroup, a.pg.Hkv);
  for (int h = blockIdx.y * a.hgroup; h < h1; ++h) {
    const u32x4 xk = *(const u32x4*)(ks + h * a.ks.h + col);
    const u32x4 xv = *(const u32x4*)(vs + h * a.vs.h + col);
    float k[8], v[8];
    Chunk<bf16>::get(xk, k);
    Chunk<bf16>::get(xv, v);
    if (turns) {
      if (INTER) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const double u = k[2 * e], w = k[2 * e + 1];
          k[2 * e] = Quant4::odd(u * c[e] - w * s[e]);
          k[2 * e + 1] = Quant4::odd(w * c[e] + u * s[e]);
        }
      } else {
        float m[8];
        Chunk<bf16>::get(*(const u32x4*)(ks + h * a.ks.h + mate), m);
#pragma unroll
        for (int e = 0; e < 8; ++e) k[e] = Quant4::odd((double)k[e] * c[e] - (double)m[e] * s[e]);
      }
    }
    const long long r = row + ((long long)h << a.pg.shift);
    uint32_t sc;
    ((uint32_t*)a.kp)[r * (a.d / 8) + ch] = Quant4::put(k, sc);
    if (ch % 4 == 0) a.ksc[r * (a.d / 32) + ch / 4] = (uint8_t)sc;
    ((uint32_t*)a.vp)[r * (a.d / 8) + ch] = Quant4::put(v, sc);
    if (ch % 4 == 0) a.vsc[r * (a.d / 32) + ch / 4] = (uint8_t)sc;
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
// such token (or no page for it). A thread moves 16 bytes of K and of V.
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
// query heads that share it (the columns of S^T = K Q^T), so each cached row is
// read once per step. Its four waves take blocks of BK keys in turn, each with
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
  float* part;                 // nsplit > 1: as decode_kernel's
  void* o;
  float* lse;
  int Hq, G, n, append, fuse_append, rows;
  int nsplit, qchunks;
  float sl2;
  int interleaved;
  int negate;                  // the scale is negative
};

typedef const __attribute__((address_space(4))) int* ConstInt;   // uniform reads by the scalar unit

template <int D, int NQ, bool Q4>
__global__ void __launch_bounds__(256, 2) paged_decode_kernel(const PagedArgs a) {
  constexpr int BK = Q4 ? 64 : 32, KB = BK / kGranule;   // keys of a block, in rows of 16
  constexpr int TD = D / 32, DB = D / 16;                // steps over d, output rows of 16
  constexpr int C = 16 * NQ;                             // query columns
  constexpr int KW = Q4 ? TD : 4 * TD;                   // 32-bit words of K per lane and row of 16
  constexpr int RB = Q4 ? D / 2 : 2 * D;                 // bytes of a row
  constexpr int NV = BK * RB / 1024;                     // 16-byte loads of V per lane
  constexpr int QS = D + 8;                              // row stride of the queries in LDS (elements)
  constexpr int VBYTES = 4 * BK * RB, OBYTES = 4 * D * C * 4, QBYTES = 2 * C * QS * 2;
  constexpr int BYTES = VBYTES > OBYTES ? VBYTES : OBYTES;
  __shared__ __attribute__((aligned(16))) unsigned char smem[BYTES > QBYTES ? BYTES : QBYTES];
  __shared__ float ml[2][4][C];
  __shared__ __attribute__((aligned(16))) float nrow[2][D];   // 4 bits: the new key and value

  const int tid = threadIdx.x, lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int split = (int)gridDim.x - 1 - (int)blockIdx.x;   // the one with the new row starts first
  const int qc = blockIdx.y % a.qchunks, bh = blockIdx.y / a.qchunks;
  const int b = bh / a.pg.Hkv, hk = bh - b * a.pg.Hkv;
  const int len = min(max(a.lens[b], 0), a.n);
  const int T_b = len + a.append;
  const unsigned tiles = (unsigned)(T_b + 4 * BK - 1) / (4 * BK);
  const int k_lo = 4 * BK * (int)(split * (size_t)tiles / a.nsplit);
  const int k_hi = min(T_b, 4 * BK * (int)((split + 1) * (size_t)tiles / a.nsplit));
  const int h0 = hk * a.G + qc * C, nq = min(C, a.G - qc * C);
  const int* table = a.pg.table + (size_t)b * a.pg.width;
  const int pos = a.pos ? a.pos[b] : T_b - 1;

  // ---- the queries, turned, as two bfloat16 each (their sum is 16 bits of the
  // result; one alone would cost L its last digits), and the new row
  bf16* qh = (bf16*)smem;
  bf16* ql = qh + C * QS;
  {
    constexpr int P = D / 2;                    // pairs of a row, or neighbours that do not turn
    const int pr = tid % P, nrot = a.rot.r / 2;
    const bool turns = pr < nrot;
    const bool halves = turns && !a.interleaved;
    const int c0 = halves ? pr : 2 * pr, c1 = halves ? pr + nrot : 2 * pr + 1;
    typedef typename std::conditional<Q4, double, float>::type R;
    R cs = 1, sn = 0;
    if (turns) turn_cs(pos, a.rot, pr, cs, sn);
    for (int r = tid / P; r < C; r += 256 / P) {
      float u = 0.f, x = 0.f;
      if (r < nq) {
        const bf16* src = (const bf16*)a.q + b * a.q_b + (size_t)(h0 + r) * D;
        u = (float)src[c0];
        x = (float)src[c1];
      }
      if (turns) {
        const float u2 = u * (float)cs - x * (float)sn;
        x = x * (float)cs + u * (float)sn;
        u = u2;
      }
      if (a.negate) u = -u, x = -x;
      const bf16 uh = (bf16)u, xh = (bf16)x;
      qh[r * QS + c0] = uh;
      qh[r * QS + c1] = xh;
      ql[r * QS + c0] = (bf16)(u - (float)uh);
      ql[r * QS + c1] = (bf16)(x - (float)xh);
    }
    // the split that holds the new row writes it; only this workgroup reads it,
    // behind the barrier
    const long long row = a.fuse_append && T_b - 1 >= k_lo && T_b - 1 < k_hi ? page_row(a.pg, table, T_b - 1) : -1;
    if (row >= 0) {
      const long long r = row + ((long long)hk << a.pg.shift);
      const bf16* kn = (const bf16*)a.k_new + b * a.k_b + (size_t)hk * D;
      const bf16* vn = (const bf16*)a.v_new + b * a.v_b + (size_t)hk * D;
      if (tid < P) {
        const R u = (R)(float)kn[c0], x = (R)(float)kn[c1];
        const R u2 = turns ? u * cs - x * sn : u, x2 = turns ? x * cs + u * sn : x;
        if constexpr (Q4) {
          nrow[0][c0] = Quant4::odd(u2);
          nrow[0][c1] = Quant4::odd(x2);
          nrow[1][c0] = (float)vn[c0];
          nrow[1][c1] = (float)vn[c1];
        } else {
          bf16 *kd = (bf16*)a.kp + r * D, *vd = (bf16*)a.vp + r * D;
          kd[c0] = turns ? (bf16)u2 : kn[c0];
          kd[c1] = turns ? (bf16)x2 : kn[c1];
          vd[c0] = vn[c0];
          vd[c1] = vn[c1];
        }
      }
      if constexpr (Q4) {
        __syncthreads();   // row is the same for the whole workgroup
        if (tid < D / 4) {
          const int which = tid / (D / 8), ch = tid % (D / 8);
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) v[e] = nrow[which][8 * ch + e];
          uint32_t sc;
          const uint32_t x = Quant4::put(v, sc);
          ((uint32_t*)(which ? a.vp : a.kp))[r * (D / 8) + ch] = x;
          if (ch % 4 == 0) (which ? a.vsc : a.ksc)[r * (D / 32) + ch / 4] = (uint8_t)sc;
        }
      }
    }
  }
  __syncthreads();
  bf16x8 qf[NQ][TD], qr[NQ][TD];
#pragma unroll
  for (int x = 0; x < NQ; ++x)
#pragma unroll
    for (int t = 0; t < TD; ++t) {
      const int at = (16 * x + c) * QS + (Q4 ? D / 4 * g + 8 * t : 32 * t + 8 * g);
      qf[x][t] = *(const bf16x8*)(qh + at);
      qr[x][t] = *(const bf16x8*)(ql + at);
    }
  __syncthreads();   // the stages below take this memory

  f32x4 oacc[NQ][DB];
  float m_use[NQ], lsum[NQ];
#pragma unroll
  for (int x = 0; x < NQ; ++x) {
    m_use[x] = -INFINITY;
    lsum[x] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[x][db] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }

  struct Block {
    uint32_t k[KB][KW];
    u32x4 v[NV];
    uint32_t ks[Q4 ? KB : 1], vs[Q4 ? KB : 1][Q4 ? TD : 1];
    int lim[KB];   // keys of each row of 16 that take part
  };
  // loads of the block at key kv0 (a multiple of 16, inside the table)
  auto load = [&](Block& x, int kv0) __attribute__((always_inline)) {
    long long row[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const int p = kv0 + kGranule * kb;
      x.lim[kb] = 0;
      row[kb] = 0;   // the first rows of page 0, which exist: never used
      if (p < k_hi) {
        const int page = ((ConstInt)(uintptr_t)table)[p >> a.pg.shift];
        if (page_ok(a.pg, page)) {
          row[kb] = (((long long)page * a.pg.Hkv + hk) << a.pg.shift) + (p & ((1 << a.pg.shift) - 1));
          x.lim[kb] = min(k_hi - p, kGranule);
        }
      }
    }
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const unsigned char* src = (const unsigned char*)a.kp + row[kb] * RB + c * RB + (Q4 ? RB / 4 * g : 16 * g);
      if constexpr (!Q4) {
#pragma unroll
        for (int t = 0; t < TD; ++t) {
          const u32x4 y = *(const u32x4*)(src + 64 * t);
#pragma unroll
          for (int e = 0; e < 4; ++e) x.k[kb][4 * t + e] = y[e];
        }
      } else {
        if constexpr (TD == 4) {
          const u32x4 y = *(const u32x4*)src;
#pragma unroll
          for (int e = 0; e < 4; ++e) x.k[kb][e] = y[e];
        } else if constexpr (TD == 2) {
          const u32x2 y = *(const u32x2*)src;
          x.k[kb][0] = y[0];
          x.k[kb][1] = y[1];
        } else {
          x.k[kb][0] = *(const uint32_t*)src;
        }
        x.ks[kb] = a.ksc[(row[kb] + c) * TD + g * TD / 4];
        const unsigned char* vs = a.vsc + (row[kb] + 4 * g) * TD;
        if constexpr (TD == 4) {
          const u32x4 y = *(const u32x4*)vs;
#pragma unroll
          for (int e = 0; e < 4; ++e) x.vs[kb][e] = y[e];
        } else if constexpr (TD == 2) {
          const u32x2 y = *(const u32x2*)vs;
          x.vs[kb][0] = y[0];
          x.vs[kb][1] = y[1];
        } else {
          x.vs[kb][0] = *(const uint32_t*)vs;
        }
      }
    }
    // V: 1 KB per load, the block's rows one after the other
#pragma unroll
    for (int m = 0; m < NV; ++m) {
      constexpr int RPL = 1024 / RB;   // rows of a load
      const int r = RPL * m + lane / (64 / RPL);
      long long base = row[RPL * m / kGranule];
      if constexpr (RPL > kGranule) {
#pragma unroll
        for (int kb = 1; kb < RPL / kGranule; ++kb)
          base = r / kGranule == RPL * m / kGranule + kb ? row[RPL * m / kGranule + kb] : base;
      }
      x.v[m] = *(const u32x4*)((const unsigned char*)a.vp + (base + r % kGranule) * RB + 16 * (lane % (64 / RPL)));
    }
  };

  unsigned char* vst = smem + w * (BK * RB);
  const float sl2 = a.sl2;
  auto step = [&](Block& x) __attribute__((always_inline)) {
    bool whole = true;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) whole = whole && x.lim[kb] == kGranule;
    // V to LDS; rows that take no part as zeros, so that P's zeros meet no NaN
#pragma unroll
    for (int m = 0; m < NV; ++m) {
      constexpr int RPL = 1024 / RB, CPR = 64 / RPL;
      const int r = RPL * m + lane / CPR, ch = lane % CPR;
      u32x4 y = x.v[m];
      if constexpr (!Q4) {
        if (!whole) {
          int lim = x.lim[0];
#pragma unroll
          for (int kb = 1; kb < KB; ++kb) lim = r / kGranule == kb ? x.lim[kb] : lim;
          if (r % kGranule >= lim) y = (u32x4){0u, 0u, 0u, 0u};
        }
        *(u32x4*)(vst + r * RB + 16 * (ch ^ swz16<D>(r))) = y;
      } else {
        // 8-byte pieces; the eight rows that a half-wave's transposed read takes
        // at one place of a 256-byte line get different pieces of it
        const int f = D == 128 ? ((r >> 4) & 3) * 2 + ((r >> 2) & 1) : D == 64 ? (r >> 4) & 3 : (r >> 4) & 1;
        *(u32x2*)(vst + r * RB + 8 * ((2 * ch) ^ f)) = (u32x2){y[0], y[1]};
        *(u32x2*)(vst + r * RB + 8 * ((2 * ch + 1) ^ f)) = (u32x2){y[2], y[3]};
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    f32x4 s[NQ][KB];
#pragma unroll
    for (int q = 0; q < NQ; ++q)
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) s[q][kb] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int t = 0; t < TD; ++t) {
        bf16x8 kf;
        if constexpr (Q4) kf = Quant4::get(x.k[kb][t], __uint_as_float(x.ks[kb] << 23));
        else kf = __builtin_bit_cast(bf16x8, (u32x4){x.k[kb][4 * t], x.k[kb][4 * t + 1], x.k[kb][4 * t + 2], x.k[kb][4 * t + 3]});
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          mma16(s[q][kb], kf, qf[q][t]);
          if (a.rot.r) mma16(s[q][kb], kf, qr[q][t]);
        }
      }
    if (!whole) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
#pragma unroll
          for (int q = 0; q < NQ; ++q) s[q][kb][i] = 4 * g + i < x.lim[kb] ? s[q][kb][i] : -INFINITY;
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
      bf16x8 pf[NQ];
#pragma unroll
      for (int q = 0; q < NQ; ++q) pf[q] = frag16(s[q][0], s[q][1]);
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const bf16x8 vf = tr_read16<D, BK>((const bf16*)vst, 0, db, g, c);
#pragma unroll
        for (int q = 0; q < NQ; ++q) mma16(oacc[q][db], vf, pf[q]);
      }
    } else {
      if (!whole) {   // scales of rows that take no part
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int t = 0; t < TD; ++t) {
            // byte k of the words together is row k / TD, block k % TD
            const int keep = max(0, min(x.lim[kb] - 4 * g, 4)) * TD - 4 * t;   // bytes of this word
            x.vs[kb][t] &= keep >= 4 ? ~0u : keep <= 0 ? 0u : (1u << (8 * keep)) - 1;
          }
      }
      const int rr = 16 * (c >> 2) + 4 * g + (c & 3);   // the row whose columns this lane fetches
      const int f = D == 128 ? ((rr >> 4) & 3) * 2 + ((rr >> 2) & 1) : D == 64 ? (rr >> 4) & 3 : (rr >> 4) & 1;
#pragma unroll
      for (int dg = 0; dg < TD; ++dg) {
        bf16x8 pf[NQ][2];
        f32x4 sc[KB];
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int k = i * TD + dg;
            sc[kb][i] = __uint_as_float(((x.vs[kb][k / 4] >> (8 * (k % 4))) & 255u) << 23);
          }
#pragma unroll
        for (int q = 0; q < NQ; ++q) {
          pf[q][0] = frag16(s[q][0] * sc[0], s[q][1] * sc[1]);
          pf[q][1] = frag16(s[q][2] * sc[2], s[q][3] * sc[3]);
        }
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
          }
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  };

  {
    Block A, B2;
    int kv = k_lo + BK * w;
    if (kv < k_hi) load(A, kv);
    while (kv < k_hi) {
      const bool more = kv + 4 * BK < k_hi;
      if (more) load(B2, kv + 4 * BK);
      step(A);
      if (!more) break;
      kv += 8 * BK;
      if (kv < k_hi) load(A, kv);
      step(B2);
    }
  }

  // ---- merge the waves through LDS: O parts [4][D][C], maxima and sums [4][C]
  __syncthreads();
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
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int i = 0; i < 4; ++i) ow[(w * D + 16 * db + 4 * g + i) * C + 16 * q + c] = oacc[q][db][i];
  }
  __syncthreads();
  for (int it = tid; it < C * (D / 4); it += 256) {
    const int col = it % C, d4 = it / C;
    if (col >= nq) continue;
    float M = -INFINITY, l = 0.f;
#pragma unroll
    for (int v = 0; v < 4; ++v) M = fmaxf(M, ml[0][v][col]);
    f32x4 acc = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int v = 0; v < 4; ++v) {
      const float f = M == -INFINITY ? 0.f : exp2_fast(ml[0][v][col] - M);
      l += f * ml[1][v][col];
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] += f * ow[(v * D + 4 * d4 + i) * C + col];
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

}  // namespace attn
