// C ABI of the rotary positions and the paged key/value cache (declared in
// include/attn_mi355x.h): argument validation, plans and launches. As in attn.hip,
// everything is validated on the host before any HIP call.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
#include <cmath>
#include <cstdint>
#include <type_traits>
#include <utility>

#include "attn_mi355x.h"
#include "launch.hpp"
#include "paged.hpp"

namespace {

using attn::bf16;
using attn::Strides;
using attn::writable;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

bool good_d(int d) { return d == 32 || d == 64 || d == 128; }

// The rotation's arguments; `freqs` null: none.
int check_rotation(const double* freqs, int r, int d, float amplitude, int interleaved) {
  if (interleaved != 0 && interleaved != 1) return ATTN_E_ARG;
  if (!freqs) return ATTN_OK;
  if (!std::isfinite(amplitude)) return ATTN_E_ARG;
  if (r < 16 || r > d || r % 16 != 0) return ATTN_E_UNSUPPORTED;
  return aligned(freqs, 8) ? ATTN_OK : ATTN_E_ALIGN;
}
attn::Rotation rotation(const double* freqs, int r, float amplitude) {
  attn::Rotation rot{};
  rot.freqs = freqs;
  rot.r = freqs ? r : 0;
  rot.amplitude = amplitude;
  return rot;
}

// The caller's strides (sequence, head, token), or those of a dense [B, H, n, d].
// That of an axis of one entry says nothing.
Strides strides_of(const long long* s, int B, int H, int n, int d) {
  Strides r = {(long long)H * n * d, (long long)n * d, d};
  if (s) r = {s[0], s[1], s[2]};
  if (B == 1) r.b = 0;
  if (H == 1) r.h = 0;
  if (n == 1) r.t = 0;
  return r;
}
// Rows start at multiples of 16 bytes.
bool aligned(const Strides& s, int elem) {
  const int m = 16 / elem;
  return s.b % m == 0 && s.h % m == 0 && s.t % m == 0;
}
bool fits(const Strides& s, int B, int H, int n) {   // offsets in 62 bits
  __int128 far = 0;
  for (const auto& [step, size] : {std::pair<long long, int>{s.b, B}, {s.h, H}, {s.t, n}}) {
    if (step < 0) return false;
    far += (__int128)step * (size - 1);
  }
  return far < ((__int128)1 << 60);
}

// Workgroups of 256 threads for `rows` rows, `per` to a workgroup; a launch has fewer
// than 2^32 threads along an axis.
long long blocks_for(long long rows, int per) { return (rows + per - 1) / per; }
bool launches(long long rows, int per) { return blocks_for(rows, per) < 1LL << 24; }

// Heads per workgroup: a thread's sines and cosines serve all of them, so as many,
// up to 8, as leave four workgroups per compute unit (rotation of 2 x 64 heads, n = 16384:
// 197 us, one head each 228, up to 16 211; append of 16000 tokens of 8 heads in 4 bits 23.8,
// one head each 42.6, up to 4 24.4).
int heads_per_group(long long token_blocks, int heads) {
  const long long want = attn::kXcds * attn::kCusPerXcd * 4;
  return (int)std::max<long long>(1, std::min<long long>({8, heads, token_blocks * heads / want}));
}

template <typename T> void launch_rope(attn::RopeArgs a, bool interleaved, hipStream_t st) {
  const unsigned blocks = (unsigned)blocks_for(a.tokens, 512 * attn::Chunk<T>::N / a.d);
  a.hgroup = heads_per_group(blocks, a.Hq + a.Hk);
  const dim3 grid(blocks, (a.Hq + a.Hk + a.hgroup - 1) / a.hgroup);
  if (interleaved) hipLaunchKernelGGL((attn::rope_kernel<T, true>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((attn::rope_kernel<T, false>), grid, dim3(256), 0, st, a);
}

int rope(const void* q, const void* k, void* q_out, void* k_out, const long long* strides, const double* freqs,
         const int* positions, long long pos_stride, int start, int B, int Hq, int Hk, int n, int d, int r,
         float amplitude, int interleaved, int dtype, void* stream, float sign) {
  if (!q || !q_out || !freqs || (k == nullptr) != (k_out == nullptr)) return ATTN_E_NULL;
  if (!k) Hk = 0;
  if (B < 1 || Hq < 1 || (k && Hk < 1) || n < 1) return ATTN_E_SHAPE;
  if (dtype != ATTN_BF16 && dtype != ATTN_F32) return ATTN_E_UNSUPPORTED;
  if (!good_d(d)) return ATTN_E_UNSUPPORTED;
  if (const int rc = check_rotation(freqs, r, d, amplitude, interleaved)) return rc;
  const int elem = dtype == ATTN_BF16 ? 2 : 4;
  if ((long long)B * n > INT_MAX || !launches((long long)B * n, 8192 / elem / d) || (long long)Hq + Hk > 65535)
    return ATTN_E_SHAPE;
  if (positions ? pos_stride < 0 || pos_stride > LLONG_MAX / B : start > INT_MAX - n) return ATTN_E_SHAPE;
  attn::RopeArgs a{};
  a.q = q; a.k = k; a.qo = q_out; a.ko = k_out;
  a.qs = strides_of(strides, B, Hq, n, d);
  a.qos = strides_of(strides ? strides + 6 : nullptr, B, Hq, n, d);
  if (!fits(a.qs, B, Hq, n) || !fits(a.qos, B, Hq, n)) return ATTN_E_SHAPE;
  if (!aligned(q, 16) || !aligned(q_out, 16) || !aligned(a.qs, elem) || !aligned(a.qos, elem) ||
      (positions && !aligned(positions, 4)))
    return ATTN_E_ALIGN;
  if (!writable(a.qos, B, Hq, n, d)) return ATTN_E_ARG;
  if (k) {
    a.ks = strides_of(strides ? strides + 3 : nullptr, B, Hk, n, d);
    a.kos = strides_of(strides ? strides + 9 : nullptr, B, Hk, n, d);
    if (!fits(a.ks, B, Hk, n) || !fits(a.kos, B, Hk, n)) return ATTN_E_SHAPE;
    if (!aligned(k, 16) || !aligned(k_out, 16) || !aligned(a.ks, elem) || !aligned(a.kos, elem)) return ATTN_E_ALIGN;
    if (!writable(a.kos, B, Hk, n, d)) return ATTN_E_ARG;
    const long long apart = (reinterpret_cast<intptr_t>(k_out) - reinterpret_cast<intptr_t>(q_out)) / elem;
    if (attn::rows_meet(a.qos, Hq, a.kos, Hk, B, n, d, apart)) return ATTN_E_ARG;
  }
  a.pos = positions;
  a.pos_stride = pos_stride;
  a.start = start;
  a.rot = rotation(freqs, r, amplitude);
  a.Hq = Hq; a.Hk = Hk; a.n = n; a.d = d;
  a.tokens = B * n;
  a.sign = sign;
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (dtype == ATTN_BF16) launch_rope<bf16>(a, interleaved, st);
  else launch_rope<float>(a, interleaved, st);
  return hipGetLastError() == hipSuccess ? ATTN_OK : ATTN_E_HIP;
}

// A pool and its tables.
int check_pages(const void* kp, const void* vp, const void* ksc, const void* vsc, const int* table, const int* lens,
                int B, int Hkv, int num_pages, int page_size, int width, int d, int dtype) {
  if (!kp || !vp || !table || !lens || (ksc == nullptr) != (vsc == nullptr)) return ATTN_E_NULL;
  if (B < 1 || Hkv < 1 || num_pages < 1 || width < 1) return ATTN_E_SHAPE;
  if (dtype != ATTN_BF16 || !good_d(d)) return ATTN_E_UNSUPPORTED;
  if (page_size < attn::kGranule || page_size > (1 << 20) || (page_size & (page_size - 1)) != 0) return ATTN_E_UNSUPPORTED;
  if ((__int128)num_pages * Hkv * page_size * d > ((__int128)1 << 46)) return ATTN_E_SHAPE;
  if (B > 65535 || Hkv > 65535) return ATTN_E_SHAPE;   // grid limits
  if (!aligned(kp, 16) || !aligned(vp, 16) || !aligned(ksc, 16) || !aligned(vsc, 16) || !aligned(table, 4) ||
      !aligned(lens, 4))
    return ATTN_E_ALIGN;
  return ATTN_OK;
}
attn::Pages pages_of(const int* table, int Hkv, int num_pages, int page_size, int width) {
  attn::Pages p{};
  p.table = table;
  p.width = width;
  p.num_pages = num_pages;
  while ((1 << p.shift) < page_size) ++p.shift;
  p.Hkv = Hkv;
  return p;
}

template <int D> void launch_append4(const attn::AppendArgs& a, const dim3& grid, bool interleaved, hipStream_t st) {
  if (interleaved) hipLaunchKernelGGL((attn::append4_kernel<D, true>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((attn::append4_kernel<D, false>), grid, dim3(256), 0, st, a);
}
int append_tokens(int d, bool q4) { return 256 / (d / (q4 ? 8 : 16)); }   // per workgroup
void launch_append(attn::AppendArgs a, bool interleaved, hipStream_t st) {
  const bool q4 = a.ksc != nullptr;
  const unsigned blocks = (unsigned)blocks_for(a.tokens, append_tokens(a.d, q4));
  a.hgroup = heads_per_group(blocks, a.pg.Hkv);
  const dim3 grid(blocks, (a.pg.Hkv + a.hgroup - 1) / a.hgroup);
  if (q4) {
    if (a.d == 32) launch_append4<32>(a, grid, interleaved, st);
    else if (a.d == 64) launch_append4<64>(a, grid, interleaved, st);
    else launch_append4<128>(a, grid, interleaved, st);
  } else {
    if (interleaved) hipLaunchKernelGGL(attn::append_kernel<true>, grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL(attn::append_kernel<false>, grid, dim3(256), 0, st, a);
  }
}

// Decode: a workgroup owns (sequence, cache head, up to 32 query heads, one split
// of the keys). Times are a step's, merge included, back to back in a captured graph.
//
// Up to 256 groups the keys are split, a block for each of its four waves at least, into as
// many parts as leave no more than two workgroups per compute unit, so that all run at once
// (160 groups of 1900 tokens in 4 bits 15.9 us in three parts, 19.3 in four, 640
// workgroups; one sequence of 131072 tokens in 4 bits 33, up to 768 workgroups 37). From 257
// to 511 groups they are split in two, up to 1022 workgroups, which even each other out
// (384 groups of 2000 tokens, bfloat16, 68.5 us, undivided 77). From 512 on they are not
// split: two parts cost 2 to 10 % where the lengths are alike (512 groups of 4096 tokens,
// bfloat16 169 us, 172 in two; 4 bits 54 and 58). The price is a batch of which one sequence
// is far longer than the rest, whose step takes as long as that one's workgroup (64
// sequences of 8 heads, one of 16000 tokens, the others of 500: bfloat16 222 us, 119 in two
// parts; 4 bits 76, 46).
//
// Merging the splits costs a launch and 2.7 to 4.7 us, so up to a number of blocks
// the keys stay undivided: few where many parts would share them (d = 128, 600 tokens in
// 4 bits, 64 groups: 9.4 us, in two parts 10.5), more for three (160 groups of 1200
// tokens in 4 bits 12.2, 13.7) and most where two workgroups of a compute unit would
// only halve what one has to itself (256 groups of 1900 tokens in 4 bits 17.4, 20.1;
// bfloat16, 1500: 35.1, 37.2). Beyond, sequences of different lengths need the
// splits (176 groups of 8000 to 16000 tokens in 4 bits 74 us, undivided 78). At d = 64 and 32
// the numbers of blocks are those of d = 128: they save less there (256 groups of 1500
// tokens, bfloat16: d = 64 18.5 us, 20.8 in two parts, d = 32 11.7, 14.0), and in few groups of
// bfloat16 they split too early (16 groups of 600 tokens, d = 32: 6.6 us, undivided 6.0).
//
// More than 16 query heads of a cache head are two columns of 16, which read the keys
// once (220 groups of 8000 tokens, 32 heads, d = 64: 60.5 us in 4 bits, 68.0 by workgroups
// of one column; bfloat16 84, 159), or, with so few blocks that latency counts, workgroups
// of one column each (2 groups of 1500 tokens, d = 64, 4 bits 8.8 us, two columns 9.9;
// bfloat16, d = 128, 500 tokens 9.1, 10.6). In 4 bits at d = 128 always the latter: two
// columns need more registers than there are, and what is spilled comes back behind the next
// block's loads (16 groups of 8000 tokens 16.9 us, 27.1; 220 of 1500 28.3, 38.2).
constexpr long long kWorkgroups = 2 * attn::kXcds * attn::kCusPerXcd;
struct PagedPlan {
  int nq;        // query columns of a workgroup / 16
  int qchunks, nsplit;
};
PagedPlan paged_plan(int B, int Hq, int Hkv, int n, int d, int append, bool q4) {
  PagedPlan p;
  const int G = Hq / Hkv, block = q4 ? 64 : 32;
  const long long blocks = ((long long)n + append + block - 1) / block;
  const long long pairs = (long long)B * Hkv * ((G + 31) / 32);
  p.nq = G > 16 && !(q4 && d == 128) && pairs * blocks > (q4 ? 2048 : 512) ? 2 : 1;
  p.qchunks = (G + 16 * p.nq - 1) / (16 * p.nq);
  const long long groups = (long long)B * Hkv * p.qchunks;
  const bool crowded = 2 * groups > kWorkgroups;
  const long long parts = groups >= kWorkgroups ? 1 : crowded ? 2 : kWorkgroups / groups;
  const long long undivided = parts > 3 ? (q4 ? 16 : 12) : parts == 3 || crowded ? (q4 ? 32 : 16) : (q4 ? 128 : 64);
  p.nsplit = blocks <= undivided ? 1 : (int)std::min(parts, blocks / 4);
  return p;
}

template <int D, int NQ, int REP, bool Q4> void launch_decode(const attn::PagedArgs& a, const dim3& grid, hipStream_t st) {
  constexpr int block = Q4 ? 64 : 32;
  if (1 << a.pg.shift >= block)
    hipLaunchKernelGGL((attn::paged_decode_kernel<D, NQ, REP, Q4, block>), grid, dim3(256), 0, st, a);
  else
    hipLaunchKernelGGL((attn::paged_decode_kernel<D, NQ, REP, Q4, attn::kGranule>), grid, dim3(256), 0, st, a);
}
template <int D> void launch_decode(const attn::PagedArgs& a, const dim3& grid, int nq, hipStream_t st) {
  if (!a.ksc) {
    nq == 1 ? launch_decode<D, 1, 1, false>(a, grid, st) : launch_decode<D, 2, 1, false>(a, grid, st);
  } else if (D < 128 && nq == 2) {
    launch_decode<D < 128 ? D : 64, 2, 1, true>(a, grid, st);
  } else if (D == 128 && a.G <= 4) {   // as often in the 16 columns as the heads go into them
    launch_decode<D, 1, D / 32, true>(a, grid, st);
  } else if (D >= 64 && a.G <= 8) {
    launch_decode<D, 1, D == 32 ? 1 : 2, true>(a, grid, st);
  } else {
    launch_decode<D, 1, 1, true>(a, grid, st);
  }
}

// One wave per row while it can have the loads of all splits in flight at once, otherwise
// eight (a step of 3 heads in 512 splits at d = 128: 15.1 us, with one wave 32.6; of 32 heads
// in 8 splits 9.0, with eight waves and their join through LDS 9.6).
template <int D> void launch_combine(const attn::PagedArgs& a, hipStream_t st) {
  if (a.nsplit <= 8 * 256 / D)
    hipLaunchKernelGGL((attn::paged_combine_kernel<D, 1>), dim3(a.rows), dim3(64), 0, st, a.part, a.o, a.lse, a.rows, a.nsplit);
  else
    hipLaunchKernelGGL((attn::paged_combine_kernel<D, 8>), dim3(a.rows), dim3(512), 0, st, a.part, a.o, a.lse, a.rows, a.nsplit);
}

}  // namespace

extern "C" {

int attn_rope(const void* q, const void* k, void* q_out, void* k_out, const long long* strides, const double* freqs,
              const int* positions, long long pos_stride, int start, int B, int Hq, int Hk, int n, int d, int r,
              float amplitude, int interleaved, int dtype, void* stream) {
  return rope(q, k, q_out, k_out, strides, freqs, positions, pos_stride, start, B, Hq, Hk, n, d, r, amplitude,
              interleaved, dtype, stream, 1.f);
}

int attn_rope_bwd(const void* dq, const void* dk, void* dq_in, void* dk_in, const long long* strides, const double* freqs,
                  const int* positions, long long pos_stride, int start, int B, int Hq, int Hk, int n, int d, int r,
                  float amplitude, int interleaved, int dtype, void* stream) {
  return rope(dq, dk, dq_in, dk_in, strides, freqs, positions, pos_stride, start, B, Hq, Hk, n, d, r, amplitude,
              interleaved, dtype, stream, -1.f);
}

int attn_paged_append(const void* k_new, const void* v_new, const long long* strides, void* k_pages, void* v_pages,
                      void* k_scales, void* v_scales, const int* block_table, const int* lens, const int* new_lens,
                      const double* freqs, const int* positions, int B, int Hkv, int T, int num_pages, int page_size,
                      int table_width, int d, int r, float amplitude, int interleaved, int dtype, void* stream) {
  if (!k_new || !v_new) return ATTN_E_NULL;
  if (const int rc = check_pages(k_pages, v_pages, k_scales, v_scales, block_table, lens, B, Hkv, num_pages, page_size,
                                 table_width, d, dtype))
    return rc;
  if (T < 1 || (long long)B * T > INT_MAX || !launches((long long)B * T, append_tokens(d, k_scales != nullptr)))
    return ATTN_E_SHAPE;
  if (const int rc = check_rotation(freqs, r, d, amplitude, interleaved)) return rc;
  attn::AppendArgs a{};
  a.k_new = k_new; a.v_new = v_new;
  a.ks = strides_of(strides, B, Hkv, T, d);
  a.vs = strides_of(strides ? strides + 3 : nullptr, B, Hkv, T, d);
  if (!fits(a.ks, B, Hkv, T) || !fits(a.vs, B, Hkv, T)) return ATTN_E_SHAPE;
  if (!aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(a.ks, 2) || !aligned(a.vs, 2) ||
      !aligned(new_lens, 4) || !aligned(positions, 4))
    return ATTN_E_ALIGN;
  a.kp = k_pages; a.vp = v_pages;
  a.ksc = static_cast<uint8_t*>(k_scales); a.vsc = static_cast<uint8_t*>(v_scales);
  a.pg = pages_of(block_table, Hkv, num_pages, page_size, table_width);
  a.lens = lens; a.new_lens = new_lens;
  a.pos = positions;
  a.rot = rotation(freqs, r, amplitude);
  a.T = T; a.d = d; a.tokens = B * T;
  (void)hipGetLastError();
  launch_append(a, interleaved, static_cast<hipStream_t>(stream));
  return hipGetLastError() == hipSuccess ? ATTN_OK : ATTN_E_HIP;
}

int attn_paged_gather(const void* k_pages, const void* v_pages, const void* k_scales, const void* v_scales,
                      const int* block_table, const int* lens, const int* starts, void* K, void* V, int B, int Hkv,
                      int n, int num_pages, int page_size, int table_width, int d, int dtype, void* stream) {
  if (!K || !V) return ATTN_E_NULL;
  if (const int rc = check_pages(k_pages, v_pages, k_scales, v_scales, block_table, lens, B, Hkv, num_pages, page_size,
                                 table_width, d, dtype))
    return rc;
  const int per = 256 / (d / 8);
  if (n < 1 || !launches(n, per) || (__int128)B * Hkv * n * d > ((__int128)1 << 46)) return ATTN_E_SHAPE;
  if (!aligned(K, 16) || !aligned(V, 16) || !aligned(starts, 4)) return ATTN_E_ALIGN;
  attn::GatherArgs a{};
  a.kp = k_pages; a.vp = v_pages;
  a.ksc = static_cast<const uint8_t*>(k_scales); a.vsc = static_cast<const uint8_t*>(v_scales);
  a.pg = pages_of(block_table, Hkv, num_pages, page_size, table_width);
  a.lens = lens; a.starts = starts;
  a.k = K; a.v = V;
  a.n = n; a.d = d;
  const dim3 grid((unsigned)blocks_for(n, per), Hkv, B);
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  if (k_scales) hipLaunchKernelGGL(attn::gather_kernel<true>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(attn::gather_kernel<false>, grid, dim3(256), 0, st, a);
  return hipGetLastError() == hipSuccess ? ATTN_OK : ATTN_E_HIP;
}

size_t attn_paged_decode_workspace_bytes(int B, int Hq, int Hkv, int n, int d, int append, int bits) {
  if (B < 1 || Hq < 1 || Hkv < 1 || Hq % Hkv != 0 || n < 0 || !good_d(d) || (bits != 16 && bits != 4)) return 0;
  const PagedPlan p = paged_plan(B, Hq, Hkv, n, d, append ? 1 : 0, bits == 4);
  if (p.nsplit == 1) return 0;
  return (size_t)B * Hq * p.nsplit * (size_t)(d + 2) * sizeof(float);
}

int attn_paged_decode(const void* q, const void* k_new, const void* v_new, const long long* strides, void* k_pages,
                      void* v_pages, void* k_scales, void* v_scales, const int* block_table, const int* lens,
                      const double* freqs, const int* positions, void* O, float* L, void* workspace,
                      size_t workspace_bytes, int B, int Hq, int Hkv, int n, int num_pages, int page_size,
                      int table_width, int d, int r, float amplitude, int interleaved, float scale, int dtype,
                      void* stream) {
  if (!q || !O || (k_new == nullptr) != (v_new == nullptr)) return ATTN_E_NULL;
  if (const int rc = check_pages(k_pages, v_pages, k_scales, v_scales, block_table, lens, B, Hkv, num_pages, page_size,
                                 table_width, d, dtype))
    return rc;
  const int append = k_new ? 1 : 0;
  const bool q4 = k_scales != nullptr;
  if (Hq < 1 || Hq % Hkv != 0 || n < 0 || n > INT_MAX - 1024) return ATTN_E_SHAPE;
  if ((long long)n + append > (long long)table_width * page_size) return ATTN_E_SHAPE;
  if ((long long)B * Hq > INT_MAX) return ATTN_E_SHAPE;
  if (!std::isfinite(scale)) return ATTN_E_ARG;
  if (const int rc = check_rotation(freqs, r, d, amplitude, interleaved)) return rc;
  // elements between sequences; with one of them the caller's say nothing
  const bool given = strides && B > 1;
  const long long row_q = given ? strides[0] : (long long)Hq * d, row_k = given ? strides[1] : (long long)Hkv * d,
                  row_v = given ? strides[2] : (long long)Hkv * d;
  for (const long long s : {row_q, row_k, row_v}) {
    if (s < 0 || s > (1LL << 44)) return ATTN_E_SHAPE;
    if (s % 8 != 0) return ATTN_E_ALIGN;
  }
  if (!aligned(q, 16) || !aligned(k_new, 16) || !aligned(v_new, 16) || !aligned(O, 16) || !aligned(L, 4) ||
      !aligned(positions, 4))
    return ATTN_E_ALIGN;
  const PagedPlan plan = paged_plan(B, Hq, Hkv, n, d, append, q4);
  if ((long long)B * Hkv * plan.qchunks > 65535) return ATTN_E_SHAPE;   // grid y limit
  const size_t need = attn_paged_decode_workspace_bytes(B, Hq, Hkv, n, d, append, q4 ? 4 : 16);
  if (need > 0) {
    if (!workspace) return ATTN_E_NULL;
    if (!aligned(workspace, 16)) return ATTN_E_ALIGN;
    if (workspace_bytes < need) return ATTN_E_WORKSPACE;
  }
  attn::PagedArgs a{};
  a.q = q; a.k_new = k_new; a.v_new = v_new;
  a.q_b = row_q; a.k_b = row_k; a.v_b = row_v;
  a.kp = k_pages; a.vp = v_pages;
  a.ksc = static_cast<uint8_t*>(k_scales); a.vsc = static_cast<uint8_t*>(v_scales);
  a.pg = pages_of(block_table, Hkv, num_pages, page_size, table_width);
  a.lens = lens; a.pos = positions;
  a.rot = rotation(freqs, r, amplitude);
  a.part = static_cast<float*>(workspace);
  a.o = O; a.lse = L;
  a.Hq = Hq; a.G = Hq / Hkv; a.n = n; a.append = append; a.rows = B * Hq;
  a.nsplit = plan.nsplit; a.qchunks = plan.qchunks;
  // a zero scale would turn masked scores into NaN: see split_scale in attn.hip
  a.sl2 = std::fmax(std::fabs(scale) * attn::kLog2e, 1e-30f);
  a.interleaved = interleaved;
  a.negate = scale < 0.f;
  hipStream_t st = static_cast<hipStream_t>(stream);
  (void)hipGetLastError();
  const dim3 grid(plan.nsplit, B * Hkv * plan.qchunks);
  if (d == 32) launch_decode<32>(a, grid, plan.nq, st);
  else if (d == 64) launch_decode<64>(a, grid, plan.nq, st);
  else launch_decode<128>(a, grid, plan.nq, st);
  if (plan.nsplit > 1) d == 32 ? launch_combine<32>(a, st) : d == 64 ? launch_combine<64>(a, st) : launch_combine<128>(a, st);
  return hipGetLastError() == hipSuccess ? ATTN_OK : ATTN_E_HIP;
}

}  // extern "C"
