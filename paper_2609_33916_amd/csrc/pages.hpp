// Addresses in the paged key/value cache, on the host and the device (no HIP
// headers needed, so that they can be checked on the CPU).
//
// A pool is [num_pages, Hkv, page_size, d]: a page holds page_size consecutive
// tokens of one sequence, every cache head's rows together. Sequence b's token
// p lies in page table[b, p / page_size], row p % page_size. page_size is a power
// of two of at least 16, so 16 tokens starting at a multiple of 16 are 16
// consecutive rows of one page: the unit the attention kernel reads.
#pragma once

#include "grid.hpp"

namespace attn {

constexpr int kGranule = 16;

struct Pages {
  const int* table;   // [B, width] page numbers
  int width;          // table entries per sequence
  int num_pages;
  int shift;          // log2(page_size)
  int Hkv;
};

// Whether `page` is one of the pool. Entries behind a sequence's pages may hold
// anything; one within its length that is no page is skipped: its tokens are
// neither read nor written.
ATTN_HD bool page_ok(const Pages& a, int page) { return (unsigned)page < (unsigned)a.num_pages; }

// Row of the pool (rows of all heads and pages counted through) that holds
// token p of a sequence in cache head 0, -1 if it has none; head h's is
// h << shift further. `table`: the sequence's entries.
ATTN_HD long long page_row(const Pages& a, const int* table, int p) {
  if (p < 0 || (p >> a.shift) >= a.width) return -1;
  const int page = table[p >> a.shift];
  if (!page_ok(a, page)) return -1;
  return (((long long)page * a.Hkv) << a.shift) + (p & ((1 << a.shift) - 1));
}

}  // namespace attn
