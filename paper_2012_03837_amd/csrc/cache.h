// The paged cache of keys and values in 8 bits, as its kernels see it.
//
// Pages of 2^shift tokens (16 or more): keys [n_pages][Hkv][tokens][dh], values [n_pages][Hkv][dh][tokens], e4m3, with a scale in fp32
// for every page and head.  Values stand transposed, because the token is the index over which attention sums them: sixteen tokens of
// one column are then one access and the operand of two matrix instructions, as sixteen columns of one token are for the keys.
// dh is a multiple of 16, so that every run of sixteen bytes of either pool is whole and aligned.
//
// Scales that the library writes are powers of two: a quotient by them is exact, so that a code is one rounding of the
// stored value whatever else its page holds, and a page's codes move to a larger scale without a second rounding but for those
// below 2^-6 of it.  In 8 bits of floating point a scale between two powers of two would buy nothing but range.
#pragma once
#include "common.h"

namespace lp {

struct CacheView {
  const int32_t *starts, *lens, *table;
  uint8_t *k, *v;
  float *ks, *vs;
  int B, T, rows, Hkv, dh, shift, max_pages, n_pages;
};
// A sequence's new rows, first .. first + n - 1, are its last positions, len - n .. len - 1.
struct Sequence { int first, n, len; };

__device__ __forceinline__ Sequence sequence_of(const CacheView& c, int b) {
  Sequence s;
  const int64_t most = (int64_t)c.max_pages << c.shift;
  const int len = c.lens[b];
  s.len = len < 0 ? 0 : (len < most ? len : (int)most);
  if (c.starts) {
    const int lo = c.starts[b], hi = c.starts[b + 1];
    const bool there = lo >= 0 && hi >= lo && hi <= c.rows && hi - lo <= c.T;
    s.first = there ? lo : 0;
    s.n = there ? hi - lo : 0;
  } else {
    s.first = b * c.T;
    s.n = c.T;
  }
  return s;
}
// Page number of a sequence's slot; -1 where there is none.
__device__ __forceinline__ int page_of(const CacheView& c, int b, int slot) {
  if (slot < 0 || slot >= c.max_pages) return -1;
  const int p = c.table[(int64_t)b * c.max_pages + slot];
  return (unsigned)p < (unsigned)c.n_pages ? p : -1;
}

}  // namespace lp
