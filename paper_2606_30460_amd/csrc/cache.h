// Index arithmetic and token ranges of the paged K/V cache shared by its kernels and, built for the host, by the tests.
#pragma once

#include <cstdint>

#if defined(__HIPCC__)
#include <hip/hip_runtime.h>
#define HSAP_CACHE_HD __host__ __device__ __forceinline__
#else
#define HSAP_CACHE_HD inline
#endif

namespace hsap {

// Page that holds position pos of a sequence whose table row is `row` (table_width entries): -1 where the position lies
// behind the table or the entry is no page.
HSAP_CACHE_HD int32_t cache_page(const int32_t* row, int32_t table_width, int32_t num_pages, int32_t page_size, int32_t pos) {
  if (pos < 0) return -1;
  const int32_t at = (int32_t)((uint32_t)pos / (uint32_t)page_size);
  if (at >= table_width) return -1;
  const int32_t page = row[at];
  return page >= 0 && page < num_pages ? page : -1;
}

// Element offset of (page, head, slot, 0) in the codes [num_pages, heads, page_size, head_dim].
HSAP_CACHE_HD int64_t cache_row(int64_t page, int32_t heads, int32_t head, int32_t page_size, int32_t slot, int32_t head_dim) {
  return ((page * heads + head) * page_size + slot) * head_dim;
}

// Ragged work lists.  Sequence s has new tokens cu[s] .. cu[s + 1] - 1; its T tokens need up to T * num / den + add items
// (rounded down).  Its items are numbered from item_base(cu[s], s): bases of successive sequences are far enough
// apart for any split of the tokens, since floor(a + b) >= floor(a) + floor(b).  An item number maps back to the last
// sequence whose base is not above it.
HSAP_CACHE_HD int64_t item_base(int64_t cu, int64_t num, int64_t den, int64_t add, int64_t s) { return cu * num / den + add * s; }

// Workgroups of 256 threads that a launch can have: the runtime counts its threads in 32 bits.
constexpr int64_t kMaxBlocks256 = (int64_t(1) << 32) / 256 - 1;

// e of a page's scale 2^e: the smallest exponent with amax <= 448 * 2^e, within [-100, 120].  448 = 1.75 * 2^8, so e is
// amax's own exponent less 8, and one more where its significand is above 1.75.
constexpr int kMinScaleExp = -100, kMaxScaleExp = 120;
HSAP_CACHE_HD int scale_exponent(uint32_t amax_bits) {
  const int e = (int)((amax_bits >> 23) & 255) - 127 - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return e < kMinScaleExp ? kMinScaleExp : e > kMaxScaleExp ? kMaxScaleExp : e;
}

// Token ranges that the rows at positions plo .. phi of one sequence see, in steps of STEP: the sinks' from 0 on, then the
// windows'.  Tokens at or behind cap are in no page.
template <int STEP>
struct Steps {
  int32_t sinks;   // sink steps
  int32_t win0;    // first token of the window steps (a multiple of STEP)
  int32_t lo;      // first token of a window, win0 or less than STEP behind it
  int32_t total;

  HSAP_CACHE_HD int32_t first(int32_t s) const { return s < sinks ? STEP * s : win0 + STEP * (s - sinks); }
  // Of a step's tokens up to the last row's position some row sees those from the first window on and the sinks, so all of
  // them behind the first window step; in the steps before that and in it, a place that no row sees may hold anything, NaN
  // included.
  HSAP_CACHE_HD bool edge(int32_t s) const { return s <= sinks; }
  HSAP_CACHE_HD bool seen(int32_t all_sinks, int32_t from, int32_t to) const {  // a token of from .. to
    return (to >= lo) | (from < all_sinks);
  }
  // Whether the page of sixteen tokens from `from` on is looked up (top: last token any row sees): the entries of pages
  // without a token that some row sees may be those of pages handed back.
  HSAP_CACHE_HD bool looked_up(int32_t all_sinks, int32_t from, int32_t top) const {
    return (from <= top) & seen(all_sinks, from, from + 15);
  }
};

template <int STEP>
HSAP_CACHE_HD Steps<STEP> cache_steps(int32_t plo, int32_t phi, int32_t cap, int32_t window, int32_t sinks) {
  phi = phi < cap - 1 ? phi : cap - 1;
  if (phi < 0) return Steps<STEP>{0, 0, 0, 0};
  const int32_t back = (plo > 0 ? plo : 0) - (window - 1), lo = back > 0 ? back : 0;
  const int32_t win0 = (lo <= phi ? lo : phi + 1) & ~(STEP - 1);
  const int32_t ns = ((sinks < win0 ? sinks : win0) + STEP - 1) / STEP;
  return Steps<STEP>{ns, win0, lo, ns + (phi >= win0 ? (phi - win0) / STEP + 1 : 0)};
}

}  // namespace hsap
