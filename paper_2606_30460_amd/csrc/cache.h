// Index arithmetic of the paged K/V cache shared by its kernels and, built for the host, by the tests.
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

// e of a page's scale 2^e: the smallest exponent with amax <= 448 * 2^e, within [-100, 120].  448 = 1.75 * 2^8, so e is
// amax's own exponent less 8, and one more where its significand is above 1.75.
constexpr int kMinScaleExp = -100, kMaxScaleExp = 120;
HSAP_CACHE_HD int scale_exponent(uint32_t amax_bits) {
  const int e = (int)((amax_bits >> 23) & 255) - 127 - 8 + ((amax_bits & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  return e < kMinScaleExp ? kMinScaleExp : e > kMaxScaleExp ? kMaxScaleExp : e;
}

}  // namespace hsap
