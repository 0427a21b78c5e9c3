// Index arithmetic and token ranges of the paged K/V cache shared by its kernels and, built for the host, by the tests.
#pragma once

#include <algorithm>
#include <cstdint>

#include "hsap_internal.h"

#if defined(__HIPCC__)
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

constexpr int kChunkRows = 128;  // rows of a workgroup of cache_chunk_kernel
constexpr int kMaxSplits = 128;  // of a row tile's tokens

// How a call is cut: row tiles, and splits of a tile's tokens so that the grid fills the chip, each of at least 256 tokens.
struct CacheCut {
  int rows;  // of a tile: 16 or 32 (cache_attn_kernel), kChunkRows (cache_chunk_kernel)
  bool once;  // cache_attn_kernel's ONCE
  int64_t tiles;
  int32_t splits;
};

// Workgroups of cache_attn_kernel to aim at: twice what the chip holds at once (64 sequences of 8k tokens: 129 us with 512,
// 128 with 1024, 127 with 2048).  At most 128 splits (one sequence of 128k tokens, two K/V heads, pass in us: 64 splits
// 24.5, 128 19.4, 256 22.0: more partials to join).
constexpr int64_t kCacheGrid = 1024;

// Two 16-row blocks where the sequences have more than 16 rows (28 x 50 rows x 8 of 64 heads of 128, us: 28, one block 34,
// four 48).  128 rows, where the sequences have more than 64 and the grid can be filled: at head_dim 64 always (us, 32 -> 128
// rows: 3 x 700 x 4 over 12000 tokens 44 -> 38; 4 x 300 x 4 over 6000 50 -> 48; 400 x 5 over 200000 445 -> 344), at 128
// over many tokens, since it needs splits sooner and their partials are twice as large (2048 x 8 over 30000 787 -> 665,
// 512 x 4 over 16000 217 -> 188, but 512 x 4, twice, over 8000 103 -> 116 and 32 x 8, 64 times, over 3125 94 -> 119).
constexpr int64_t kChunkGrid = 2 * kComputeUnits, kChunkSplits = 16, kChunkTokens128 = 12000;

// `tokens` is the table's capacity: the lengths are the device's, and the window is not looked at, so that a workspace is
// enough for every window.  A table much wider than its sequences, or a window far below them, gives splits without work (one
// token, window 1024, table of 131072: 94 of 128).
inline CacheCut cache_cut(const hsap_cache_desc& d, int32_t heads_q, int64_t total_q, bool one_each, int64_t tokens) {
  CacheCut c;
  const int64_t group = heads_q / d.heads_kv;
  const int64_t rows = one_each ? group : (total_q * group + d.num_seqs - 1) / std::max(d.num_seqs, 1);
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(kMaxSplits, tokens / 256));
  // workgroups of 128 rows without splits (c.tiles counts a tile more per sequence, which does nothing)
  const int64_t full = (total_q * group + kChunkRows - 1) / kChunkRows * d.heads_kv;
  const bool chunk = rows > 64 && full * std::min(most, kChunkSplits) >= kChunkGrid && (d.head_dim == 64 || tokens >= kChunkTokens128);
  c.rows = chunk ? kChunkRows : rows > 16 ? 32 : 16;
  c.once = one_each && c.rows == 16 && 2 * d.num_seqs * tokens * d.heads_kv * d.head_dim > (int64_t(256) << 20);
  c.tiles = one_each ? (int64_t)d.num_seqs * ((group + c.rows - 1) / c.rows) : item_base(total_q, group, c.rows, 1, d.num_seqs);
  if (!chunk) {
    c.splits = (int32_t)std::min(most, std::max<int64_t>(1, kCacheGrid / std::max<int64_t>(1, c.tiles * d.heads_kv)));
    return c;
  }
  // Splits that make whole rounds of the chip's 512 workgroups, in ns: a round's steps of 64 tokens (2.2 us, head_dim 64 1.5)
  // and its beginning and end, a join and the partials written and read (2048 x 8 rows over 30000 tokens: one split 1086,
  // three 760, two 665).
  c.splits = 1;
  int64_t least = INT64_MAX;
  for (int64_t s = 1; s <= std::min(most, kChunkSplits); ++s) {
    const int64_t rounds = (full * s + kChunkGrid - 1) / kChunkGrid;
    const int64_t steps = (tokens + 64 * s - 1) / (64 * s);
    const int64_t ns = rounds * (steps * (d.head_dim == 64 ? 1500 : 2200) + 6000) +
                       (s > 1 ? 4000 + total_q * heads_q * d.head_dim * 8 * s / 4000 : 0);
    if (ns < least) {
      least = ns;
      c.splits = (int32_t)s;
    }
  }
  return c;
}

}  // namespace hsap
