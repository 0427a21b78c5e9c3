// What the attention kernels over the paged cache share: arguments, row tiles, decoding, the masks of drafted tokens.
#pragma once

#include <type_traits>

#include "cache.h"
#include "hsap_internal.h"
#include "mfma.h"
#include "window.h"

namespace hsap {

struct CacheAttnArgs {
  hsap_cache_desc d;
  hsap_cache c;
  const __bf16* q;
  int64_t q_stride;
  const int32_t* cu;
  int64_t total_q;
  __bf16* o;
  float* lse;      // may be NULL
  float* part_o;   // [splits, total_q, Hq, d], normalised
  float* part_lse; // [splits, total_q, Hq], log2 units
  int32_t heads_q;
  int32_t group;
  int32_t page_shift;  // log2 of the page size
  int32_t window;
  int32_t sinks;
  int32_t splits;
  float scale_log2;
  const uint64_t* mask;      // TREE kernels: [total_q, words]
  const int32_t* positions;  // TREE kernels: [total_q]
  int32_t words;
  int32_t furthest;  // TREE kernels: rows behind this position count as at it
};

// Steps of each split, of `total` steps dealt to `splits` (the last ones may have none).
__device__ __forceinline__ int32_t steps_per_split(int32_t total, int32_t splits) { return (total + splits - 1) / splits; }

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// four e4m3 codes times a power of two to bf16 (exact within bf16's range)
__device__ __forceinline__ void decode4(uint32_t w, float pow2, bf16x2& lo, bf16x2& hi) {
  lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, pow2, false);
  hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, pow2, true);
}

__device__ __forceinline__ f32x4 mfma16(const bf16x8& a, const bf16x8& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// The sequence, first row and rows of a row tile; false where the tile is empty.
struct RowTile {
  int32_t seq, t0, count, row0;  // row0: first row (token * group + head) of the tile within the sequence
  int32_t len;                   // tokens of the sequence
};
__device__ __forceinline__ bool row_tile(const CacheAttnArgs& a, int32_t tile, int rows, RowTile& t) {
  if (!a.cu) {
    const int32_t per = (a.group + rows - 1) / rows;
    t.seq = tile / per;
    t.t0 = t.seq;
    t.count = 1;
    t.row0 = (tile - t.seq * per) * rows;
    if (t.seq >= a.d.num_seqs) return false;
    t.len = max(0, a.c.seq_lens[t.seq]);
    return true;
  }
  const Sequence q = sequence_of(a.cu, a.d.num_seqs, a.group, rows, 1, tile, a.c.seq_lens);
  t.seq = q.s;
  t.t0 = q.begin;
  t.count = (int32_t)min((int64_t)q.end, a.total_q) - t.t0;
  t.len = max(0, q.value);
  const int64_t row0 = (tile - item_base(t.t0, a.group, rows, 1, q.s)) * rows;
  t.row0 = (int32_t)row0;
  return t.count > 0 && row0 < (int64_t)t.count * a.group;
}

// Trees.  A row sees the tokens before the drafted ones, from `base` places on, by its position (window, sinks) and the
// drafted ones that its mask names.  Bits of drafted tokens from .. from + 63 (from may be below 0) of a row's mask:
__device__ __forceinline__ uint64_t mask_bits(const uint64_t* mask, int32_t words, int32_t from) {
  if (from <= -64) return 0;
  if (from < 0) return mask[0] << -from;
  const int32_t w = from >> 6, sh = from & 63;
  uint64_t x = w < words ? mask[w] >> sh : 0;
  if (sh && w + 1 < words) x |= mask[w + 1] << (64 - sh);
  return x;
}
__device__ __forceinline__ uint64_t bits_from(int64_t n) { return n <= 0 ? ~uint64_t(0) : n >= 64 ? 0 : ~uint64_t(0) << n; }
// Places j0 .. j0 + 63 that a row at position pos, with that mask, sees; `base` places come before the drafted tokens, `top`
// is the last.  deep: a window may end among the drafted tokens.  (base, j0, top and deep are the same on every lane.)
__device__ __forceinline__ uint64_t seen_bits(const CacheAttnArgs& a, const RowTile& rt, const uint64_t* mask, int32_t pos, int32_t base,
                                              int32_t j0, int32_t top, bool deep, int lane) {
  const uint64_t drafted = bits_from((int64_t)base - j0);
  uint64_t m = (bits_from((int64_t)pos - a.window + 1 - j0) | ~bits_from((int64_t)a.sinks - j0)) & ~drafted;
  if (drafted) {
    uint64_t n = mask_bits(mask, a.words, j0 - base) & drafted;
    if (deep) {
      const int32_t first = max(0, base - j0), last = min(63, min(top, base + rt.count - 1) - j0);
      const int32_t mine = a.positions[rt.t0 + min(max(j0 + lane - base, 0), rt.count - 1)];  // of place j0 + lane
#pragma unroll 1
      for (int32_t x = first; x <= last; ++x) {
        const int32_t at = __builtin_amdgcn_readlane(mine, x);
        if (!((int64_t)pos - at < a.window || at < a.sinks)) n &= ~(uint64_t(1) << x);
      }
    }
    m |= n;
  }
  return pos < 0 ? 0 : m & ~bits_from((int64_t)top + 1 - j0);
}
// A row's position.  A window of 2^31 - 1 ends nothing, not even place 0 for a row at 2^31 - 1: it counts as at the position before.
__device__ __forceinline__ int32_t row_position(const CacheAttnArgs& a, int32_t row) { return min(a.positions[row], a.furthest); }
// Least and largest position of the rows that see anything (a position below 0 sees nothing): over the lanes that differ in
// the bits of LANES.
template <int LANES>
__device__ __forceinline__ void position_range(int32_t& lo, int32_t& hi) {
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) {
    lo = min(lo, __shfl_xor(lo, o));
    hi = max(hi, __shfl_xor(hi, o));
  }
}
// Whether a window may end among the drafted tokens of a sequence with a row at position phi.
__device__ __forceinline__ bool drafts_end(const CacheAttnArgs& a, const RowTile& rt, int32_t phi, int lane) {
  if (a.window == INT32_MAX) return false;
  int32_t lo = INT32_MAX, hi = 0;
  for (int32_t i = lane; i < rt.count; i += 64) {
    const int32_t p = a.positions[rt.t0 + i];
    lo = min(lo, p < 0 ? INT32_MAX : p);
  }
  position_range<64>(lo, hi);
  return phi - uniform(lo) >= a.window;
}
// Steps of a tile whose rows' positions are plo .. phi (none: phi < 0): the sinks', then from the first window, or from the
// drafted tokens where that is behind them, to the last token.
template <int STEP>
__device__ __forceinline__ Steps<STEP> tree_steps(int32_t plo, int32_t phi, int32_t base, int32_t len, int32_t cap, int32_t window,
                                                  int32_t sinks) {
  const int64_t most = (int64_t)max(base, 0) + window - 1;
  return cache_steps<STEP>((int32_t)min((int64_t)plo, most), phi < 0 ? -1 : len - 1, cap, window, sinks);
}

// The kernels for many rows of a tree (cache_tree.hip): tiles of 128 rows at head_dim 128, 64 at 64.
void launch_tree(const CacheAttnArgs& a, int64_t blocks, hipStream_t s);

}  // namespace hsap
