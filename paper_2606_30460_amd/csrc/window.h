// Device helpers of the window-attention kernels: document bounds of a wave's positions, the row of a position in
// sharded order, and the direct-to-LDS transfer of a 64-row tile.  What comes before them, the choices of a call's kernels and
// index arithmetic, also builds without HIP.
#pragma once

#include <algorithm>

#include "hsap_internal.h"

#if defined(__HIPCC__)
#include "mfma.h"
#endif

namespace hsap {

// Key row that the dQ kernel reads for position x when it forms delta of a wave's short rows, whose windows begin at lo or
// behind it and whose sinks before position g0, the wave's first row, are far .. far_end - 1.  A place that none of them
// sees is g0's own instead: the rows that no query of the shard sees are not read.  (Positions from g0 to `last` are the
// shard's own rows.)
HSAP_HD inline int32_t short_row_key(int32_t x, int32_t g0, int32_t lo, int32_t far, int32_t far_end, int32_t last) {
  if (x < lo && (x < far || x >= far_end)) return g0;
  return x < last ? x : last;
}

// 32-row blocks of a workgroup's four waves: four, or fewer, each then taken by several waves that share its steps as
// streams, so that a small grid has more and shorter workgroups.  `tiles`: workgroups that four blocks would give.  A split
// pays as long as all its workgroups are resident at once: one per CU at head_dim 128, two at 64 (their LDS).
// Measured on one document, us, four blocks -> two -> one:
//   forward, d 64, window 300:   64 tiles 14.0 -> 9.2, 256 tiles 14.8 -> 11.7, 282 tiles 17.6 -> 18.9
//   forward, d 128, window 300:  128 tiles 17.9 -> 13.6, 256 tiles 19.2 -> 24.8
//   whole backward by dK/dV's choice, d 64:   64 tiles 72 -> 49 -> 39, 128 tiles 72 -> 50 -> 45, 256 tiles 94 -> 77 -> 85,
//     512 tiles 130 -> 132 -> 151
//   d 128:  64 tiles 112 -> 73 -> 62, 128 tiles 119 -> 80 -> 96, 256 tiles 157 -> 164 -> 195
inline int window_row_blocks(int64_t tiles, int head_dim) {
  const int64_t resident = kComputeUnits * (head_dim == 64 ? 2 : 1);
  return 4 * tiles <= resident ? 1 : 2 * tiles <= resident ? 2 : 4;
}
// Blocks of the kernels by query tiles (forward, dQ): two or four (one block in four streams gains nothing over two in two).
inline int window_query_blocks(const Geom& g, int heads_q, int head_dim) {
  return window_row_blocks(g.n / g.m * ((g.m + 127) / 128) * heads_q, head_dim) < 4 ? 2 : 4;
}
// Key tiles of dK/dV: of the chunks' keys, those that the shard's windows reach.
inline int64_t window_key_tiles(const Geom& g, int heads_kv, int64_t window) {
  const int64_t keys = g.n / g.m * (g.m + window);
  return (keys < g.N ? keys : g.N) / 128 * heads_kv;
}

// Queries of a sink chunk: a workgroup per CU over all chunks and K/V heads, at least 256 (8192 rows x 8 heads: chunks of 256
// 33 us, of 1024 177 us; 16384 rows x 16 heads: 256 58 us, 1024 26 us).
inline int32_t sink_chunk(const hsap_attn_desc* d, const Geom& g) {
  int32_t c = 256;
  while (c < 4096 && g.n * d->heads_kv > c * kComputeUnits) c *= 2;
  return c;
}

// Sink chunks per segment; 0 where no chunk begins inside a document that has a sink further than a window from its queries.
inline int32_t sink_chunks(const hsap_attn_desc* d, const Geom& g, int32_t window, int32_t sinks) {
  if (sinks == 0 || window >= g.Ns) return 0;
  const int32_t c = sink_chunk(d, g), per = (int32_t)((g.m + c - 1) / c);
  return per == 1 && g.P == 1 && g.layout == HSAP_LAYOUT_CONTIGUOUS ? 0 : per;
}

// Up to so many chunks per segment the dK/dV kernel adds a document's partials itself.
constexpr int32_t kDirectChunks = 8;

// Workgroups that share a key tile's heads: while all stay resident at once and each keeps at least eight steps, its parts
// within 64 MiB.
inline int32_t head_split(const hsap_attn_desc* d, const Geom& g, int32_t window) {
  const int grp = d->heads_q / d->heads_kv;
  const int64_t tiles = window_key_tiles(g, d->heads_kv, window);
  const int blocks = window_row_blocks(tiles, d->head_dim);
  if (blocks == 4 || grp == 1) return 1;
  const int64_t resident = kComputeUnits * (d->head_dim == 64 ? 2 : 1);
  const int64_t per_head = (std::min<int64_t>(window, g.m) + 32 * blocks) / 32;  // 32-query steps of one head
  const int64_t steps = per_head * grp * blocks / 4;                             // a stream's
  const int64_t bytes = (int64_t)g.P * g.n * d->heads_kv * 2 * d->head_dim * 4;
  const int64_t most = std::min<int64_t>(std::min<int64_t>(grp, steps / 8),
                                         std::min(resident / std::max<int64_t>(1, tiles * 4 / blocks), (int64_t(64) << 20) / bytes));
  return (int32_t)std::max<int64_t>(1, most);
}

#if defined(__HIPCC__)
// Shard segments: local rows in pieces of consecutive positions, one (CONTIGUOUS) or two (ZIGZAG) per sequence of the
// batch, each of geom.m rows.  Segment sg holds local rows sg * m .. sg * m + m - 1.
__host__ __device__ inline int32_t segments_per_sequence(const Geom& g) { return g.layout == HSAP_LAYOUT_CONTIGUOUS ? 1 : 2; }

// Most sink tokens per document that the backward takes: one workgroup holds them all (4 waves x 32 keys).
constexpr int32_t kMaxBwdSinks = 128;

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// First position of segment sg of chunk x.
__device__ __forceinline__ int32_t segment_start(const Geom& g, int32_t x, int32_t sg) {
  return (int32_t)global_pos(g, x, (int64_t)sg * g.m);
}

// Storage of keys in sharded order as runs of consecutive positions: [lo, hi) are the positions whose row is
// position + delta.  One chunk of a contiguous layout of one shard holds everything.
struct KeySpan {
  int32_t lo, hi;
  int32_t delta;
};

__device__ __forceinline__ KeySpan key_span(const Geom& g, int32_t pos) {
  if (g.P == 1 && g.layout == HSAP_LAYOUT_CONTIGUOUS) return KeySpan{0, (int32_t)g.N, 0};
  const uint32_t Ns = (uint32_t)g.Ns, m = (uint32_t)g.m;
  const uint32_t b = (uint32_t)pos / Ns, at = (uint32_t)pos - b * Ns;
  const uint32_t piece = at / m;
  const uint32_t P = (uint32_t)g.P;
  uint32_t row = b * (uint32_t)g.ns;  // first row of the piece within its chunk
  uint32_t chunk = piece;
  if (g.layout != HSAP_LAYOUT_CONTIGUOUS && piece >= P) {
    chunk = 2 * P - 1 - piece;
    row += m;
  }
  const int32_t lo = (int32_t)(b * Ns + piece * m);
  return KeySpan{lo, lo + (int32_t)m, (int32_t)(chunk * (uint32_t)g.n + row) - lo};
}

// Document [start, end) of this lane's position gq, for a wave whose lanes 0..31 hold positions that rise by at most one
// from lane to lane (lane l ^ 32 holds the position of lane l).  A position at or behind the last boundary cu[nd]
// has none: start = end = INT32_MAX.  One 64-entry window of boundaries serves the wave unless documents without
// tokens fill it; then each lane searches.
struct DocSpan {
  int32_t start, end;
};

__device__ __forceinline__ DocSpan doc_span(const int32_t* cu, int32_t nd, int32_t gq, int lane) {
  const DocWindow r = doc_window(nullptr, cu, nd, gq, lane);
  const int32_t lo = __popcll(__builtin_amdgcn_ballot_w64(r.w <= r.g_lo)) - 1;
  const int32_t last = __popcll(__builtin_amdgcn_ballot_w64(r.w <= r.g_hi)) - 1;
  if (last >= 63) {
    int32_t l = 0, h = nd + 1;  // cu[l] <= gq, cu[h] > gq (cu[nd + 1] standing for infinity)
    while (h - l > 1) {
      const int32_t mid = (l + h) >> 1;
      if (cu[mid] <= gq) l = mid;
      else h = mid;
    }
    if (l == nd) return DocSpan{INT32_MAX, INT32_MAX};
    return DocSpan{cu[l], cu[l + 1]};
  }
  DocSpan d{__builtin_amdgcn_readlane(r.w, lo), INT32_MAX};
  for (int32_t j = lo + 1; j <= last + 1; ++j) {
    const int32_t b = __builtin_amdgcn_readlane(r.w, j);
    if (gq >= b) d.start = b;
    else d.end = min(d.end, b);
  }
  return d;
}

// Transfers of a [R][D] bf16 tile (R = 64 by default) from global memory to a swizzled LDS tile (mfma.h), WAVES waves, 64
// 16-byte chunks per instruction.  Issued from asm and ordered by the kernels' own vmcnt waits (vm_wait_barrier): the compiler would
// wait for every transfer before any later LDS read.
template <int D, int WAVES, int R = 64>
struct TileStage {
  static constexpr int CPR = D / 8, WCH = R * CPR / WAVES, U = WCH / 64;
  static_assert(WCH % 64 == 0, "a wave moves whole instructions");
  uint32_t off[U];  // byte offset of this lane's chunk of instruction u from the tile's first row
  uint32_t lds0;    // the wave's first chunk within a tile, in bytes
  int first;        // this lane's chunk of instruction 0

  __device__ __forceinline__ void init(int wave, int lane, int64_t row_bytes) {
    first = WCH * wave + lane;
    lds0 = (uint32_t)(WCH * 16 * wave);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int p = first + 64 * u, row = p / CPR;
      off[u] = (uint32_t)(row * row_bytes + swz_chunk<CPR>(row, p % CPR) * 16);
    }
  }
  // R readable rows at src, row_bytes apart; src and dst uniform over the wave
  __device__ __forceinline__ void rows(const void* src, const __bf16* dst) const {
    typedef __attribute__((address_space(3))) void* lds_void;
    const uint32_t lds = (uint32_t)(uintptr_t)(lds_void)dst + lds0;
#pragma unroll
    for (int u = 0; u < U; ++u)
      asm volatile("global_load_lds_dwordx4 %0, %1" ::"v"(off[u]), "s"(src), "{m0}"(lds + 1024 * u));
  }
  // row r at address row(r), any order (rows may repeat)
  template <typename F>
  __device__ __forceinline__ void gather(F row, const __bf16* dst) const {
    typedef __attribute__((address_space(3))) void* lds_void;
    const uint32_t lds = (uint32_t)(uintptr_t)(lds_void)dst + lds0;
#pragma unroll 1  // (the rare path: one address at a time, the kernels have no registers to spare)
    for (int u = 0; u < U; ++u) {
      const int p = first + 64 * u, r = p / CPR;
      const char* src = (const char*)row(r) + swz_chunk<CPR>(r, p % CPR) * 16;
      asm volatile("global_load_lds_dwordx4 %0, off" ::"v"(src), "{m0}"(lds + 1024 * u));
    }
  }
};

// Operand addresses in a swizzled [rows][D] tile (mfma.h).  Row reads (row l32 of a 32-row block, chunk 2 kk + hi) and
// transpose reads (rows 8 k + tr_row of a 16-row block, columns 32 mb + tr_col) of one lane differ by an exclusive or
// in the chunk's bits alone, so a base each gives them all.  fresh() keeps the compiler from holding the sixteen
// addresses in registers through a loop that has none to spare.
template <int D>
struct TileReads {
  int row, tr0, tr1;  // elements

  __device__ __forceinline__ void init(int lane) {
    constexpr int CPR = D / 8;
    const int l32 = lane & 31, hi = lane >> 5;
    const int tr_row = 4 * hi + ((lane & 15) >> 2), tr_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
    row = swz<CPR>(l32, 8 * hi);
    tr0 = swz<CPR>(tr_row, tr_col);
    tr1 = swz<CPR>(8 + tr_row, tr_col);
  }
  __device__ __forceinline__ void fresh() { asm volatile("" : "+v"(row), "+v"(tr0), "+v"(tr1)); }
  // row l32 of the block at `tile`, sixteen columns kk
  __device__ __forceinline__ bf16x8 rows(const __bf16* tile, int kk) const { return *(const bf16x8*)(tile + (row ^ (16 * kk))); }
  // columns 32 mb .. +31 of the sixteen rows at `tile`, transposed
  __device__ __forceinline__ bf16x8 turned(const __bf16* tile, int mb) const {
    return cat4(ds_read_tr16(tile + (tr0 ^ (32 * mb))), ds_read_tr16(tile + (tr1 ^ (32 * mb))));
  }
};

// Uniform copy of a value that is the same on every lane.
__device__ __forceinline__ int32_t uniform(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }

// Stages keys j0 .. j0 + 63 (clamped to jmax) of one K/V head: `base` is the head's row 0, rows `row_bytes` apart.
// `span` is the run of positions that held the last tile's first key.
template <int D, int WAVES>
__device__ __forceinline__ void stage_keys(const TileStage<D, WAVES>& st, const Geom& g, KeySpan& span, int32_t j0,
                                           int32_t jmax, const __bf16* base, int64_t row_elems, const __bf16* dst) {
  if (j0 < span.lo || j0 >= span.hi) {
    const KeySpan s = key_span(g, j0);
    span = KeySpan{uniform(s.lo), uniform(s.hi), uniform(s.delta)};
  }
  if (__builtin_expect(j0 + 63 <= jmax && j0 + 63 < span.hi, 1)) {
    st.rows(base + (int64_t)(j0 + span.delta) * row_elems, dst);
  } else {
    // A step has keys of one run or, mostly, two: the second one's place is found once, not per row (3168 tokens in 16
    // pieces, two of them a shard, 5 heads of 128, window 1588: forward 41 -> 36 us).
    int32_t hi2 = span.hi, delta2 = 0;
    if (__builtin_expect(hi2 <= min(j0 + 63, jmax), 0)) {
      const KeySpan next = key_span(g, hi2);
      hi2 = uniform(next.hi);
      delta2 = uniform(next.delta);
    }
    st.gather(
        [&](int r) {
          const int32_t pos = min(j0 + r, jmax);
          int32_t delta = pos < span.hi ? span.delta : delta2;
          if (__builtin_expect(pos >= hi2, 0)) delta = key_span(g, pos).delta;
          return base + (int64_t)(pos + delta) * row_elems;
        },
        dst);
  }
}

#endif

}  // namespace hsap
