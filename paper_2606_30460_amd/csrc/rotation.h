// Rotation of rows by positions of one or several axes.
//
// A row of one head is D / 16 units, each two runs of eight values D / 2 apart or, where halves are rotated, rot / 2 apart
// (eight pairs), so that the lanes of a row read and write it in whole lines.  A thread holds a unit.  Every operation of
// (a cos - b sin, b cos + a sin) is rounded to fp32 by itself.
#pragma once

#include "cache_codes.h"

namespace hsap {

constexpr int kMaxAxes = 4;

// hsap_rotation as a kernel takes it.
struct Turns {
  const float* cos_sin;
  int64_t rows;
  const int32_t* positions;  // [axes, stride]; NULL: the token's place in its sequence
  int64_t stride;
  int32_t rot;
  int32_t interleaved;
  int32_t axes;
  uint32_t axis[4];  // two bits per pair
};

struct Unit {
  f32x8 a, b;  // the two runs
};

// Unit u of a row: the first values of its two runs of eight.  rot: values of the row that are rotated as halves (0: none).
template <int D>
__device__ __forceinline__ void unit_at(int rot, int u, int (&at)[2]) {
  const int base = 16 * u < rot ? 0 : rot, width = 16 * u < rot ? rot : D - rot;
  at[0] = base + 8 * (u - base / 16);
  at[1] = at[0] + width / 2;
}

__device__ __forceinline__ f32x8 load8(const float* p) {  // (16-byte aligned)
  const f32x4 x = *(const f32x4*)p, y = *(const f32x4*)(p + 4);
  return f32x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
}

// Cosines and sines of a unit's eight pairs: of halves pairs 8 u .. 8 u + 7 (both runs), interleaved pairs 4 u .. + 3 (the
// first run) and 4 u + D / 4 .. + 3 (the second).
struct UnitTurn {
  f32x8 c, s;
};

// Positions of a token on every axis; false where one has no row in the table.
struct Place {
  int32_t p0, p1, p2, p3;
};
__device__ __forceinline__ bool place_of(const Turns& r, int64_t t, Place& x) {
  static_assert(kMaxAxes == 4, "one member per axis");
  const int32_t* p = r.positions + t;
  x.p0 = p[0];
  x.p1 = r.axes > 1 ? p[r.stride] : x.p0;
  x.p2 = r.axes > 2 ? p[2 * r.stride] : x.p0;
  x.p3 = r.axes > 3 ? p[3 * r.stride] : x.p0;
  return min(min(x.p0, x.p1), min(x.p2, x.p3)) >= 0 && max(max(x.p0, x.p1), max(x.p2, x.p3)) < r.rows;
}

// (by value: a choice between members would be one between their addresses, in memory)
template <typename T>
__device__ __forceinline__ T pick(uint32_t i, T x0, T x1, T x2, T x3) {
  const T lo = i & 1 ? +x1 : +x0, hi = i & 1 ? +x3 : +x2;
  return i & 2 ? +hi : +lo;
}
__device__ __forceinline__ int32_t place_on(const Place& x, uint32_t axis) { return pick(axis, x.p0, x.p1, x.p2, x.p3); }

// cos and sin of the four pairs from `pair` on (a multiple of 4): one row where they share an axis
__device__ __forceinline__ void load_pairs(const Turns& r, const Place& x, int pair, f32x4& c, f32x4& s) {
  const uint32_t bits = (pick((uint32_t)pair >> 4, r.axis[0], r.axis[1], r.axis[2], r.axis[3]) >> (2 * (pair & 15))) & 255u;
  if (bits == (bits & 3u) * 0x55u) {
    const float* row = r.cos_sin + (int64_t)place_on(x, bits & 3u) * r.rot + pair;
    c = *(const f32x4*)row;
    s = *(const f32x4*)(row + r.rot / 2);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float* row = r.cos_sin + (int64_t)place_on(x, (bits >> (2 * e)) & 3u) * r.rot + pair + e;
      c[e] = row[0];
      s[e] = row[r.rot / 2];
    }
  }
}

template <int D>
__device__ __forceinline__ UnitTurn load_turn(const Turns& r, const Place& x, int u) {
  f32x4 c[2] = {f32x4{}, f32x4{}}, s[2] = {f32x4{}, f32x4{}};
#pragma unroll
  for (int y = 0; y < 2; ++y) {
    const int pair = r.interleaved ? 4 * u + y * (D / 4) : 8 * u + 4 * y;
    if (pair < r.rot / 2) load_pairs(r, x, pair, c[y], s[y]);
  }
  return UnitTurn{f32x8{c[0][0], c[0][1], c[0][2], c[0][3], c[1][0], c[1][1], c[1][2], c[1][3]},
                  f32x8{s[0][0], s[0][1], s[0][2], s[0][3], s[1][0], s[1][1], s[1][2], s[1][3]}};
}

// four interleaved pairs by the cosines and sines c and s
__device__ __forceinline__ f32x8 turn_pairs(const f32x8& v, const f32x4& c, const f32x4& s) {
#pragma clang fp contract(off)
  return f32x8{v[0] * c[0] - v[1] * s[0], v[1] * c[0] + v[0] * s[0], v[2] * c[1] - v[3] * s[1], v[3] * c[1] + v[2] * s[1],
               v[4] * c[2] - v[5] * s[2], v[5] * c[2] + v[4] * s[2], v[6] * c[3] - v[7] * s[3], v[7] * c[3] + v[6] * s[3]};
}

template <int D>
__device__ __forceinline__ Unit turn(int rot, int interleaved, int u, const UnitTurn& t, Unit r) {
#pragma clang fp contract(off)
  if (interleaved) {
    if (4 * u < rot / 2) r.a = turn_pairs(r.a, __builtin_shufflevector(t.c, t.c, 0, 1, 2, 3), __builtin_shufflevector(t.s, t.s, 0, 1, 2, 3));
    if (4 * u + D / 4 < rot / 2) r.b = turn_pairs(r.b, __builtin_shufflevector(t.c, t.c, 4, 5, 6, 7), __builtin_shufflevector(t.s, t.s, 4, 5, 6, 7));
  } else if (16 * u < rot) {
    const f32x8 x = r.a, y = r.b;
    r.a = x * t.c - y * t.s;
    r.b = y * t.c + x * t.s;
  }
  return r;
}

template <int D>
__device__ __forceinline__ Unit load_bf16(const __bf16* row, int rot, int u) {
  int at[2];
  unit_at<D>(rot, u, at);
  return Unit{__builtin_convertvector(*(const bf16x8*)(row + at[0]), f32x8),
              __builtin_convertvector(*(const bf16x8*)(row + at[1]), f32x8)};
}

template <int D>
__device__ __forceinline__ void store_bf16(__bf16* row, int rot, int u, const Unit& r) {
  int at[2];
  unit_at<D>(rot, u, at);
  *(bf16x8*)(row + at[0]) = __builtin_convertvector(r.a, bf16x8);
  *(bf16x8*)(row + at[1]) = __builtin_convertvector(r.b, bf16x8);
}

// A token's rows of `heads` heads by one unit's cosines and sines, `lanes` rows of a wave at a time from `sub` on, FLIGHT of them
// in flight: a lane forms them once for all heads.
template <int D, int FLIGHT, typename Load, typename Store>
__device__ __forceinline__ void turn_heads(const Turns& t, const UnitTurn& by, int heads, int sub, int lanes, int u, Load load, Store store) {
  for (int h0 = sub; h0 < heads; h0 += FLIGHT * lanes) {
    Unit r[FLIGHT];
#pragma unroll
    for (int y = 0; y < FLIGHT; ++y)
      if (h0 + y * lanes < heads) r[y] = load(h0 + y * lanes);
#pragma unroll
    for (int y = 0; y < FLIGHT; ++y)
      if (h0 + y * lanes < heads) store(h0 + y * lanes, turn<D>(t.rot, t.interleaved, u, by, r[y]));
  }
}
// Rows of a token that a wave takes at a time: a power of two up to the rows that its lanes hold.
inline int32_t rows_at_a_time(int32_t heads, int32_t head_dim) {
  int32_t n = 1;
  while (n < heads && n < 64 / (head_dim / 16)) n *= 2;
  return n;
}

// Checks a rotation and fills in all of `out` but the positions (ops of hsap_rotate and hsap_cache_append_at).
hsap_status check_rotation(const hsap_rotation* r, int32_t head_dim, Turns* out);

}  // namespace hsap
