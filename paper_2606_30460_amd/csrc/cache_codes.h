// e4m3 codes and scales of a cache page: what appends and moves of tokens share.
#pragma once

#include "cache.h"
#include "mfma.h"

namespace hsap {

typedef float f32x8 __attribute__((ext_vector_type(8)));

// e4m3 of x (nearest even, saturating at 448; NaN stays NaN)
__device__ __forceinline__ float clamp448(float x) {
  const float c = fminf(fmaxf(x, -448.f), 448.f);
  return x == x ? c : x;
}
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(clamp448(a), clamp448(b), 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(clamp448(c), clamp448(d), w, true);
  return (uint32_t)w;
}

__device__ __forceinline__ uint2 encode8(const f32x8& x) {
  return make_uint2(encode4(x[0], x[1], x[2], x[3]), encode4(x[4], x[5], x[6], x[7]));
}

__device__ __forceinline__ uint32_t recode4(uint32_t x, float ratio) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true);
  return encode4(lo[0] * ratio, lo[1] * ratio, hi[0] * ratio, hi[1] * ratio);
}

// 16 codes encoded anew for a scale 1 / ratio times as large
__device__ __forceinline__ uint4 recoded16(const uint4& w, float ratio) {
  return make_uint4(recode4(w.x, ratio), recode4(w.y, ratio), recode4(w.z, ratio), recode4(w.w, ratio));
}
__device__ __forceinline__ void recode16(uint8_t* p, float ratio) { *(uint4*)p = recoded16(*(const uint4*)p, ratio); }

// The page's new scale; `kept` tokens before the new ones stay.  Sets inv to its reciprocal and ratio to what their codes
// are multiplied by (1: they stay as they are).
__device__ __forceinline__ float page_scale(float amax, bool kept, float old, float& inv, float& ratio) {
  const int e = scale_exponent(__float_as_uint(amax));
  float s = __uint_as_float((uint32_t)(e + 127) << 23);
  inv = __uint_as_float((uint32_t)(127 - e) << 23);
  ratio = 1.f;
  if (kept) {
    if (old > s) {
      s = old;
      inv = 1.f / old;
    } else if (old < s) {
      ratio = old * inv;
    }
  }
  return s;
}

}  // namespace hsap
