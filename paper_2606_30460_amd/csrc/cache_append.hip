// New tokens into the paged 8-bit K/V cache, with the rotation of their positions on the way.
//
// Rotation of a pair (a, b) by the row (cos, sin) of the token's position: (a cos - b sin, b cos + a sin), in fp32,
// every operation rounded by itself.  K's codes are e4m3 of the rotated fp32 values, V's of the values, both divided
// by the scale of (page, head).  Scales are powers of two: 2^e with the smallest e for which the page's largest value
// is at most 448 2^e.  A page that fills token by token starts with its first token's scale; a later, larger token
// raises it and the page's older codes are encoded anew -- by a power of two, so exactly, but for what falls under
// e4m3's smallest normal number.
//
// A row of one head is D / 16 units, each two runs of eight values D / 2 apart or, where halves are rotated, rot / 2 apart
// (eight pairs), so that the lanes of a row read and write it in whole lines.  A thread holds a unit.
//
// Bound by memory: k, v (and q) are read once, codes (and q_out, k_out) written once, a page's values held in registers
// between its maximum and its codes.  16 prompts of 19269 tokens in all, 32 heads over 8 of 128: 102 us, 4.6 TB/s (a
// copy reaches 5.1).  64 sequences' new tokens: 3.8 us, one: 2.7, a launch and the chain position, page, scale, codes.
#include <algorithm>

#include "cache.h"
#include "hsap_internal.h"
#include "mfma.h"

namespace hsap {

struct AppendArgs {
  hsap_cache_desc d;
  hsap_cache c;
  const __bf16* k;
  const __bf16* v;
  const __bf16* q;
  int64_t k_stride, v_stride, q_stride;
  const int32_t* cu;  // new tokens per sequence, cumulative; NULL: one each
  int64_t total_new;
  const float* cos_sin;
  int64_t rows;  // positions that cos_sin has
  int32_t rot;
  int32_t interleaved;
  __bf16* k_out;
  __bf16* q_out;
  int32_t heads_q;
  int32_t kv_blocks;  // workgroups of the cache's part; the others rotate Q
};

typedef float f32x8 __attribute__((ext_vector_type(8)));
struct Unit {
  f32x8 a, b;  // the two runs
};

// Unit u of a row: the first values of its two runs of eight.
template <int D>
__device__ __forceinline__ void unit_at(const AppendArgs& a, int u, bool turn, int (&at)[2]) {
  const int rot = turn && !a.interleaved ? a.rot : 0;
  const int base = 16 * u < rot ? 0 : rot, width = 16 * u < rot ? rot : D - rot;
  at[0] = base + 8 * (u - base / 16);
  at[1] = at[0] + width / 2;
}

template <int D>
__device__ __forceinline__ Unit load_unit(const AppendArgs& a, const __bf16* row, int u, bool turn) {
  int at[2];
  unit_at<D>(a, u, turn, at);
  return Unit{__builtin_convertvector(*(const bf16x8*)(row + at[0]), f32x8),
              __builtin_convertvector(*(const bf16x8*)(row + at[1]), f32x8)};
}

__device__ __forceinline__ f32x8 load8(const float* p) {  // (16-byte aligned)
  const f32x4 x = *(const f32x4*)p, y = *(const f32x4*)(p + 4);
  return f32x8{x[0], x[1], x[2], x[3], y[0], y[1], y[2], y[3]};
}

// four interleaved pairs by the cosines and sines at c and s
__device__ __forceinline__ f32x8 turn_pairs(const f32x8& v, const float* cos, const float* sin) {
#pragma clang fp contract(off)
  const f32x4 c = *(const f32x4*)cos, s = *(const f32x4*)sin;
  return f32x8{v[0] * c[0] - v[1] * s[0], v[1] * c[0] + v[0] * s[0], v[2] * c[1] - v[3] * s[1], v[3] * c[1] + v[2] * s[1],
               v[4] * c[2] - v[5] * s[2], v[5] * c[2] + v[4] * s[2], v[6] * c[3] - v[7] * s[3], v[7] * c[3] + v[6] * s[3]};
}

template <int D>
__device__ __forceinline__ Unit turn_unit(const AppendArgs& a, int u, int64_t pos, Unit r) {
#pragma clang fp contract(off)
  const float* cs = a.cos_sin + pos * a.rot;
  if (a.interleaved) {
    const int first = 4 * u, second = first + D / 4;  // first pairs of the runs
    if (first < a.rot / 2) r.a = turn_pairs(r.a, cs + first, cs + a.rot / 2 + first);
    if (second < a.rot / 2) r.b = turn_pairs(r.b, cs + second, cs + a.rot / 2 + second);
  } else if (16 * u < a.rot) {
    const f32x8 c = load8(cs + 8 * u), s = load8(cs + a.rot / 2 + 8 * u);
    const f32x8 x = r.a, y = r.b;
    r.a = x * c - y * s;
    r.b = y * c + x * s;
  }
  return r;
}

template <int D>
__device__ __forceinline__ void store_bf16(const AppendArgs& a, __bf16* row, int u, bool turn, const Unit& r) {
  int at[2];
  unit_at<D>(a, u, turn, at);
  *(bf16x8*)(row + at[0]) = __builtin_convertvector(r.a, bf16x8);
  *(bf16x8*)(row + at[1]) = __builtin_convertvector(r.b, bf16x8);
}

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

template <int D>
__device__ __forceinline__ void store_codes(const AppendArgs& a, uint8_t* row, int u, bool turn, const Unit& r, float inv) {
  int at[2];
  unit_at<D>(a, u, turn, at);
  *(uint2*)(row + at[0]) = encode8(r.a * inv);
  *(uint2*)(row + at[1]) = encode8(r.b * inv);
}

// largest finite magnitude of a unit
__device__ __forceinline__ float unit_max(const Unit& r) {
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float x = fabsf(r.a[e]), y = fabsf(r.b[e]);
    m = fmaxf(m, fmaxf(x < __builtin_inff() ? x : 0.f, y < __builtin_inff() ? y : 0.f));
  }
  return m;
}

__device__ __forceinline__ uint32_t recode4(uint32_t x, float ratio) {
  const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true);
  return encode4(lo[0] * ratio, lo[1] * ratio, hi[0] * ratio, hi[1] * ratio);
}

// 16 codes at p, encoded anew for a scale 1 / ratio times as large
__device__ __forceinline__ void recode16(uint8_t* p, float ratio) {
  const uint4 w = *(const uint4*)p;
  *(uint4*)p = make_uint4(recode4(w.x, ratio), recode4(w.y, ratio), recode4(w.z, ratio), recode4(w.w, ratio));
}

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

// One rotated Q row unit per thread.
template <int D>
__device__ __forceinline__ void rotate_q(const AppendArgs& a, int64_t item) {
  constexpr int UNITS = D / 16;
  const int u = (int)(item % UNITS);
  const int64_t row = item / UNITS;
  const int64_t t = row / a.heads_q;
  const int h = (int)(row - t * a.heads_q);
  if (t >= a.total_new || (a.cu && t >= a.cu[a.d.num_seqs])) return;  // (behind the last sequence: not read)
  Unit x = load_unit<D>(a, a.q + t * a.q_stride + (int64_t)h * D, u, true);  // (under way while the position is looked up)
  int64_t pos;
  if (a.cu) {
    int32_t l = 0, r = a.d.num_seqs;  // cu[l] <= t < cu[r]
    while (r - l > 1) {
      const int32_t mid = (l + r) >> 1;
      if (a.cu[mid] <= t) l = mid;
      else r = mid;
    }
    pos = (int64_t)a.c.seq_lens[l] - (a.cu[l + 1] - t);
  } else {
    pos = (int64_t)a.c.seq_lens[t] - 1;
  }
  if (pos < 0 || (a.rot && pos >= a.rows)) return;
  if (a.rot) x = turn_unit<D>(a, u, pos, x);
  store_bf16<D>(a, a.q_out + (t * a.heads_q + h) * D, u, true, x);
}

// One new token per sequence: D / 16 lanes per (sequence, head, K or V).
template <int D>
__global__ __launch_bounds__(256) void cache_append_one_kernel(AppendArgs a) {
  constexpr int UNITS = D / 16;
  if ((int)blockIdx.x >= a.kv_blocks) {
    rotate_q<D>(a, (int64_t)(blockIdx.x - a.kv_blocks) * 256 + threadIdx.x);
    return;
  }
  const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int u = (int)(item % UNITS);
  const int64_t row = item / UNITS;
  const bool is_v = row & 1;
  const int64_t s = (row >> 1) / a.d.heads_kv;
  const int h = (int)((row >> 1) - s * a.d.heads_kv);
  if (s >= a.d.num_seqs) return;
  const __bf16* src = is_v ? a.v + s * a.v_stride : a.k + s * a.k_stride;
  Unit x = load_unit<D>(a, src + (int64_t)h * D, u, !is_v);
  const int32_t pos = a.c.seq_lens[s] - 1;
  if (pos < 0 || (a.rot && pos >= a.rows)) return;
  if (!is_v && a.rot) x = turn_unit<D>(a, u, pos, x);
  if (!is_v && a.k_out) store_bf16<D>(a, a.k_out + (s * a.d.heads_kv + h) * D, u, true, x);
  const int32_t page = cache_page(a.c.page_table + s * a.d.table_width, a.d.table_width, a.d.num_pages, a.d.page_size, pos);
  if (page < 0) return;
  const int32_t slot = pos & (a.d.page_size - 1);
  float* scale = (is_v ? a.c.v_scale : a.c.k_scale) + (int64_t)page * a.d.heads_kv + h;
  uint8_t* codes = (is_v ? a.c.v_codes : a.c.k_codes) + cache_row(page, a.d.heads_kv, h, a.d.page_size, 0, D);
  const float old = slot > 0 ? *scale : 0.f;
  float amax = unit_max(x);
#pragma unroll
  for (int o = 1; o < UNITS; o <<= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
  float inv, ratio;
  const float now = page_scale(amax, slot > 0, old, inv, ratio);
  // (token after token: 64 new tokens that raise the scales of pages of 16, 64, 128 take 15, 33, 58 us, of none 10, event to
  // event)
  if (ratio != 1.f)
    for (int32_t t = 0; t < slot; ++t) recode16(codes + t * D + 16 * u, ratio);
  store_codes<D>(a, codes + slot * D, u, !is_v, x, inv);
  if (u == 0) *scale = now;
}

// Any number of new tokens: one workgroup per (page that a sequence's new tokens reach, head, K or V); the page's new
// values are held in registers between the reduction of their maximum and their encoding.
// PER: units of a page per thread.
template <int D, int PER>
__global__ __launch_bounds__(256) void cache_append_kernel(AppendArgs a) {
  constexpr int UNITS = D / 16;
  if ((int)blockIdx.x >= a.kv_blocks) {
    rotate_q<D>(a, (int64_t)(blockIdx.x - a.kv_blocks) * 256 + threadIdx.x);
    return;
  }
  __shared__ float wave_max[4], old_scale;
  const int tid = threadIdx.x;
  const bool is_v = blockIdx.x & 1;
  const int32_t pair = (int32_t)(blockIdx.x >> 1);
  const int h = pair % a.d.heads_kv;
  const int64_t item = pair / a.d.heads_kv;
  const int32_t ps = a.d.page_size;
  // the sequence whose pages this item is one of
  int32_t s = 0, r = a.d.num_seqs;
  while (r - s > 1) {
    const int32_t mid = (s + r) >> 1;
    if (item_base(a.cu[mid], 1, ps, 2, mid) <= item) s = mid;
    else r = mid;
  }
  const int32_t t0 = a.cu[s], count = a.cu[s + 1] - t0, len = a.c.seq_lens[s];
  if (count <= 0 || len <= 0) return;
  const int64_t pos0 = (int64_t)len - count;  // position of the first new token
  const int64_t first = pos0 > 0 ? pos0 : 0;
  const int64_t at = first / ps + (item - item_base(t0, 1, ps, 2, s));
  const int64_t lo = max(first, at * ps);
  int64_t end = min((int64_t)len, (at + 1) * ps);
  if (a.rot) end = min(end, a.rows);
  end = min(end, pos0 + a.total_new - t0);
  if (lo >= end) return;
  const int32_t page = cache_page(a.c.page_table + (int64_t)s * a.d.table_width, a.d.table_width, a.d.num_pages, ps, (int32_t)lo);
  const int32_t slot0 = (int32_t)(lo - at * ps), units = (int32_t)(end - lo) * UNITS;
  const __bf16* src = (is_v ? a.v : a.k) + (int64_t)h * D;
  const int64_t stride = is_v ? a.v_stride : a.k_stride;
  Unit x[PER] = {};
  float amax = 0.f;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int unit = tid + 256 * i;
    if (unit < units) {
      const int64_t pos = lo + unit / UNITS, t = t0 + (pos - pos0);
      x[i] = load_unit<D>(a, src + t * stride, unit % UNITS, !is_v);
      if (!is_v && a.rot) x[i] = turn_unit<D>(a, unit % UNITS, pos, x[i]);
      amax = fmaxf(amax, unit_max(x[i]));
      if (!is_v && a.k_out) store_bf16<D>(a, a.k_out + (t * a.d.heads_kv + h) * D, unit % UNITS, true, x[i]);
    }
  }
  if (page < 0) return;
  float* scale = (is_v ? a.c.v_scale : a.c.k_scale) + (int64_t)page * a.d.heads_kv + h;
  uint8_t* codes = (is_v ? a.c.v_codes : a.c.k_codes) + cache_row(page, a.d.heads_kv, h, ps, 0, D);
  if (tid == 0) old_scale = slot0 > 0 ? *scale : 0.f;  // (read by the thread that writes it)
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
  if ((tid & 63) == 0) wave_max[tid >> 6] = amax;
  __syncthreads();
  amax = fmaxf(fmaxf(wave_max[0], wave_max[1]), fmaxf(wave_max[2], wave_max[3]));
  float inv, ratio;
  const float now = page_scale(amax, slot0 > 0, old_scale, inv, ratio);
  if (ratio != 1.f)
    for (int e = tid; e < slot0 * UNITS; e += 256) recode16(codes + 16 * e, ratio);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int unit = tid + 256 * i;
    if (unit < units) store_codes<D>(a, codes + (slot0 + unit / UNITS) * D, unit % UNITS, !is_v, x[i], inv);
  }
  if (tid == 0) *scale = now;
}

hsap_status check_cache_desc(const hsap_cache_desc* d, bool pages) {
  if (!d) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "cache descriptor is NULL");
  if ((pages && d->num_pages < 1) || d->heads_kv < 1 || d->num_seqs < 0 || d->table_width < 1)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "bad cache: num_pages %d, heads_kv %d, num_seqs %d, table_width %d", d->num_pages,
              d->heads_kv, d->num_seqs, d->table_width);
  if (d->page_size != 16 && d->page_size != 32 && d->page_size != 64 && d->page_size != 128)
    HSAP_FAIL(HSAP_ERR_UNSUPPORTED, "page_size %d not supported (16, 32, 64 or 128)", d->page_size);
  if (d->head_dim != 64 && d->head_dim != 128)
    HSAP_FAIL(HSAP_ERR_UNSUPPORTED, "head_dim %d not supported (64 or 128)", d->head_dim);
  if ((int64_t)d->table_width * d->page_size > INT32_MAX)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "table_width %d x page_size %d beyond 2^31-1 positions", d->table_width, d->page_size);
  return HSAP_OK;
}

hsap_status check_cache(const hsap_cache_desc* d, const hsap_cache* c) {
  const hsap_status st = check_cache_desc(d, true);
  if (st != HSAP_OK) return st;
  if (!c) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "cache descriptor is NULL");
  if (!c->k_codes || !c->v_codes || !c->k_scale || !c->v_scale)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "NULL pointer in the cache");
  if (d->num_seqs > 0 && (!c->page_table || !c->seq_lens)) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "NULL page_table or seq_lens");
  if (((uintptr_t)c->k_codes | (uintptr_t)c->v_codes) & 15) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "codes must be 16-byte aligned");
  return HSAP_OK;
}

static hsap_status check_rows(const char* what, const void* p, int64_t stride, int64_t row) {
  if (!p) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "NULL %s", what);
  if (((uintptr_t)p & 15) || stride % 8 || stride < row)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "%s must be 16-byte aligned, its row stride (%lld) a multiple of 8 and at least %lld", what,
              (long long)stride, (long long)row);
  return HSAP_OK;
}

}  // namespace hsap

using namespace hsap;

extern "C" hsap_status hsap_cache_append(const hsap_cache_desc* desc, const hsap_cache* cache, const void* k, int64_t k_stride,
                                         const void* v, int64_t v_stride, const int32_t* cu_new, int64_t total_new,
                                         const float* cos_sin, int64_t cos_sin_rows, int32_t rot_dim, int32_t interleaved,
                                         void* k_out, const void* q, int64_t q_stride, int32_t heads_q, void* q_out,
                                         void* hip_stream) {
  clear_error();
  hsap_status st = check_cache(desc, cache);
  if (st != HSAP_OK) return st;
  const int d = desc->head_dim;
  if (total_new < 0 || total_new > INT32_MAX) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "bad total_new %lld", (long long)total_new);
  if (!cu_new && total_new != desc->num_seqs)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "without cu_new every sequence has one new token: total_new %lld, num_seqs %d",
              (long long)total_new, desc->num_seqs);
  if (rot_dim < 0 || rot_dim > d || rot_dim % 16)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "rot_dim %d must be a multiple of 16 up to head_dim %d", rot_dim, d);
  if (rot_dim && (!cos_sin || cos_sin_rows < 1 || ((uintptr_t)cos_sin & 15)))
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "rot_dim without a 16-byte aligned cos_sin table");
  if ((q != nullptr) != (q_out != nullptr)) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "q and q_out come together");
  if (total_new == 0 || desc->num_seqs == 0) return HSAP_OK;
  if ((st = check_rows("k", k, k_stride, (int64_t)desc->heads_kv * d)) != HSAP_OK) return st;
  if ((st = check_rows("v", v, v_stride, (int64_t)desc->heads_kv * d)) != HSAP_OK) return st;
  if (q) {
    if (heads_q < 1) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "heads_q %d < 1", heads_q);
    if ((st = check_rows("q", q, q_stride, (int64_t)heads_q * d)) != HSAP_OK) return st;
  }
  if (((uintptr_t)k_out | (uintptr_t)q_out) & 15) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "k_out and q_out must be 16-byte aligned");
  AppendArgs a{};
  a.d = *desc;
  a.c = *cache;
  a.k = (const __bf16*)k;
  a.v = (const __bf16*)v;
  a.q = (const __bf16*)q;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_stride = q_stride;
  a.cu = cu_new;
  a.total_new = total_new;
  a.cos_sin = cos_sin;
  a.rows = cos_sin_rows;
  a.rot = rot_dim;
  a.interleaved = interleaved != 0;
  a.k_out = (__bf16*)k_out;
  a.q_out = (__bf16*)q_out;
  a.heads_q = heads_q;
  const int64_t units = d / 16;
  const int64_t kv = cu_new ? (item_base(total_new, 1, desc->page_size, 2, desc->num_seqs)) * desc->heads_kv * 2
                            : ((int64_t)desc->num_seqs * desc->heads_kv * 2 * units + 255) / 256;
  const int64_t blocks = kv + (q ? (total_new * heads_q * units + 255) / 256 : 0);
  if (blocks > kMaxBlocks256) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "too many tokens x heads");
  a.kv_blocks = (int32_t)kv;
  hipStream_t s = (hipStream_t)hip_stream;
  const dim3 grid((unsigned)blocks), block(256);
  if (cu_new) {
    const int per = desc->page_size * (d / 16) / 256;
    if (d == 128) {
      if (per <= 1) hipLaunchKernelGGL((cache_append_kernel<128, 1>), grid, block, 0, s, a);
      else if (per == 2) hipLaunchKernelGGL((cache_append_kernel<128, 2>), grid, block, 0, s, a);
      else hipLaunchKernelGGL((cache_append_kernel<128, 4>), grid, block, 0, s, a);
    } else {
      if (per <= 1) hipLaunchKernelGGL((cache_append_kernel<64, 1>), grid, block, 0, s, a);
      else hipLaunchKernelGGL((cache_append_kernel<64, 2>), grid, block, 0, s, a);
    }
  } else {
    if (d == 128) hipLaunchKernelGGL(cache_append_one_kernel<128>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(cache_append_one_kernel<64>, grid, block, 0, s, a);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) HSAP_FAIL(HSAP_ERR_HIP, "cache_append launch: %s", hipGetErrorString(e));
  return HSAP_OK;
}
