// New tokens into the paged 8-bit K/V cache, with the rotation of their positions on the way.
//
// Rotation of a pair (a, b) by the row (cos, sin) of the token's position: (a cos - b sin, b cos + a sin), in fp32,
// every operation rounded by itself.  K's codes are e4m3 of the rotated fp32 values, V's of the values, both divided
// by the scale of (page, head).  Scales are powers of two: 2^e with the smallest e for which the page's largest value
// is at most 448 2^e.  A page that fills token by token starts with its first token's scale; a later, larger token
// raises it and the page's older codes are encoded anew -- by a power of two, so exactly, but for what falls under
// e4m3's smallest normal number.
//
// Units of rows, rotation: rotation.h; codes and scales: cache_codes.h.  A thread holds a unit.
//
// Bound by memory: k, v (and q) are read once, codes (and q_out, k_out) written once, a page's values held in registers
// between its maximum and its codes.  16 prompts of 19269 tokens in all, 32 heads over 8 of 128: 99 us, 4.8 TB/s (a
// copy reaches 5.1).  64 sequences' new tokens: 3.8 us, one: 2.7, a launch and the chain position, page, scale, codes; at positions
// of three axes given 4.9 and 3.6.
#include <algorithm>

#include "cache.h"
#include "cache_codes.h"
#include "hsap_internal.h"
#include "mfma.h"
#include "rotation.h"

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
  Turns turn;     // (positions: of AT kernels alone)
  __bf16* k_out;
  __bf16* q_out;
  int32_t heads_q;
  int32_t kv_blocks;  // workgroups of the cache's part; the others rotate Q
  int32_t q_lanes;    // AT: rows of Q that a wave takes at a time
};

// Values of a row that are rotated as halves.
__device__ __forceinline__ int halves(const AppendArgs& a, bool turned) { return turned && !a.turn.interleaved ? a.turn.rot : 0; }

// Whether new token t, at place pos of its sequence, is taken, and its unit's cosines and sines.  AT: by the positions given.
template <int D, bool AT>
__device__ __forceinline__ bool place(const AppendArgs& a, int64_t t, int64_t pos, Place& x) {
  if (pos < 0) return false;
  if constexpr (AT) return place_of(a.turn, t, x);
  else return a.turn.rot == 0 || pos < a.turn.rows;
}
template <int D, bool AT>
__device__ __forceinline__ UnitTurn turn_of(const AppendArgs& a, const Place& x, int64_t pos, int u) {
  if constexpr (AT) return load_turn<D>(a.turn, x, u);
  else {
    // (one position for every pair)
    const float* cs = a.turn.cos_sin + pos * a.turn.rot;
    const int half = a.turn.rot / 2;
    UnitTurn t{};
    if (a.turn.interleaved) {
      const int first = 4 * u, second = first + D / 4;  // first pairs of the runs
      f32x4 c[2] = {f32x4{}, f32x4{}}, s[2] = {f32x4{}, f32x4{}};
      if (first < half) {
        c[0] = *(const f32x4*)(cs + first);
        s[0] = *(const f32x4*)(cs + half + first);
      }
      if (second < half) {
        c[1] = *(const f32x4*)(cs + second);
        s[1] = *(const f32x4*)(cs + half + second);
      }
      t.c = __builtin_shufflevector(c[0], c[1], 0, 1, 2, 3, 4, 5, 6, 7);
      t.s = __builtin_shufflevector(s[0], s[1], 0, 1, 2, 3, 4, 5, 6, 7);
    } else if (16 * u < a.turn.rot) {
      t.c = load8(cs + 8 * u);
      t.s = load8(cs + half + 8 * u);
    }
    return t;
  }
}
template <int D, bool AT>
__device__ __forceinline__ Unit turned_unit(const AppendArgs& a, const Place& x, int64_t pos, int u, const Unit& r) {
  return turn<D>(a.turn.rot, a.turn.interleaved, u, turn_of<D, AT>(a, x, pos, u), r);
}

template <int D>
__device__ __forceinline__ void store_codes(uint8_t* row, int rot, int u, const Unit& r, float inv) {
  int at[2];
  unit_at<D>(rot, u, at);
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

// AT: a wave takes a token's Q rows, several tokens' where it has few heads, so that their cosines and sines are formed once
// (32 x 24 drafted tokens, 32 heads over 8 of 128, three axes: kernel 8.4 us with a thread per unit, 7.0; four images of 2500
// tokens 24, 4.7 TB/s of rows and codes).
template <int D>
__device__ __forceinline__ void rotate_q_at(const AppendArgs& a, int64_t wave) {
  constexpr int UNITS = D / 16, G = 64 / UNITS;
  const int lane = threadIdx.x & 63, u = lane % UNITS, g = lane / UNITS;
  const int per = G / a.q_lanes, sub = g & (a.q_lanes - 1);
  const int64_t first = wave * per, t = first + g / a.q_lanes;
  if (first >= a.total_new) return;
  int64_t pos;
  if (a.cu) {
    Sequence q = sequence_of(a.cu, a.d.num_seqs, 1, 1, 0, first, a.c.seq_lens);  // q.begin <= first
    if (t >= a.total_new) return;
    if (t >= q.end) {
      int32_t r = a.d.num_seqs;
      if (t >= a.cu[r]) return;  // (behind the last sequence: not read)
      while (r - q.s > 1) {
        const int32_t mid = (q.s + r) >> 1;
        if (a.cu[mid] <= t) q.s = mid;
        else r = mid;
      }
      q.end = a.cu[q.s + 1];
      q.value = a.c.seq_lens[q.s];
    }
    pos = (int64_t)q.value - (q.end - t);
  } else {
    if (t >= a.total_new) return;
    pos = (int64_t)a.c.seq_lens[t] - 1;
  }
  Place at;
  if (pos < 0 || !place_of(a.turn, t, at)) return;
  const UnitTurn by = load_turn<D>(a.turn, at, u);
  const int rot = halves(a, true);
  turn_heads<D, 2>(
      a.turn, by, a.heads_q, sub, a.q_lanes, u, [&](int h) { return load_bf16<D>(a.q + t * a.q_stride + (int64_t)h * D, rot, u); },
      [&](int h, const Unit& r) { store_bf16<D>(a.q_out + (t * a.heads_q + h) * D, rot, u, r); });
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
  const int rot = halves(a, true);
  Unit x = load_bf16<D>(a.q + t * a.q_stride + (int64_t)h * D, rot, u);  // (under way while the position is looked up)
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
  Place at;
  if (!place<D, false>(a, t, pos, at)) return;
  if (a.turn.rot) x = turned_unit<D, false>(a, at, pos, u, x);
  store_bf16<D>(a.q_out + (t * a.heads_q + h) * D, rot, u, x);
}

// One new token per sequence: D / 16 lanes per (sequence, head, K or V).
template <int D, bool AT>
__global__ __launch_bounds__(256) void cache_append_one_kernel(AppendArgs a) {
  constexpr int UNITS = D / 16;
  if ((int)blockIdx.x >= a.kv_blocks) {
    const int64_t block = blockIdx.x - a.kv_blocks;
    if constexpr (AT) rotate_q_at<D>(a, block * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    else rotate_q<D>(a, block * 256 + threadIdx.x);
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
  const int rot = halves(a, !is_v);
  Unit x = load_bf16<D>(src + (int64_t)h * D, rot, u);
  const int32_t pos = a.c.seq_lens[s] - 1;
  Place at;
  if (!place<D, AT>(a, s, pos, at)) return;  // (a place that may hold a token already: the page keeps its scale)
  if (!is_v && a.turn.rot) x = turned_unit<D, AT>(a, at, pos, u, x);
  if (!is_v && a.k_out) store_bf16<D>(a.k_out + (s * a.d.heads_kv + h) * D, rot, u, x);
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
  store_codes<D>(codes + slot * D, rot, u, x, inv);
  if (u == 0) *scale = now;
}

// Any number of new tokens: one workgroup per (page that a sequence's new tokens reach, head, K or V); the page's new
// values are held in registers between the reduction of their maximum and their encoding.
// PER: units of a page per thread.
template <int D, int PER, bool AT>
__global__ __launch_bounds__(256) void cache_append_kernel(AppendArgs a) {
  constexpr int UNITS = D / 16;
  if ((int)blockIdx.x >= a.kv_blocks) {
    const int64_t block = blockIdx.x - a.kv_blocks;
    if constexpr (AT) rotate_q_at<D>(a, block * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6));
    else rotate_q<D>(a, block * 256 + threadIdx.x);
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
  const Sequence q = sequence_of(a.cu, a.d.num_seqs, 1, ps, 2, item, a.c.seq_lens);
  const int32_t s = q.s, t0 = q.begin, count = q.end - t0, len = q.value;
  if (count <= 0 || len <= 0) return;
  const int64_t pos0 = (int64_t)len - count;  // position of the first new token
  const int64_t first = pos0 > 0 ? pos0 : 0;
  const int64_t at = first / ps + (item - item_base(t0, 1, ps, 2, s));
  const int64_t lo = max(first, at * ps);
  int64_t end = min((int64_t)len, (at + 1) * ps);
  if (!AT && a.turn.rot) end = min(end, a.turn.rows);
  end = min(end, pos0 + a.total_new - t0);
  if (lo >= end) return;
  const int32_t page = cache_page(a.c.page_table + (int64_t)s * a.d.table_width, a.d.table_width, a.d.num_pages, ps, (int32_t)lo);
  const int32_t slot0 = (int32_t)(lo - at * ps), units = (int32_t)(end - lo) * UNITS;
  const __bf16* src = (is_v ? a.v : a.k) + (int64_t)h * D;
  const int64_t stride = is_v ? a.v_stride : a.k_stride;
  const int rot = halves(a, !is_v);
  Unit x[PER] = {};
  uint32_t taken = 0;
  float amax = AT ? -1.f : 0.f;  // (AT: tokens without a row in the table are left out, all of them maybe)
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int unit = tid + 256 * i;
    if (unit < units) {
      const int64_t pos = lo + unit / UNITS, t = t0 + (pos - pos0);
      x[i] = load_bf16<D>(src + t * stride, rot, unit % UNITS);
      Place at;
      if (AT && !place<D, AT>(a, t, pos, at)) continue;
      taken |= 1u << i;
      if (!is_v && a.turn.rot) x[i] = turned_unit<D, AT>(a, at, pos, unit % UNITS, x[i]);
      amax = fmaxf(amax, unit_max(x[i]));
      if (!is_v && a.k_out) store_bf16<D>(a.k_out + (t * a.d.heads_kv + h) * D, rot, unit % UNITS, x[i]);
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
  if (AT && amax < 0.f) return;  // (places that may hold tokens already: the page keeps its scale)
  float inv, ratio;
  const float now = page_scale(amax, slot0 > 0, old_scale, inv, ratio);
  if (ratio != 1.f)
    for (int e = tid; e < slot0 * UNITS; e += 256) recode16(codes + 16 * e, ratio);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int unit = tid + 256 * i;
    if (AT ? (taken >> i & 1) != 0 : unit < units) store_codes<D>(codes + (slot0 + unit / UNITS) * D, rot, unit % UNITS, x[i], inv);
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

template <int D, bool AT>
static void launch_append(const AppendArgs& a, int64_t blocks, hipStream_t s) {
  const dim3 grid((unsigned)blocks), block(256);
  const int per = a.d.page_size * (D / 16) / 256;
  if (!a.cu) hipLaunchKernelGGL((cache_append_one_kernel<D, AT>), grid, block, 0, s, a);
  else if (per <= 1) hipLaunchKernelGGL((cache_append_kernel<D, 1, AT>), grid, block, 0, s, a);
  else if (per == 2) hipLaunchKernelGGL((cache_append_kernel<D, 2, AT>), grid, block, 0, s, a);
  else if constexpr (D == 128) hipLaunchKernelGGL((cache_append_kernel<D, 4, AT>), grid, block, 0, s, a);
}

// Everything of an append but what its rotation says.
static hsap_status append(const hsap_cache_desc* desc, const hsap_cache* cache, const void* k, int64_t k_stride, const void* v,
                          int64_t v_stride, const int32_t* cu_new, int64_t total_new, const Turns& turn, void* k_out,
                          const void* q, int64_t q_stride, int32_t heads_q, void* q_out, void* hip_stream) {
  hsap_status st;
  const int d = desc->head_dim;
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
  a.turn = turn;
  a.k_out = (__bf16*)k_out;
  a.q_out = (__bf16*)q_out;
  a.heads_q = heads_q;
  const int64_t units = d / 16;
  const int64_t kv = cu_new ? (item_base(total_new, 1, desc->page_size, 2, desc->num_seqs)) * desc->heads_kv * 2
                            : ((int64_t)desc->num_seqs * desc->heads_kv * 2 * units + 255) / 256;
  a.q_lanes = rows_at_a_time(heads_q, d);
  const int64_t q_tokens = 4 * (64 / units / a.q_lanes);  // AT: of a workgroup
  const int64_t blocks = kv + (!q ? 0 : turn.positions ? (total_new + q_tokens - 1) / q_tokens : (total_new * heads_q * units + 255) / 256);
  if (blocks > kMaxBlocks256) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "too many tokens x heads");
  a.kv_blocks = (int32_t)kv;
  hipStream_t s = (hipStream_t)hip_stream;
  if (turn.positions) {
    if (d == 128) launch_append<128, true>(a, blocks, s);
    else launch_append<64, true>(a, blocks, s);
  } else {
    if (d == 128) launch_append<128, false>(a, blocks, s);
    else launch_append<64, false>(a, blocks, s);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) HSAP_FAIL(HSAP_ERR_HIP, "cache_append launch: %s", hipGetErrorString(e));
  return HSAP_OK;
}

static hsap_status check_new(const hsap_cache_desc* desc, const int32_t* cu_new, int64_t total_new) {
  if (total_new < 0 || total_new > INT32_MAX) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "bad total_new %lld", (long long)total_new);
  if (!cu_new && total_new != desc->num_seqs)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "without cu_new every sequence has one new token: total_new %lld, num_seqs %d",
              (long long)total_new, desc->num_seqs);
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
  if ((st = check_new(desc, cu_new, total_new)) != HSAP_OK) return st;
  if (rot_dim < 0 || rot_dim > desc->head_dim || rot_dim % 16)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "rot_dim %d must be a multiple of 16 up to head_dim %d", rot_dim, desc->head_dim);
  if (rot_dim && (!cos_sin || cos_sin_rows < 1 || ((uintptr_t)cos_sin & 15)))
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "rot_dim without a 16-byte aligned cos_sin table");
  Turns t{};
  t.cos_sin = cos_sin;
  t.rows = cos_sin_rows;
  t.rot = rot_dim;
  t.interleaved = interleaved != 0;
  return append(desc, cache, k, k_stride, v, v_stride, cu_new, total_new, t, k_out, q, q_stride, heads_q, q_out, hip_stream);
}

extern "C" hsap_status hsap_cache_append_at(const hsap_cache_desc* desc, const hsap_cache* cache, const void* k,
                                            int64_t k_stride, const void* v, int64_t v_stride, const int32_t* cu_new,
                                            int64_t total_new, const hsap_rotation* rotation, const int32_t* positions,
                                            void* k_out, const void* q, int64_t q_stride, int32_t heads_q, void* q_out,
                                            void* hip_stream) {
  clear_error();
  hsap_status st = check_cache(desc, cache);
  if (st != HSAP_OK) return st;
  if ((st = check_new(desc, cu_new, total_new)) != HSAP_OK) return st;
  Turns t{};
  if ((st = check_rotation(rotation, desc->head_dim, &t)) != HSAP_OK) return st;
  if (!positions && total_new > 0 && desc->num_seqs > 0) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "NULL positions");
  t.positions = positions;
  t.stride = total_new;
  return append(desc, cache, k, k_stride, v, v_stride, cu_new, total_new, t, k_out, q, q_stride, heads_q, q_out, hip_stream);
}
