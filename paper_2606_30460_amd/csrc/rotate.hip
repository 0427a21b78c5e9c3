// Rotation of rows by positions of several axes, and back (the gradient's).
//
//   (a, b) of pair i  ->  (a cos - b sin, b cos + a sin),   cos | sin = row positions[axis(i), t] of the table, entry i
//
// and with the sine's sign turned for the inverse, which is the transpose: the gradient of the rotated rows goes back by it.
// Bound by memory: every row is read and written once (32768 tokens, 32 heads and 8 of 128: 148 us, 4.8 TB/s where a copy reaches
// 5.0; with fp32 rows in 189 us, out 216, both 250: 5.3, 4.7, 5.4 TB/s; 1999 tokens of 6 and 2 heads of 64: 4.6 us).  A wave takes one token's rows of all heads (several tokens where it
// has few), so that a lane forms its unit's cosines and sines, whose rows differ from pair to pair, once for all heads, and
// has the rows of several heads in flight.
#include "hsap_internal.h"
#include "rotation.h"

namespace hsap {

struct RotateArgs {
  Turns turn;
  hsap_token_rows x[2];
  int64_t total;
  int32_t lanes;  // rows of one token that a wave takes at a time: a power of two up to 64 / (D / 16)
  int32_t inverse;
};

template <int D>
__device__ __forceinline__ Unit load_row(const hsap_token_rows& x, int64_t at, int rot, int u) {
  if (!x.in_f32) return load_bf16<D>((const __bf16*)x.in + at, rot, u);
  int p[2];
  unit_at<D>(rot, u, p);
  const float* row = (const float*)x.in + at;
  return Unit{load8(row + p[0]), load8(row + p[1])};
}

__device__ __forceinline__ void store8(float* p, const f32x8& v) {
  *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]};
  *(f32x4*)(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}

template <int D>
__device__ __forceinline__ void store_row(const hsap_token_rows& x, int64_t at, int rot, int u, const Unit& r) {
  if (!x.out_f32) return store_bf16<D>((__bf16*)x.out + at, rot, u, r);
  int p[2];
  unit_at<D>(rot, u, p);
  float* row = (float*)x.out + at;
  store8(row + p[0], r.a);
  store8(row + p[1], r.b);
}

template <int D>
__global__ __launch_bounds__(256) void rotate_kernel(RotateArgs a) {
  constexpr int UNITS = D / 16, G = 64 / UNITS;
  const int lane = threadIdx.x & 63, u = lane % UNITS, g = lane / UNITS;
  const int64_t wave = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int sub = g & (a.lanes - 1);
  const int64_t t = wave * (G / a.lanes) + g / a.lanes;
  if (t >= a.total) return;
  Place at;
  if (!place_of(a.turn, t, at)) return;
  UnitTurn turned = load_turn<D>(a.turn, at, u);
  if (a.inverse) turned.s = -turned.s;
  const int rot = a.turn.interleaved ? 0 : a.turn.rot;
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const hsap_token_rows& x = a.x[n];
    turn_heads<D, 4>(
        a.turn, turned, x.heads, sub, a.lanes, u, [&](int h) { return load_row<D>(x, t * x.in_stride + (int64_t)h * D, rot, u); },
        [&](int h, const Unit& r) { store_row<D>(x, t * x.out_stride + (int64_t)h * D, rot, u, r); });
  }
}

hsap_status check_rotation(const hsap_rotation* r, int32_t head_dim, Turns* out) {
  if (!r) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "rotation is NULL");
  if (r->rot_dim < 16 || r->rot_dim > head_dim || r->rot_dim % 16)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "rot_dim %d must be a multiple of 16 from 16 to head_dim %d", r->rot_dim, head_dim);
  if (r->axes < 1 || r->axes > kMaxAxes) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "axes %d: 1 to %d", r->axes, kMaxAxes);
  if (!r->cos_sin || r->rows < 1 || ((uintptr_t)r->cos_sin & 15))
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "rotation without a 16-byte aligned cos_sin table");
  Turns t{};
  t.cos_sin = r->cos_sin;
  t.rows = r->rows;
  t.rot = r->rot_dim;
  t.interleaved = r->interleaved != 0;
  t.axes = r->axes;
  for (int i = 0; i < r->rot_dim / 2; ++i) {
    if (r->pair_axis[i] >= r->axes) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "pair %d has axis %d of %d", i, r->pair_axis[i], r->axes);
    t.axis[i / 16] |= (uint32_t)r->pair_axis[i] << (2 * (i % 16));
  }
  *out = t;
  return HSAP_OK;
}

static hsap_status check_token_rows(const char* what, const hsap_token_rows& x, int64_t row) {
  if (x.heads < 1) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "%s: heads %d < 1", what, x.heads);
  if (!x.in || !x.out) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "%s: NULL pointer", what);
  if (((uintptr_t)x.in | (uintptr_t)x.out) & 15) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "%s: rows must be 16-byte aligned", what);
  if (x.in_stride % 8 || x.out_stride % 8 || x.in_stride < x.heads * row || x.out_stride < x.heads * row)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "%s: row strides (%lld, %lld) must be multiples of 8 and at least %lld", what,
              (long long)x.in_stride, (long long)x.out_stride, (long long)(x.heads * row));
  if (x.in == x.out && (x.in_stride != x.out_stride || !x.in_f32 != !x.out_f32))
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "%s: in place rows have one type and stride", what);
  return HSAP_OK;
}

}  // namespace hsap

using namespace hsap;

extern "C" hsap_status hsap_rotate(const hsap_rotation* rotation, int32_t head_dim, const int32_t* positions, int64_t total,
                                   const hsap_token_rows* q, const hsap_token_rows* k, int32_t inverse, void* hip_stream) {
  clear_error();
  if (head_dim != 64 && head_dim != 128) HSAP_FAIL(HSAP_ERR_UNSUPPORTED, "head_dim %d not supported (64 or 128)", head_dim);
  RotateArgs a{};
  hsap_status st = check_rotation(rotation, head_dim, &a.turn);
  if (st != HSAP_OK) return st;
  if (total < 0 || total > INT32_MAX) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "bad total %lld", (long long)total);
  if (!q) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "q is NULL");
  if (total == 0) return HSAP_OK;
  if (!positions) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "NULL positions");
  if ((st = check_token_rows("q", *q, head_dim)) != HSAP_OK) return st;
  if (k && (st = check_token_rows("k", *k, head_dim)) != HSAP_OK) return st;
  a.turn.positions = positions;
  a.turn.stride = total;
  a.x[0] = *q;
  if (k) a.x[1] = *k;
  a.total = total;
  a.inverse = inverse != 0;
  const int32_t most = 64 / (head_dim / 16);
  a.lanes = rows_at_a_time(q->heads > a.x[1].heads ? q->heads : a.x[1].heads, head_dim);
  const int64_t per = 4 * (most / a.lanes), blocks = (total + per - 1) / per;
  if (blocks > kMaxBlocks256) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "too many tokens");
  hipStream_t s = (hipStream_t)hip_stream;
  if (head_dim == 128) hipLaunchKernelGGL(rotate_kernel<128>, dim3((unsigned)blocks), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(rotate_kernel<64>, dim3((unsigned)blocks), dim3(256), 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) HSAP_FAIL(HSAP_ERR_HIP, "rotate launch: %s", hipGetErrorString(e));
  return HSAP_OK;
}
