// Window attention with sinks, forward: one shard's queries against the keys of their document that are at most
// window - 1 positions back or among the document's first `sinks` tokens.
//
//   O_i = sum_j p_ij v_j,  p_ij = exp(scale q_i . k_j - LSE_i),  LSE_i = ln sum_j exp(scale q_i . k_j)
//
// One workgroup per (q-tile of 32 WAVES consecutive positions, query head), one pass over the tile's keys in steps
// of 64 with a running maximum and sum: first the sinks of the first row's document that lie before every window
// of the tile, then the keys from the first row's window (or document start) to the last row.  A later row's
// document starts inside the tile, so its sinks are among the second set.  No plan: the ranges follow from
// cu_seqlens in the kernel.
//
// Per step: S^T = K Q^T with Q in registers (a lane holds one query and 16 keys of each 32-key block, so the row
// statistics need only the lane and lane l ^ 32), then O^T += V^T P^T with P straight from registers and V^T by
// LDS transpose reads.  K and V go from global memory to LDS directly, K two steps ahead and V one; the scores
// of step s + 1 are formed beside the exponentials of step s.  P is rounded to bf16 for the second product (2^-8
// relative at most, summed in fp32; the row sum takes the unrounded values); O is rounded once, at the end.
//
// Bound by the products and, beside them, the softmax's vector work (per 64-key step and wave, head_dim 128: 32 products,
// 32 exponentials, 115 other vector instructions; with two waves per SIMD they come close to a sum).  65536 tokens,
// 16 heads of 128, window 4096: 2080 us, 1014 TFLOP/s (library product 1314).  4096 of 32768 tokens, 32 heads, window 1024:
// 95 to 98 us, where a workgroup's beginning and end are 8 of its 47 us.  2048 tokens, 4 heads of 64: 9.8 us, latency alone.
#include <algorithm>
#include <type_traits>

#include "window.h"

namespace hsap {

struct WindowFwdArgs {
  const __bf16* q;
  const __bf16* k;
  const __bf16* v;
  const int32_t* cu;
  __bf16* o;
  float* lse;
  Geom geom;
  int32_t num_docs;
  int32_t shard;
  int32_t hq;
  int32_t hkv;
  int32_t window;
  int32_t sinks;
  int32_t tiles;  // q-tiles per segment
  float scale_log2;
};

template <int D, int WAVES, int KS>
__global__ __launch_bounds__(64 * WAVES * KS, KS * D > 128 ? 1 : D == 64 && KS == 1 ? 3 : 2) void window_fwd_kernel(WindowFwdArgs a) {
  constexpr int KB = 64, CPR = D / 8, TILE = KB * D, BM = 32 * WAVES;
  constexpr float NEG_INF = -__builtin_inff();
  constexpr float RESCALE_SLACK = 8.f;  // log2 units a row maximum may rise before O is rescaled
  __shared__ __attribute__((aligned(16))) __bf16 rings[KS * 4 * TILE];  // per stream: K slots 0, 1, then V slots 0, 1
  __shared__ int32_t tile_start;
  static_assert(KS == 1 || KS * 4 * TILE * 2 >= (KS - 1) * WAVES * (D / 2 + 2) * 256, "room for the streams' results");

  const int tid = threadIdx.x;
  const int lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
  const int w = uniform(tid >> 6) % WAVES, ks = uniform(tid >> 6) / WAVES;  // 32-row slice, key stream
  __bf16* const ring = rings + ks * 4 * TILE;
  auto Ks = [&](int slot) { return ring + slot * TILE; };
  auto Vs = [&](int slot) { return ring + (2 + slot) * TILE; };
  int t, h;
  run_and_head(blockIdx.x, a.hq, a.hkv, t, h);
  // the last q-tiles of every segment first: with a wide window they have the most keys
  const int32_t segs = (int32_t)(a.geom.n / a.geom.m);
  const int32_t seg = t % segs, qt = a.tiles - 1 - t / segs;
  const int g = h / (a.hq / a.hkv);
  const int64_t n = a.geom.n;
  const int32_t m = (int32_t)a.geom.m;
  const int32_t p0 = uniform(segment_start(a.geom, a.shard, seg));  // the segment's first position
  const int32_t i0 = p0 + qt * BM;
  const int32_t gq = min(i0 + 32 * w + l32, p0 + m - 1);
  const DocSpan doc = doc_span(a.cu, a.num_docs, gq, lane);
  // positions of the tile's rows that are queries: i0 .. i1; rows behind the last document are left alone
  const int32_t i1 = min(min(i0 + BM - 1, p0 + m - 1), a.cu[a.num_docs] - 1);
  if (i1 < i0) return;
  const bool valid = i0 + 32 * w + l32 <= i1;
  const int64_t qrow = (int64_t)seg * m + (min(gq, i1) - p0);

  bf16x8 qf[D / 16];
  {
    const __bf16* qp = a.q + (qrow * a.hq + h) * D + 8 * hi;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) qf[kk] = *(const bf16x8*)(qp + 16 * kk);
  }
  if (tid == 0) tile_start = doc.start;
  __syncthreads();
  const int32_t start0 = uniform(tile_start);
  // window keys from win_lo, sinks before them from start0 to sink_hi - 1
  const int32_t win_lo = max(start0, i0 - (a.window - 1));
  const int32_t sink_hi = start0 + min(a.sinks, win_lo - start0);
  const int32_t sink_steps = (sink_hi - start0 + KB - 1) / KB;
  const int32_t steps = sink_steps + (i1 - win_lo + KB) / KB;
  const int32_t total = KS == 1 ? steps : (steps - ks + KS - 1) / KS;  // this stream's: ks, ks + KS, ...
  // this lane's keys: wlo .. gq, and start .. start + slen - 1 (its sinks before the window)
  const int32_t wlo = max(doc.start, gq - (a.window - 1));
  const int32_t slen = min(a.sinks, wlo - doc.start);

  const int64_t rstride = (int64_t)a.hkv * D;
  const __bf16* kbase = a.k + (int64_t)g * D;
  const __bf16* vbase = a.v + (int64_t)g * D;
  TileStage<D, WAVES> st;
  st.init(w, lane, rstride * 2);
  KeySpan kspan{0, 0, 0}, vspan{0, 0, 0};
  auto at = [&](int s) { return KS * s + ks; };  // of all steps
  auto step_key = [&](int s) { return at(s) < sink_steps ? start0 + KB * at(s) : win_lo + KB * (at(s) - sink_steps); };
  auto step_max = [&](int s) { return at(s) < sink_steps ? sink_hi - 1 : i1; };  // last key that exists for it
  auto stage_k = [&](int s, int slot) {
    stage_keys<D, WAVES>(st, a.geom, kspan, step_key(s), step_max(s), kbase, rstride, Ks(slot));
  };
  auto stage_v = [&](int s, int slot) {
    stage_keys<D, WAVES>(st, a.geom, vspan, step_key(s), step_max(s), vbase, rstride, Vs(slot));
  };

  const int tr_row = 4 * hi + ((lane & 15) >> 2);
  const int tr_col = 16 * ((lane >> 4) & 1) + 4 * (lane & 3);
  int rowoff[D / 16], troff[D / 32][2];
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) rowoff[kk] = swz<CPR>(l32, 16 * kk + 8 * hi);
#pragma unroll
  for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
    for (int k = 0; k < 2; ++k) troff[mb][k] = swz<CPR>(8 * k + tr_row, 32 * mb + tr_col) - 8 * k * D;

  // S^T of the step's 32-key block nb
  auto scores = [&](const __bf16* K, f32x16 (&sc)[KB / 32], int nb) __attribute__((always_inline)) {
    bf16x8 kf[D / 16];
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) kf[kk] = *(const bf16x8*)(K + 32 * nb * D + rowoff[kk]);
    sc[nb] = f32x16{};
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) sc[nb] = mfma32(kf[kk], qf[kk], sc[nb]);
  };

  float m_run = NEG_INF, l_run = 0.f;
  f32x16 o[D / 32];
#pragma unroll
  for (int mb = 0; mb < D / 32; ++mb) o[mb] = f32x16{};

  if (KS == 1 || total > 0) {
    stage_k(0, 0);
    stage_v(0, 0);
  }
  if (total > 1) stage_k(1, 1);
  vm_wait_barrier<0>();
  f32x16 sc[KB / 32];
#pragma unroll
  for (int nb = 0; nb < KB / 32; ++nb) scores(Ks(0), sc, nb);
  hsap_lds_barrier();

  // Instruction order asked of the compiler for the block of a step (head_dim 128): four K reads ahead, then per score
  // MFMA one LDS read and four vector instructions (this step's exponentials, sums and conversions), then per PV MFMA
  // two V^T reads and three vector ones.
  auto block_order = []() __attribute__((always_inline)) {
    __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);  // LDS reads
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);  // MFMA
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x406, 4, 0);  // VALU, SALU, transcendental
    }
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x406, 3, 0);
    }
  };
  // one 64-key step: softmax and PV of step s from `sc`, the scores of step s + 1 into `sn` (`par` is s % 2 as a
  // compile-time constant; the last step's next scores read a slot that nothing refills and are dropped)
  auto step = [&](int s, auto par, f32x16 (&sc)[KB / 32], f32x16 (&sn)[KB / 32]) __attribute__((always_inline)) {
    constexpr int S0 = decltype(par)::value, S1 = S0 ^ 1;
    if (s + 2 < total) stage_k(s + 2, S0);
    if (s + 1 < total) stage_v(s + 1, S1);

    // A step that every query of the wave sees whole needs no per-key mask.  Keys of a sink step at or behind the first
    // window belong to the window steps.
    const bool sink_step = at(s) < sink_steps;
    const int32_t j0 = step_key(s);
    const uint32_t wlen = sink_step || !valid ? 0u : (uint32_t)(gq - wlo + 1);
    const uint32_t sl = !valid ? 0u : (uint32_t)(sink_step ? min(slen, max(sink_hi - doc.start, 0)) : slen);
    const int32_t rw = j0 - wlo, rs = j0 - doc.start;  // offsets of the step's first key in the two ranges
    const bool all = !valid || (rw >= 0 && rw + KB <= (int32_t)wlen);
    if (__builtin_amdgcn_ballot_w64(!all) != 0) {
      const int32_t rw0 = rw + 4 * hi, rs0 = rs + 4 * hi;
#pragma unroll
      for (int nb = 0; nb < KB / 32; ++nb)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int c = 32 * nb + c_row(j, 0);
          if ((uint32_t)(rw0 + c) >= wlen && (uint32_t)(rs0 + c) >= sl) sc[nb][j] = NEG_INF;
        }
    }
    float mx = sc[0][0];
#pragma unroll
    for (int nb = 0; nb < KB / 32; ++nb)
#pragma unroll
      for (int j = 0; j < 16; ++j) mx = fmaxf(mx, sc[nb][j]);
    const float m_new = fmaxf(m_run, pair_max(mx) * a.scale_log2);
    if (__builtin_amdgcn_ballot_w64(m_new > m_run + RESCALE_SLACK) != 0) {
      const float alpha = fast_exp2(m_run - (m_new == NEG_INF ? 0.f : m_new));
      l_run *= alpha;
#pragma unroll
      for (int mb = 0; mb < D / 32; ++mb) o[mb] *= alpha;
      m_run = m_new;
    }
    const float m_use = m_run == NEG_INF ? 0.f : m_run;  // (a row that has seen no key yet)
    __builtin_amdgcn_s_setprio(1);
    float rsum = 0.f;
    bf16x8 pb[KB / 32][2];
#pragma unroll
    for (int nb = 0; nb < KB / 32; ++nb) {
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float p = fast_exp2(__builtin_fmaf(sc[nb][j], a.scale_log2, -m_use));
        rsum += p;
        pb[nb][j >> 3][j & 7] = (__bf16)p;
      }
      scores(Ks(S1), sn, nb);
    }
    l_run += rsum;
    const __bf16* V = Vs(S0);
#pragma unroll
    for (int nb = 0; nb < KB / 32; ++nb)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int rb = (32 * nb + 16 * half) * D;
#pragma unroll
        for (int mb = 0; mb < D / 32; ++mb)
          o[mb] = mfma32(cat4(ds_read_tr16(V + rb + troff[mb][0]), ds_read_tr16(V + rb + 8 * D + troff[mb][1])),
                         pb[nb][half], o[mb]);
      }
    if constexpr (D == 128) block_order();
    __builtin_amdgcn_s_setprio(0);
    vm_wait_barrier<0>();
  };
  if constexpr (KS > 1) {
    // every stream takes part in the barriers of the longest one (the first)
    const int most = (steps + KS - 1) / KS;
    f32x16 sn[KB / 32];
    for (int s = 0; s < most; s += 2) {
      if (s < total) step(s, std::integral_constant<int, 0>{}, sc, sn);
      else vm_wait_barrier<0>();
      if (s + 1 < most) {
        if (s + 1 < total) step(s + 1, std::integral_constant<int, 1>{}, sn, sc);
        else vm_wait_barrier<0>();
      }
    }
    // the streams' maxima, sums and O to LDS, register by register (no bank conflict), joined in stream order
    float* const res = (float*)rings;
    if (ks > 0) {
      float* const mine = res + ((ks - 1) * WAVES + w) * (D / 2 + 2) * 64 + lane;
#pragma unroll
      for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
        for (int j = 0; j < 16; ++j) mine[(16 * mb + j) * 64] = o[mb][j];
      mine[(D / 2) * 64] = m_run;
      mine[(D / 2 + 1) * 64] = l_run;
    }
    hsap_lds_barrier();
    if (ks > 0) return;
    for (int x = 1; x < KS; ++x) {
      const float* const other = res + ((x - 1) * WAVES + w) * (D / 2 + 2) * 64 + lane;
      const float m2 = other[(D / 2) * 64], l2 = other[(D / 2 + 1) * 64];
      const float m = fmaxf(m_run, m2), m_use = m == NEG_INF ? 0.f : m;
      const float f1 = fast_exp2(m_run - m_use), f2 = fast_exp2(m2 - m_use);
      l_run = l_run * f1 + l2 * f2;
      m_run = m;
#pragma unroll
      for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
        for (int j = 0; j < 16; ++j) o[mb][j] = o[mb][j] * f1 + other[(16 * mb + j) * 64] * f2;
    }
  } else if constexpr (D == 64) {
    // one score array: each 32-key half is replaced once its exponentials are formed
    for (int s = 0; s < total; s += 2) {
      step(s, std::integral_constant<int, 0>{}, sc, sc);
      if (s + 1 < total) step(s + 1, std::integral_constant<int, 1>{}, sc, sc);
    }
  } else {
    f32x16 sn[KB / 32];
    for (int s = 0; s < total; s += 2) {
      step(s, std::integral_constant<int, 0>{}, sc, sn);
      if (s + 1 < total) step(s + 1, std::integral_constant<int, 1>{}, sn, sc);
    }
  }

  if (!valid) return;
  l_run = pair_sum(l_run);
  const float inv = 1.f / l_run;  // a row always sees itself: l_run > 0
  __bf16* op = a.o + (qrow * a.hq + h) * D + 4 * hi;
#pragma unroll
  for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
    for (int grp = 0; grp < 4; ++grp)
      *(bf16x4*)(op + 32 * mb + 8 * grp) = bf16x4{(__bf16)(o[mb][4 * grp] * inv), (__bf16)(o[mb][4 * grp + 1] * inv),
                                                  (__bf16)(o[mb][4 * grp + 2] * inv), (__bf16)(o[mb][4 * grp + 3] * inv)};
  if (hi == 0) a.lse[(int64_t)h * n + qrow] = (m_run + __log2f(l_run)) * kLn2;
}

hsap_status check_window(const hsap_attn_desc* desc, int32_t window, int32_t sinks, const int32_t* cu, int32_t num_docs,
                         Geom* g) {
  if (!desc) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "attention descriptor is NULL");
  hsap_attn_desc d = *desc;
  d.shard.block_m = d.shard.block_n = 1;  // no tile lists here: any row count
  const hsap_status st = check_attn(&d, g);
  if (st != HSAP_OK) return st;
  if (window < 1) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "window %d < 1 (a query always sees itself)", window);
  if (sinks < 0) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "sinks %d < 0", sinks);
  if ((int64_t)desc->heads_q * desc->head_dim * 128 > INT32_MAX)
    HSAP_FAIL(HSAP_ERR_UNSUPPORTED, "heads_q %d too large", desc->heads_q);
  if (num_docs < 1) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "num_docs %d < 1", num_docs);
  if (!cu) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "NULL cu_seqlens");
  return HSAP_OK;
}

template <int D, int WAVES, int KS>
static hsap_status launch_window_fwd(WindowFwdArgs& a, hipStream_t stream) {
  constexpr int BM = 32 * WAVES;
  a.tiles = (int32_t)((a.geom.m + BM - 1) / BM);
  const int64_t blocks = a.geom.n / a.geom.m * a.tiles * a.hq;
  if (blocks > INT32_MAX) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "too many rows x heads");
  hipLaunchKernelGGL((window_fwd_kernel<D, WAVES, KS>), dim3((unsigned)blocks), dim3(64 * WAVES * KS), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) HSAP_FAIL(HSAP_ERR_HIP, "window_attn_fwd launch: %s", hipGetErrorString(e));
  return HSAP_OK;
}

template <int D>
static hsap_status dispatch_window_fwd(WindowFwdArgs& a, hipStream_t stream) {
  if (window_query_blocks(a.geom, a.hq, D) == 2) return launch_window_fwd<D, 2, 2>(a, stream);
  return launch_window_fwd<D, 4, 1>(a, stream);
}

}  // namespace hsap

using namespace hsap;

extern "C" hsap_status hsap_window_attn_fwd(const hsap_attn_desc* desc, int32_t window, int32_t sinks, const void* q,
                                            const void* k, const void* v, const int32_t* cu_seqlens, int32_t num_docs,
                                            void* o_out, float* lse_out, void* hip_stream) {
  clear_error();
  WindowFwdArgs a{};
  const hsap_status st = check_window(desc, window, sinks, cu_seqlens, num_docs, &a.geom);
  if (st != HSAP_OK) return st;
  if (!q || !k || !v || !o_out || !lse_out) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "NULL pointer argument");
  if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v) & 15)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "q, k and v must be 16-byte aligned");
  if ((uintptr_t)o_out & 7) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "o_out must be 8-byte aligned");
  a.q = (const __bf16*)q;
  a.k = (const __bf16*)k;
  a.v = (const __bf16*)v;
  a.cu = cu_seqlens;
  a.o = (__bf16*)o_out;
  a.lse = lse_out;
  a.num_docs = num_docs;
  a.shard = desc->shard.shard_id;
  a.hq = desc->heads_q;
  a.hkv = desc->heads_kv;
  a.window = (int32_t)std::min<int64_t>(window, a.geom.Ns);
  a.sinks = (int32_t)std::min<int64_t>(sinks, a.geom.Ns);
  a.scale_log2 = desc->softmax_scale * kLog2e;
  hipStream_t s = (hipStream_t)hip_stream;
  return desc->head_dim == 128 ? dispatch_window_fwd<128>(a, s) : dispatch_window_fwd<64>(a, s);
}
