// Window attention with sinks, backward.  With P_ij = exp(scale q_i . k_j - LSE_i) over the pairs the forward allows
// and delta_i = sum_d dO_id O_id:
//
//   dV_j = sum_i P_ij dO_i,   dS_ij = P_ij (dO_i . v_j - delta_i),
//   dQ_i = scale sum_j dS_ij k_j,   dK_j = scale sum_i dS_ij q_i   (dK, dV over the query heads of the K/V head)
//
// Every gradient row has one owner, which forms it whole in registers and stores it once: no atomics, the same bits
// each time.  S and dP are formed by the dQ and by the dK/dV kernel: 14 d flops per pair instead of 10 d, where adding dQ up
// across key tiles would need fp32 atomics or partials.  P and dS are rounded to bf16 for the second products (2^-8 relative
// at most, summed in fp32), each gradient once, at the end.
//
// Bound by LDS reads, products and exponentials following one another in a wave.  16384 of 65536 tokens, 16 heads over 16 of
// 128, window 2048: dQ 423 us (0.75 of the library product's rate, counting what is executed), dK/dV 678 (0.63), sinks 36.
// 8192 tokens, 32 heads over 8, window 1024: 211, 270, 35.  Three times 1999 tokens, 6 heads over 2 of 64, window 200: 20,
// 19, 12, each the longest chain of its grid.
//
// Two to five launches:
//   dQ       one workgroup per (128-row q-tile, query head), over the tile's keys as in the forward; delta first
//   sinks    a document's sinks are seen by all its later queries, far more than a window's worth.  The shard's rows
//            are cut into chunks (256 queries or more); one workgroup per (chunk, K/V head) forms what the chunk's queries
//            give to the sinks of the document that reaches into it from before (outside their windows): fp32 partials
//   sum      where a segment has many chunks: those of one document added up, in order, into the first one's partial
//   dK, dV   one workgroup per (128 consecutive keys, K/V head), over the queries whose window holds one of them --
//            and, for sinks, over the queries of their own chunk -- for every query head of the group; a sink's
//            partials are added before the gradient is rounded
//   heads    where that grid is small and a group large, the group's heads are dealt to several workgroups, whose fp32
//            gradients this one adds up in order
// Sinks and sum run only where some query can be further than a window from a sink.
#include <algorithm>
#include <type_traits>

#include "window.h"

namespace hsap {

hsap_status check_window(const hsap_attn_desc* desc, int32_t window, int32_t sinks, const int32_t* cu, int32_t num_docs,
                         Geom* g);

struct WindowBwdArgs {
  const __bf16* q;
  const __bf16* k;
  const __bf16* v;
  const __bf16* d_o;
  const __bf16* o;
  const float* lse;
  float* delta;    // [Hq, n]
  float* partial;  // [chunks, Hkv, sinks, 2, D]: dK (unscaled) and dV of the sinks per chunk of queries
  const int32_t* cu;
  __bf16* dq;
  void* dk;
  void* dv;
  Geom geom;
  int32_t num_docs;
  int32_t shard;
  int32_t hq;
  int32_t hkv;
  int32_t window;
  int32_t sinks;
  int32_t tiles;   // q-tiles (dQ) or key tiles (dK, dV) per segment
  int32_t chunk;   // queries of a sink chunk, a power of two
  int32_t chunks;  // sink chunks per segment; 0: no sink pass
  int32_t summed;  // a document's partials are summed up in its first chunk's
  int32_t dkv_f32;
  int32_t head_split;  // workgroups per key tile and K/V head, each with some of the group's heads
  float* heads_part;   // [head_split, P * n, Hkv, 2, D], head_split > 1: dK (unscaled) and dV of each
  float scale;
  float scale_log2;
};

// Adds the streams' sums onto stream 0's, in stream order, through LDS (register by register: no bank conflict).
template <int N, int WAVES, int KS>
__device__ __forceinline__ void join_streams(f32x16 (&sum)[N], float* res, int w, int ks, int lane) {
  if (ks > 0) {
    float* const mine = res + ((ks - 1) * WAVES + w) * N * 16 * 64 + lane;
#pragma unroll
    for (int mb = 0; mb < N; ++mb)
#pragma unroll
      for (int j = 0; j < 16; ++j) mine[(16 * mb + j) * 64] = sum[mb][j];
  }
  hsap_lds_barrier();
  if (ks == 0) {
    for (int x = 1; x < KS; ++x) {
      const float* const other = res + ((x - 1) * WAVES + w) * N * 16 * 64 + lane;
#pragma unroll
      for (int mb = 0; mb < N; ++mb)
#pragma unroll
        for (int j = 0; j < 16; ++j) sum[mb][j] += other[(16 * mb + j) * 64];
    }
  }
}

// The compiler, short of registers, reads an operand from LDS right before its product and waits for it.  The loops below
// read a few products ahead instead and keep the order of reads and products (vector instructions may still move).
constexpr int kAhead = 3;
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0x406); }

// ---------------------------------------------------------------------------
// dQ: the forward's ranges, three products per 64-key step (S, dP and dS K).  dP - delta is formed by the matrix
// product itself, whose accumulator starts at -delta.
// ---------------------------------------------------------------------------
template <int D, int WAVES, int KS>
__global__ __launch_bounds__(64 * WAVES * KS, KS * D > 128 ? 1 : 2) void window_dq_kernel(WindowBwdArgs a) {
  constexpr int KB = 64, TILE = KB * D, BM = 32 * WAVES;
  constexpr float NEG_INF = -__builtin_inff();
  __shared__ __attribute__((aligned(16))) __bf16 rings[KS * 4 * TILE];  // per stream: K slots 0, 1, then V slots 0, 1
  __shared__ int32_t tile_start;
  static_assert(KS == 1 || KS * 4 * TILE * 2 >= (KS - 1) * WAVES * (D / 2) * 256, "room for the streams' results");

  const int tid = threadIdx.x;
  const int lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
  const int w = uniform(tid >> 6) % WAVES, ks = uniform(tid >> 6) / WAVES;  // 32-row slice, key stream
  __bf16* const ring = rings + ks * 4 * TILE;
  auto Ks = [&](int slot) { return ring + slot * TILE; };
  auto Vs = [&](int slot) { return ring + (2 + slot) * TILE; };
  int t, h;
  run_and_head(blockIdx.x, a.hq, a.hkv, t, h);
  const int32_t segs = (int32_t)(a.geom.n / a.geom.m);
  const int32_t seg = t % segs, qt = a.tiles - 1 - t / segs;
  const int g = h / (a.hq / a.hkv);
  const int64_t n = a.geom.n;
  const int32_t m = (int32_t)a.geom.m;
  const int32_t p0 = uniform(segment_start(a.geom, a.shard, seg));
  const int32_t i0 = p0 + qt * BM;
  const int32_t gq = min(i0 + 32 * w + l32, p0 + m - 1);
  const DocSpan doc = doc_span(a.cu, a.num_docs, gq, lane);
  const int32_t i1 = min(min(i0 + BM - 1, p0 + m - 1), a.cu[a.num_docs] - 1);
  if (i1 < i0) return;
  const bool valid = i0 + 32 * w + l32 <= i1;
  const int64_t qrow = (int64_t)seg * m + (min(gq, i1) - p0);

  bf16x8 qf[D / 16], df[D / 16];
  float delta = 0.f;
  {
    const int64_t at = (qrow * a.hq + h) * D + 8 * hi;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      qf[kk] = *(const bf16x8*)(a.q + at + 16 * kk);
      df[kk] = *(const bf16x8*)(a.d_o + at + 16 * kk);
      const bf16x8 of = *(const bf16x8*)(a.o + at + 16 * kk);
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = __builtin_fmaf((float)df[kk][e], (float)of[e], delta);
    }
  }
  delta = pair_sum(delta);
  const float lse2 = a.lse[(int64_t)h * n + qrow] * kLog2e;
  if (tid == 0) tile_start = doc.start;
  __syncthreads();
  const int32_t start0 = uniform(tile_start);
  const int32_t win_lo = max(start0, i0 - (a.window - 1));
  const int32_t sink_hi = start0 + min(a.sinks, win_lo - start0);
  const int32_t sink_steps = (sink_hi - start0 + KB - 1) / KB;
  const int32_t steps = sink_steps + (i1 - win_lo + KB) / KB;
  const int32_t total = KS == 1 ? steps : (steps - ks + KS - 1) / KS;  // this stream's: ks, ks + KS, ...
  const int32_t wlo = max(doc.start, gq - (a.window - 1));
  const int32_t slen = min(a.sinks, wlo - doc.start);

  const int64_t rstride = (int64_t)a.hkv * D;
  const __bf16* kbase = a.k + (int64_t)g * D;
  const __bf16* vbase = a.v + (int64_t)g * D;
  // delta from O carries O's rounding, which dS = P (dP - delta) feels where a row has few keys (one key: dS is 0, but
  // for that rounding).  Rows of fewer than 32 keys take delta = sum_j P_ij dP_ij instead, over the 64 positions up
  // to the wave's last row and the sinks of its first row's document, read straight from global memory (a place of those
  // that no short row sees: the wave's first row instead).
  const bool few = valid && gq - wlo + 1 + slen < 32;
  const uint64_t short_rows = __builtin_amdgcn_ballot_w64(few);
  if (short_rows != 0) {
    const int32_t g0 = __builtin_amdgcn_readlane(gq, 0), far = __builtin_amdgcn_readlane(doc.start, 0);
    // (windows begin later from row to row, and a later row of a document has as many sinks before its window or more)
    const int32_t lo = __builtin_amdgcn_readlane(wlo, __builtin_ctzll(short_rows));
    const uint32_t of_far = (uint32_t)__builtin_amdgcn_ballot_w64(few && doc.start == far);
    const int32_t far_end = far + (of_far ? __builtin_amdgcn_readlane(slen, 31 - __builtin_clz(of_far)) : 0);
    const bool sinks = __builtin_amdgcn_ballot_w64(few && slen > 0 && doc.start < g0 - 32) != 0;
    float sum = 0.f;
    for (int b = 0; b < (sinks ? 3 : 2); ++b) {
      const int32_t j0 = b == 2 ? far : g0 - 32 + 32 * b;
      const int32_t j = short_row_key(j0 + l32, g0, lo, far, far_end, i1);  // this lane's key row
      const int64_t at = ((int64_t)(j + key_span(a.geom, j).delta) * a.hkv + g) * D + 8 * hi;
      f32x16 sc = f32x16{}, dp = f32x16{};
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) sc = mfma32(*(const bf16x8*)(a.k + at + 16 * kk), qf[kk], sc);
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) dp = mfma32(*(const bf16x8*)(a.v + at + 16 * kk), df[kk], dp);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int32_t x = j0 + c_row(e, hi);
        const bool in = x >= wlo && x <= gq, sink = x >= doc.start && x < doc.start + slen;
        // (the sinks of the third block: those before the other two)
        const bool see = b == 2 ? sink && x < g0 - 32 : in || sink;
        sum += see ? fast_exp2(__builtin_fmaf(sc[e], a.scale_log2, -lse2)) * dp[e] : 0.f;
      }
    }
    sum = pair_sum(sum);
    if (few) delta = sum;
  }
  if (hi == 0 && valid && ks == 0) a.delta[(int64_t)h * n + qrow] = delta;

  TileStage<D, WAVES> st;
  st.init(w, lane, rstride * 2);
  KeySpan span{0, 0, 0};
  auto stage = [&](int i, int slot) {
    const int s = KS * i + ks;
    const int32_t j0 = s < sink_steps ? start0 + KB * s : win_lo + KB * (s - sink_steps);
    const int32_t jmax = s < sink_steps ? sink_hi - 1 : i1;
    stage_keys<D, WAVES>(st, a.geom, span, j0, jmax, kbase, rstride, Ks(slot));
    stage_keys<D, WAVES>(st, a.geom, span, j0, jmax, vbase, rstride, Vs(slot));
  };
  TileReads<D> rd;
  rd.init(lane);

  f32x16 dq[D / 32];
#pragma unroll
  for (int mb = 0; mb < D / 32; ++mb) dq[mb] = f32x16{};
  f32x16 minus_delta;
#pragma unroll
  for (int j = 0; j < 16; ++j) minus_delta[j] = -delta;

  if (KS == 1 || total > 0) stage(0, 0);
  // (the compiler sees no wait inside asm: without this use it would wait for these rows at their first use in the
  // loop, every time, and so for the transfers under way)
#pragma unroll
  for (int kk = 0; kk < D / 16; ++kk) asm volatile("" ::"v"(qf[kk]), "v"(df[kk]));
  vm_wait_barrier<0>();
  auto step = [&](int i, auto par) __attribute__((always_inline)) {
    constexpr int S0 = decltype(par)::value, S1 = S0 ^ 1;
    if (i + 1 < total) stage(i + 1, S1);
    const int s = KS * i + ks;
    const bool sink_step = s < sink_steps;
    const int32_t j0 = sink_step ? start0 + KB * s : win_lo + KB * (s - sink_steps);
    const uint32_t wlen = sink_step || !valid ? 0u : (uint32_t)(gq - wlo + 1);
    const uint32_t sl = !valid ? 0u : (uint32_t)(sink_step ? min(slen, max(sink_hi - doc.start, 0)) : slen);
    const int32_t rw = j0 - wlo, rs = j0 - doc.start;
    const bool all = !valid || (rw >= 0 && rw + KB <= (int32_t)wlen);
    const bool masked = __builtin_amdgcn_ballot_w64(!all) != 0;
    const __bf16 *K = Ks(S0), *V = Vs(S0);
#pragma unroll
    for (int nb = 0; nb < KB / 32; ++nb) {
      const __bf16 *Kb = K + 32 * nb * D, *Vb = V + 32 * nb * D;
      f32x16 sc = f32x16{}, dp = minus_delta;
      bf16x8 fa[kAhead];
      auto read = [&](int i) __attribute__((always_inline)) {
        if (i < D / 8) fa[i % kAhead] = i < D / 16 ? rd.rows(Kb, i) : rd.rows(Vb, i - D / 16);
      };
#pragma unroll
      for (int i = 0; i < kAhead; ++i) read(i);
#pragma unroll
      for (int i = 0; i < D / 8; ++i) {
        if (i < D / 16) sc = mfma32(fa[i % kAhead], qf[i], sc);
        else dp = mfma32(fa[i % kAhead], df[i - D / 16], dp);
        read(i + kAhead);
        keep_order();
      }
      if (masked) {
        const int32_t rw0 = rw + 4 * hi, rs0 = rs + 4 * hi;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int c = 32 * nb + c_row(j, 0);
          if ((uint32_t)(rw0 + c) >= wlen && (uint32_t)(rs0 + c) >= sl) sc[j] = NEG_INF;
        }
      }
      bf16x8 ft[kAhead], ds[2];
      auto read_turned = [&](int i) __attribute__((always_inline)) {
        if (i < D / 16) ft[i % kAhead] = rd.turned(Kb + 16 * (i / (D / 32)) * D, i % (D / 32));
      };
#pragma unroll
      for (int i = 0; i < kAhead; ++i) read_turned(i);
      keep_order();
#pragma unroll
      for (int j = 0; j < 16; ++j) ds[j >> 3][j & 7] = (__bf16)(fast_exp2(__builtin_fmaf(sc[j], a.scale_log2, -lse2)) * dp[j]);
#pragma unroll
      for (int i = 0; i < D / 16; ++i) {
        dq[i % (D / 32)] = mfma32(ft[i % kAhead], ds[i / (D / 32)], dq[i % (D / 32)]);
        read_turned(i + kAhead);
        keep_order();
      }
    }
    vm_wait_barrier<0>();
  };
  // every stream takes part in the barriers of the longest one (the first)
  const int most = KS == 1 ? total : (steps + KS - 1) / KS;
  for (int s = 0; s < most; s += 2) {
    if (KS == 1 || s < total) step(s, std::integral_constant<int, 0>{});
    else vm_wait_barrier<0>();
    if (s + 1 < most) {
      if (KS == 1 || s + 1 < total) step(s + 1, std::integral_constant<int, 1>{});
      else vm_wait_barrier<0>();
    }
  }
  if constexpr (KS > 1) join_streams<D / 32, WAVES, KS>(dq, (float*)rings, w, ks, lane);
  if (KS > 1 && ks > 0) return;

  if (!valid) return;
  __bf16* op = a.dq + (qrow * a.hq + h) * D + 4 * hi;
#pragma unroll
  for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
    for (int grp = 0; grp < 4; ++grp)
      *(bf16x4*)(op + 32 * mb + 8 * grp) =
          bf16x4{(__bf16)(dq[mb][4 * grp] * a.scale), (__bf16)(dq[mb][4 * grp + 1] * a.scale),
                 (__bf16)(dq[mb][4 * grp + 2] * a.scale), (__bf16)(dq[mb][4 * grp + 3] * a.scale)};
}

// ---------------------------------------------------------------------------
// dK, dV.  Wave w holds 32 keys (K and V rows in registers as the products' B operand, key = column), the workgroup
// walks the queries in steps of 64 rows (32 at head_dim 128 or with four streams) staged in LDS, head by head.  Per 32
// queries: S and dP (rows = queries), then dV^T += dO^T P and dK^T += Q^T dS with P and dS straight from registers and dO^T, Q^T by LDS transpose reads.
//
// Queries of key j in segment [a0, b0): j .. j + len - 1, where len ends with the window or the document -- a sink's
// with its chunk or the window, whichever is later (pairs of a sink with queries behind both are the sink pass's).
//
// SINKS: the keys are the sinks, up to the chunk's first position, of the document that holds that position and began
// before it; the queries those of the chunk outside the window.
// ---------------------------------------------------------------------------
template <int D, bool SINKS, int WAVES, int KS>
__global__ __launch_bounds__(64 * WAVES * KS, KS * D > 128 && D == 128 ? 1 : 2) void window_dkv_kernel(WindowBwdArgs a) {
  constexpr int BN = 32 * WAVES, CPR = D / 8;
  constexpr bool VLDS = D == 128;       // V in LDS: its fragments, K's and the two sums do not fit the registers together
  constexpr int QB = VLDS || WAVES == 1 ? 32 : 64, TILE = QB * D;
  constexpr float NEG_INF = -__builtin_inff();
  static_assert(KS == 1 || KS * 4 * TILE * 2 >= (KS - 1) * WAVES * (D / 2) * 256, "room for the streams' results");
  __shared__ __attribute__((aligned(16))) __bf16 vtile[VLDS ? BN * D : 8];
  __shared__ __attribute__((aligned(16))) __bf16 rings[KS * 4 * TILE];  // per stream: Q slots 0, 1, then dO slots 0, 1
  __shared__ __attribute__((aligned(16))) float rows_all[KS][2][2][QB];   // [slot][LSE in log2 units, -delta]
  __shared__ int32_t last_s[WAVES][2];
  __shared__ int32_t key_s[SINKS ? 1 : WAVES][4][32];  // what the end needs of the keys: row (-1: none), position, document

  const int tid = threadIdx.x;
  const int lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
  const int w = uniform(tid >> 6) % WAVES, ks = uniform(tid >> 6) / WAVES;  // 32 keys, stream of query steps
  const int sid = tid - 64 * WAVES * ks;                                    // thread of the stream
  __bf16* const ring = rings + ks * 4 * TILE;
  auto& rows_s = rows_all[ks];
  const int grp = a.hq / a.hkv;
  const int g = blockIdx.x % a.hkv;
  const int32_t rest = blockIdx.x / a.hkv;
  const int hs = SINKS ? 0 : rest % a.head_split;
  const int32_t tile = SINKS ? rest : rest / a.head_split;
  const int h0 = SINKS ? 0 : hs * grp / a.head_split, h1 = SINKS ? grp : (hs + 1) * grp / a.head_split;  // heads of the group
  const int64_t n = a.geom.n;
  const int32_t m = (int32_t)a.geom.m;
  const int32_t per_seq = segments_per_sequence(a.geom);

  // this lane's key: position, row, and its queries [qlo, qlo + len[x]) in the shard's segment x of the sequence
  int32_t key, qlo, first_seg;
  int64_t krow;
  bool key_ok;
  int32_t len[2] = {0, 0}, seg_lo[2] = {0, 0}, seg_hi[2] = {0, 0};
  DocSpan doc;
  int32_t t_doc = 0;  // SINKS: the document's start
  if constexpr (SINKS) {
    first_seg = tile / a.chunks;
    const int32_t a0 = uniform(segment_start(a.geom, a.shard, first_seg));
    const int32_t c0 = a0 + (tile - first_seg * a.chunks) * a.chunk;
    doc = doc_span(a.cu, a.num_docs, c0, lane);
    if (c0 >= a.cu[a.num_docs]) return;
    t_doc = uniform(doc.start);
    const int32_t doc_end = uniform(doc.end);
    const int32_t count = min(a.sinks, c0 - t_doc);
    if (count <= 0) return;  // the document begins here: its sinks' far queries are other chunks'
    key_ok = 32 * w + l32 < count;
    key = t_doc + min(32 * w + l32, count - 1);
    krow = key + key_span(a.geom, key).delta;
    seg_lo[0] = c0;
    seg_hi[0] = min(min(c0 + a.chunk, a0 + m), doc_end);
    qlo = max(c0, (int32_t)min((int64_t)key + a.window, (int64_t)INT32_MAX));
    len[0] = key_ok ? max(seg_hi[0] - qlo, 0) : 0;
  } else {
    // tile of 128 rows within a run of consecutive positions of the sharded order
    const int32_t run = tile / a.tiles, at = (tile - run * a.tiles) * BN;
    const int32_t runs = (int32_t)(n / m);  // per chunk
    const int32_t chunk = run / runs, rseg = run - chunk * runs;
    const int32_t r0 = uniform(segment_start(a.geom, chunk, rseg));
    const int32_t j0 = r0 + at;
    key = min(j0 + 32 * w + l32, r0 + m - 1);
    doc = doc_span(a.cu, a.num_docs, key, lane);
    const int32_t jl = min(min(j0 + BN - 1, r0 + m - 1), a.cu[a.num_docs] - 1);
    if (jl < j0) return;
    key_ok = j0 + 32 * w + l32 <= jl;
    krow = (int64_t)chunk * n + (int64_t)rseg * m + (min(key, jl) - r0);
    qlo = key;
    const int32_t b = rseg / per_seq;  // sequence of the batch
    first_seg = b * per_seq;
    const int32_t near = (int32_t)min((int64_t)doc.end, (int64_t)key + a.window);  // end of the queries whose window holds it
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      if (x >= per_seq) break;
      const int32_t a0 = uniform(segment_start(a.geom, a.shard, first_seg + x)), b0 = a0 + m;
      int32_t end = near;
      if (key - doc.start < a.sinks && key >= a0 && key < b0)
        end = max(end, a.chunks ? min(doc.end, a0 + ((key - a0) / a.chunk + 1) * a.chunk) : doc.end);
      len[x] = key_ok ? max(min(end, b0) - key, 0) : 0;
      seg_lo[x] = max(a0, j0);
      seg_hi[x] = b0;
    }
  }
  // the workgroup's queries per segment: from the first that any key has to the last
  if constexpr (!SINKS) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      int32_t e = key_ok ? key + len[x] : 0;
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) e = max(e, __shfl_xor(e, o));
      if (lane == 0 && ks == 0) last_s[w][x] = e;
    }
    if (hi == 0 && ks == 0) {  // (kept here: the loop has no registers to spare)
      key_s[w][0][l32] = key_ok ? (int32_t)krow : -1;
      key_s[w][1][l32] = key;
      key_s[w][2][l32] = doc.start;
      key_s[w][3][l32] = doc.end;
    }
    __syncthreads();
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      int32_t e = last_s[0][x];
      for (int y = 1; y < WAVES; ++y) e = max(e, last_s[y][x]);
      seg_hi[x] = min(seg_hi[x], uniform(e));
    }
  } else {
    seg_lo[0] = max(seg_lo[0], (int32_t)min((int64_t)t_doc + a.window, (int64_t)INT32_MAX));
  }
  const int32_t cnt0 = max(0, (seg_hi[0] - seg_lo[0] + QB - 1) / QB);
  const int32_t cnt1 = SINKS ? 0 : max(0, (seg_hi[1] - seg_lo[1] + QB - 1) / QB);
  const int32_t steps = (cnt0 + cnt1) * (h1 - h0);
  const int32_t total = KS == 1 ? steps : (steps - ks + KS - 1) / KS;  // this stream's: ks, ks + KS, ...

  f32x16 dk[D / 32], dv[D / 32];
#pragma unroll
  for (int mb = 0; mb < D / 32; ++mb) dk[mb] = dv[mb] = f32x16{};

  if (steps > 0) {
    bf16x8 kf[D / 16], vf[VLDS ? 1 : D / 16];
    {
      const int64_t at = (krow * a.hkv + g) * D + 8 * hi;
      // (the row of a key that no query of the shard sees may hold anything)
      const bool seen = (len[0] > 0 && qlo + len[0] > seg_lo[0]) || (len[1] > 0 && qlo + len[1] > seg_lo[1]);
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        kf[kk] = seen ? *(const bf16x8*)(a.k + at + 16 * kk) : bf16x8{};
        const bf16x8 x = seen ? *(const bf16x8*)(a.v + at + 16 * kk) : bf16x8{};
        if constexpr (VLDS) *(bf16x8*)(vtile + 32 * w * D + swz<CPR>(l32, 16 * kk + 8 * hi)) = x;  // (the streams' are the same)
        else vf[kk] = x;
      }
    }
    const int64_t rstride = (int64_t)a.hq * D;
    TileStage<D, WAVES, QB> st;
    st.init(w, lane, rstride * 2);
    // step i: segment x, head hh of the group, 64 queries from position pos; segment by segment, head by head
    struct Step {
      int32_t x, hh, s;
    };
    auto advance = [&](Step& p, int by) {
      for (int y = 0; y < by; ++y) {
        if (++p.s < (p.x ? cnt1 : cnt0)) continue;
        p.s = 0;
        if (++p.hh < h1) continue;
        p.hh = h0;
        ++p.x;
      }
    };
    float row_next = 0.f;  // the next step's LSE (the stream's threads 0 .. QB - 1) or delta (the next QB) of a row
    auto stage = [&](const Step& p, int slot) {
      const int32_t lo = p.x ? seg_lo[1] : seg_lo[0], top = p.x ? seg_hi[1] : seg_hi[0];
      const int32_t pos = lo + QB * p.s;
      const int32_t a0 = segment_start(a.geom, a.shard, first_seg + p.x);
      const int64_t r0 = (int64_t)(first_seg + p.x) * m + (pos - a0);  // local row of the step's first query
      const int h = g * grp + p.hh;
      const __bf16* qb = a.q + (r0 * a.hq + h) * D;
      const __bf16* ob = a.d_o + (r0 * a.hq + h) * D;
      const int32_t most = top - 1 - pos;  // rows behind the last query repeat it (masked)
      if (most >= QB - 1) {
        st.rows(qb, ring + slot * TILE);
        st.rows(ob, ring + (2 + slot) * TILE);
      } else {
        st.gather([&](int r) { return qb + min(r, most) * rstride; }, ring + slot * TILE);
        st.gather([&](int r) { return ob + min(r, most) * rstride; }, ring + (2 + slot) * TILE);
      }
      if (sid < 2 * QB) row_next = (sid < QB ? a.lse : a.delta)[(int64_t)h * n + r0 + min(sid % QB, most)];
    };
    auto store_rows = [&](int slot) {
      if (sid < 2 * QB) rows_s[slot][sid / QB][sid % QB] = sid < QB ? row_next * kLog2e : -row_next;
    };
    TileReads<D> rd;
    rd.init(lane);

    Step cur{cnt0 > 0 ? 0 : 1, h0, 0};
    if (KS == 1 || total > 0) {
      advance(cur, ks);
      stage(cur, 0);
      store_rows(0);
    }
    // (as in the dQ kernel: no wait for these rows inside the loop)
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) {
      asm volatile("" ::"v"(kf[kk]));
      if constexpr (!VLDS) asm volatile("" ::"v"(vf[kk]));
    }
    vm_wait_barrier<0>();
    Step nxt = cur;
    if (total > 1) advance(nxt, KS);
    auto step = [&](int i, auto par) __attribute__((always_inline)) {
      constexpr int S0 = decltype(par)::value, S1 = S0 ^ 1;
      if (i + 1 < total) stage(nxt, S1);
      const __bf16 *Q = ring + S0 * TILE, *O = ring + (2 + S0) * TILE;
      const int32_t pos = (cur.x ? seg_lo[1] : seg_lo[0]) + QB * cur.s;
      const uint32_t ln = (uint32_t)(cur.x ? len[1] : len[0]);
#pragma unroll
      for (int nb = 0; nb < QB / 32; ++nb) {
        const int32_t r = pos + 32 * nb - qlo;  // first query of the block relative to the key's first
        const bool some = r < (int32_t)ln && r + 31 >= 0;
        const bool all = !key_ok || (r >= 0 && r + 32 <= (int32_t)ln);
        if (__builtin_amdgcn_ballot_w64(some) == 0) continue;
        rd.fresh();
        // S and dP: 2 D / 16 products, each operand read kAhead products before its use
        const __bf16 *Qb = Q + 32 * nb * D, *Ob = O + 32 * nb * D;
        f32x16 sc = f32x16{}, dp;
#pragma unroll
        for (int j = 0; j < 16; ++j) dp[j] = rows_s[S0][1][32 * nb + c_row(j, hi)];
        bf16x8 fa[kAhead], fv[kAhead];
        auto read = [&](int i) __attribute__((always_inline)) {
          if (i >= D / 8) return;
          fa[i % kAhead] = i < D / 16 ? rd.rows(Qb, i) : rd.rows(Ob, i - D / 16);
          if (VLDS && i >= D / 16) fv[i % kAhead] = rd.rows(vtile + 32 * w * D, i - D / 16);
        };
#pragma unroll
        for (int i = 0; i < kAhead; ++i) read(i);
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          if (i < D / 16) sc = mfma32(fa[i % kAhead], kf[i], sc);
          else dp = mfma32(fa[i % kAhead], VLDS ? fv[i % kAhead] : vf[VLDS ? 0 : i - D / 16], dp);
          read(i + kAhead);
          keep_order();
        }
        if (__builtin_amdgcn_ballot_w64(!all) != 0) {
          const int32_t r4 = r + 4 * hi;
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if ((uint32_t)(r4 + c_row(j, 0)) >= ln) sc[j] = NEG_INF;
        }
        // the sums' operands: per sixteen queries and 32 columns dO^T (for dV), then Q^T (for dK)
        bf16x8 ft[kAhead], pb[2], ds[2];
        auto read_turned = [&](int i) __attribute__((always_inline)) {
          if (i < D / 8) ft[i % kAhead] = rd.turned((i & 1 ? Qb : Ob) + 16 * (i / (D / 16)) * D, i / 2 % (D / 32));
        };
        float lse2[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) lse2[j] = rows_s[S0][0][32 * nb + c_row(j, hi)];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) read_turned(i);
        keep_order();
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const float p = fast_exp2(__builtin_fmaf(sc[j], a.scale_log2, -lse2[j]));
          pb[j >> 3][j & 7] = (__bf16)p;
          ds[j >> 3][j & 7] = (__bf16)(p * dp[j]);
        }
#pragma unroll
        for (int i = 0; i < D / 8; ++i) {
          const int half = i / (D / 16), mb = i / 2 % (D / 32);
          if (i & 1) dk[mb] = mfma32(ft[i % kAhead], ds[half], dk[mb]);
          else dv[mb] = mfma32(ft[i % kAhead], pb[half], dv[mb]);
          read_turned(i + kAhead);
          keep_order();
        }
      }
      if (i + 1 < total) store_rows(S1);
      vm_wait_barrier<0>();
      cur = nxt;
      if (i + 2 < total) advance(nxt, KS);
    };
    // every stream takes part in the barriers of the longest one (the first)
    const int most = KS == 1 ? total : (steps + KS - 1) / KS;
    for (int i = 0; i < most; i += 2) {
      if (KS == 1 || i < total) step(i, std::integral_constant<int, 0>{});
      else vm_wait_barrier<0>();
      if (i + 1 < most) {
        if (KS == 1 || i + 1 < total) step(i + 1, std::integral_constant<int, 1>{});
        else vm_wait_barrier<0>();
      }
    }
    if constexpr (KS > 1) {
      join_streams<D / 32, WAVES, KS>(dk, (float*)rings, w, ks, lane);
      hsap_lds_barrier();
      join_streams<D / 32, WAVES, KS>(dv, (float*)rings, w, ks, lane);
    }
  }
  if (KS > 1 && ks > 0) return;

  if constexpr (SINKS) {
    // every sink of the document; those at or behind the chunk's first position are zeros
    const int32_t s = 32 * w + l32;
    if (s >= a.sinks) return;
    float* out = a.partial + (((int64_t)tile * a.hkv + g) * a.sinks + s) * (2 * D) + 4 * hi;
#pragma unroll
    for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        f32x4 x{dk[mb][4 * q], dk[mb][4 * q + 1], dk[mb][4 * q + 2], dk[mb][4 * q + 3]};
        f32x4 y{dv[mb][4 * q], dv[mb][4 * q + 1], dv[mb][4 * q + 2], dv[mb][4 * q + 3]};
        if (!key_ok) x = y = f32x4{};  // (a lane without a key repeats the last one's, unmasked)
        *(f32x4*)(out + 32 * mb + 8 * q) = x;
        *(f32x4*)(out + D + 32 * mb + 8 * q) = y;
      }
  } else {
    const int32_t row = key_s[w][0][l32], start = key_s[w][2][l32], doc_end = key_s[w][3][l32];
    if (row < 0) return;
    const int32_t s = key_s[w][1][l32] - start;
    if (s < a.sinks && a.chunks && hs == 0) {
      // the partials of the document's chunks, or their sum, in each of the shard's segments
      for (int x = 0; x < per_seq; ++x) {
        const int32_t a0 = segment_start(a.geom, a.shard, first_seg + x);
        const int32_t first = start < a0 ? 0 : (start - a0) / a.chunk + 1;  // first chunk that begins inside it
        const int32_t end = (int32_t)((min((int64_t)doc_end, (int64_t)a0 + m) - a0 + a.chunk - 1) / a.chunk);
        for (int32_t c = first; c < (a.summed ? min(end, first + 1) : end); ++c) {
          const float* in = a.partial + ((((int64_t)(first_seg + x) * a.chunks + c) * a.hkv + g) * a.sinks + s) * (2 * D) + 4 * hi;
#pragma unroll
          for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const f32x4 y = *(const f32x4*)(in + 32 * mb + 8 * q), z = *(const f32x4*)(in + D + 32 * mb + 8 * q);
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                dk[mb][4 * q + e] += y[e];
                dv[mb][4 * q + e] += z[e];
              }
            }
        }
      }
    }
    if (a.head_split > 1) {
      float* out = a.heads_part + (((int64_t)hs * a.geom.P * n + row) * a.hkv + g) * (2 * D) + 4 * hi;
#pragma unroll
      for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          *(f32x4*)(out + 32 * mb + 8 * q) = f32x4{dk[mb][4 * q], dk[mb][4 * q + 1], dk[mb][4 * q + 2], dk[mb][4 * q + 3]};
          *(f32x4*)(out + D + 32 * mb + 8 * q) = f32x4{dv[mb][4 * q], dv[mb][4 * q + 1], dv[mb][4 * q + 2], dv[mb][4 * q + 3]};
        }
      return;
    }
    const int64_t at = ((int64_t)row * a.hkv + g) * D + 4 * hi;
#pragma unroll
    for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const f32x4 x{dk[mb][4 * q] * a.scale, dk[mb][4 * q + 1] * a.scale, dk[mb][4 * q + 2] * a.scale, dk[mb][4 * q + 3] * a.scale};
        const f32x4 y{dv[mb][4 * q], dv[mb][4 * q + 1], dv[mb][4 * q + 2], dv[mb][4 * q + 3]};
        const int64_t e = at + 32 * mb + 8 * q;
        if (a.dkv_f32) {
          *(f32x4*)((float*)a.dk + e) = x;
          *(f32x4*)((float*)a.dv + e) = y;
        } else {
          *(bf16x4*)((__bf16*)a.dk + e) = bf16x4{(__bf16)x[0], (__bf16)x[1], (__bf16)x[2], (__bf16)x[3]};
          *(bf16x4*)((__bf16*)a.dv + e) = bf16x4{(__bf16)y[0], (__bf16)y[1], (__bf16)y[2], (__bf16)y[3]};
        }
      }
  }
}

// Sum of the sink partials of one document over a segment's chunks, in order, into the first one's: one workgroup per
// (chunk, K/V head), idle unless its chunk is a document's first.
__global__ __launch_bounds__(256) void window_sink_sum_kernel(WindowBwdArgs a, int elems) {
  const int lane = threadIdx.x & 63;
  const int g = blockIdx.x % a.hkv;
  const int32_t tile = blockIdx.x / a.hkv;
  const int32_t seg = tile / a.chunks, c = tile - seg * a.chunks;
  const int32_t a0 = segment_start(a.geom, a.shard, seg);
  const int64_t c0 = (int64_t)a0 + (int64_t)c * a.chunk;
  if (c0 >= a.cu[a.num_docs]) return;
  const DocSpan doc = doc_span(a.cu, a.num_docs, (int32_t)c0, lane);
  if (doc.start >= c0 || (c > 0 && doc.start < c0 - a.chunk)) return;
  const int64_t end = min((int64_t)doc.end, a0 + a.geom.m);
  const int32_t more = (int32_t)((end - 1 - c0) / a.chunk);  // chunks of the document behind this one
  if (more == 0) return;
  const int64_t step = (int64_t)a.hkv * elems;
  float* p = a.partial + ((int64_t)tile * a.hkv + g) * elems;
  for (int e = 4 * threadIdx.x; e < elems; e += 4 * 256) {
    f32x4 sum = *(const f32x4*)(p + e);
    int x = 1;
    for (; x + 7 <= more; x += 8) {  // eight loads in flight
      f32x4 part[8];
#pragma unroll
      for (int y = 0; y < 8; ++y) part[y] = *(const f32x4*)(p + (x + y) * step + e);
#pragma unroll
      for (int y = 0; y < 8; ++y) sum += part[y];
    }
    for (; x <= more; ++x) sum += *(const f32x4*)(p + x * step + e);
    *(f32x4*)(p + e) = sum;
  }
}

// dK and dV as the sum of the head splits' fp32 parts, in order: a thread per four values of each.
__global__ __launch_bounds__(256) void window_heads_sum_kernel(WindowBwdArgs a, int d) {
  const int64_t item = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t rows = (int64_t)a.geom.P * a.geom.n, per_row = (int64_t)a.hkv * (d / 4);
  const int64_t row = item / per_row;
  if (row >= rows) return;
  const int32_t at = (int32_t)(item - row * per_row), g = at / (d / 4), e = 4 * (at - g * (d / 4));
  const int32_t chunk = (int32_t)(row / a.geom.n);
  if (global_pos(a.geom, chunk, row - (int64_t)chunk * a.geom.n) >= a.cu[a.num_docs]) return;  // padding
  const float* p = a.heads_part + (row * a.hkv + g) * (2 * d) + e;
  const int64_t step = rows * a.hkv * (2 * d);
  f32x4 dk = *(const f32x4*)p, dv = *(const f32x4*)(p + d);
  for (int x = 1; x < a.head_split; ++x) {
    dk += *(const f32x4*)(p + x * step);
    dv += *(const f32x4*)(p + x * step + d);
  }
  dk *= a.scale;
  const int64_t out = (row * a.hkv + g) * d + e;
  if (a.dkv_f32) {
    *(f32x4*)((float*)a.dk + out) = dk;
    *(f32x4*)((float*)a.dv + out) = dv;
  } else {
    *(bf16x4*)((__bf16*)a.dk + out) = bf16x4{(__bf16)dk[0], (__bf16)dk[1], (__bf16)dk[2], (__bf16)dk[3]};
    *(bf16x4*)((__bf16*)a.dv + out) = bf16x4{(__bf16)dv[0], (__bf16)dv[1], (__bf16)dv[2], (__bf16)dv[3]};
  }
}

static hsap_status check_launch_window(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) HSAP_FAIL(HSAP_ERR_HIP, "%s launch: %s", what, hipGetErrorString(e));
  return HSAP_OK;
}

static int64_t delta_bytes(const hsap_attn_desc* d, const Geom& g) { return (4 * g.n * d->heads_q + 255) / 256 * 256; }

static int64_t heads_bytes(const hsap_attn_desc* d, const Geom& g, int32_t window) {
  const int64_t split = head_split(d, g, window);
  return split > 1 ? split * g.P * g.n * d->heads_kv * 2 * d->head_dim * 4 : 0;
}

static int64_t bwd_workspace(const hsap_attn_desc* d, const Geom& g, int32_t window, int32_t sinks) {
  return delta_bytes(d, g) + heads_bytes(d, g, window) +
         g.n / g.m * sink_chunks(d, g, window, sinks) * d->heads_kv * sinks * 2 * d->head_dim * 4;
}

template <int D, int WAVES, int KS>
static hsap_status launch_dq(WindowBwdArgs& a, hipStream_t s) {
  a.tiles = (int32_t)((a.geom.m + 32 * WAVES - 1) / (32 * WAVES));
  const int64_t blocks = a.geom.n / a.geom.m * a.tiles * a.hq;
  if (blocks > INT32_MAX) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "too many rows x heads");
  hipLaunchKernelGGL((window_dq_kernel<D, WAVES, KS>), dim3((unsigned)blocks), dim3(64 * WAVES * KS), 0, s, a);
  return check_launch_window("window_attn_bwd dQ");
}

template <int D, bool SINKS, int WAVES, int KS>
static hsap_status launch_dkv(WindowBwdArgs& a, hipStream_t s) {
  const int64_t segs = a.geom.n / a.geom.m;
  a.tiles = (int32_t)((a.geom.m + 32 * WAVES - 1) / (32 * WAVES));
  const int64_t blocks = (SINKS ? segs * a.chunks : segs * a.geom.P * a.tiles * a.head_split) * a.hkv;
  if (blocks > INT32_MAX) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "too many rows x heads");
  hipLaunchKernelGGL((window_dkv_kernel<D, SINKS, WAVES, KS>), dim3((unsigned)blocks), dim3(64 * WAVES * KS), 0, s, a);
  return check_launch_window(SINKS ? "window_attn_bwd sinks" : "window_attn_bwd dK/dV");
}

template <int D>
static hsap_status launch_window_bwd(WindowBwdArgs& a, hipStream_t s) {
  hsap_status st = window_query_blocks(a.geom, a.hq, D) == 2 ? launch_dq<D, 2, 2>(a, s) : launch_dq<D, 4, 1>(a, s);
  if (st != HSAP_OK) return st;
  if (a.chunks) {
    // as many key blocks as there are sinks; the other waves are streams over the queries
    st = a.sinks <= 32 ? launch_dkv<D, true, 1, 4>(a, s) : a.sinks <= 64 ? launch_dkv<D, true, 2, 2>(a, s) : launch_dkv<D, true, 4, 1>(a, s);
    if (st != HSAP_OK) return st;
    if (a.summed) {
      const int64_t blocks = a.geom.n / a.geom.m * a.chunks * a.hkv;
      hipLaunchKernelGGL(window_sink_sum_kernel, dim3((unsigned)blocks), dim3(256), 0, s, a, a.sinks * 2 * D);
      st = check_launch_window("window_attn_bwd sink sum");
      if (st != HSAP_OK) return st;
    }
  }
  switch (window_row_blocks(window_key_tiles(a.geom, a.hkv, a.window), D)) {
    case 1: st = launch_dkv<D, false, 1, 4>(a, s); break;
    case 2: st = launch_dkv<D, false, 2, 2>(a, s); break;
    default: return launch_dkv<D, false, 4, 1>(a, s);
  }
  if (st != HSAP_OK || a.head_split == 1) return st;
  const int64_t blocks = ((int64_t)a.geom.P * a.geom.n * a.hkv * (D / 4) + 255) / 256;
  hipLaunchKernelGGL(window_heads_sum_kernel, dim3((unsigned)blocks), dim3(256), 0, s, a, D);
  return check_launch_window("window_attn_bwd head sum");
}

}  // namespace hsap

using namespace hsap;

extern "C" int64_t hsap_window_attn_bwd_workspace(const hsap_attn_desc* desc, int32_t window, int32_t sinks) {
  clear_error();
  Geom g;
  static const int32_t none = 0;
  if (check_window(desc, window, sinks, &none, 1, &g) != HSAP_OK) return -1;
  const int32_t s = (int32_t)std::min<int64_t>(sinks, g.Ns);
  return bwd_workspace(desc, g, (int32_t)std::min<int64_t>(window, g.Ns), s);
}

extern "C" hsap_status hsap_window_attn_bwd(const hsap_attn_desc* desc, int32_t window, int32_t sinks, const void* q,
                                            const void* k, const void* v, const void* d_o, const void* o, const float* lse,
                                            const int32_t* cu_seqlens, int32_t num_docs, void* dq, void* dk, void* dv,
                                            int32_t dkv_f32, void* workspace, int64_t workspace_bytes, void* hip_stream) {
  clear_error();
  WindowBwdArgs a{};
  hsap_status st = check_window(desc, window, sinks, cu_seqlens, num_docs, &a.geom);
  if (st != HSAP_OK) return st;
  a.window = (int32_t)std::min<int64_t>(window, a.geom.Ns);
  a.sinks = (int32_t)std::min<int64_t>(sinks, a.geom.Ns);
  a.chunks = sink_chunks(desc, a.geom, a.window, a.sinks);
  a.chunk = sink_chunk(desc, a.geom);
  a.summed = a.chunks > kDirectChunks;
  if (a.chunks && a.sinks > kMaxBwdSinks)
    HSAP_FAIL(HSAP_ERR_UNSUPPORTED, "sinks %d above %d in the backward", sinks, kMaxBwdSinks);
  if (!q || !k || !v || !d_o || !o || !lse || !dq || !dk || !dv || !workspace)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "NULL pointer argument");
  if (((uintptr_t)q | (uintptr_t)k | (uintptr_t)v | (uintptr_t)d_o | (uintptr_t)o | (uintptr_t)workspace) & 15)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "q, k, v, d_o, o and workspace must be 16-byte aligned");
  if (((uintptr_t)dq & 7) || (((uintptr_t)dk | (uintptr_t)dv) & (dkv_f32 ? 15 : 7)))
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "dq, dk and dv must be 8-byte aligned (16-byte as fp32)");
  if (workspace_bytes < bwd_workspace(desc, a.geom, a.window, a.sinks))
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes,
              (long long)bwd_workspace(desc, a.geom, a.window, a.sinks));
  a.q = (const __bf16*)q;
  a.k = (const __bf16*)k;
  a.v = (const __bf16*)v;
  a.d_o = (const __bf16*)d_o;
  a.o = (const __bf16*)o;
  a.lse = lse;
  a.delta = (float*)workspace;
  a.head_split = head_split(desc, a.geom, a.window);
  a.heads_part = (float*)((char*)workspace + delta_bytes(desc, a.geom));
  a.partial = (float*)((char*)a.heads_part + heads_bytes(desc, a.geom, a.window));
  a.cu = cu_seqlens;
  a.dq = (__bf16*)dq;
  a.dk = dk;
  a.dv = dv;
  a.num_docs = num_docs;
  a.shard = desc->shard.shard_id;
  a.hq = desc->heads_q;
  a.hkv = desc->heads_kv;
  a.dkv_f32 = dkv_f32 != 0;
  a.scale = desc->softmax_scale;
  a.scale_log2 = desc->softmax_scale * kLog2e;
  return desc->head_dim == 128 ? launch_window_bwd<128>(a, (hipStream_t)hip_stream)
                               : launch_window_bwd<64>(a, (hipStream_t)hip_stream);
}
