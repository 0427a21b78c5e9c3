// Trees of drafted tokens: masks and positions from each one's parent, and the attention of many rows.
//
// A token's mask names itself and its ancestors among the drafted tokens of its sequence, its position is that of its
// depth: the drafted tokens stand behind `base` tokens, a token without a parent at position base.  A thread forms one word
// of a token's mask, and walks the token's whole chain of parents for it (their numbers fall, so every walk ends): of a sequence
// 256 words at a time, each as many dependent reads of LDS as its token is deep.  A launch for the trees of a batch (32 of 24 in
// one word 2.8 us, 32 chains of 64: 3.9), but the longer part of a step with long ones: eight of 300 tokens in five words, parents
// within eight 17 us, chains 60; of 1024 in sixteen words 430, chains 1800.
#include <algorithm>

#include "cache_attn.h"

namespace hsap {

__global__ __launch_bounds__(256) void tree_masks_kernel(const int32_t* seq_lens, const int32_t* cu, int64_t total, const int32_t* parents,
                                                         int32_t words, uint64_t* mask, int32_t* positions) {
  __shared__ int32_t parent[64 * kMaxMaskWords];
  const int32_t s = blockIdx.x, tid = threadIdx.x;
  const int32_t t0 = cu ? cu[s] : s;
  const int32_t count = cu ? (int32_t)min((int64_t)cu[s + 1], total) - t0 : 1;
  if (count <= 0) return;
  const int32_t base = (int32_t)max((int64_t)seq_lens[s] - count, (int64_t)INT32_MIN);
  const int32_t named = min(count, 64 * words);  // tokens that a mask has a bit for
  for (int32_t j = tid; j < named; j += 256) {
    const int32_t p = cu ? parents[t0 + j] : -1;
    parent[j] = p < j ? p : -1;
  }
  __syncthreads();
  for (int64_t i = tid; i < (int64_t)count * words; i += 256) {
    const int32_t j = (int32_t)(i / words), x = (int32_t)(i - (int64_t)j * words);
    uint64_t bits = 0;
    int32_t depth = 0;
    if (j < named) {
      for (int32_t at = j; at >= 0; at = parent[at]) {
        if (at >> 6 == x) bits |= uint64_t(1) << (at & 63);
        ++depth;
      }
    }
    mask[(int64_t)(t0 + j) * words + x] = bits;
    if (x == 0) positions[t0 + j] = j < named ? base + depth - 1 : -1;
  }
}

// Many rows of a sequence's tree against its tokens: every code is decoded once for the 32 RB rows of a workgroup.  A step's
// codes come to registers a step ahead and go as bf16 (which e4m3 fits exactly; V times its scale's power of two) into LDS;
// then every wave takes 32 rows and 32 tokens (two waves share a row's tokens where RB = 2): 32x32x16 products
// S^T = K Q^T, O^T += V^T P^T with V^T by transpose reads, Q from LDS too.  One copy of the tiles and few registers, so that
// three workgroups share a compute unit and decode, multiply and wait at different times.  P is rounded to bf16 for the second
// product (2^-8 relative at most, summed in fp32), O once at the end.  Steps before the drafted tokens and inside every row's
// window have no masks; the others (few) form a row's bits once.
//
// Bound by no one pipe.  8 sequences of up to 64 drafted tokens over up to 32768, 32 heads over 8 of 128: 150 us with the join,
// 521 TFLOP/s (an 8192^3 product 1248); of the cycles of compute units with work the matrix pipes take 0.29, the vector units 0.42
// (the issue of products among them), LDS 0.43, and waves wait for 0.35 of theirs, at a step's two barriers, for codes and for LDS.
// Tiles are not full either: a wave without rows only loads and decodes (82 % of the waves' steps multiply), 74 % of the rows that
// are multiplied are a sequence's, and a sequence of more than 128 has its tokens decoded twice (1.5 times on average).  32 of up
// to 24 over up to 4096: 83 us, 54 % of the waves' steps and 41 % of the rows; 5 of 100 through a window of 1024, head_dim 64: 16.
// (Three registers are spilled at head_dim 128; a variant without was no faster.)
// Order of N products with two LDS reads each: the reads of three are under way before the first.  (Left to itself the
// compiler, short of registers, waits for each product's reads.)
template <int N>
__device__ __forceinline__ void reads_ahead() {
  constexpr int READ = 0x100, PRODUCT = 0x8;
  __builtin_amdgcn_sched_group_barrier(READ, 6, 0);
#pragma unroll
  for (int i = 0; i < N - 3; ++i) {
    __builtin_amdgcn_sched_group_barrier(PRODUCT, 1, 0);
    __builtin_amdgcn_sched_group_barrier(READ, 2, 0);
  }
  __builtin_amdgcn_sched_group_barrier(PRODUCT, 3, 0);
}

template <int D, int RB>
__global__ __launch_bounds__(256, D == 64 ? 4 : 3) void cache_tree_kernel(CacheAttnArgs a) {
  constexpr int KB = RB == 4 ? 32 : 64;                          // tokens of a step: a block of 32 for every wave
  constexpr int CPR = D / 8, ROWS = 32 * RB, U = KB * D / 4096;  // U: runs of 16 codes per thread
  constexpr int SLOT = (2 + D / 2) * 64;                         // floats of a wave's results
  constexpr float NEG_INF = -__builtin_inff(), TINY = 1.17549435e-38f;
  constexpr float RESCALE_SLACK = 8.f;
  __shared__ __attribute__((aligned(16))) union {
    struct {
      __bf16 k[KB * D], v[KB * D], q[ROWS * D];
    };
    float join[2 * SLOT];
  } lds;
  __shared__ __attribute__((aligned(16))) float scales[2][4];        // [K's times the softmax's, V's rest][16 tokens]
  __shared__ uint32_t named[2 * kMaxMaskWords];                      // drafted tokens that some row of the tile names

  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = blockIdx.x % a.d.heads_kv;
  const int32_t rest = blockIdx.x / a.d.heads_kv;
  const int32_t split = rest % a.splits, tile = rest / a.splits;
  RowTile rt;
  if (!row_tile(a, tile, ROWS, rt)) return;
  const int32_t len = rt.len;
  const int32_t ps = a.d.page_size, cap = a.d.table_width * ps;
  const int32_t nrows = rt.count * a.group;
  const int32_t last_row = min(rt.row0 + ROWS, nrows) - 1;
  const int32_t base = len - rt.count;  // place of the sequence's first drafted token
  int32_t plo = INT32_MAX, phi = -1, least = INT32_MAX;  // positions of the tile's rows
#pragma unroll
  for (int r = 0; r < ROWS; r += 64) {
    const int32_t p = row_position(a, rt.t0 + min(rt.row0 + r + lane, last_row) / a.group);
    least = min(least, p);
    plo = min(plo, p < 0 ? INT32_MAX : p);
    phi = max(phi, p);
  }
  const bool plive = __builtin_amdgcn_ballot_w64(least < 0) == 0;  // all of them see something
  position_range<64>(plo, phi);
  plo = uniform(plo);
  phi = uniform(phi);
  const bool deep = drafts_end(a, rt, phi, lane);
  const Steps<KB> steps = tree_steps<KB>(plo, phi, base, len, cap, a.window, a.sinks);
  const int32_t per = steps_per_split(steps.total, a.splits);
  const int32_t s_begin = split * per, s_end = min(steps.total, s_begin + per);
  if (s_begin >= s_end && a.splits > 1) {  // nothing here for the join
    const int32_t r = rt.row0 + tid, t = r / a.group;
    if (tid < ROWS && r < nrows)
      a.part_lse[((int64_t)split * a.total_q + rt.t0 + t) * a.heads_q + g * a.group + (r - t * a.group)] = NEG_INF;
    return;
  }
  // the wave's rows, and its first block of a step's tokens
  const int rb = RB == 2 ? w & 1 : w, b0 = RB == 2 ? w >> 1 : 0;
  const bool busy = rt.row0 + 32 * rb <= last_row;
  const int32_t row = min(rt.row0 + 32 * rb + l32, last_row), tok = row / a.group;
  const int32_t pos = row_position(a, rt.t0 + tok);
  const int h = g * a.group + (row - tok * a.group);
#pragma unroll
  for (int i = 0; i < ROWS * CPR / 256; ++i) {
    const int at = tid + 256 * i, r = min(rt.row0 + at / CPR, last_row), t = r / a.group;
    *(bf16x8*)(lds.q + swz<CPR>(at / CPR, 8 * (at % CPR))) =
        *(const bf16x8*)(a.q + (int64_t)(rt.t0 + t) * a.q_stride + (int64_t)(g * a.group + (r - t * a.group)) * D + 8 * (at % CPR));
  }
  const int32_t* table = a.c.page_table + (int64_t)rt.seq * a.d.table_width;
  const int32_t top = min(len - 1, cap - 1);  // last token any row sees

  // Steps whose places are all some row's, and every row's: behind the sinks' and every window's beginning, before the drafts.
  const int64_t inside = max((int64_t)phi - a.window + 1, (int64_t)steps.win0) - steps.win0;
  const int32_t hot0 = steps.sinks + (int32_t)min((inside + KB - 1) / KB, (int64_t)steps.total);
  const int32_t hot1 = plive ? steps.sinks + max(base - steps.win0, 0) / KB : 0;

  // Thread's codes of a step: those of 16-token group group_of(u) (one page each), 16 codes of a token.  What is formed of a
  // page's number is formed on the vector units, which have its multiplication and addition in one, and which do not make
  // every wait for LDS one for memory, as scalar loads would.
  auto group_of = [&](int u) { return D == 64 ? w : (w >> 1) + 2 * u; };
  const int slot_in = D == 64 ? (lane >> 2) : 8 * (w & 1) + (lane >> 3);  // token within the group
  const int column = 16 * (D == 64 ? lane & 3 : lane & 7);
  int zero;
  asm volatile("v_mov_b32 %0, 0" : "=v"(zero));
  const uint32_t page_bytes = (uint32_t)a.d.heads_kv << a.page_shift;  // (times D)
  const int64_t first_row = ((int64_t)g << a.page_shift) + slot_in;
  const uint8_t* k_at = a.c.k_codes + first_row * D + column;
  const uint8_t* v_at = a.c.v_codes + first_row * D + column;
  struct Codes {
    uint4 k[U], v[U];
    float ks[U], vs[U];
    bool held[U];  // the group lies in a page
  };
  struct Where {
    int32_t page[U];
  };
  // (steps behind the last are its own again)
  auto look_up = [&](int32_t s) __attribute__((always_inline)) {
    Where x;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int32_t j = steps.first(min(s, s_end - 1)) + 16 * group_of(u);
      const bool any = steps.looked_up(a.sinks, j, top);
      x.page[u] = table[(any ? j >> a.page_shift : 0) + zero];
      if (!any) x.page[u] = -1;
    }
    return x;
  };
  auto load = [&](int32_t s, const Where& where, Codes& x) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int32_t j = steps.first(min(s, s_end - 1)) + 16 * group_of(u);
      x.held[u] = (uint32_t)where.page[u] < (uint32_t)a.d.num_pages;
      const uint32_t page = x.held[u] ? where.page[u] : 0;
      const uint64_t scale = (uint64_t)page * (uint32_t)a.d.heads_kv + g;
      x.ks[u] = a.c.k_scale[scale];
      x.vs[u] = a.c.v_scale[scale];
      const uint64_t at = ((uint64_t)page * page_bytes + (uint32_t)(j & (ps - 1))) * D;
      x.k[u] = *(const uint4*)(k_at + at);
      x.v[u] = *(const uint4*)(v_at + at);
    }
  };
  auto decode = [&](const uint4& c, float pow2, __bf16* out0, __bf16* out1) __attribute__((always_inline)) {
    bf16x2 p[8];
    decode4(c.x, pow2, p[0], p[1]);
    decode4(c.y, pow2, p[2], p[3]);
    decode4(c.z, pow2, p[4], p[5]);
    decode4(c.w, pow2, p[6], p[7]);
    *(bf16x8*)out0 = bf16x8{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
    *(bf16x8*)out1 = bf16x8{p[4][0], p[4][1], p[5][0], p[5][1], p[6][0], p[6][1], p[7][0], p[7][1]};
  };
  auto store = [&](int32_t s, Codes& x) __attribute__((always_inline)) {
    bool held = true;
#pragma unroll
    for (int u = 0; u < U; ++u) held &= x.held[u];
    float vpow[U];
#pragma unroll
    for (int u = 0; u < U; ++u) vpow[u] = __uint_as_float(__float_as_uint(x.vs[u]) & 0x7F800000u);
    if (__builtin_expect(s < hot0 || s >= hot1 || __builtin_amdgcn_ballot_w64(!held) != 0, 0)) {  // places that no row sees may hold anything
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int32_t j = steps.first(s) + 16 * group_of(u) + slot_in;
        bool unseen = (j > top) | !x.held[u] | ((j < steps.lo) & (j >= a.sinks));
        if (j >= base) unseen |= j - base >= 64 * a.words || !(named[(j - base) >> 5] >> ((j - base) & 31) & 1);
        if (unseen) {
          x.k[u] = x.v[u] = uint4{0, 0, 0, 0};
          vpow[u] = 1.f;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int token = 16 * group_of(u) + slot_in;
      const int at0 = swz<CPR>(token, column), at1 = swz<CPR>(token, column + 8);
      decode(x.k[u], 1.f, lds.k + at0, lds.k + at1);
      decode(x.v[u], vpow[u], lds.v + at0, lds.v + at1);
      // (a scale of 0 stands for no page; at least the smallest normal number, so that -inf times it stays -inf)
      if (lane == 0) {
        scales[0][group_of(u)] = x.held[u] ? fmaxf(x.ks[u] * a.scale_log2, TINY) : 0.f;
        scales[1][group_of(u)] = __uint_as_float((__float_as_uint(x.vs[u]) & 0x007FFFFFu) | 0x3F800000u);
      }
    }
  };

  TileReads<D> rd;
  rd.init(lane);
  float m_run = NEG_INF, l_run = 0.f;
  f32x16 o[D / 32];
#pragma unroll
  for (int mb = 0; mb < D / 32; ++mb) o[mb] = f32x16{};

  auto compute = [&](int32_t s) __attribute__((always_inline)) {
    float sl[2], vrest[2];
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      sl[q] = scales[0][2 * b0 + q];
      vrest[q] = scales[1][2 * b0 + q];
    }
    f32x16 sc{};
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) sc = mfma32(rd.rows(lds.k + 32 * b0 * D, kk), rd.rows(lds.q + 32 * rb * D, kk), sc);
    reads_ahead<D / 16>();
    if (__builtin_expect(s < hot0 || s >= hot1 || __builtin_amdgcn_ballot_w64(!(fminf(sl[0], sl[1]) > 0.f)) != 0, 0)) {
      const int32_t jb = steps.first(s) + 32 * b0;
      const uint32_t m = (uint32_t)seen_bits(a, rt, a.mask + (int64_t)(rt.t0 + tok) * a.words, pos, base, jb, top, deep, lane) &
                         ((sl[0] > 0.f ? 0xFFFFu : 0u) | (sl[1] > 0.f ? 0xFFFF0000u : 0u));
#pragma unroll
      for (int j = 0; j < 16; ++j) sc[j] = (m >> (4 * hi)) & (1u << c_row(j, 0)) ? sc[j] : NEG_INF;
#pragma unroll
      for (int q = 0; q < 2; ++q) sl[q] = fmaxf(sl[q], TINY);
    }
    float mx = NEG_INF;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      float x = sc[8 * q];
#pragma unroll
      for (int j = 1; j < 8; ++j) x = fmaxf(x, sc[8 * q + j]);
      mx = fmaxf(mx, x * sl[q]);
    }
    // (the two lanes of a row join their maxima only when some row's rose by more than the slack)
    if (__builtin_amdgcn_ballot_w64(mx > m_run + RESCALE_SLACK) != 0) {
      const float m_new = fmaxf(m_run, pair_max(mx));
      const float alpha = m_run == NEG_INF ? 0.f : fast_exp2(m_run - m_new);
      l_run *= alpha;
#pragma unroll
      for (int mb = 0; mb < D / 32; ++mb) o[mb] *= alpha;
      m_run = m_new;
    }
    const float m_use = m_run == NEG_INF ? 0.f : m_run;
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const float p = fast_exp2(__builtin_fmaf(sc[j], sl[j >> 3], -m_use));
      l_run += p;
      sc[j] = p;
    }
    if (__builtin_amdgcn_ballot_w64(vrest[0] != 1.f || vrest[1] != 1.f) != 0) {
#pragma unroll
      for (int j = 0; j < 16; ++j) sc[j] *= vrest[j >> 3];
    }
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      bf16x8 pb;
#pragma unroll
      for (int j = 0; j < 8; ++j) pb[j] = (__bf16)sc[8 * q + j];
#pragma unroll
      for (int mb = 0; mb < D / 32; ++mb) o[mb] = mfma32(rd.turned(lds.v + 16 * (2 * b0 + q) * D, mb), pb, o[mb]);
    }
    reads_ahead<D / 16>();
  };

  // (the first barrier comes before the first of them is read)
  for (int i = tid; i < 2 * a.words; i += 256) named[i] = 0;
  if (s_begin < s_end) {
    Codes x;
    load(s_begin, look_up(s_begin), x);
    Where next = look_up(s_begin + 1);
    __syncthreads();
    const int32_t first = rt.row0 / a.group, count = last_row / a.group - first + 1;
    for (int i = tid; i < count * a.words; i += 256) {
      const int32_t t = i / a.words, at = i - t * a.words;
      const uint64_t m = a.mask[(int64_t)(rt.t0 + first + t) * a.words + at];
      if ((uint32_t)m) atomicOr(&named[2 * at], (uint32_t)m);
      if (m >> 32) atomicOr(&named[2 * at + 1], (uint32_t)(m >> 32));
    }
    __syncthreads();
    for (int32_t s = s_begin; s < s_end; ++s) {
      store(s, x);
      const Where after = look_up(s + 2);
      load(s + 1, next, x);
      next = after;
      hsap_lds_barrier();
      if (busy) compute(s);
      hsap_lds_barrier();
    }
  }
  l_run = pair_sum(l_run);
  if constexpr (RB == 2) {  // the second block's wave hands its results to the first's
    float* join = lds.join + rb * SLOT + lane;
    __syncthreads();  // (without steps nobody has waited for Q's rows)
    if (b0 == 1) {
      join[0] = m_run;
      join[64] = l_run;
#pragma unroll
      for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
        for (int e = 0; e < 16; ++e) join[64 * (2 + 16 * mb + e)] = o[mb][e];
    }
    __syncthreads();
    if (b0 == 1) return;
    const float m2 = join[0], l2 = join[64], m = fmaxf(m_run, m2), m_use = m == NEG_INF ? 0.f : m;
    const float f1 = fast_exp2(m_run - m_use), f2 = fast_exp2(m2 - m_use);
    l_run = l_run * f1 + l2 * f2;
    m_run = m;
#pragma unroll
    for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[mb][e] = o[mb][e] * f1 + join[64 * (2 + 16 * mb + e)] * f2;
  }
  if (rt.row0 + 32 * rb + l32 > last_row) return;
  const float inv = l_run > 0.f ? 1.f / l_run : 0.f;
  const float lse2 = l_run > 0.f ? m_run + __log2f(l_run) : NEG_INF;
  const int64_t out = (int64_t)(rt.t0 + tok) * a.heads_q + h;
  if (a.splits == 1) {
    __bf16* op = a.o + out * D + 4 * hi;
#pragma unroll
    for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *(bf16x4*)(op + 32 * mb + 8 * q) = bf16x4{(__bf16)(o[mb][4 * q] * inv), (__bf16)(o[mb][4 * q + 1] * inv),
                                                  (__bf16)(o[mb][4 * q + 2] * inv), (__bf16)(o[mb][4 * q + 3] * inv)};
    if (hi == 0 && a.lse) a.lse[(int64_t)h * a.total_q + rt.t0 + tok] = lse2 * 0.69314718055994530942f;
  } else {
    const int64_t at = (int64_t)split * a.total_q * a.heads_q + out;
    float* op = a.part_o + at * D + 4 * hi;
#pragma unroll
    for (int mb = 0; mb < D / 32; ++mb)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *(f32x4*)(op + 32 * mb + 8 * q) = f32x4{o[mb][4 * q] * inv, o[mb][4 * q + 1] * inv, o[mb][4 * q + 2] * inv, o[mb][4 * q + 3] * inv};
    if (hi == 0) a.part_lse[at] = lse2;
  }
}

void launch_tree(const CacheAttnArgs& a, int64_t blocks, hipStream_t s) {
  const dim3 grid((unsigned)blocks), block(256);
  if (a.d.head_dim == 64) hipLaunchKernelGGL((cache_tree_kernel<64, 2>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((cache_tree_kernel<128, 4>), grid, block, 0, s, a);
}

}  // namespace hsap

using namespace hsap;

extern "C" hsap_status hsap_tree_masks(int32_t num_seqs, const int32_t* seq_lens, const int32_t* cu_new, int64_t total_new,
                                       const int32_t* parents, int32_t mask_words, uint64_t* mask, int32_t* positions,
                                       void* hip_stream) {
  clear_error();
  if (num_seqs < 0 || num_seqs > kMaxBlocks256) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "bad num_seqs %d", num_seqs);
  if (total_new < 0 || total_new > INT32_MAX) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "bad total_new %lld", (long long)total_new);
  if (!cu_new && total_new != num_seqs)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "without cu_new every sequence has one new token: total_new %lld, num_seqs %d",
              (long long)total_new, num_seqs);
  if (mask_words < 1 || mask_words > kMaxMaskWords) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "mask_words %d: 1 to %d", mask_words, kMaxMaskWords);
  if (total_new == 0 || num_seqs == 0) return HSAP_OK;
  if (!seq_lens || (cu_new && !parents) || !mask || !positions || ((uintptr_t)mask & 7))
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "NULL pointer argument, or mask not 8-byte aligned");
  hipLaunchKernelGGL(tree_masks_kernel, dim3((unsigned)num_seqs), dim3(256), 0, (hipStream_t)hip_stream, seq_lens, cu_new, total_new,
                     parents, mask_words, mask, positions);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) HSAP_FAIL(HSAP_ERR_HIP, "tree_masks launch: %s", hipGetErrorString(e));
  return HSAP_OK;
}
