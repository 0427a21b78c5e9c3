// Attention of the newest tokens over the paged 8-bit K/V cache.
//
//   s_j = scale ks(page of j) q . k8_j,   O = sum_j exp(s_j - LSE) vs(page of j) v8_j
//
// Few rows against many cached tokens: bound by reading the codes, 2 d bytes per token and K/V head.  So the query
// heads of a K/V head (and a sequence's several new tokens) share one pass: rows r = (token, head of the group) in
// tiles of 16 MT, one workgroup per (row tile, K/V head, split of the tile's tokens), a running maximum and sum per
// wave, the waves' results joined in LDS, the splits' by a second launch over fp32 partials.  64 sequences of up to 8192
// tokens, 32 heads over 8 of 128: 115 us for the codes (5.5 TB/s; a large sum reads at 6.0) and 4.5 for the join.  One of
// 131072 tokens, 16 heads over 2: 16 and 4 us, a chain of table, codes, eight or nine steps per wave and joins.
//
// A wave takes 32 tokens at a time (its workgroup's four waves take turns), with the next ones' codes in flight in
// registers: no LDS on the way.  S^T = K Q^T by 16x16x32 products, tokens as rows: lane l holds row l % 16 of K and
// of Q, sixteen of a token's values at a time (the order of d is the same for both, so any will do).  The result
// has query l % 16 on lane l and tokens 4 (l / 16) .. +3 of each 16, which is the layout of the B operand of
// O^T += V^T P^T if its eight tokens per lane are 4 (l / 16) + 0..3 of both halves; V's rows are loaded by those tokens
// and turned in registers, two codes of two tokens at a time (v_perm, then the conversion to bf16, which e4m3 fits
// exactly).  P is rounded to bf16 for the second product (2^-8 relative at most, summed in fp32), O once at the end.
#include <algorithm>

#include "cache_attn.h"

namespace hsap {

hsap_status check_cache_desc(const hsap_cache_desc* d, bool pages);
hsap_status check_cache(const hsap_cache_desc* d, const hsap_cache* c);

template <typename T, bool ONCE>
__device__ __forceinline__ T read_codes(const uint8_t* p) {
  typedef uint32_t words __attribute__((ext_vector_type(sizeof(T) / 4)));
  if constexpr (ONCE) return __builtin_bit_cast(T, __builtin_nontemporal_load((const words*)p));
  else return *(const T*)p;
}

// ONCE: every code is read by one workgroup of the call alone and the cache is larger than the 256 MB behind the L2s: the
// loads are marked as streaming (64 sequences of 8k tokens, 8 heads of 128: 128 -> 119 us; with several row tiles per
// sequence 46 -> 49 us, with 67 MB of codes, which the next call finds there again, 21.8 -> 22.5 us).
// TREE: drafted tokens by masks.  A step's places that no row of the tile sees are found by ballots over its rows.
template <int D, int MT, bool ONCE, bool TREE>
__global__ __launch_bounds__(256, 2) void cache_attn_kernel(CacheAttnArgs a) {
  constexpr int KX = D / 64, CB = D / 16, ROWS = 16 * MT;  // 16-byte loads per K row and lane; d values per lane of V
  constexpr float NEG_INF = -__builtin_inff();
  constexpr float RESCALE_SLACK = 8.f;
  using VT = typename std::conditional<D == 128, uint2, uint32_t>::type;  // a lane's CB codes of a V row
  constexpr int SLOT = MT * (CB * 4 + 2) * 64;                          // floats of one wave's results
  __shared__ float join[2 * SLOT];

  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, grp = lane >> 4;
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
  const int32_t pos0 = len - rt.count;  // position of the sequence's first new token
  int32_t plo = pos0 + rt.row0 / a.group, phi = pos0 + last_row / a.group;
  if constexpr (TREE) {
    plo = INT32_MAX;
    phi = -1;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const int32_t p = row_position(a, rt.t0 + min(rt.row0 + 16 * mt + l16, last_row) / a.group);
      plo = min(plo, p < 0 ? INT32_MAX : p);
      phi = max(phi, p);
    }
    position_range<16>(plo, phi);
    plo = uniform(plo);
    phi = uniform(phi);
  }
  const bool deep = TREE && drafts_end(a, rt, phi, lane);
  const Steps<32> steps = TREE ? tree_steps<32>(plo, phi, pos0, len, cap, a.window, a.sinks)
                               : cache_steps<32>(plo, phi, cap, a.window, a.sinks);
  const int32_t per = steps_per_split(steps.total, a.splits);
  const int32_t s_begin = split * per, s_end = min(steps.total, s_begin + per);
  if (s_begin >= s_end && a.splits > 1) {  // nothing here for the join
    const int32_t r = rt.row0 + tid, t = r / a.group;
    if (tid < ROWS && r < nrows)
      a.part_lse[((int64_t)split * a.total_q + rt.t0 + t) * a.heads_q + g * a.group + (r - t * a.group)] = NEG_INF;
    return;
  }

  // this lane's query of each 16-row block: row, position, Q fragments
  int32_t pos[MT];
  bf16x8 qf[MT][2 * KX];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int32_t r = min(rt.row0 + 16 * mt + l16, nrows - 1);
    const int32_t t = r / a.group;
    pos[mt] = TREE ? row_position(a, rt.t0 + t) : pos0 + t;
    const __bf16* qp = a.q + (int64_t)(rt.t0 + t) * a.q_stride + (int64_t)(g * a.group + (r - t * a.group)) * D + 16 * grp;
#pragma unroll
    for (int x = 0; x < KX; ++x) {
      qf[mt][2 * x] = *(const bf16x8*)(qp + 64 * x);
      qf[mt][2 * x + 1] = *(const bf16x8*)(qp + 64 * x + 8);
    }
  }
  const int32_t* table = a.c.page_table + (int64_t)rt.seq * a.d.table_width;
  const int32_t top = min(TREE ? len - 1 : phi, cap - 1);  // last token any row sees
  const bool live = !TREE || __builtin_amdgcn_ballot_w64(MT == 1 ? pos[0] < 0 : pos[0] < 0 || pos[MT - 1] < 0) == 0;

  struct Tokens {
    uint4 k[2][KX];
    VT v[8];
    float ks[2], vs[2];
    int32_t j0;
    bool held[2];  // each half of 16 tokens lies in a page
  };
  // Pages of a step's halves (-1: none), looked up a step before its codes are asked for, those a step before their use.
  struct Where {
    int32_t page[2];
  };
  auto look_up = [&](int32_t s) __attribute__((always_inline)) {
    Where x{{-1, -1}};
    if (s < s_end) {
      const int32_t j0 = steps.first(s);
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const int32_t at = (j0 + 16 * half) >> a.page_shift;
        if (steps.looked_up(a.sinks, j0 + 16 * half, top)) x.page[half] = table[at];  // (top is below the table's capacity)
      }
    }
    return x;
  };
  auto load = [&](int32_t s, const Where& where, Tokens& x) __attribute__((always_inline)) {
    x.j0 = steps.first(s);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int32_t j = x.j0 + 16 * half;
      x.held[half] = (uint32_t)where.page[half] < (uint32_t)a.d.num_pages;
      const int32_t page = x.held[half] ? where.page[half] : 0;
      const int64_t at = (int64_t)page * a.d.heads_kv + g;
      x.ks[half] = x.held[half] ? a.c.k_scale[at] : 0.f;
      x.vs[half] = x.held[half] ? a.c.v_scale[at] : 0.f;
      const int64_t row = (at << a.page_shift) + (j & (ps - 1));
      const uint8_t* kp = a.c.k_codes + (row + l16) * D + 16 * grp;
#pragma unroll
      for (int y = 0; y < KX; ++y) x.k[half][y] = read_codes<uint4, ONCE>(kp + 64 * y);
      const uint8_t* vp = a.c.v_codes + (row + 4 * grp) * D + CB * l16;
#pragma unroll
      for (int y = 0; y < 4; ++y) x.v[4 * half + y] = read_codes<VT, ONCE>(vp + y * D);
    }
  };

  float m_run[MT], l_run[MT];
  f32x4 o[MT][CB];
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    m_run[mt] = NEG_INF;
    l_run[mt] = 0.f;
#pragma unroll
    for (int c = 0; c < CB; ++c) o[mt][c] = f32x4{};
  }

  auto compute = [&](const Tokens& x, int32_t s) __attribute__((always_inline)) {
    // K operand: eight codes of a token per product
    bf16x8 kf[2][2 * KX];
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int y = 0; y < KX; ++y) {
        const uint32_t c[4] = {x.k[half][y].x, x.k[half][y].y, x.k[half][y].z, x.k[half][y].w};
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          bf16x2 p0, p1, p2, p3;
          decode4(c[2 * e], 1.f, p0, p1);
          decode4(c[2 * e + 1], 1.f, p2, p3);
          kf[half][2 * y + e] = bf16x8{p0[0], p0[1], p1[0], p1[1], p2[0], p2[1], p3[0], p3[1]};
        }
      }
    const int32_t jl = x.j0 + 31;
    const int32_t sinks = s < steps.sinks ? min(a.sinks, steps.win0) : a.sinks;
    const int32_t near = s < steps.sinks ? 0 : a.window;
    // every row of the tile sees every token of the step
    const bool all = x.held[0] && x.held[1] && (TREE ? live && jl < pos0 : jl <= plo) && (phi - x.j0 < near || jl < sinks);
    uint32_t sees[TREE ? MT : 1], some = 0;  // the step's tokens that the lane's rows see, that any row does
    if constexpr (TREE) {
      if (__builtin_expect(!all, 0)) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
          const int32_t t = min(rt.row0 + 16 * mt + l16, nrows - 1) / a.group;
          sees[mt] = (uint32_t)seen_bits(a, rt, a.mask + (int64_t)(rt.t0 + t) * a.words, pos[mt], pos0, x.j0, top, deep, lane);
          sees[mt] &= (x.held[0] ? 0xFFFFu : 0u) | (x.held[1] ? 0xFFFF0000u : 0u);
          some |= sees[mt];
        }
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) some |= __shfl_xor(some, o);
      }
    }
    // V's scale: its power of two goes into the conversion of the codes, what is left of it (1 for the scales that an
    // append makes) into P
    float vpow[2], vrest[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      vpow[half] = __uint_as_float(__float_as_uint(x.vs[half]) & 0x7F800000u);
      vrest[half] = __uint_as_float((__float_as_uint(x.vs[half]) & 0x007FFFFFu) | 0x3F800000u);
    }
    const bool rest = vrest[0] != 1.f || vrest[1] != 1.f;
    bf16x8 pf[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      f32x4 sc[2] = {f32x4{}, f32x4{}};
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int kk = 0; kk < 2 * KX; ++kk) sc[half] = mfma16(kf[half][kk], qf[mt][kk], sc[half]);
      const float sl[2] = {fmaxf(x.ks[0] * a.scale_log2, 1.17549435e-38f), fmaxf(x.ks[1] * a.scale_log2, 1.17549435e-38f)};
      if (TREE ? __builtin_expect(!all, 0) : !all) {
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int32_t j = x.j0 + 16 * half + 4 * grp + e;
            const bool see = TREE ? (sees[TREE ? mt : 0] >> (4 * grp)) & (1u << (16 * half + e))
                                  : j <= pos[mt] && (pos[mt] - j < near || j < sinks) && x.held[half];
            if (!see) sc[half][e] = NEG_INF;
          }
      }
      // (scales are positive; at least the smallest normal number, so that -inf stays -inf)
      float mx = fmaxf(fmaxf(fmaxf(sc[0][0], sc[0][1]), fmaxf(sc[0][2], sc[0][3])) * sl[0],
                       fmaxf(fmaxf(sc[1][0], sc[1][1]), fmaxf(sc[1][2], sc[1][3])) * sl[1]);
      // a row's tokens lie on four lanes; its maximum is joined only when some lane's rose by more than the slack
      if (__builtin_amdgcn_ballot_w64(mx > m_run[mt] + RESCALE_SLACK) != 0) {
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float m_new = fmaxf(m_run[mt], mx);
        const float alpha = m_run[mt] == NEG_INF ? 0.f : fast_exp2(m_run[mt] - m_new);
        l_run[mt] *= alpha;
#pragma unroll
        for (int c = 0; c < CB; ++c) o[mt][c] *= alpha;
        m_run[mt] = m_new;
      }
      const float m_use = m_run[mt] == NEG_INF ? 0.f : m_run[mt];
      float pr[8];
#pragma unroll
      for (int half = 0; half < 2; ++half)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p = fast_exp2(__builtin_fmaf(sc[half][e], sl[half], -m_use));
          l_run[mt] += p;
          pr[4 * half + e] = p;
        }
      if (rest) {
#pragma unroll
        for (int e = 0; e < 8; ++e) pr[e] *= vrest[e >> 2];
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) pf[mt][e] = (__bf16)pr[e];
    }
    // V operand: rows d = CB l16 + c, the lane's eight tokens
    VT v[8];
#pragma unroll
    for (int y = 0; y < 8; ++y) v[y] = x.v[y];
    if (TREE && __builtin_expect(!all, 0)) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (!((some >> (4 * grp)) & (1u << (16 * half + e)))) v[4 * half + e] = VT{};
        // (of sixteen tokens that no row sees the page's scale may be anything too)
        if (!(some & (0xFFFFu << (16 * half)))) vpow[half] = 1.f;
      }
    }
    if (!TREE && (jl > top || !x.held[0] || !x.held[1] || steps.edge(s))) {  // P is 0 there, V whatever the page holds
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        const int32_t j = x.j0 + 16 * (y >> 2) + 4 * grp + (y & 3);
        if (j > top || !x.held[y >> 2] || !steps.seen(a.sinks, j, j)) v[y] = VT{};
      }
    }
#pragma unroll
    for (int c4 = 0; c4 < CB / 4; ++c4) {
      bf16x2 turned[4][4];  // [column][token pair]
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        uint32_t u0, u1;
        if constexpr (D == 128) {
          u0 = c4 ? v[2 * y].y : v[2 * y].x;
          u1 = c4 ? v[2 * y + 1].y : v[2 * y + 1].x;
        } else {
          u0 = v[2 * y];
          u1 = v[2 * y + 1];
        }
        // bytes (u0.0, u1.0, u0.1, u1.1) and (u0.2, u1.2, u0.3, u1.3): v_perm selects 0..3 from its second operand
        const uint32_t lo = __builtin_amdgcn_perm(u1, u0, 0x05010400u), hi = __builtin_amdgcn_perm(u1, u0, 0x07030602u);
        decode4(lo, vpow[y >> 1], turned[0][y], turned[1][y]);
        decode4(hi, vpow[y >> 1], turned[2][y], turned[3][y]);
      }
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const bf16x8 vf{turned[c][0][0], turned[c][0][1], turned[c][1][0], turned[c][1][1],
                        turned[c][2][0], turned[c][2][1], turned[c][3][0], turned[c][3][1]};
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) o[mt][4 * c4 + c] = mfma16(vf, pf[mt], o[mt][4 * c4 + c]);
      }
    }
  };

  int32_t s = s_begin + w;
  if (s < s_end) {
    Tokens x, y;
    load(s, look_up(s), x);
    Where next = look_up(s + 4);
    for (;;) {
      const bool more = s + 4 < s_end;
      if (more) load(s + 4, next, y);
      next = look_up(s + 8);
      compute(x, s);
      if (!more) break;
      s += 4;
      x = y;
    }
  }

  // join the four waves: 2 and 3 hand theirs to 0 and 1, then 1 to 0
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    l_run[mt] += __shfl_xor(l_run[mt], 16);
    l_run[mt] += __shfl_xor(l_run[mt], 32);
  }
#pragma unroll
  for (int turn = 0; turn < 2; ++turn) {
    const int half = turn == 0 ? 2 : 1;
    if (w >= half && w < 2 * half) {
      float* out = join + (w - half) * SLOT + lane;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        out[(mt * (CB * 4 + 2)) * 64] = m_run[mt];
        out[(mt * (CB * 4 + 2) + 1) * 64] = l_run[mt];
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) out[(mt * (CB * 4 + 2) + 2 + 4 * c + e) * 64] = o[mt][c][e];
      }
    }
    __syncthreads();
    if (w < half) {
      const float* in = join + w * SLOT + lane;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const float m2 = in[(mt * (CB * 4 + 2)) * 64], l2 = in[(mt * (CB * 4 + 2) + 1) * 64];
        const float m = fmaxf(m_run[mt], m2), m_use = m == NEG_INF ? 0.f : m;
        const float f1 = fast_exp2(m_run[mt] - m_use), f2 = fast_exp2(m2 - m_use);
        l_run[mt] = l_run[mt] * f1 + l2 * f2;
        m_run[mt] = m;
#pragma unroll
        for (int c = 0; c < CB; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[mt][c][e] = o[mt][c][e] * f1 + in[(mt * (CB * 4 + 2) + 2 + 4 * c + e) * 64] * f2;
      }
    }
    __syncthreads();
  }
  if (w != 0) return;
#pragma unroll
  for (int mt = 0; mt < MT; ++mt) {
    const int32_t r = rt.row0 + 16 * mt + l16;
    if (r >= nrows) continue;
    const int32_t t = r / a.group;
    const int64_t tok = rt.t0 + t;
    const int h = g * a.group + (r - t * a.group);
    const float inv = l_run[mt] > 0.f ? 1.f / l_run[mt] : 0.f;
    const float lse2 = l_run[mt] > 0.f ? m_run[mt] + __log2f(l_run[mt]) : NEG_INF;
    const int64_t row = tok * a.heads_q + h;
    if (a.splits == 1) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        __bf16* op = a.o + row * D + CB * (4 * grp + e);
#pragma unroll
        for (int c = 0; c < CB; c += 4)
          *(bf16x4*)(op + c) = bf16x4{(__bf16)(o[mt][c][e] * inv), (__bf16)(o[mt][c + 1][e] * inv),
                                      (__bf16)(o[mt][c + 2][e] * inv), (__bf16)(o[mt][c + 3][e] * inv)};
      }
      if (grp == 0 && a.lse) a.lse[(int64_t)h * a.total_q + tok] = lse2 * 0.69314718055994530942f;
    } else {
      const int64_t at = (int64_t)split * a.total_q * a.heads_q + row;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float* op = a.part_o + at * D + CB * (4 * grp + e);
#pragma unroll
        for (int c = 0; c < CB; c += 4)
          *(f32x4*)(op + c) = f32x4{o[mt][c][e] * inv, o[mt][c + 1][e] * inv, o[mt][c + 2][e] * inv, o[mt][c + 3][e] * inv};
      }
      if (grp == 0) a.part_lse[at] = lse2;
    }
  }
}

// Many rows of a sequence (a prompt's chunk): bound by products and exponentials, no longer by the codes, so a workgroup
// takes 128 rows, a wave 32 of them, and every step's 64 tokens are decoded once for all: codes to registers a step ahead,
// from there as bf16 (which e4m3 fits exactly; V times its scale's power of two) into the tiles of the window kernels, and
// 32x32x16 products S^T = K Q^T, O^T += V^T P^T with V^T by transpose reads.  P is rounded to bf16 for the second product,
// as in the window kernels.  2048 rows x 8 heads over 30000 tokens, head_dim 128: 680 us, 765 TFLOP/s (a step's products,
// exponentials and decoding add up in a wave: matrix cores 0.31 busy).  head_dim 64: three workgroups per CU (185 -> 167 us).
template <int D>
__global__ __launch_bounds__(256, D == 64 ? 3 : 2) void cache_chunk_kernel(CacheAttnArgs a) {
  constexpr int KB = 64, CPR = D / 8, TILE = KB * D, ROWS = kChunkRows, U = D / 64;  // U: runs of 16 codes per thread
  constexpr float NEG_INF = -__builtin_inff(), TINY = 1.17549435e-38f;
  constexpr float RESCALE_SLACK = 8.f;
  __shared__ __attribute__((aligned(16))) __bf16 tiles[2][2][TILE];  // [slot][K, V]
  __shared__ __attribute__((aligned(16))) float scales[2][2][4];     // [slot][K's times the softmax's, V's rest][16 tokens]

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
  const int32_t pos0 = len - rt.count;
  const int32_t plo = pos0 + rt.row0 / a.group, phi = pos0 + last_row / a.group;
  const Steps<KB> steps = cache_steps<KB>(plo, phi, cap, a.window, a.sinks);
  const int32_t per = steps_per_split(steps.total, a.splits);
  const int32_t s_begin = split * per, s_end = min(steps.total, s_begin + per);
  if (s_begin >= s_end && a.splits > 1) {  // nothing here for the join
    const int32_t r = rt.row0 + tid, t = r / a.group;
    if (tid < ROWS && r < nrows)
      a.part_lse[((int64_t)split * a.total_q + rt.t0 + t) * a.heads_q + g * a.group + (r - t * a.group)] = NEG_INF;
    return;
  }
  // this lane's query, and the first and last position of the wave's
  const bool busy = rt.row0 + 32 * w <= last_row;
  const int32_t row = min(rt.row0 + 32 * w + l32, last_row), tok = row / a.group;
  const int32_t pos = pos0 + tok;
  const int32_t wlo = pos0 + min(rt.row0 + 32 * w, last_row) / a.group;
  const int32_t whi = pos0 + min(rt.row0 + 32 * w + 31, last_row) / a.group;
  const int h = g * a.group + (row - tok * a.group);
  bf16x8 qf[D / 16];
  {
    const __bf16* qp = a.q + (int64_t)(rt.t0 + tok) * a.q_stride + (int64_t)h * D + 8 * hi;
#pragma unroll
    for (int kk = 0; kk < D / 16; ++kk) qf[kk] = *(const bf16x8*)(qp + 16 * kk);
  }
  const int32_t* table = a.c.page_table + (int64_t)rt.seq * a.d.table_width;
  const int32_t top = min(phi, cap - 1);  // last token any row sees

  // Thread's codes of a step: of the 64 tokens those of 16-token group group_of(u) (one page each), 16 codes of a token.
  auto group_of = [&](int u) { return D == 64 ? w : (w >> 1) + 2 * u; };
  const int slot_in = D == 64 ? (lane >> 2) : 8 * (w & 1) + (lane >> 3);  // token within the group
  const int column = 16 * (D == 64 ? lane & 3 : lane & 7);
  // Pages and scales are read as vectors: a scalar load, which may come back out of order, would make every wait for an LDS
  // read a wait for memory.
  int zero;
  asm volatile("v_mov_b32 %0, 0" : "=v"(zero));
  struct Codes {
    uint4 k[U], v[U];
    float ks[U], vs[U];
    bool held[U];  // the group lies in a page
  };
  struct Where {
    int32_t page[U];
  };
  auto look_up = [&](int32_t s) __attribute__((always_inline)) {
    Where x;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int32_t j = steps.first(s) + 16 * group_of(u);
      x.page[u] = (s < s_end) & steps.looked_up(a.sinks, j, top) ? table[(j >> a.page_shift) + zero] : -1;
    }
    return x;
  };
  auto load = [&](int32_t s, const Where& where, Codes& x) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int32_t j = steps.first(s) + 16 * group_of(u);
      const int32_t page = uniform(where.page[u]);
      x.held[u] = (uint32_t)page < (uint32_t)a.d.num_pages;
      const int64_t at = (int64_t)(x.held[u] ? page : 0) * a.d.heads_kv + g;
      x.ks[u] = (a.c.k_scale + at)[zero];
      x.vs[u] = (a.c.v_scale + at)[zero];
      const int64_t first = ((at << a.page_shift) + (j & (ps - 1)) + slot_in) * D + column;
      x.k[u] = *(const uint4*)(a.c.k_codes + first);
      x.v[u] = *(const uint4*)(a.c.v_codes + first);
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
  auto store = [&](int32_t s, Codes& x, int slot) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int token = 16 * group_of(u) + slot_in;
      const int32_t j = steps.first(s) + token;
      float vpow = __uint_as_float(__float_as_uint(x.vs[u]) & 0x7F800000u);
      if (j > top || !x.held[u] || (steps.edge(s) && !steps.seen(a.sinks, j, j))) {  // anything may be there
        x.k[u] = x.v[u] = uint4{0, 0, 0, 0};
        vpow = 1.f;
      }
      const int at0 = swz<CPR>(token, column), at1 = swz<CPR>(token, column + 8);
      decode(x.k[u], 1.f, tiles[slot][0] + at0, tiles[slot][0] + at1);
      decode(x.v[u], vpow, tiles[slot][1] + at0, tiles[slot][1] + at1);
      // (a scale of 0 stands for no page; at least the smallest normal number, so that -inf times it stays -inf)
      if (lane == 0) {
        scales[slot][0][group_of(u)] = x.held[u] ? fmaxf(x.ks[u] * a.scale_log2, TINY) : 0.f;
        scales[slot][1][group_of(u)] = __uint_as_float((__float_as_uint(x.vs[u]) & 0x007FFFFFu) | 0x3F800000u);
      }
    }
  };

  TileReads<D> rd;
  rd.init(lane);
  float m_run = NEG_INF, l_run = 0.f;
  f32x16 o[D / 32];
#pragma unroll
  for (int mb = 0; mb < D / 32; ++mb) o[mb] = f32x16{};

  auto compute = [&](int32_t s, int slot) __attribute__((always_inline)) {
    const int32_t j0 = steps.first(s);
    const f32x4 sl = *(const f32x4*)scales[slot][0], vrest = *(const f32x4*)scales[slot][1];
    f32x16 sc[2];
#pragma unroll
    for (int nb = 0; nb < 2; ++nb) {
      bf16x8 kf[D / 16];
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) kf[kk] = rd.rows(tiles[slot][0] + 32 * nb * D, kk);
      sc[nb] = f32x16{};
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) sc[nb] = mfma32(kf[kk], qf[kk], sc[nb]);
    }
    const int32_t sinks = s < steps.sinks ? min(a.sinks, steps.win0) : a.sinks;
    const int32_t near = s < steps.sinks ? 0 : a.window;
    const bool held = sl[0] > 0.f && sl[1] > 0.f && sl[2] > 0.f && sl[3] > 0.f;
    // every row of the wave sees every token of the step
    const bool all = __builtin_amdgcn_ballot_w64(!held) == 0 && j0 + KB - 1 <= wlo && (whi - j0 < near || j0 + KB - 1 < sinks);
    if (!all) {
#pragma unroll
      for (int nb = 0; nb < 2; ++nb)
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const int32_t t = j0 + 32 * nb + c_row(j, hi);
          const bool see = (t <= pos) & (((int32_t)((uint32_t)pos - (uint32_t)t) < near) | (t < sinks)) & (sl[2 * nb + (j >> 3)] > 0.f);
          sc[nb][j] = see ? sc[nb][j] : NEG_INF;
        }
    }
    float mx = NEG_INF;
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      float x = sc[q >> 1][8 * (q & 1)];
#pragma unroll
      for (int j = 1; j < 8; ++j) x = fmaxf(x, sc[q >> 1][8 * (q & 1) + j]);
      mx = fmaxf(mx, x * fmaxf(sl[q], TINY));
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
    for (int q = 0; q < 4; ++q) {
      const float x = fmaxf(sl[q], TINY);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float p = fast_exp2(__builtin_fmaf(sc[q >> 1][8 * (q & 1) + j], x, -m_use));
        l_run += p;
        sc[q >> 1][8 * (q & 1) + j] = p;
      }
    }
    if (__builtin_amdgcn_ballot_w64(vrest[0] != 1.f || vrest[1] != 1.f || vrest[2] != 1.f || vrest[3] != 1.f) != 0) {
#pragma unroll
      for (int j = 0; j < 32; ++j) sc[j >> 4][j & 15] *= vrest[j >> 3];
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      bf16x8 pb;
#pragma unroll
      for (int j = 0; j < 8; ++j) pb[j] = (__bf16)sc[q >> 1][8 * (q & 1) + j];
#pragma unroll
      for (int mb = 0; mb < D / 32; ++mb) o[mb] = mfma32(rd.turned(tiles[slot][1] + 16 * q * D, mb), pb, o[mb]);
    }
  };

  if (s_begin < s_end) {
    Codes x;
    load(s_begin, look_up(s_begin), x);
    store(s_begin, x, 0);
    Where next = look_up(s_begin + 1);
    hsap_lds_barrier();
    for (int32_t s = s_begin; s < s_end; ++s) {
      const int slot = (s - s_begin) & 1;
      const bool more = s + 1 < s_end;
      if (more) load(s + 1, next, x);
      next = look_up(s + 2);
      const int32_t j0 = steps.first(s);
      if (busy && j0 <= whi && (s < steps.sinks || j0 + KB - 1 >= max(wlo, 0) - (a.window - 1) || j0 < a.sinks)) compute(s, slot);
      if (more) store(s + 1, x, slot ^ 1);
      hsap_lds_barrier();
    }
  }
  l_run = pair_sum(l_run);
  if (rt.row0 + 32 * w + l32 > last_row) return;
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

// Joins the splits of every row by their LSE.  Up to eight: D / 4 lanes per row, four values each, every load of a row
// in flight together (4.5 us for 64 rows x 32 heads x 2 splits, of which about 3 are the launch).
template <int D>
__global__ __launch_bounds__(256) void cache_join_few_kernel(CacheAttnArgs a) {
  constexpr float NEG_INF = -__builtin_inff();
  constexpr int LANES = D / 4, MOST = 8;
  const int64_t rows = a.total_q * a.heads_q;
  const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LANES;
  const int x = threadIdx.x % LANES;
  if (row >= rows) return;
  const int64_t tok = row / a.heads_q;
  if (a.cu && tok >= a.cu[a.d.num_seqs]) return;  // a row of no sequence
  float l[MOST], m = NEG_INF, sum = 0.f;
#pragma unroll
  for (int s = 0; s < MOST; ++s) {
    l[s] = s < a.splits ? a.part_lse[s * rows + row] : NEG_INF;
    m = fmaxf(m, l[s]);
  }
  f32x4 acc = f32x4{};
#pragma unroll
  for (int s = 0; s < MOST; ++s) {
    const float f = l[s] == NEG_INF ? 0.f : fast_exp2(l[s] - m);
    sum += f;
    if (f > 0.f) acc += f * *(const f32x4*)(a.part_o + (s * rows + row) * D + 4 * x);
  }
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
  *(bf16x4*)(a.o + row * D + 4 * x) = bf16x4{(__bf16)(acc[0] * inv), (__bf16)(acc[1] * inv), (__bf16)(acc[2] * inv),
                                             (__bf16)(acc[3] * inv)};
  if (x == 0 && a.lse)
    a.lse[(row - tok * a.heads_q) * a.total_q + tok] = sum > 0.f ? (m + __log2f(sum)) * 0.69314718055994530942f : NEG_INF;
}

// More splits: a workgroup per row.  Every wave forms the weights of all splits (up to 128, two to a lane); the
// 256 / (D / 4) groups of lanes then take every so manieth split and are added up in LDS.
template <int D>
__global__ __launch_bounds__(256) void cache_join_many_kernel(CacheAttnArgs a) {
  constexpr float NEG_INF = -__builtin_inff();
  constexpr int LANES = D / 4, GROUPS = 256 / LANES;
  __shared__ float weight[kMaxSplits];
  __shared__ f32x4 part[GROUPS][LANES];
  const int64_t rows = a.total_q * a.heads_q, row = blockIdx.x;
  const int64_t tok = row / a.heads_q;
  if (a.cu && tok >= a.cu[a.d.num_seqs]) return;
  const int tid = threadIdx.x, lane = tid & 63, x = tid % LANES, grp = tid / LANES;
  float l[kMaxSplits / 64], m = NEG_INF, sum = 0.f;
#pragma unroll
  for (int y = 0; y < kMaxSplits / 64; ++y) {
    const int s = 64 * y + lane;
    l[y] = s < a.splits ? a.part_lse[s * rows + row] : NEG_INF;
    m = fmaxf(m, l[y]);
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
#pragma unroll
  for (int y = 0; y < kMaxSplits / 64; ++y) {
    const float f = l[y] == NEG_INF ? 0.f : fast_exp2(l[y] - m);
    sum += f;
    if (tid < 64) weight[64 * y + lane] = f;
  }
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) sum += __shfl_xor(sum, o);
  __syncthreads();
  f32x4 acc = f32x4{};
  for (int s0 = grp; s0 < a.splits; s0 += 8 * GROUPS) {  // eight loads in flight
    f32x4 o[8];
    float f[8];
#pragma unroll
    for (int y = 0; y < 8; ++y) {
      const int s = min(s0 + y * GROUPS, a.splits - 1);
      f[y] = s0 + y * GROUPS < a.splits ? weight[s] : 0.f;
      o[y] = *(const f32x4*)(a.part_o + (s * rows + row) * D + 4 * x);
    }
#pragma unroll
    for (int y = 0; y < 8; ++y)
      if (f[y] > 0.f) acc += f[y] * o[y];  // (the rows of an idle split are not written)
  }
  part[grp][x] = acc;
  __syncthreads();
  if (grp > 0) return;
  for (int y = 1; y < GROUPS; ++y) acc += part[y][x];
  const float inv = sum > 0.f ? 1.f / sum : 0.f;
  *(bf16x4*)(a.o + row * D + 4 * x) = bf16x4{(__bf16)(acc[0] * inv), (__bf16)(acc[1] * inv), (__bf16)(acc[2] * inv),
                                             (__bf16)(acc[3] * inv)};
  if (x == 0 && a.lse)
    a.lse[(row - tok * a.heads_q) * a.total_q + tok] = sum > 0.f ? (m + __log2f(sum)) * 0.69314718055994530942f : NEG_INF;
}

static int64_t cache_workspace(const CacheCut& c, int32_t heads_q, int64_t total_q, int head_dim) {
  return c.splits == 1 ? 0 : (int64_t)c.splits * total_q * heads_q * (head_dim + 1) * 4;
}

static hsap_status check_attn_rows(const hsap_cache_desc& d, int32_t heads_q, int64_t total_q) {
  if (heads_q < 1 || heads_q % d.heads_kv)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "heads_q=%d must be a positive multiple of heads_kv=%d", heads_q, d.heads_kv);
  if (total_q < 0 || total_q > INT32_MAX / heads_q) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "bad total_q %lld", (long long)total_q);
  return HSAP_OK;
}

template <typename Cut>
static int64_t workspace_of(Cut cut, const hsap_cache_desc* desc, int32_t heads_q, int64_t total_q, int32_t one_each) {
  clear_error();
  if (check_cache_desc(desc, false) != HSAP_OK || check_attn_rows(*desc, heads_q, total_q) != HSAP_OK) return -1;
  const CacheCut c = cut(*desc, heads_q, total_q, one_each != 0, (int64_t)desc->table_width * desc->page_size);
  return std::max<int64_t>(16, cache_workspace(c, heads_q, total_q, desc->head_dim));
}

template <int D>
static void launch_cache_attn(const CacheAttnArgs& a, const CacheCut& c, int64_t blocks, hipStream_t s) {
  const dim3 grid((unsigned)blocks), block(256);
  if (c.rows == kChunkRows) hipLaunchKernelGGL(cache_chunk_kernel<D>, grid, block, 0, s, a);
  else if (c.rows == 32) hipLaunchKernelGGL((cache_attn_kernel<D, 2, false, false>), grid, block, 0, s, a);
  else if (c.once) hipLaunchKernelGGL((cache_attn_kernel<D, 1, true, false>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((cache_attn_kernel<D, 1, false, false>), grid, block, 0, s, a);
}

template <int D>
static void launch_tree_attn(const CacheAttnArgs& a, const CacheCut& c, int64_t blocks, hipStream_t s) {
  const dim3 grid((unsigned)blocks), block(256);
  if (c.rows >= 64) launch_tree(a, blocks, s);
  else if (D == 128 && c.rows == 32) hipLaunchKernelGGL((cache_attn_kernel<128, 2, false, true>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((cache_attn_kernel<D, 1, false, true>), grid, block, 0, s, a);
}

// A call's rows, without or with a tree's masks and positions.
static hsap_status attend(const char* name, const hsap_cache_desc* desc, const hsap_cache* cache, int32_t heads_q,
                          float softmax_scale, int32_t window, int32_t sinks, const void* q, int64_t q_stride, const int32_t* cu_new,
                          int64_t total_q, bool tree, const uint64_t* mask, int32_t words, const int32_t* positions, void* o_out,
                          float* lse_out, void* workspace, int64_t workspace_bytes, void* hip_stream) {
  hsap_status st = check_cache(desc, cache);
  if (st != HSAP_OK) return st;
  const int d = desc->head_dim;
  if ((st = check_attn_rows(*desc, heads_q, total_q)) != HSAP_OK) return st;
  if (!(softmax_scale > 0.f) || softmax_scale > 1e30f) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "softmax_scale must be positive and finite");
  if (window < 1) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "window %d < 1 (a query always sees itself)", window);
  if (sinks < 0) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "sinks %d < 0", sinks);
  if (!cu_new && total_q != desc->num_seqs)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "without cu_new every sequence has one row: total_q %lld, num_seqs %d", (long long)total_q,
              desc->num_seqs);
  if (tree && (words < 1 || words > kMaxMaskWords)) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "mask_words %d: 1 to %d", words, kMaxMaskWords);
  if (total_q == 0 || desc->num_seqs == 0) return HSAP_OK;
  if (!q || !o_out || !workspace) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "NULL pointer argument");
  if (tree && (!mask || !positions || ((uintptr_t)mask & 7)))
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "a tree's mask (8-byte aligned) and positions are needed");
  if (((uintptr_t)q | (uintptr_t)o_out | (uintptr_t)workspace) & 15)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "q, o_out and workspace must be 16-byte aligned");
  if (q_stride % 8 || q_stride < (int64_t)heads_q * d)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "q_stride %lld must be a multiple of 8 and at least %lld", (long long)q_stride,
              (long long)heads_q * d);
  const int64_t tokens = (int64_t)desc->table_width * desc->page_size;
  CacheCut c = (tree ? tree_cut : cache_cut)(*desc, heads_q, total_q, !cu_new, tokens);
  const int64_t need = cache_workspace(c, heads_q, total_q, d);
  if (workspace_bytes < need)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)need);
  if (tree) {  // fewer splits where a window leaves little
    const int64_t near = std::min(tokens, (int64_t)window + sinks + 64 * words);
    c.splits = std::min(c.splits, tree_cut(*desc, heads_q, total_q, !cu_new, near).splits);
  }
  CacheAttnArgs a{};
  a.d = *desc;
  a.c = *cache;
  a.q = (const __bf16*)q;
  a.q_stride = q_stride;
  a.cu = cu_new;
  a.total_q = total_q;
  a.o = (__bf16*)o_out;
  a.lse = lse_out;
  a.part_o = (float*)workspace;
  a.part_lse = a.part_o + (int64_t)c.splits * total_q * heads_q * d;
  a.heads_q = heads_q;
  a.group = heads_q / desc->heads_kv;
  a.page_shift = __builtin_ctz((unsigned)desc->page_size);
  a.window = window;
  a.sinks = sinks;
  a.splits = c.splits;
  a.scale_log2 = softmax_scale * 1.44269504088896340736f;
  a.mask = mask;
  a.positions = positions;
  a.words = words;
  a.furthest = window == INT32_MAX ? INT32_MAX - 1 : INT32_MAX;
  const int64_t blocks = c.tiles * c.splits * desc->heads_kv;
  if (blocks > kMaxBlocks256) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "too many rows x heads");
  hipStream_t s = (hipStream_t)hip_stream;
  if (tree) {
    if (d == 128) launch_tree_attn<128>(a, c, blocks, s);
    else launch_tree_attn<64>(a, c, blocks, s);
  } else {
    if (d == 128) launch_cache_attn<128>(a, c, blocks, s);
    else launch_cache_attn<64>(a, c, blocks, s);
  }
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) HSAP_FAIL(HSAP_ERR_HIP, "%s launch: %s", name, hipGetErrorString(e));
  if (c.splits > 1) {
    const int64_t rows = total_q * heads_q;
    const dim3 few((unsigned)((rows * (d / 4) + 255) / 256)), many((unsigned)rows), block(256);
    if (c.splits <= 8) {
      if (d == 128) hipLaunchKernelGGL(cache_join_few_kernel<128>, few, block, 0, s, a);
      else hipLaunchKernelGGL(cache_join_few_kernel<64>, few, block, 0, s, a);
    } else {
      if (d == 128) hipLaunchKernelGGL(cache_join_many_kernel<128>, many, block, 0, s, a);
      else hipLaunchKernelGGL(cache_join_many_kernel<64>, many, block, 0, s, a);
    }
    e = hipGetLastError();
    if (e != hipSuccess) HSAP_FAIL(HSAP_ERR_HIP, "%s join launch: %s", name, hipGetErrorString(e));
  }
  return HSAP_OK;
}

}  // namespace hsap

using namespace hsap;

extern "C" int64_t hsap_cache_attn_workspace(const hsap_cache_desc* desc, int32_t heads_q, int64_t total_q, int32_t one_each) {
  return workspace_of(cache_cut, desc, heads_q, total_q, one_each);
}

extern "C" hsap_status hsap_cache_attn(const hsap_cache_desc* desc, const hsap_cache* cache, int32_t heads_q, float softmax_scale,
                                       int32_t window, int32_t sinks, const void* q, int64_t q_stride, const int32_t* cu_new,
                                       int64_t total_q, void* o_out, float* lse_out, void* workspace, int64_t workspace_bytes,
                                       void* hip_stream) {
  clear_error();
  return attend("cache_attn", desc, cache, heads_q, softmax_scale, window, sinks, q, q_stride, cu_new, total_q, false, nullptr, 0,
                nullptr, o_out, lse_out, workspace, workspace_bytes, hip_stream);
}

extern "C" int64_t hsap_cache_tree_attn_workspace(const hsap_cache_desc* desc, int32_t heads_q, int64_t total_q, int32_t one_each) {
  return workspace_of(tree_cut, desc, heads_q, total_q, one_each);
}

extern "C" hsap_status hsap_cache_tree_attn(const hsap_cache_desc* desc, const hsap_cache* cache, int32_t heads_q,
                                            float softmax_scale, int32_t window, int32_t sinks, const void* q, int64_t q_stride,
                                            const int32_t* cu_new, int64_t total_q, const uint64_t* mask, int32_t mask_words,
                                            const int32_t* positions, void* o_out, float* lse_out, void* workspace,
                                            int64_t workspace_bytes, void* hip_stream) {
  clear_error();
  return attend("cache_tree_attn", desc, cache, heads_q, softmax_scale, window, sinks, q, q_stride, cu_new, total_q, true, mask,
                mask_words, positions, o_out, lse_out, workspace, workspace_bytes, hip_stream);
}
