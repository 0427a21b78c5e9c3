// Kept tokens of every sequence moved together, in place or into fresh pages.
//
// Token i of a sequence's list goes to place first + i.  A page's moved codes come from pages of other scales: the new scale
// is the smallest that holds their largest value (and at least the old one where the page keeps tokens before them), and every
// code is multiplied by old over new scale, powers of two: exact but for what falls under e4m3's smallest normal number.
//
// In place one workgroup takes a sequence's pages of one head in order: a list is ascending, so no place is written before
// what it held has been read.  Into fresh pages every page is a workgroup's own.  Bound by memory: codes read and written
// once.  A thread holds 16 codes of a token.
#include <algorithm>

#include "cache.h"
#include "cache_codes.h"
#include "hsap_internal.h"

namespace hsap {

hsap_status check_cache(const hsap_cache_desc* d, const hsap_cache* c);

struct CompactArgs {
  hsap_cache_desc d;
  hsap_cache c;
  const int32_t* keep;
  const int32_t* cu;
  int64_t total;
  const int32_t* first;  // may be NULL: 0
  const int32_t* dst_table;
  int32_t* new_lens;  // may be NULL
};

// Largest finite magnitude of 16 codes (times their scale, which is positive).
__device__ __forceinline__ float codes_max(const uint4& w) {
  const uint32_t c[4] = {w.x, w.y, w.z, w.w};
  float m = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)c[i], true);
    // (fmaxf takes the other operand of a NaN)
    m = fmaxf(fmaxf(m, fabsf(lo[0])), fmaxf(fabsf(lo[1]), fmaxf(fabsf(hi[0]), fabsf(hi[1]))));
  }
  return m;
}

// A workgroup moves K's and V's codes of a page and head, whose tokens it looks up once (16 sequences of 8k tokens, half of
// them into fresh pages: 49 us with a workgroup each, 46 with one for both, 39 since it holds no decoded values, so that seven
// share a compute unit: 4.0 TB/s; a chain of list, table, codes and a maximum, four trips to memory).  PER: units of 16 codes of a page per thread.
template <int D, int PER, bool FRESH>
__global__ __launch_bounds__(256) void cache_compact_kernel(CompactArgs a) {
  constexpr int UNITS = D / 16;
  __shared__ float wave_max[2][4], old_scale[2];
  const int tid = threadIdx.x;
  const int h = blockIdx.x % a.d.heads_kv;
  const int64_t item = blockIdx.x / a.d.heads_kv;
  const int32_t ps = a.d.page_size;
  int32_t s = (int32_t)item, i0, i1, first;
  if constexpr (FRESH) {
    const Sequence q = sequence_of(a.cu, a.d.num_seqs, 1, ps, 2, item, a.first);
    s = q.s;
    i0 = q.begin;
    i1 = q.end;
    first = max(q.value, 0);
  } else {
    i0 = a.cu[s];
    i1 = a.cu[s + 1];
    first = a.first ? max(a.first[s], 0) : 0;
  }
  const int64_t count = min((int64_t)i1, a.total) - i0;
  const int64_t nth = FRESH ? item - item_base(i0, 1, ps, 2, s) : 0;  // page of the list's
  if (a.new_lens && h == 0 && nth == 0 && tid == 0) a.new_lens[s] = first + (int32_t)max(count, (int64_t)0);
  if (count <= 0) return;
  const int32_t* row = a.c.page_table + (int64_t)s * a.d.table_width;
  const int32_t* out_row = FRESH ? a.dst_table + (int64_t)s * a.d.table_width : row;
  uint8_t* const all[2] = {a.c.k_codes, a.c.v_codes};
  float* const scales[2] = {a.c.k_scale, a.c.v_scale};
  const int64_t end = (int64_t)first + count;
  int64_t at = first / ps + nth;
  for (int64_t lo = max((int64_t)first, at * ps); lo < end; lo = ++at * ps) {
    const int64_t hi = min(end, (at + 1) * ps);
    const int32_t page = lo <= INT32_MAX ? cache_page(out_row, a.d.table_width, a.d.num_pages, ps, (int32_t)lo) : -1;
    const int32_t slot0 = (int32_t)(lo - at * ps), units = (int32_t)(hi - lo) * UNITS;
    uint4 w[2][PER];
    float scale[2][PER], amax[2] = {0.f, 0.f};
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int unit = tid + 256 * i;
      w[0][i] = w[1][i] = uint4{0, 0, 0, 0};
      scale[0][i] = scale[1][i] = 0.f;
      if (unit < units) {
        const int32_t src = a.keep[i0 + (lo - first) + unit / UNITS];
        const int32_t from = cache_page(row, a.d.table_width, a.d.num_pages, ps, src);
        if (from >= 0) {
          const int64_t of = (int64_t)from * a.d.heads_kv + h;
          const int64_t place = cache_row(from, a.d.heads_kv, h, ps, src & (ps - 1), D) + 16 * (unit % UNITS);
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            scale[x][i] = scales[x][of];
            w[x][i] = *(const uint4*)(all[x] + place);
          }
        }
      }
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        amax[x] = fmaxf(amax[x], codes_max(w[x][i]) * scale[x][i]);
        // (decoded again below: sixteen values a unit, held until then, would take the registers of more workgroups)
        asm volatile("" : "+v"(w[x][i].x), "+v"(w[x][i].y), "+v"(w[x][i].z), "+v"(w[x][i].w));
      }
      if (page >= 0 && tid == 0) old_scale[x] = slot0 > 0 ? scales[x][(int64_t)page * a.d.heads_kv + h] : 0.f;
#pragma unroll
      for (int o = 1; o < 64; o <<= 1) amax[x] = fmaxf(amax[x], __shfl_xor(amax[x], o));
      if ((tid & 63) == 0) wave_max[x][tid >> 6] = amax[x];
    }
    __syncthreads();  // (everything that this page's places held has been read)
    float now[2], inv[2], ratio[2];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const float m = fmaxf(fmaxf(wave_max[x][0], wave_max[x][1]), fmaxf(wave_max[x][2], wave_max[x][3]));
      now[x] = page_scale(m, slot0 > 0, old_scale[x], inv[x], ratio[x]);
    }
    if (!FRESH) __syncthreads();  // (the next page's come to the same places)
    if (page >= 0) {
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        uint8_t* codes = all[x] + cache_row(page, a.d.heads_kv, h, ps, 0, D);
        if (ratio[x] != 1.f)
          for (int e = tid; e < slot0 * UNITS; e += 256) recode16(codes + 16 * e, ratio[x]);
#pragma unroll
        for (int i = 0; i < PER; ++i) {
          const int unit = tid + 256 * i;
          if (unit < units) {
            // (a code that is not 0 has at most 448 2^9 times the new scale; a page of zeros may have had any)
            const float by = fminf(scale[x][i] * inv[x], 0x1p20f);
            *(uint4*)(codes + (slot0 * UNITS + unit) * 16) = by == 1.f ? w[x][i] : recoded16(w[x][i], by);
          }
        }
        if (tid == 0) scales[x][(int64_t)page * a.d.heads_kv + h] = now[x];
      }
    }
    if (FRESH) break;
  }
}

template <int D, bool FRESH>
static void launch_compact(const CompactArgs& a, int64_t blocks, hipStream_t s) {
  const dim3 grid((unsigned)blocks), block(256);
  const int per = a.d.page_size * (D / 16) / 256;
  if (per <= 1) hipLaunchKernelGGL((cache_compact_kernel<D, 1, FRESH>), grid, block, 0, s, a);
  else if (per == 2) hipLaunchKernelGGL((cache_compact_kernel<D, 2, FRESH>), grid, block, 0, s, a);
  else if constexpr (D == 128) hipLaunchKernelGGL((cache_compact_kernel<D, 4, FRESH>), grid, block, 0, s, a);
}

}  // namespace hsap

using namespace hsap;

extern "C" hsap_status hsap_cache_compact(const hsap_cache_desc* desc, const hsap_cache* cache, const int32_t* keep,
                                          const int32_t* cu_keep, int64_t total_keep, const int32_t* first, const int32_t* dst_table,
                                          int32_t* new_lens, void* hip_stream) {
  clear_error();
  const hsap_status st = check_cache(desc, cache);
  if (st != HSAP_OK) return st;
  if (total_keep < 0 || total_keep > INT32_MAX) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "bad total_keep %lld", (long long)total_keep);
  if (desc->num_seqs == 0) return HSAP_OK;
  if (!cu_keep || (total_keep && !keep)) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "NULL pointer argument");
  // (head 0's workgroups write new_lens while others still read first)
  const uintptr_t lens = (uintptr_t)new_lens, kept = (uintptr_t)first, bytes = (uintptr_t)desc->num_seqs * sizeof(int32_t);
  if (new_lens && first && lens < kept + bytes && kept < lens + bytes)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "first and new_lens must not overlap");
  CompactArgs a{*desc, *cache, keep, cu_keep, total_keep, first, dst_table, new_lens};
  const int64_t items = dst_table ? item_base(total_keep, 1, desc->page_size, 2, desc->num_seqs) : desc->num_seqs;
  const int64_t blocks = items * desc->heads_kv;
  if (blocks > kMaxBlocks256) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "too many tokens x heads");
  hipStream_t s = (hipStream_t)hip_stream;
  if (dst_table) {
    if (desc->head_dim == 128) launch_compact<128, true>(a, blocks, s);
    else launch_compact<64, true>(a, blocks, s);
  } else {
    if (desc->head_dim == 128) launch_compact<128, false>(a, blocks, s);
    else launch_compact<64, false>(a, blocks, s);
  }
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) HSAP_FAIL(HSAP_ERR_HIP, "cache_compact launch: %s", hipGetErrorString(e));
  return HSAP_OK;
}
