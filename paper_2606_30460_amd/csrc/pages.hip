// Pages of a cache: rows of a page table that become other rows (sequences that fork, end or go back), pages for new
// tokens, copies of pages.
//
// refs[p] counts the entries of the table that are page p: 0, the page is free.  All counts are whole numbers that atomics
// add to, and the lowest free pages go to the first places, so results do not depend on the order of anything.  All
// three kernels are bound by their launch and a few dependent reads, the copy of many pages by memory (64 rows of 33 pages: fork
// 3, reservation 9 us; 48 pages of 128 KB of K and of V copied: 5 us a layer, 4.9 TB/s).
#include <algorithm>

#include "cache.h"
#include "hsap_internal.h"

namespace hsap {

hsap_status check_cache_desc(const hsap_cache_desc* d, bool pages);
hsap_status check_cache(const hsap_cache_desc* d, const hsap_cache* c);

struct PagesArgs {
  hsap_cache_desc d;
  int32_t* table;
  int32_t* lens;
  int32_t* refs;
  const int32_t* source;  // may be NULL
  const int32_t* cu;
  int64_t total;
  int32_t* pairs;
  int32_t* missing;
  int32_t* work;
  int64_t items;
  int32_t window;
  int32_t sinks;
  int32_t columns;
  int32_t with_lens;
};

__device__ __forceinline__ bool is_page(const hsap_cache_desc& d, int32_t p) { return p >= 0 && p < d.num_pages; }

// Row whose tokens row s goes on with (-1: none).
__device__ __forceinline__ int32_t source_of(const PagesArgs& a, int32_t s) {
  const int32_t x = a.source ? a.source[s] : s;
  return x >= 0 && x < a.d.num_seqs ? x : -1;
}

constexpr int kForkEntries = 16384;  // of the table, that a workgroup holds: columns for all rows
constexpr int kForkThreads = 1024;

// A workgroup takes some columns of all rows, so that rows can change places.  One that takes them all writes the lengths too
// (a second launch would: 8 rows of 63 pages 4.1 us in two, 2.0 in one).
__global__ __launch_bounds__(kForkThreads) void pages_fork_kernel(PagesArgs a) {
  extern __shared__ int32_t held[];
  const int32_t c0 = (int32_t)blockIdx.x * a.columns, width = min(a.columns, a.d.table_width - c0);
  const int32_t n = a.d.num_seqs * width, ps = a.d.page_size;
  const int32_t* lens = a.lens;
  if (a.with_lens) {
    int32_t* lens_held = held + n;
    for (int32_t s = threadIdx.x; s < a.d.num_seqs; s += kForkThreads) lens_held[s] = a.lens[s];
    lens = lens_held;
  }
  for (int32_t i = threadIdx.x; i < n; i += kForkThreads) {
    const int32_t s = i / width, c = i - s * width;
    held[i] = a.table[(int64_t)s * a.d.table_width + c0 + c];
  }
  __syncthreads();
  for (int32_t i = threadIdx.x; i < n; i += kForkThreads) {
    const int32_t s = i / width, c = i - s * width;
    const int32_t from = source_of(a, s), old = held[i];
    int32_t now = -1;
    if (from >= 0) {
      const int64_t len = lens[from], first = (int64_t)(c0 + c) * ps;
      // (the next token is at position len)
      const bool seen = len - (first + ps - 1) < a.window || first < a.sinks;
      if (first < len && seen) now = held[from * width + c];
    }
    if (!is_page(a.d, now)) now = -1;
    if (now == old) continue;
    if (is_page(a.d, old)) atomicAdd(a.refs + old, -1);
    if (now >= 0) atomicAdd(a.refs + now, 1);
    a.table[(int64_t)s * a.d.table_width + c0 + c] = now;
  }
  if (a.with_lens)
    for (int32_t s = threadIdx.x; s < a.d.num_seqs; s += kForkThreads) {
      const int32_t from = source_of(a, s);
      a.lens[s] = from < 0 ? 0 : lens[from];
    }
}

// The lengths of the rows, after the pages (whose kernel reads the old ones).
__global__ __launch_bounds__(256) void pages_lens_kernel(PagesArgs a) {
  extern __shared__ int32_t held[];
  for (int32_t s = threadIdx.x; s < a.d.num_seqs; s += 256) held[s] = a.lens[s];
  __syncthreads();
  for (int32_t s = threadIdx.x; s < a.d.num_seqs; s += 256) {
    const int32_t from = source_of(a, s);
    a.lens[s] = from < 0 ? 0 : held[from];
  }
}

// Place of an item (numbered as an append's): a page that new tokens of sequence s are written to.
struct Item {
  int32_t s;
  int64_t entry;  // in the table
  bool part;      // the page holds older tokens of the sequence
};
// Page nth of those that the `count` new tokens from t0 on of sequence s, len tokens long, are written to; false: there is none.
__device__ __forceinline__ bool place_of(const PagesArgs& a, int32_t s, int32_t t0, int32_t count, int32_t len, int64_t nth, Item& x) {
  const int32_t ps = a.d.page_size;
  if (count <= 0 || len <= 0) return false;
  const int64_t pos0 = (int64_t)len - count, first = max(pos0, (int64_t)0), at = first / ps + nth;
  const int64_t lo = max(first, at * ps), end = min(min((int64_t)len, (at + 1) * ps), pos0 + a.total - t0);
  if (lo >= end || at >= a.d.table_width) return false;
  x.s = s;
  x.entry = (int64_t)s * a.d.table_width + at;
  x.part = lo > at * ps;
  return true;
}
__device__ __forceinline__ bool item_of(const PagesArgs& a, const int32_t* cu, int64_t item, Item& x) {
  const int32_t ps = a.d.page_size;
  int32_t s = 0, t0, count;
  int64_t nth = 0;
  if (cu) {
    int32_t r = a.d.num_seqs;
    while (r - s > 1) {
      const int32_t mid = (s + r) >> 1;
      if (item_base(cu[mid], 1, ps, 2, mid) <= item) s = mid;
      else r = mid;
    }
    t0 = cu[s];
    count = cu[s + 1] - t0;
    nth = item - item_base(t0, 1, ps, 2, s);
  } else {
    s = (int32_t)item;
    t0 = s;
    count = 1;
  }
  return place_of(a, s, t0, count, a.lens[s], nth, x);
}

__device__ __forceinline__ int32_t count_now(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Exclusive sum over the workgroup's threads, and the total.
__device__ __forceinline__ int32_t block_scan(int32_t x, int32_t* waves, int32_t& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  int32_t sum = x;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int32_t y = __shfl_up(sum, o);
    if (lane >= o) sum += y;
  }
  __syncthreads();  // (the last call's sums have been read)
  if (lane == 63) waves[w] = sum;
  __syncthreads();
  int32_t before = 0;
  total = 0;
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int32_t y = waves[i];
    if (i < w) before += y;
    total += y;
  }
  return before + sum - x;
}

constexpr int kReserveSeqs = 8192;  // searched in LDS (one new token of each of 4000: 167 us from memory, 125)

// One workgroup.  Every place that is written and has a page takes its count off that page; where nobody else is left the
// last of those places keeps it (refs holds -(item + 1) meanwhile), all others need a free one.
__global__ __launch_bounds__(1024) void pages_reserve_kernel(PagesArgs a) {
  __shared__ int32_t waves[16], held[kReserveSeqs + 1];
  constexpr int KEEP = -1, NONE = -2;  // of `work`: the place's page stays; nothing is written there
  const int tid = threadIdx.x;
  const int32_t* cu = a.cu;
  if (a.cu && a.d.num_seqs <= kReserveSeqs) {
    for (int32_t s = tid; s <= a.d.num_seqs; s += 1024) held[s] = a.cu[s];
    cu = held;
    __syncthreads();
  }
  for (int32_t s = tid; s < 2 * a.d.num_seqs; s += 1024) a.pairs[s] = -1;
  for (int64_t i = tid; i < a.items; i += 1024) {
    Item x;
    if (item_of(a, cu, i, x) && is_page(a.d, a.table[x.entry])) atomicAdd(a.refs + a.table[x.entry], -1);
  }
  __syncthreads();
  for (int64_t i = tid; i < a.items; i += 1024) {
    Item x;
    if (item_of(a, cu, i, x) && is_page(a.d, a.table[x.entry]) && count_now(a.refs + a.table[x.entry]) <= 0)
      atomicMin(a.refs + a.table[x.entry], -(int32_t)(i + 1));
  }
  __syncthreads();
  int32_t need = 0;
  for (int64_t i0 = 0; i0 < a.items; i0 += 1024) {
    const int64_t i = i0 + tid;
    Item x;
    int32_t what = NONE;
    if (i < a.items && item_of(a, cu, i, x)) {
      const int32_t page = a.table[x.entry];
      what = is_page(a.d, page) && count_now(a.refs + page) == -(int32_t)(i + 1) ? KEEP : 0;
    }
    int32_t total;
    const int32_t nth = block_scan(what == 0, waves, total);
    if (i < a.items) a.work[i] = what == 0 ? need + nth : what;
    need += total;
  }
  // the first `need` free pages
  int32_t* list = a.work + a.items;
  int32_t found = 0;
  for (int64_t p0 = 0; p0 < a.d.num_pages && found < need; p0 += 1024 * 16) {
    const int64_t p = p0 + 16 * tid;
    uint32_t free = 0;
#pragma unroll
    for (int y = 0; y < 16; ++y)
      if (p + y < a.d.num_pages && a.refs[p + y] == 0) free |= 1u << y;
    int32_t total;
    int32_t at = found + block_scan(__popc(free), waves, total);
    for (; free && at < need; free &= free - 1) list[at++] = (int32_t)p + __ffs(free) - 1;
    found += total;
  }
  __syncthreads();
  const int32_t short_of = max(0, need - found);
  if (tid == 0) *a.missing = short_of;
  if (short_of) {  // as if nothing had been asked
    for (int64_t i = tid; i < a.items; i += 1024) {
      Item x;
      if (a.work[i] == KEEP && item_of(a, cu, i, x)) atomicExch(a.refs + a.table[x.entry], 0);
    }
    __syncthreads();
    for (int64_t i = tid; i < a.items; i += 1024) {
      Item x;
      if (a.work[i] != NONE && item_of(a, cu, i, x) && is_page(a.d, a.table[x.entry])) atomicAdd(a.refs + a.table[x.entry], 1);
    }
    return;
  }
  for (int64_t i = tid; i < a.items; i += 1024) {
    const int32_t what = a.work[i];
    Item x;
    if (what == NONE || !item_of(a, cu, i, x)) continue;
    const int32_t old = a.table[x.entry];
    if (what == KEEP) {
      atomicExch(a.refs + old, 1);
      continue;
    }
    const int32_t page = list[what];
    atomicExch(a.refs + page, 1);
    a.table[x.entry] = page;
    if (x.part && is_page(a.d, old)) {  // (a sequence has at most one such page)
      a.pairs[2 * x.s] = old;
      a.pairs[2 * x.s + 1] = page;
    }
  }
}

// The same where every thread has one item at most: sequences and lengths in LDS, places held in registers, and the sequences
// that write a shared page found by comparison, so that nothing is written before it is known that the free pages are enough.
constexpr int kFewItems = 1024;
__global__ __launch_bounds__(1024) void pages_reserve_few_kernel(PagesArgs a) {
  __shared__ int32_t waves[16], cu[kFewItems + 1], lens[kFewItems], list[kFewItems];
  __shared__ __attribute__((aligned(16))) int32_t shared[kFewItems];  // each item's page where it is shared, else -1
  const int tid = threadIdx.x, ps = a.d.page_size;
  const int32_t n = a.d.num_seqs, items = (int32_t)a.items;
  // (free pages of the first stretch, under way while the places are found)
  uint32_t free = 0;
  const int32_t p0 = 16 * tid;
  const bool wide = ((uintptr_t)a.refs & 15) == 0;
  int4 r[4];
#pragma unroll
  for (int y = 0; y < 4; ++y) {
    const int32_t p = p0 + 4 * y;
    r[y] = int4{1, 1, 1, 1};
    if (wide && p + 3 < a.d.num_pages) r[y] = *(const int4*)(a.refs + p);
    else {
      if (p < a.d.num_pages) r[y].x = a.refs[p];
      if (p + 1 < a.d.num_pages) r[y].y = a.refs[p + 1];
      if (p + 2 < a.d.num_pages) r[y].z = a.refs[p + 2];
      if (p + 3 < a.d.num_pages) r[y].w = a.refs[p + 3];
    }
  }
  if (tid < n) {
    lens[tid] = a.lens[tid];
    a.pairs[2 * tid] = a.pairs[2 * tid + 1] = -1;
  }
  if (a.cu)
    for (int32_t i = tid; i <= n; i += 1024) cu[i] = a.cu[i];
  __syncthreads();
  Item x{};
  int32_t page = -1, count = 0;
  bool mine = false;
  if (tid < items) {
    int32_t s = tid, t0 = tid, new_count = 1;
    int64_t nth = 0;
    if (a.cu) {
      int32_t hi = n;
      s = 0;
      while (hi - s > 1) {
        const int32_t mid = (s + hi) >> 1;
        if (item_base(cu[mid], 1, ps, 2, mid) <= tid) s = mid;
        else hi = mid;
      }
      t0 = cu[s];
      new_count = cu[s + 1] - t0;
      nth = tid - item_base(t0, 1, ps, 2, s);
    }
    mine = place_of(a, s, t0, new_count, lens[s], nth, x);
    if (mine) {
      page = a.table[x.entry];
      if (is_page(a.d, page)) count = a.refs[page];
      else page = -1;
    }
  }
  shared[tid] = count > 1 ? page : -1;
  __syncthreads();
  bool need = mine && page < 0;
  if (count > 1) {
    int32_t writers = 0;
    bool last = true;
#pragma unroll 4
    for (int32_t i = 0; i < items; i += 4) {
      const int4 x4 = *(const int4*)(shared + i);
      const int32_t p4[4] = {x4.x, x4.y, x4.z, x4.w};
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool same = p4[e] == page;
        writers += same;
        last &= !same | (i + e <= tid);
      }
    }
    need = writers < count || !last;
  }
  int32_t wanted, total;
  const int32_t nth = block_scan(need, waves, wanted);
#pragma unroll
  for (int y = 0; y < 4; ++y)
    free |= (uint32_t)((r[y].x == 0) | (r[y].y == 0) << 1 | (r[y].z == 0) << 2 | (r[y].w == 0) << 3) << (4 * y);
  int32_t at = block_scan(__popc(free), waves, total), found = total;
  for (int64_t p = p0;;) {
    for (; free && at < wanted; free &= free - 1) list[at++] = (int32_t)p + __ffs(free) - 1;
    p += 1024 * 16;
    if (found >= wanted || p - p0 >= a.d.num_pages) break;
    free = 0;
#pragma unroll
    for (int y = 0; y < 16; ++y)
      if (p + y < a.d.num_pages && a.refs[p + y] == 0) free |= 1u << y;
    at = found + block_scan(__popc(free), waves, total);
    found += total;
  }
  __syncthreads();
  if (tid == 0) *a.missing = max(0, wanted - found);
  if (found < wanted || !need) return;
  const int32_t to = list[nth];
  if (page >= 0) atomicAdd(a.refs + page, -1);
  a.refs[to] = 1;
  a.table[x.entry] = to;
  if (x.part && page >= 0) {
    a.pairs[2 * x.s] = page;
    a.pairs[2 * x.s + 1] = to;
  }
}

constexpr int kCopyBytes = 16384;  // of a page, per workgroup

__global__ __launch_bounds__(256) void copy_pages_kernel(hsap_cache_desc d, hsap_cache c, const int32_t* pairs, int32_t parts) {
  const int32_t part = (int32_t)(blockIdx.x % (2 * parts));
  const int64_t n = blockIdx.x / (2 * parts);
  const int32_t from = pairs[2 * n], to = pairs[2 * n + 1];
  if (!is_page(d, from) || !is_page(d, to) || from == to) return;
  const bool is_v = part & 1;
  const int64_t bytes = (int64_t)d.heads_kv * d.page_size * d.head_dim;
  uint8_t* codes = is_v ? c.v_codes : c.k_codes;
  const int64_t lo = (int64_t)(part >> 1) * kCopyBytes, hi = min(bytes, lo + kCopyBytes);
  typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
  const u32x4* src = (const u32x4*)(codes + from * bytes + lo);
  u32x4* dst = (u32x4*)(codes + to * bytes + lo);
  const int32_t count = (int32_t)((hi - lo) / 16);
  u32x4 x[kCopyBytes / 16 / 256];
#pragma unroll
  for (int i = 0; i < kCopyBytes / 16 / 256; ++i) x[i] = src[min((int32_t)threadIdx.x + 256 * i, count - 1)];
#pragma unroll
  for (int i = 0; i < kCopyBytes / 16 / 256; ++i)
    if ((int)threadIdx.x + 256 * i < count) dst[threadIdx.x + 256 * i] = x[i];
  if (part >> 1 == 0) {
    float* scale = is_v ? c.v_scale : c.k_scale;
    for (int h = threadIdx.x; h < d.heads_kv; h += 256) scale[(int64_t)to * d.heads_kv + h] = scale[(int64_t)from * d.heads_kv + h];
  }
}

static hsap_status launched(const char* name) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) HSAP_FAIL(HSAP_ERR_HIP, "%s launch: %s", name, hipGetErrorString(e));
  return HSAP_OK;
}

static int64_t reserve_items(const hsap_cache_desc& d, bool one_each, int64_t total_new) {
  return one_each ? d.num_seqs : item_base(total_new, 1, d.page_size, 2, d.num_seqs);
}

static hsap_status check_reserve(const hsap_cache_desc* desc, int64_t total_new, bool pages) {
  const hsap_status st = check_cache_desc(desc, pages);
  if (st != HSAP_OK) return st;
  if (total_new < 0 || total_new > INT32_MAX) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "bad total_new %lld", (long long)total_new);
  // (numbers of places are int32, negative ones mark pages, and loops go on by 1024)
  if (reserve_items(*desc, false, total_new) > (int64_t(1) << 29))
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "too many places: %lld tokens of %d sequences", (long long)total_new, desc->num_seqs);
  return HSAP_OK;
}

}  // namespace hsap

using namespace hsap;

extern "C" hsap_status hsap_pages_fork(const hsap_cache_desc* desc, int32_t* page_table, int32_t* seq_lens, int32_t* refs,
                                       const int32_t* source, int32_t window, int32_t sinks, void* hip_stream) {
  clear_error();
  hsap_status st = check_cache_desc(desc, true);
  if (st != HSAP_OK) return st;
  if (window < 1) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "window %d < 1 (a query always sees itself)", window);
  if (sinks < 0) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "sinks %d < 0", sinks);
  if (desc->num_seqs > kForkEntries) HSAP_FAIL(HSAP_ERR_UNSUPPORTED, "num_seqs %d: at most %d", desc->num_seqs, kForkEntries);
  if (desc->num_seqs == 0) return HSAP_OK;
  if (!page_table || !seq_lens || !refs) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "NULL pointer argument");
  PagesArgs a{};
  a.d = *desc;
  a.table = page_table;
  a.lens = seq_lens;
  a.refs = refs;
  a.source = source;
  a.window = window;
  a.sinks = sinks;
  const int64_t all = (int64_t)desc->num_seqs * desc->table_width;
  a.columns = std::min(all <= kForkEntries / 4 ? desc->table_width : std::min(32, desc->table_width), kForkEntries / desc->num_seqs);
  a.with_lens = source && a.columns == desc->table_width && desc->num_seqs <= (kForkEntries - all);
  hipStream_t s = (hipStream_t)hip_stream;
  const unsigned blocks = (unsigned)((desc->table_width + a.columns - 1) / a.columns);
  if (blocks > kMaxBlocks256 / (kForkThreads / 256)) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "table too wide for its rows");
  const size_t lds = (size_t)desc->num_seqs * (a.columns + a.with_lens) * 4;
  hipLaunchKernelGGL(pages_fork_kernel, dim3(blocks), dim3(kForkThreads), lds, s, a);
  if ((st = launched("pages_fork")) != HSAP_OK || !source || a.with_lens) return st;
  hipLaunchKernelGGL(pages_lens_kernel, dim3(1), dim3(256), (size_t)desc->num_seqs * 4, s, a);
  return launched("pages_fork lengths");
}

extern "C" int64_t hsap_pages_reserve_workspace(const hsap_cache_desc* desc, int64_t total_new) {
  clear_error();
  if (check_reserve(desc, total_new, false) != HSAP_OK) return -1;
  return std::max<int64_t>(16, 8 * std::max(reserve_items(*desc, false, total_new), reserve_items(*desc, true, total_new)));
}

extern "C" hsap_status hsap_pages_reserve(const hsap_cache_desc* desc, int32_t* page_table, const int32_t* seq_lens, int32_t* refs,
                                          const int32_t* cu_new, int64_t total_new, int32_t* pairs, int32_t* missing,
                                          void* workspace, int64_t workspace_bytes, void* hip_stream) {
  clear_error();
  const hsap_status st = check_reserve(desc, total_new, true);
  if (st != HSAP_OK) return st;
  if (!cu_new && total_new != desc->num_seqs)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "without cu_new every sequence has one new token: total_new %lld, num_seqs %d",
              (long long)total_new, desc->num_seqs);
  if (desc->num_seqs > 0 && (!page_table || !seq_lens || !refs || !pairs)) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "NULL pointer argument");
  if (!missing || !workspace || ((uintptr_t)workspace & 15))
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "missing and a 16-byte aligned workspace are needed");
  PagesArgs a{};
  a.d = *desc;
  a.table = page_table;
  a.lens = const_cast<int32_t*>(seq_lens);  // (not written)
  a.refs = refs;
  a.cu = cu_new;
  a.total = total_new;
  a.pairs = pairs;
  a.missing = missing;
  a.work = (int32_t*)workspace;
  a.items = desc->num_seqs ? reserve_items(*desc, !cu_new, total_new) : 0;
  if (desc->num_seqs == 0) {  // (the kernel writes missing; arrays that may be NULL then are not read)
    a.d.num_pages = 0;
    a.cu = nullptr;
  }
  if (workspace_bytes < 8 * a.items)
    HSAP_FAIL(HSAP_ERR_INVALID_ARG, "workspace of %lld bytes, %lld needed", (long long)workspace_bytes, (long long)(8 * a.items));
  if (a.items <= kFewItems && desc->num_seqs <= kFewItems)
    hipLaunchKernelGGL(pages_reserve_few_kernel, dim3(1), dim3(1024), 0, (hipStream_t)hip_stream, a);
  else hipLaunchKernelGGL(pages_reserve_kernel, dim3(1), dim3(1024), 0, (hipStream_t)hip_stream, a);
  return launched("pages_reserve");
}

extern "C" hsap_status hsap_cache_copy_pages(const hsap_cache_desc* desc, const hsap_cache* cache, const int32_t* pairs, int64_t count,
                                             void* hip_stream) {
  clear_error();
  const hsap_status st = check_cache(desc, cache);
  if (st != HSAP_OK) return st;
  if (count < 0 || count > INT32_MAX) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "bad count %lld", (long long)count);
  if (count == 0) return HSAP_OK;
  if (!pairs) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "NULL pairs");
  const int64_t parts = ((int64_t)desc->heads_kv * desc->page_size * desc->head_dim + kCopyBytes - 1) / kCopyBytes;
  if (2 * parts > kMaxBlocks256 / count) HSAP_FAIL(HSAP_ERR_INVALID_ARG, "too many pages x heads");
  hipLaunchKernelGGL(copy_pages_kernel, dim3((unsigned)(2 * parts * count)), dim3(256), 0, (hipStream_t)hip_stream, *desc, *cache,
                     pairs, (int32_t)parts);
  return launched("cache_copy_pages");
}
