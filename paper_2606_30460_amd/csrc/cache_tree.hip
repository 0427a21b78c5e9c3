// Masks and positions of drafted tokens from each one's parent.
//
// A token's mask names itself and its ancestors among the drafted tokens of its sequence, its position is that of its
// depth: the drafted tokens stand behind `base` tokens, a token without a parent at position base.  A thread walks one
// chain of parents (their numbers fall, so every walk ends) and collects one word of a mask: a launch and as many reads
// of LDS as the tree is deep.
#include <algorithm>

#include "cache.h"
#include "hsap_internal.h"

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
