// Trees of drafted tokens: the masks and positions that rollout_attn_decode_tree and the rotary
// table need, from the nodes' parents, and the walk of the target's tokens down the tree.
//
// A node's mask is itself and its ancestors. Parents come before their children, so the walk up
// from a node visits bits of falling index: one 64-bit word is gathered at a time and stored
// when the walk leaves it, and no node's mask waits for another's.
//
// The walk down: cur = 0, the root; the next node is the first child of cur whose token is the
// one chosen at cur. A wave a row looks at 64 nodes at a time.
//
// Bound by latency: some 30 bytes a node, a few dependent steps each. 8 rows of up to 16 nodes:
// mask 2.8 us, walk 3.2; 512 rows of 48 to 64 nodes: 4.9 and 5.2; of chains of 64 that are accepted
// as a whole 6.4 and 25.7; 8 chains of 1,024: 255 and 361. A workgroup a row and all of its parents in
// LDS: a step of the walk up is an LDS read, one of the walk down a load of the token chosen there
// and then LDS reads, 0.35 us.
#include "ra_device.h"
#include "ra_internal.h"

namespace ra {
namespace {

constexpr int kMaskThreads = 256;

// Row b's nodes: first packed node and how many, inside the caller's arrays.
__device__ __forceinline__ void draft_row(const int32_t *cu_q, int b, int32_t total_q,
                                          int32_t max_q_len, int &first, int &T) {
  first = min(max(cu_q[b], 0), total_q);
  T = min(min(max(cu_q[b + 1] - first, 0), max_q_len), total_q - first);
}

__global__ __launch_bounds__(kMaskThreads) void draft_mask_kernel(
    const int32_t *parents, const int32_t *cu_q, const int32_t *ctx_lens, int32_t total_q,
    int32_t max_q_len, int32_t words, uint64_t *tree_mask, int32_t *positions) {
  __shared__ int16_t up[kMaxDraftNodes];
  const int b = blockIdx.x;
  int first, T;
  draft_row(cu_q, b, total_q, max_q_len, first, T);
  for (int i = threadIdx.x; i < T; i += kMaskThreads) {
    const int p = parents[first + i];
    up[i] = p >= 0 && p < i ? (int16_t)p : (int16_t)-1;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < T; i += kMaskThreads) {
    uint64_t *row = tree_mask + (size_t)(first + i) * words;
    int word = words - 1, depth = -1;
    uint64_t bits = 0;
    for (int j = i; j >= 0; j = up[j], ++depth) {
      for (; word > (j >> 6); --word) row[word] = bits, bits = 0;
      bits |= 1ull << (j & 63);
    }
    for (; word >= 0; --word) row[word] = bits, bits = 0;
    if (positions) positions[first + i] = (ctx_lens ? ctx_lens[b] : 0) + depth;
  }
}

__global__ __launch_bounds__(kWave) void draft_accept_kernel(
    const int32_t *parents, const int32_t *draft_tokens, const int32_t *chosen,
    const int32_t *cu_q, const int32_t *ctx_lens, int32_t total_q, int32_t max_q_len,
    int32_t *path, int32_t *tokens, int32_t *accepted, int32_t *kv_lens, int32_t *next_tokens) {
  __shared__ int32_t up[kMaxDraftNodes], held[kMaxDraftNodes];
  const int b = blockIdx.x, lane = threadIdx.x;
  int first, T;
  draft_row(cu_q, b, total_q, max_q_len, first, T);
  for (int i = lane; i < T; i += kWave) {
    up[i] = parents[first + i];
    held[i] = draft_tokens[first + i];
  }
  __syncthreads();
  int count = 0, last = -1;
  for (int cur = T > 0 ? 0 : -1; cur >= 0;) {
    last = chosen[first + cur];
    if (lane == 0) {
      path[first + count] = cur;
      tokens[first + count] = last;
    }
    ++count;
    int next = -1;
    for (int j0 = cur + 1; j0 < T && next < 0; j0 += kWave) {
      const int j = j0 + lane;
      const bool fits = j < T && last >= 0 && up[j] == cur && held[j] == last;
      const uint64_t any = __ballot(fits);
      if (any) next = j0 + __ffsll((unsigned long long)any) - 1;
    }
    cur = next;
  }
  for (int i = count + lane; i < T; i += kWave) path[first + i] = tokens[first + i] = -1;
  if (lane == 0) {
    accepted[b] = count;
    kv_lens[b] = ctx_lens[b] + count;
    next_tokens[b] = last;
  }
}

}  // namespace

hipError_t launch_draft_mask(const int32_t *parents, const int32_t *cu_q, const int32_t *ctx_lens,
                             int32_t B, int32_t total_q, int32_t max_q_len, int32_t words,
                             uint64_t *tree_mask, int32_t *positions, hipStream_t stream) {
  draft_mask_kernel<<<B, kMaskThreads, 0, stream>>>(parents, cu_q, ctx_lens, total_q, max_q_len,
                                                    words, tree_mask, positions);
  return hipGetLastError();
}

hipError_t launch_draft_accept(const int32_t *parents, const int32_t *draft_tokens,
                               const int32_t *chosen, const int32_t *cu_q,
                               const int32_t *ctx_lens, int32_t B, int32_t total_q,
                               int32_t max_q_len, int32_t *path, int32_t *tokens,
                               int32_t *accepted, int32_t *kv_lens, int32_t *next_tokens,
                               hipStream_t stream) {
  draft_accept_kernel<<<B, kWave, 0, stream>>>(parents, draft_tokens, chosen, cu_q, ctx_lens,
                                               total_q, max_q_len, path, tokens, accepted, kv_lens,
                                               next_tokens);
  return hipGetLastError();
}

}  // namespace ra
