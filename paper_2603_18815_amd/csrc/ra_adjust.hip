// Logits before a token is drawn: penalties for repeated tokens, biases, and masks of the tokens
// that a grammar allows (token_logits_adjust).
//
// A workgroup takes a chunk of the vocabulary for some rows of logits. It counts the row's
// history in LDS, one word a logit of the chunk (bit 31: in the prompt, below it how often in
// the answer; whole numbers, so the order of the atomics does not matter), and the place of
// each token's last bias, then passes over the chunk once. The rows of one tree share the
// history's counts, with the tokens of each node's path added and taken off again.
//
// Bound by HBM: each logit read and written once (in place: only those that change), the
// history once for every chunk, mostly from the L2.
#include "ra_device.h"
#include "ra_internal.h"

namespace ra {
namespace {

constexpr int kThreads = 512;
constexpr int kChunk = 8192;               // logits of a chunk
constexpr uint32_t kPrompt = 1u << 31;

template <bool kBf16>
struct Element {
  using type = uint32_t;
  static __device__ __forceinline__ float value(type x) { return __uint_as_float(x); }
  static __device__ __forceinline__ type round(float x) { return __float_as_uint(x); }
};
template <>
struct Element<true> {
  using type = uint16_t;
  static __device__ __forceinline__ float value(type x) { return __uint_as_float((uint32_t)x << 16); }
  static __device__ __forceinline__ type round(float x) {
    return __builtin_bit_cast(uint16_t, (__bf16)x);
  }
};

__device__ __forceinline__ float param(const float *p, int b, float off, bool positive) {
  if (!p) return off;
  const float x = p[b];
  return isfinite(x) && (!positive || x > 0.f) ? x : off;
}

template <bool kBf16>
__global__ __launch_bounds__(kThreads) void adjust_kernel(AdjustArgs a, int32_t chunks,
                                                          int32_t rows_per_group) {
  using E = Element<kBf16>;
  using T = typename E::type;
  constexpr int kVec = 16 / sizeof(T);
  extern __shared__ uint32_t lds[];
  uint32_t *const count = lds;                                          // [kChunk]
  int32_t *const bias_at = reinterpret_cast<int32_t *>(lds + kChunk);   // [kChunk] with biases
  const int tid = threadIdx.x;
  const int group = blockIdx.x / chunks, chunk = blockIdx.x - group * chunks;
  const int c0 = chunk * kChunk, c1 = min(a.V, c0 + kChunk);
  const int n0 = group * rows_per_group, n1 = min(a.N, n0 + rows_per_group);
  int held = -1;                                                        // the row counted in LDS
  float rep = 1.f, freq = 0.f, pres = 0.f;
  for (int n = n0; n < n1; ++n) {
    int b = n, first = 0, nodes = 0;
    if (a.cu_rows) {
      b = wave_search(a.B, n, [&](int i) { return a.cu_rows[i]; });
      first = max(a.cu_rows[b], 0);
      nodes = min(a.cu_rows[b + 1], a.N) - first;
      if (n < first || n >= first + nodes) continue;                    // behind the last row
    }
    if (b != held) {
      held = b;
      rep = param(a.repetition, b, 1.f, true);
      freq = param(a.frequency, b, 0.f, false);
      pres = param(a.presence, b, 0.f, false);
      __syncthreads();
      for (int i = tid; i < kChunk; i += kThreads) count[i] = 0;
      if (a.bias_tokens)
        for (int i = tid; i < kChunk; i += kThreads) bias_at[i] = -1;
      __syncthreads();
      if (a.history) {
        const int32_t *h = a.history + (int64_t)b * a.history_stride;
        const int len = (int)min((int64_t)max(a.history_lens[b], 0), a.history_stride);
        const int prompt = a.prompt_lens ? a.prompt_lens[b] : 0;
        for (int t = tid; t < len; t += kThreads) {
          const int v = h[t];
          if (v < c0 || v >= c1) continue;
          if (t < prompt)
            atomicOr(&count[v - c0], kPrompt);
          else
            atomicAdd(&count[v - c0], 1u);
        }
      }
      if (a.bias_tokens)
        for (int e = a.cu_bias[b] + tid; e < a.cu_bias[b + 1]; e += kThreads) {
          const int v = a.bias_tokens[e];
          if (v >= c0 && v < c1) atomicMax(&bias_at[v - c0], e);        // the last one counts
        }
    }
    // the tokens on the way to node n
    auto path = [&](uint32_t step) {
      if (!a.draft_tokens) return;
      for (int j = tid; j < min(nodes, 64 * a.mask_words); j += kThreads) {
        if (!(a.tree_mask[(int64_t)n * a.mask_words + (j >> 6)] >> (j & 63) & 1)) continue;
        const int v = a.draft_tokens[first + j];
        if (v >= c0 && v < c1) atomicAdd(&count[v - c0], step);
      }
    };
    path(1u);
    __syncthreads();

    const T *in = static_cast<const T *>(a.logits) + n * a.row_stride;
    T *out = static_cast<T *>(a.out) + n * a.out_stride;
    const uint32_t *allowed = nullptr;
    if (a.allowed) {
      const int m = a.allowed_rows ? a.allowed_rows[n] : n;
      if (m >= 0 && m < a.num_allowed) allowed = a.allowed + (int64_t)m * a.allowed_stride;
    }
    // a logit's new bits, and whether they differ from the old ones
    auto adjust = [&](int v, T x, bool ok) {
      const uint32_t c = count[v - c0];
      const int at = a.bias_tokens ? bias_at[v - c0] : -1;
      if (!ok) return E::round(-INFINITY);
      if (c == 0 && at < 0) return x;
      float z = E::value(x);
      if (c) {
        z = z > 0.f ? z / rep : z * rep;
        const uint32_t times = c & ~kPrompt;
        if (times) z = z - freq * (float)times - pres;
      }
      if (at >= 0) z += a.bias_values[at];
      return E::round(z);
    };
    auto bit = [&](int v) { return !allowed || (allowed[v >> 5] >> (v & 31) & 1); };
    const int shift = (int)((reinterpret_cast<uintptr_t>(in + c0) / sizeof(T)) % kVec);
    const bool same = in == out;
    const bool aligned = (reinterpret_cast<uintptr_t>(out + c0) / sizeof(T)) % kVec == (unsigned)shift;
    for (int e = c0 - shift + tid * kVec; e < c1; e += kThreads * kVec) {
      if (aligned && e >= c0 && e + kVec <= c1) {
        if (same) {
          bool any = false;
#pragma unroll
          for (int i = 0; i < kVec; ++i)
            any |= count[e + i - c0] || (a.bias_tokens && bias_at[e + i - c0] >= 0) || !bit(e + i);
          if (!any) continue;
        }
        u32x4 w = *reinterpret_cast<const u32x4 *>(in + e);
        T x[kVec];
        __builtin_memcpy(x, &w, 16);
#pragma unroll
        for (int i = 0; i < kVec; ++i) x[i] = adjust(e + i, x[i], bit(e + i));
        __builtin_memcpy(&w, x, 16);
        *reinterpret_cast<u32x4 *>(out + e) = w;
      } else {
        for (int v = max(e, c0); v < min(e + kVec, c1); ++v) out[v] = adjust(v, in[v], bit(v));
      }
    }
    if (a.draft_tokens) {
      __syncthreads();
      path(~0u);                                                        // taken off again
    }
  }
}

}  // namespace

// Rows of logits that a workgroup takes: several where the rows of a tree share their history's
// counts and there are workgroups enough.
static int32_t adjust_rows(int32_t N, int32_t chunks, bool trees) {
  const int64_t items = (int64_t)N * chunks;
  return trees ? (int32_t)min((int64_t)16, max((int64_t)1, items / 2048)) : 1;
}

static int32_t adjust_chunks(int32_t V) { return (V + kChunk - 1) / kChunk; }

int64_t adjust_groups(int32_t N, int32_t V, bool trees) {
  const int32_t chunks = adjust_chunks(V);
  const int64_t rows = adjust_rows(N, chunks, trees);
  return (N + rows - 1) / rows * chunks;
}

hipError_t launch_adjust(const AdjustArgs &a, bool bf16, hipStream_t stream) {
  const int32_t chunks = adjust_chunks(a.V);
  const size_t lds = kChunk * (a.bias_tokens ? 8 : 4);
  const int32_t rows = adjust_rows(a.N, chunks, a.cu_rows != nullptr);
  const unsigned grid = (unsigned)adjust_groups(a.N, a.V, a.cu_rows != nullptr);
  if (bf16)
    adjust_kernel<true><<<grid, kThreads, lds, stream>>>(a, chunks, rows);
  else
    adjust_kernel<false><<<grid, kThreads, lds, stream>>>(a, chunks, rows);
  return hipGetLastError();
}

}  // namespace ra
