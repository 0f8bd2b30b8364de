// Logits before a token is drawn: penalties for repeated tokens, biases, and masks of the tokens
// that a grammar allows (token_logits_adjust).
//
// A workgroup takes a chunk of the vocabulary for some rows of logits. It counts the row's
// history in LDS, one word a logit of the chunk (bit 31: in the prompt, below it how often in
// the answer; whole numbers, so the order of the atomics does not matter), and the place of
// each token's last bias, then passes over the chunk once, 16 bytes a thread and load. The rows
// of one tree share the history's counts: the tokens of each node's path are added, and taken
// off with the next node's. (Where rows are not a multiple of 16 bytes apart, the logits' places in
// LDS shift from row to row and the history is counted anew for each.) All that a row needs is
// loaded while the row before is worked on.
//
// Logit z of a token that the history names, n times in the answer: z / rep where z > 0 and
// z rep elsewhere, then z - n freq - pres if n > 0, then z + bias; -inf where the mask forbids it.
// All in fp32; a bf16 result is rounded once.
//
// Bound by HBM: each logit read and written once (in place: only those that change), the
// history once for every chunk, mostly from the L2. Measured: one row of 32,000, 10.8 us a call
// (the launch and the host); 64 rows of 151,936 fp32 with 4k to 32k tokens each, in place 23 us,
// out of place 25 (3.1 TB/s), where the counting of the histories, 19 times from the L2, takes
// most of the time; 256 rows bf16 out of place 58 us; 700 rows in 32 trees, bf16, every
// adjustment, histories of 2k to 24k, 146 us (441 MB, 3.0 TB/s; a copy of as much would take 90),
// with histories of 100 to 500 123 us.
#include "ra_device.h"
#include "ra_internal.h"

namespace ra {
namespace {

constexpr int kThreads = 512;              // (1,024: no faster; 256: 23.5 -> 36 us for the 64 rows)
constexpr int kMaxRows = 32;               // of a workgroup (16: 2,457 rows of trees 477 us, 32: 463)
// Words of LDS for a chunk and the 16-byte unit it begins in: four workgroups of them a compute
// unit. (Twice as many halve how often a history is read, but fewer workgroups are on the
// unit: 64 rows of 151,936 36 -> 42 us when that was tried. 9,984, the most that leave four:
// 64 rows in place 23.5 -> 20.8, 256 rows 65 -> 72, 3,278 rows of 32,000 176 -> 190.)
constexpr int kSlots = 8192;
constexpr int kChunk = kSlots - 8;         // logits of a chunk
constexpr int kTogether = 512;             // workgroups of several rows that are on the GPU together
constexpr int kBatch = 4;                  // loads of four tokens that a thread has in flight
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

struct RowInfo {
  int b, first, nodes, mask;       // history row (-1: none), its first logits row, how many; grammar mask
};

// kMany: several rows of logits a workgroup, of trees; otherwise one, and twice the workgroups fit.
template <bool kBf16, bool kMany>
__global__ __launch_bounds__(kThreads, kMany ? 4 : 8) void adjust_kernel(AdjustArgs a, int32_t chunks,
                                                             int32_t rows_per_group) {
  using E = Element<kBf16>;
  using T = typename E::type;
  constexpr int kVec = 16 / sizeof(T);
  constexpr int kUnits = kSlots / kVec / kThreads;                      // of a thread, in a row
  extern __shared__ uint32_t lds[];
  uint32_t *const count = lds;                                          // [kSlots]
  int32_t *const bias_at = reinterpret_cast<int32_t *>(lds + kSlots);   // [kSlots] with biases
  __shared__ RowInfo info[kMaxRows];
  const int tid = threadIdx.x;
  // (the first chunk first: a vocabulary's low ids are its frequent tokens, and counting them
  // takes longest)
  const int groups = gridDim.x / chunks, chunk = blockIdx.x / groups, group = blockIdx.x - chunk * groups;
  const int c0 = chunk * kChunk, c1 = min(a.V, c0 + kChunk);
  const int n0 = group * rows_per_group, n1 = min(a.N, n0 + rows_per_group);
  const bool in_place = a.logits == a.out;
  if (tid < n1 - n0) {
    RowInfo r = {n0 + tid, 0, 0, -1};
    if (a.cu_rows) {
      int lo = 0, hi = a.B - 1;                                         // the last row that begins by then
      while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (a.cu_rows[mid] <= n0 + tid) lo = mid; else hi = mid - 1;
      }
      r.first = max(a.cu_rows[lo], 0);
      r.nodes = min(a.cu_rows[lo + 1], a.N) - r.first;
      r.b = n0 + tid >= r.first && n0 + tid < r.first + r.nodes ? lo : -1;
    }
    if (a.allowed) {
      const int m = a.allowed_rows ? a.allowed_rows[n0 + tid] : n0 + tid;
      if (m >= 0 && m < a.num_allowed) r.mask = m;
    }
    info[tid] = r;
  }
  __syncthreads();

  // What a row needs: whole units of its logits (those that the chunk begins or ends in go one
  // logit at a time), their bits of the mask, and the token that a thread has of its path.
  // LDS word i is that of logit c0 - shift + i: the chunk from the unit on that it begins in.
  struct Loads {
    u32x4 w[kUnits];
    uint32_t bits[kUnits][2];
    uint64_t path;
    int token;
  };
  auto shift_of = [&](int n) {
    const T *row = static_cast<const T *>(a.logits) + n * a.row_stride;
    return (int)((reinterpret_cast<uintptr_t>(row + c0) / sizeof(T)) % kVec);
  };
  auto load = [&](int n, Loads &l) __attribute__((always_inline)) {
    const RowInfo r = info[n - n0];
    const T *in = static_cast<const T *>(a.logits) + n * a.row_stride;
    const int e0 = c0 - shift_of(n);
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int e = e0 + (u * kThreads + tid) * kVec;
      if (e < c0 || e + kVec > c1) continue;
      if (!in_place) l.w[u] = *reinterpret_cast<const u32x4 *>(in + e);
      if (r.mask >= 0) {
        const uint32_t *row = a.allowed + (int64_t)r.mask * a.allowed_stride;
        l.bits[u][0] = row[e >> 5];
        l.bits[u][1] = row[(e + kVec - 1) >> 5];
      }
    }
    l.path = 0;
    if (a.draft_tokens && tid < min(r.nodes, 64 * a.mask_words)) {
      l.path = a.tree_mask[(int64_t)n * a.mask_words + (tid >> 6)];
      l.token = a.draft_tokens[r.first + tid];
    }
  };
  Loads next;
  load(n0, next);
  int held = -1, held_shift = 0;                                        // the row counted in LDS
  int path_row = -1, path_word = -1;                                    // the path counted with it
  float rep = 1.f, freq = 0.f, pres = 0.f;
  for (int n = n0; n < (kMany ? n1 : n0 + 1); ++n) {
    const Loads now = next;
    if constexpr (kMany)
      if (n + 1 < n1) load(n + 1, next);
    const RowInfo r = info[n - n0];
    if (r.b < 0) continue;                                              // behind the last row
    const T *in = static_cast<const T *>(a.logits) + n * a.row_stride;
    T *out = static_cast<T *>(a.out) + n * a.out_stride;
    const int shift = shift_of(n), e0 = c0 - shift;
    if (r.b != held || shift != held_shift) {
      held = r.b;
      held_shift = shift;
      path_row = -1;
      rep = param(a.repetition, r.b, 1.f, true);
      freq = param(a.frequency, r.b, 0.f, false);
      pres = param(a.presence, r.b, 0.f, false);
      __syncthreads();
      for (int i = tid; i < kSlots / 4; i += kThreads)
        reinterpret_cast<u32x4 *>(count)[i] = u32x4{0, 0, 0, 0};
      if (a.bias_tokens)
        for (int i = tid; i < kSlots / 4; i += kThreads)
          reinterpret_cast<u32x4 *>(bias_at)[i] = u32x4{~0u, ~0u, ~0u, ~0u};
      __syncthreads();
      if (a.history) {
        const int32_t *h = a.history + (int64_t)r.b * a.history_stride;
        const int len = min(max(a.history_lens[r.b], 0), a.history_width);
        const int prompt = min(max(a.prompt_lens ? a.prompt_lens[r.b] : 0, 0), len);
        const uint32_t size = c1 - c0;
        auto one = [&](int t, int v) {
          if ((uint32_t)(v - c0) >= size) return;
          if (t < prompt)
            atomicOr(&count[v - e0], kPrompt);
          else
            atomicAdd(&count[v - e0], 1u);
        };
        // four tokens a load, but for the first that are not aligned and the last
        const int head = min(len, (int)(-(reinterpret_cast<uintptr_t>(h) / 4) & 3));
        const int units = (len - head) / 4, tail = head + 4 * units;
        if (tid < head) one(tid, h[tid]);
        if (tid < len - tail) one(tail + tid, h[tail + tid]);
        for (int u0 = 0; u0 < units; u0 += kBatch * kThreads) {
          u32x4 v[kBatch];
#pragma unroll
          for (int i = 0; i < kBatch; ++i) {
            const int u = u0 + i * kThreads + tid;
            v[i] = u32x4{~0u, ~0u, ~0u, ~0u};
            if (u < units) v[i] = *reinterpret_cast<const u32x4 *>(h + head + 4 * u);
          }
#pragma unroll
          for (int i = 0; i < kBatch; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k)
              one(head + 4 * (u0 + i * kThreads + tid) + k, (int)v[i][k]);
        }
      }
      if (a.bias_tokens)
        for (int e = max(a.cu_bias[r.b], 0) + tid; e < min(a.cu_bias[r.b + 1], a.num_bias); e += kThreads) {
          const int v = a.bias_tokens[e];
          if (v >= c0 && v < c1) atomicMax(&bias_at[v - e0], e);        // the last one counts
        }
    } else if (a.draft_tokens) {
      __syncthreads();                                                  // the row before is done
    }
    if (a.draft_tokens) {
      // nodes that a thread has beside its own, of trees with more than kThreads
      auto others = [&](int m, uint32_t step) {
        for (int j = kThreads + tid; j < min(r.nodes, 64 * a.mask_words); j += kThreads) {
          if (!(a.tree_mask[(int64_t)m * a.mask_words + (j >> 6)] >> (j & 63) & 1)) continue;
          const int v = a.draft_tokens[r.first + j];
          if (v >= c0 && v < c1) atomicAdd(&count[v - e0], step);
        }
      };
      if (path_row >= 0) {                                              // (of the same tree)
        if (path_word >= 0) atomicAdd(&count[path_word], ~0u);
        others(path_row, ~0u);
      }
      path_word = now.path >> (tid & 63) & 1 && now.token >= c0 && now.token < c1 ? now.token - e0 : -1;
      if (path_word >= 0) atomicAdd(&count[path_word], 1u);
      others(n, 1u);
      path_row = n;
    }
    __syncthreads();

    const uint32_t *allowed = r.mask >= 0 ? a.allowed + (int64_t)r.mask * a.allowed_stride : nullptr;
    auto adjust = [&](T x, uint32_t c, int at, bool ok) {
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
    const bool aligned = (reinterpret_cast<uintptr_t>(out + c0) / sizeof(T)) % kVec == (unsigned)shift;
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      const int at = (u * kThreads + tid) * kVec, e = e0 + at;          // in LDS, and of the logits
      if (e >= c1) continue;
      if (!aligned || e < c0 || e + kVec > c1) {
        for (int v = max(e, c0); v < min(e + kVec, c1); ++v)
          out[v] = adjust(in[v], count[v - e0], a.bias_tokens ? bias_at[v - e0] : -1,
                          !allowed || (allowed[v >> 5] >> (v & 31) & 1));
        continue;
      }
      uint32_t c[kVec], some = 0;
      int32_t ba[kVec];
#pragma unroll
      for (int i = 0; i < kVec; i += 4) {
        const u32x4 w = *reinterpret_cast<const u32x4 *>(count + at + i);
        u32x4 x = {~0u, ~0u, ~0u, ~0u};
        if (a.bias_tokens) x = *reinterpret_cast<const u32x4 *>(bias_at + at + i);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          c[i + k] = w[k];
          ba[i + k] = (int32_t)x[k];
          some |= w[k] | ~x[k];
        }
      }
      constexpr uint32_t kAll = (1u << kVec) - 1;
      uint32_t ok = kAll;                                               // bits of the unit's logits
      if (allowed) {
        const uint64_t bits = (uint64_t)now.bits[u][1] << 32 | now.bits[u][0];
        ok = (e & 31) + kVec > 32 ? (uint32_t)(bits >> (e & 31)) & kAll : now.bits[u][0] >> (e & 31) & kAll;
      }
      const bool any = some != 0 || ok != kAll;
      if (in_place && !any) continue;
      u32x4 w = in_place ? *reinterpret_cast<const u32x4 *>(in + e) : now.w[u];
      if (any) {
        T x[kVec];
        __builtin_memcpy(x, &w, 16);
#pragma unroll
        for (int i = 0; i < kVec; ++i) x[i] = adjust(x[i], c[i], ba[i], ok >> i & 1);
        __builtin_memcpy(&w, x, 16);
      }
      *reinterpret_cast<u32x4 *>(out + e) = w;
    }
  }
}

}  // namespace

// Rows of logits that a workgroup takes: several where the rows of a tree share their history's
// counts, and as few as let the call end with whole rounds of workgroups, one if it can. bf16 rows
// of 151,936 in trees, with this rule, one a workgroup, and as many as leave 2,048 workgroups:
// 138 rows 36, 47 and 47 us; 318 rows 73, 98 and 92; 700 rows 146, 231 and 163.
static int32_t adjust_rows(int32_t N, int32_t chunks, bool trees) {
  if (!trees) return 1;
  const int64_t least = ((int64_t)N + kMaxRows - 1) / kMaxRows;         // groups of rows
  const int64_t rounds = (least * chunks + kTogether - 1) / kTogether;
  const int64_t groups = max((int64_t)1, rounds * kTogether / chunks);
  return (int32_t)max((int64_t)1, (N + groups - 1) / groups);
}

static int32_t adjust_chunks(int32_t V) { return (V + kChunk - 1) / kChunk; }

static int64_t adjust_groups(int32_t N, int32_t V, bool trees) {
  const int32_t chunks = adjust_chunks(V);
  const int64_t rows = adjust_rows(N, chunks, trees);
  return (N + rows - 1) / rows * chunks;
}

int64_t adjust_threads(int32_t N, int32_t V, bool trees) {
  return adjust_groups(N, V, trees) * kThreads;
}

hipError_t launch_adjust(const AdjustArgs &a, bool bf16, hipStream_t stream) {
  const int32_t chunks = adjust_chunks(a.V);
  const size_t lds = kSlots * (a.bias_tokens ? 8 : 4);
  const int32_t rows = adjust_rows(a.N, chunks, a.cu_rows != nullptr);
  const unsigned grid = (unsigned)adjust_groups(a.N, a.V, a.cu_rows != nullptr);
  if (bf16 && rows > 1)
    adjust_kernel<true, true><<<grid, kThreads, lds, stream>>>(a, chunks, rows);
  else if (bf16)
    adjust_kernel<true, false><<<grid, kThreads, lds, stream>>>(a, chunks, rows);
  else if (rows > 1)
    adjust_kernel<false, true><<<grid, kThreads, lds, stream>>>(a, chunks, rows);
  else
    adjust_kernel<false, false><<<grid, kThreads, lds, stream>>>(a, chunks, rows);
  return hipGetLastError();
}

}  // namespace ra
