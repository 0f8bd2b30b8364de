// Drawing a token from a row of logits (token_sample): temperature, top-k, top-p and min-p
// filters, then the inverse of the cumulative distribution at a given uniform number.
//
// With M the row's largest logit, an element's weight is e = exp((z - M) / T) in 64-bit
// floating point. Where weights are added up by atomics or in no fixed order they are whole
// numbers of 2^-44 (0 below half a unit, 31.2 below M), so that no order changes a sum:
// a sum of V weights is off by at most V half units, and a row's stays below 2^63 for
// V <= 2^19. The other sums are taken in a fixed order.
//
// All filters keep a prefix of the order (logit descending, index ascending), so what is
// sought is where it ends. Rows are cut into chunks, a workgroup each, in three passes, and
// a workgroup per row ends the call:
//   stats   each chunk's largest and smallest logit, and its sum of weights below its own
//           largest one (rows without filters, or with top-p alone)
//   bins    counts and weights by (M - z) / T in 512 bins over the range that can hold the
//           end (rows with top-k or top-p)
//   border  from the bins: the bin or bins that hold the end. What lies above is kept:
//           each chunk sums it; the elements in them are listed
//   pick    the listed elements sorted, the end found, the chunk of the drawn token from
//           the chunks' sums, the token from the chunk's elements
// Bound by the first pass's read of the logits (the others find them in the caches) and,
// for few rows, by the launches. Without filters stats and pick are the whole call.
#include "ra_device.h"
#include "ra_internal.h"

namespace ra {
namespace {

constexpr int kThreads = 256;           // of a chunk's workgroup
constexpr int kPickThreads = 1024;
constexpr int kBins = 512;
constexpr int kMaxChunks = 256;         // of a row
constexpr int kMaxSorted = 4096;        // listed elements that the pick sorts
constexpr double kUnit = 0x1p44;
constexpr double kRange = 31.5;         // weights end before this

typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

template <typename T>
constexpr int kVector = 16 / sizeof(T);   // logits of a load

__device__ __forceinline__ float logit_value(float x) { return x; }
__device__ __forceinline__ float logit_value(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }

// NaN counts as -inf.
__device__ __forceinline__ float clean(float z) { return z == z ? z : -__builtin_inff(); }

// Order of fp32 values as that of whole numbers; -0 as 0.
__device__ __forceinline__ uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}

// exp(x) for x <= 0 (0 below -kRange and for NaN): exp(x) = 2^n exp(r), |r| <= ln 2 / 2, by
// the Taylor series of exp(r) to r^12, whose next term is below 2^-52.
__device__ __forceinline__ double weight_exp(double x) {
  const double n = __builtin_rint(x * 1.4426950408889634);
  // ln 2 in two parts, the first of 38 bits: its products with n are exact
  const double r = __builtin_fma(n, -0x1.cf79abc9e3b3ap-40, __builtin_fma(n, -0x1.62e42fefap-1, x));
  double p = 1.0 / 479001600.0;
  p = __builtin_fma(p, r, 1.0 / 39916800.0);
  p = __builtin_fma(p, r, 1.0 / 3628800.0);
  p = __builtin_fma(p, r, 1.0 / 362880.0);
  p = __builtin_fma(p, r, 1.0 / 40320.0);
  p = __builtin_fma(p, r, 1.0 / 5040.0);
  p = __builtin_fma(p, r, 1.0 / 720.0);
  p = __builtin_fma(p, r, 1.0 / 120.0);
  p = __builtin_fma(p, r, 1.0 / 24.0);
  p = __builtin_fma(p, r, 1.0 / 6.0);
  p = __builtin_fma(p, r, 0.5);
  p = __builtin_fma(p, r, 1.0);
  p = __builtin_fma(p, r, 1.0);
  return x >= -kRange ? __builtin_ldexp(p, (int)n) : 0.0;
}

// (z - top) / T, <= 0; elements at top, an infinite one too, are at 0.
__device__ __forceinline__ double scaled(float z, float top, double inv_t) {
  return z == top ? 0.0 : ((double)z - (double)top) * inv_t;
}
__device__ __forceinline__ uint64_t units(double e) { return (uint64_t)(e * kUnit + 0.5); }

struct SampleArgs {
  const void *logits;
  const float *temperature;
  const int32_t *top_k;
  const float *top_p, *min_p, *uniform;
  int32_t *tokens;
  float *logprob;
  int64_t row_stride;
  int32_t N, V, chunks, per;            // elements of a chunk: kThreads * per
  // workspace
  float *c_top, *c_low;                 // [N][chunks] largest and smallest finite logit
  uint32_t *c_first;                    // [N][chunks] lowest index of the largest one
  double *c_sum;                        // [N][chunks] sum of weights against c_top
  uint64_t *bin_mass;                   // [N][kBins]
  uint32_t *bin_count;                  // [N][kBins]
  uint64_t *c_kept;                     // [N][chunks] weight kept for certain
  uint32_t *c_listed;                   // [N][chunks] elements in the border's bins
  uint32_t *c_keys;                     // [N][chunks][2] their largest and smallest key
  uint64_t *list;                       // [N][chunks][per * 8] key << 32 | ~index
  struct Border *border;                // [N]
};
__host__ __device__ constexpr int list_cap(int per) { return per * 8; }

// What a row asks for.
struct Row {
  double inv_t, p, m;                   // p < 1: top-p, m > 0: min-p
  int k;                                // 0: no top-k
  bool greedy;
  __device__ __forceinline__ Row(const SampleArgs &a, int n) {
    const float t = a.temperature ? a.temperature[n] : 1.f;
    greedy = !(t > 0.f);
    inv_t = 1.0 / (double)t;
    k = a.top_k ? a.top_k[n] : 0;
    if (k < 0 || k >= a.V) k = 0;
    const float tp = a.top_p ? a.top_p[n] : 1.f, mp = a.min_p ? a.min_p[n] : 0.f;
    p = tp < 1.f ? (double)tp : 1.0;
    m = mp > 0.f ? (double)fminf(mp, 1.f) : 0.0;
  }
  __device__ __forceinline__ bool binned() const { return !greedy && (k > 0 || p < 1.0); }
  __device__ __forceinline__ bool filtered() const { return binned() || (!greedy && m > 0.0); }
  __device__ __forceinline__ bool needs_sums() const {
    return !greedy && (!filtered() || (p < 1.0 && k == 0));
  }
};

// Where a row's kept prefix ends: bins before `lo` are kept; the end is in lo .. hi, or (no
// top-p) in bin_k = lo = hi; with top-k and top-p, what top-k keeps of bin_k also decides.
struct Border {
  double inv_t, bin_scale, sum;         // bins an exp, sum of the weights (top-p alone)
  float top;
  int lo, hi, bin_k;                    // kBins: none
  uint32_t count_lo, count_k;           // elements before bin lo, bin_k
  uint64_t mass_lo, mass_k, mass_all;   // weights before them; of all bins
};

// The bin of a logit: non-decreasing as z falls. kBins: beyond.
__device__ __forceinline__ int bin_of(double x, double bin_scale) {
  const double b = -x * bin_scale;
  return b < kBins ? (int)b : kBins;
}

// ---- reductions over a workgroup, in a fixed order ----
template <typename V, typename Op>
__device__ __forceinline__ V wave_reduce(V x, Op op) {
#pragma unroll
  for (int d = kWave / 2; d > 0; d /= 2) x = op(x, __shfl_xor(x, d));
  return x;
}
template <int kN, typename V, typename Op>
__device__ __forceinline__ V group_reduce(V x, Op op, V *part) {
  x = wave_reduce(x, op);
  __syncthreads();
  if (threadIdx.x % kWave == 0) part[threadIdx.x / kWave] = x;
  __syncthreads();
  x = part[0];
#pragma unroll
  for (int w = 1; w < kN / kWave; ++w) x = op(x, part[w]);
  return x;
}
// Sums of the threads before this one; total for all.
template <int kN, typename V>
__device__ __forceinline__ V group_scan(V x, V &total, V *part) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  V s = x;
#pragma unroll
  for (int d = 1; d < kWave; d *= 2) {
    const V y = __shfl_up(s, d);
    if (lane >= d) s += y;
  }
  __syncthreads();
  if (lane == kWave - 1) part[wave] = s;
  __syncthreads();
  V before = 0;
  total = 0;
  for (int w = 0; w < kN / kWave; ++w) {
    if (w == wave) before = total;
    total += part[w];
  }
  return before + (s - x);
}

__device__ __forceinline__ float max_of(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float min_of(float a, float b) { return fminf(a, b); }

// Chunk c's logits of a thread: vectors tid, tid + kThreads, ...; -inf past the row.
template <typename T, int kPer>
__device__ __forceinline__ void load_chunk(const SampleArgs &a, int n, int c, float (&z)[kPer]) {
  constexpr int kVec = kVector<T>;
  const T *row = static_cast<const T *>(a.logits) + n * a.row_stride;
#pragma unroll
  for (int j = 0; j < kPer / kVec; ++j) {
    const int v0 = c * kThreads * kPer + (j * kThreads + threadIdx.x) * kVec;
    if (v0 + kVec <= a.V) {
      const u32x4_any w = *reinterpret_cast<const u32x4_any *>(row + v0);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        if constexpr (sizeof(T) == 4)
          z[j * kVec + e] = __uint_as_float(w[e]);
        else
          z[j * kVec + e] = __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
      }
    } else {
#pragma unroll
      for (int e = 0; e < kVec; ++e)
        z[j * kVec + e] = v0 + e < a.V ? logit_value(row[v0 + e]) : -__builtin_inff();
    }
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) z[i] = clean(z[i]);
}
// The index of a thread's i-th logit.
template <typename T, int kPer>
__device__ __forceinline__ int index_of(int c, int i) {
  constexpr int kVec = kVector<T>;
  return c * kThreads * kPer + (i / kVec * kThreads + threadIdx.x) * kVec + i % kVec;
}

template <typename T, int kPer>
__global__ __launch_bounds__(kThreads) void sample_stats_kernel(SampleArgs a) {
  const int n = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks, tid = threadIdx.x;
  __shared__ float part[kThreads / kWave];
  __shared__ double dpart[kThreads / kWave];
  __shared__ int ipart[kThreads / kWave];
  float z[kPer];
  load_chunk<T, kPer>(a, n, c, z);
  const Row row(a, n);
  float top = z[0], low = __builtin_inff();
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    top = fmaxf(top, z[i]);
    low = z[i] > -__builtin_inff() ? fminf(low, z[i]) : low;
  }
  top = group_reduce<kThreads>(top, max_of, part);
  const int64_t at = (int64_t)n * a.chunks + c;
  if (row.greedy) {
    int first = a.V;
#pragma unroll
    for (int i = kPer - 1; i >= 0; --i) first = z[i] == top ? index_of<T, kPer>(c, i) : first;
    first = group_reduce<kThreads>(first, [](int x, int y) { return min(x, y); }, ipart);
    if (tid == 0) a.c_first[at] = first;
  } else if (row.binned()) {
    low = group_reduce<kThreads>(low, min_of, part);
    if (tid == 0) a.c_low[at] = low;
    // the row's bins start at zero
    for (int i = c * kThreads + tid; i < kBins; i += a.chunks * kThreads) {
      a.bin_mass[(int64_t)n * kBins + i] = 0;
      a.bin_count[(int64_t)n * kBins + i] = 0;
    }
  }
  if (row.needs_sums()) {
    double sum = 0.0;
    if (top > -__builtin_inff())
#pragma unroll
      for (int i = 0; i < kPer; ++i) sum += weight_exp(scaled(z[i], top, row.inv_t));
    sum = group_reduce<kThreads>(sum, [](double x, double y) { return x + y; }, dpart);
    if (tid == 0) a.c_sum[at] = sum;
  }
  if (tid == 0) a.c_top[at] = top;
}

// The row's largest logit, from its chunks'.
template <int kN>
__device__ __forceinline__ float row_top(const SampleArgs &a, int n, float *part) {
  const int64_t at = (int64_t)n * a.chunks;
  const float x = threadIdx.x < a.chunks ? a.c_top[at + threadIdx.x] : -__builtin_inff();
  return group_reduce<kN>(x, max_of, part);
}

// The bins' range and, for top-p alone, the sum of all weights.
__device__ __forceinline__ void row_range(const SampleArgs &a, int n, const Row &row, Border &b,
                                          float *part, double *dpart) {
  const int64_t at = (int64_t)n * a.chunks;
  const int tid = threadIdx.x;
  b.inv_t = row.inv_t;
  b.top = row_top<kThreads>(a, n, part);
  const float low = group_reduce<kThreads>(tid < a.chunks ? a.c_low[at + tid] : __builtin_inff(),
                                           min_of, part);
  double range = fmin(kRange, -scaled(fminf(low, b.top), b.top, row.inv_t));
  b.sum = 0.0;
  if (row.needs_sums()) {
    double x = 0.0;
    if (tid < a.chunks)
      x = a.c_sum[at + tid] * weight_exp(scaled(a.c_top[at + tid], b.top, row.inv_t));
    b.sum = group_reduce<kThreads>(x, [](double u, double v) { return u + v; }, dpart);
    // elements lighter than (1 - p) sum / V weigh less than (1 - p) sum together: the end
    // lies before them
    if (row.p > 0.0) range = fmin(range, log((double)a.V / ((1.0 - row.p) * b.sum)) + 1e-3);
  }
  // the last element falls into the last bin
  b.bin_scale = kBins / (fmax(range, 1e-30) * (1.0 + 1e-9));
}

template <typename T, int kPer>
__global__ __launch_bounds__(kThreads) void sample_bins_kernel(SampleArgs a) {
  const int n = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks, tid = threadIdx.x;
  const Row row(a, n);
  if (!row.binned()) return;
  __shared__ float part[kThreads / kWave];
  __shared__ double dpart[kThreads / kWave];
  __shared__ uint64_t mass[kBins];
  __shared__ uint32_t count[kBins];
  float z[kPer];
  load_chunk<T, kPer>(a, n, c, z);
  for (int i = tid; i < kBins; i += kThreads) mass[i] = 0, count[i] = 0;
  Border b;
  row_range(a, n, row, b, part, dpart);   // barriers: the bins are clear
  if (b.top == -__builtin_inff()) return;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const double x = scaled(z[i], b.top, b.inv_t);
    const int bin = bin_of(x, b.bin_scale);
    if (bin < kBins) {
      if (row.k > 0) atomicAdd(&count[bin], 1u);
      if (row.p < 1.0) atomicAdd((unsigned long long *)&mass[bin], (unsigned long long)units(weight_exp(x)));
    }
  }
  __syncthreads();
  for (int i = tid; i < kBins; i += kThreads) {
    if (count[i]) atomicAdd(&a.bin_count[(int64_t)n * kBins + i], count[i]);
    if (mass[i])
      atomicAdd((unsigned long long *)&a.bin_mass[(int64_t)n * kBins + i], (unsigned long long)mass[i]);
  }
}

// The end's bins, from the row's bins.
__device__ __forceinline__ void find_border(const SampleArgs &a, int n, const Row &row, Border &b,
                                            uint64_t *mpart, uint32_t *cpart, Border *shared) {
  static_assert(kBins == 2 * kThreads, "two bins a thread");
  const int tid = threadIdx.x;
  const int64_t at = (int64_t)n * kBins + 2 * tid;
  uint64_t m0 = a.bin_mass[at], m1 = a.bin_mass[at + 1], mass_all;
  uint32_t c0 = a.bin_count[at], c1 = a.bin_count[at + 1], count_all;
  const uint64_t mass_before = group_scan<kThreads>(m0 + m1, mass_all, mpart);
  const uint32_t count_before = group_scan<kThreads>(c0 + c1, count_all, cpart);
  if (tid == 0) {
    shared->lo = shared->hi = shared->bin_k = kBins;
    shared->count_lo = shared->count_k = 0;
    shared->mass_lo = shared->mass_k = mass_all;
    shared->mass_all = mass_all;
  }
  __syncthreads();
  // bin_k: where the count reaches k
  if (row.k > 0) {
    const uint32_t k = (uint32_t)row.k;
    if (count_before < k && count_before + c0 + c1 >= k) {
      const bool second = count_before + c0 < k;
      shared->bin_k = 2 * tid + second;
      shared->count_k = count_before + (second ? c0 : 0);
      shared->mass_k = mass_before + (second ? m0 : 0);
      if (!(row.p < 1.0)) {
        shared->lo = shared->hi = shared->bin_k;
        shared->count_lo = shared->count_k;
      }
    }
    __syncthreads();
  }
  // lo, hi: where the weight reaches p of the least and of the most that top-k can keep
  if (row.p < 1.0) {
    const int bin_k = shared->bin_k;
    double least, most;
    if (row.k > 0) {
      least = (double)shared->mass_k;
      most = least + (bin_k < kBins ? (double)a.bin_mass[(int64_t)n * kBins + bin_k] : 0.0);
    } else {
      least = most = b.sum * kUnit;
    }
    least = fmax(row.p * least, 0.5);
    most = fmax(row.p * most, 0.5);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint64_t before = mass_before + (i ? m0 : 0), after = before + (i ? m1 : m0);
      if ((double)before < least && !((double)after < least) && 2 * tid + i <= bin_k) {
        shared->lo = 2 * tid + i;
        shared->mass_lo = before;
        shared->count_lo = count_before + (i ? c0 : 0);
      }
      if ((double)before < most && !((double)after < most) && 2 * tid + i <= bin_k)
        shared->hi = 2 * tid + i;
    }
    __syncthreads();
    // rounding aside the weight reaches it no later than in bin_k
    if (tid == 0) {
      if (shared->lo == kBins && bin_k < kBins) {
        shared->lo = bin_k;
        shared->mass_lo = shared->mass_k;
        shared->count_lo = shared->count_k;
      }
      if (shared->hi == kBins) shared->hi = bin_k;
    }
  }
  __syncthreads();
  const double inv_t = b.inv_t, bin_scale = b.bin_scale, sum = b.sum;
  const float top = b.top;
  b = *shared;
  b.inv_t = inv_t, b.bin_scale = bin_scale, b.sum = sum, b.top = top;
}

template <typename T, int kPer>
__global__ __launch_bounds__(kThreads) void sample_border_kernel(SampleArgs a) {
  const int n = blockIdx.x / a.chunks, c = blockIdx.x % a.chunks, tid = threadIdx.x;
  const Row row(a, n);
  if (!row.filtered()) return;
  __shared__ float part[kThreads / kWave];
  __shared__ double dpart[kThreads / kWave];
  __shared__ uint64_t mpart[kThreads / kWave];
  __shared__ uint32_t cpart[kThreads / kWave];
  __shared__ Border shared;
  __shared__ uint32_t listed, key_high, key_low;
  float z[kPer];
  load_chunk<T, kPer>(a, n, c, z);
  if (tid == 0) listed = 0, key_high = 0, key_low = 0xffffffffu;
  Border b;
  if (row.binned()) {
    row_range(a, n, row, b, part, dpart);
    find_border(a, n, row, b, mpart, cpart, &shared);
  } else {
    b = Border();
    b.inv_t = row.inv_t;
    b.top = row_top<kThreads>(a, n, part);
    b.lo = b.hi = b.bin_k = kBins;
  }
  __syncthreads();
  if (b.top == -__builtin_inff()) return;
  const int64_t at = (int64_t)n * a.chunks + c;
  uint64_t *list = a.list + at * list_cap(kPer);
  uint64_t kept = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const double x = scaled(z[i], b.top, b.inv_t);
    if (!(x >= -kRange)) continue;
    const int bin = row.binned() ? bin_of(x, b.bin_scale) : 0;
    if (bin < b.lo) {
      const double e = weight_exp(x);
      if (e >= row.m) kept += units(e);
    } else if (bin < kBins && (bin <= b.hi || bin == b.bin_k)) {
      const uint32_t slot = atomicAdd(&listed, 1u), key = key_of(z[i]);
      if (slot < (uint32_t)list_cap(kPer))
        list[slot] = (uint64_t)key << 32 | (uint32_t)~index_of<T, kPer>(c, i);
      atomicMax(&key_high, key);
      atomicMin(&key_low, key);
    }
  }
  kept = group_reduce<kThreads>(kept, [](uint64_t x, uint64_t y) { return x + y; }, mpart);
  if (tid == 0) {
    a.c_kept[at] = kept;
    a.c_listed[at] = listed;
    a.c_keys[2 * at] = key_high;
    a.c_keys[2 * at + 1] = key_low;
    if (c == 0) a.border[n] = b;
  }
}

// ---- pick -----------------------------------------------------------------------------
template <typename T>
__global__ __launch_bounds__(kPickThreads) void sample_pick_kernel(SampleArgs a) {
  const int n = blockIdx.x, tid = threadIdx.x;
  const T *logits = static_cast<const T *>(a.logits) + n * a.row_stride;
  __shared__ float part[kPickThreads / kWave];
  __shared__ double dpart[kPickThreads / kWave];
  __shared__ uint64_t mpart[kPickThreads / kWave];
  __shared__ uint32_t cpart[kPickThreads / kWave];
  __shared__ uint64_t sorted[kMaxSorted];        // the listed elements, or 256 bins of a pass
  __shared__ uint64_t kept_of[kMaxChunks];       // weight kept of each chunk
  __shared__ uint32_t ties_of[kMaxChunks];       // of each chunk: elements at the edge
  __shared__ uint64_t s_mass, s_sum;
  __shared__ uint32_t s_key, s_count, s_ties;
  __shared__ int s_chunk, s_token;
  __shared__ double s_before;

  const Row row(a, n);
  const int64_t at = (int64_t)n * a.chunks;
  const float top = row_top<kPickThreads>(a, n, part);
  if (top == -__builtin_inff()) {
    if (tid == 0) {
      a.tokens[n] = -1;
      if (a.logprob) a.logprob[n] = __builtin_nanf("");
    }
    return;
  }
  if (row.greedy) {
    int first = tid < a.chunks && a.c_top[at + tid] == top ? (int)a.c_first[at + tid] : a.V;
    first = group_reduce<kPickThreads>(first, [](int x, int y) { return min(x, y); }, (int *)cpart);
    if (tid == 0) {
      a.tokens[n] = first;
      if (a.logprob) a.logprob[n] = 0.f;
    }
    return;
  }
  float u = a.uniform[n];
  u = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
  const int chunk_len = kThreads * a.per;

  // the prefix's end: keys above `edge`, and of those at it the first `ties` by index
  // (tie_index: those up to this index)
  uint32_t edge = 0, tie_index = 0xffffffffu;
  uint64_t ties = ~0ull;                          // counted over the row; ~0: by tie_index
  Border b = Border();
  double total;
  if (!row.filtered()) {
    double x = 0.0;
    if (tid < a.chunks)
      x = a.c_sum[at + tid] * weight_exp(scaled(a.c_top[at + tid], top, row.inv_t));
    const double before = group_scan<kPickThreads>(x, total, dpart);
    const double goal = (double)u * total;
    if (tid == 0) s_chunk = -1;
    __syncthreads();
    // the last chunk whose sums begin at or before the goal and that weighs anything
    if (x > 0.0 && before <= goal) atomicMax(&s_chunk, tid);
    __syncthreads();
    if (tid == s_chunk) s_before = before;
    __syncthreads();
  } else {
    b = a.border[n];
    const uint32_t mine = tid < a.chunks ? a.c_listed[at + tid] : 0;
    const uint32_t high = tid < a.chunks && mine ? a.c_keys[2 * (at + tid)] : 0;
    const uint32_t low = tid < a.chunks && mine ? a.c_keys[2 * (at + tid) + 1] : 0xffffffffu;
    const uint32_t cap = list_cap(a.per);
    uint32_t count;
    const uint32_t first = group_scan<kPickThreads>(mine, count, cpart);
    auto umax = [](uint32_t x, uint32_t y) { return x > y ? x : y; };
    auto umin = [](uint32_t x, uint32_t y) { return x < y ? x : y; };
    const uint32_t key_high = group_reduce<kPickThreads>(high, umax, cpart);
    const uint32_t key_low = group_reduce<kPickThreads>(low, umin, cpart);
    const uint32_t longest = group_reduce<kPickThreads>(mine, umax, cpart);
    if (tid < kMaxChunks) {
      kept_of[tid] = tid < a.chunks ? a.c_kept[at + tid] : 0;
      ties_of[tid] = mine;
    }
    auto weight_of = [&](uint32_t key) { return weight_exp(scaled(value_of(key), top, row.inv_t)); };
    // the sum that top-p takes its share of, given what bin_k's listed elements add
    auto goal_of = [&](uint64_t of_bin_k) {
      const double z = row.k > 0 ? (double)(b.mass_k + of_bin_k) : b.sum * kUnit;
      return fmax(row.p * z, 0.5);
    };
    // the first r of `avail` equal elements of weight w, `before` ahead of them, that the
    // goal lets in
    auto ties_in = [](double goal, uint64_t before, uint64_t w, uint64_t avail) -> uint64_t {
      if (!((double)before < goal)) return 0;
      if (w == 0) return avail;
      const double r = __builtin_ceil((goal - (double)before) / (double)w);
      return r < 1.0 ? 1 : r >= (double)avail ? avail : (uint64_t)r;
    };
    __syncthreads();
    if (count == 0) {
      // everything in the bins is kept (min-p alone: everything)
      if (row.binned()) edge = 0xffffffffu;
    } else if (key_high == key_low) {
      // equal elements, however many
      edge = key_high;
      ties = count;
      const uint64_t w = units(weight_of(edge));
      const bool in_k = row.k > 0 && b.bin_k < kBins;
      if (in_k) ties = (uint64_t)row.k - b.count_k < ties ? (uint64_t)row.k - b.count_k : ties;
      if (row.p < 1.0) ties = ties_in(goal_of(in_k ? ties * w : 0), b.mass_lo, w, ties);
      if (tid < a.chunks) {
        const uint64_t left = ties > first ? ties - first : 0;
        if (weight_of(edge) >= row.m) kept_of[tid] += (left < mine ? left : mine) * w;
      }
    } else if (count <= kMaxSorted && longest <= cap) {
      // sort them, heaviest and then lowest index first
      for (int c = tid / kWave; c < a.chunks; c += kPickThreads / kWave) {
        const uint32_t m = a.c_listed[at + c];
        uint32_t to = 0;
        for (int i = tid % kWave; i < c; i += kWave) to += ties_of[i];
        to = wave_reduce(to, [](uint32_t x, uint32_t y) { return x + y; });
        for (uint32_t i = tid % kWave; i < m; i += kWave) sorted[to + i] = a.list[(at + c) * cap + i];
      }
      int size = 64;
      while (size < (int)count) size *= 2;
      for (int i = count + tid; i < size; i += kPickThreads) sorted[i] = 0;
      __syncthreads();
      for (int len = 2; len <= size; len *= 2)
        for (int step = len / 2; step > 0; step /= 2) {
          for (int i = tid; i < size / 2; i += kPickThreads) {
            const int lo = i / step * 2 * step + i % step, hi = lo + step;
            const uint64_t x = sorted[lo], y = sorted[hi];
            if ((x < y) == ((lo & len) == 0)) sorted[lo] = y, sorted[hi] = x;
          }
          __syncthreads();
        }
      // four neighbouring elements a thread: their weights, and the sums before them
      constexpr int kOwn = kMaxSorted / kPickThreads;
      uint64_t w[kOwn], own = 0, of_k = 0, in_p = 0;
      int bin[kOwn];
#pragma unroll
      for (int j = 0; j < kOwn; ++j) {
        const int i = tid * kOwn + j;
        w[j] = 0, bin[j] = kBins;
        if (i < (int)count) {
          const double x = scaled(value_of((uint32_t)(sorted[i] >> 32)), top, row.inv_t);
          w[j] = units(weight_exp(x));
          bin[j] = bin_of(x, b.bin_scale);
          in_p += bin[j] <= b.hi;
        }
        own += w[j];
      }
      uint64_t all, before = group_scan<kPickThreads>(own, all, mpart);
      // listed elements of bins lo .. hi come first; with both filters bin_k may lie behind
      const uint64_t n_p = group_reduce<kPickThreads>(in_p, [](uint64_t x, uint64_t y) { return x + y; }, mpart);
      const bool both = row.k > 0 && row.p < 1.0 && b.bin_k < kBins;
      // the rank of the i-th in the row's order, as far as top-k asks
      auto rank_of = [&](int i, int bin_i) -> uint64_t {
        return bin_i == b.bin_k && b.bin_k > b.hi ? (uint64_t)b.count_k + (i - n_p)
                                                  : (uint64_t)b.count_lo + i;
      };
#pragma unroll
      for (int j = 0; j < kOwn; ++j)
        if (both && bin[j] == b.bin_k && rank_of(tid * kOwn + j, bin[j]) < (uint64_t)row.k) of_k += w[j];
      of_k = group_reduce<kPickThreads>(of_k, [](uint64_t x, uint64_t y) { return x + y; }, mpart);
      const double goal = row.p < 1.0 ? goal_of(of_k) : 0.0;
      if (tid == 0) s_count = 0;
      __syncthreads();
      uint64_t run = before;
#pragma unroll
      for (int j = 0; j < kOwn; ++j) {
        const int i = tid * kOwn + j;
        if (i < (int)count && bin[j] <= b.hi &&
            !(row.k > 0 && b.bin_k < kBins && rank_of(i, bin[j]) >= (uint64_t)row.k) &&
            !(row.p < 1.0 && !((double)(b.mass_lo + run) < goal))) {
          atomicMax(&s_count, (uint32_t)i + 1);     // kept: a prefix of the sorted elements
          const uint32_t v = ~(uint32_t)sorted[i];
          if (weight_of((uint32_t)(sorted[i] >> 32)) >= row.m)
            atomicAdd((unsigned long long *)&kept_of[v / chunk_len], (unsigned long long)w[j]);
        }
        run += w[j];
      }
      __syncthreads();
      if (s_count == 0) {
        edge = 0xffffffffu, tie_index = 0;          // none of them
      } else {
        edge = (uint32_t)(sorted[s_count - 1] >> 32);
        tie_index = ~(uint32_t)sorted[s_count - 1];
      }
    } else {
      // too many: the edge by eight bits of the key a pass over the row, first that of
      // top-k, then that of top-p among what top-k keeps
      uint64_t *mass = sorted;
      uint32_t *counts = reinterpret_cast<uint32_t *>(sorted + 256);
      ties = ~0ull >> 1;
      for (int round = 0; round < 2; ++round) {
        const bool by_mass = round == 1;
        if (by_mass ? !(row.p < 1.0) : !(row.k > 0)) continue;
        double goal = 0.0;
        if (by_mass) {
          // the weight that top-k keeps
          uint64_t sum = 0, equal = 0;
          for (int v = tid; v < a.V; v += kPickThreads) {
            const uint32_t key = key_of(clean(logit_value(logits[v])));
            if (key > edge) sum += units(weight_of(key));
            equal += key == edge;
          }
          auto add = [](uint64_t x, uint64_t y) { return x + y; };
          sum = group_reduce<kPickThreads>(sum, add, mpart);
          equal = group_reduce<kPickThreads>(equal, add, mpart);
          if (edge) sum += (equal < ties ? equal : ties) * units(weight_of(edge));
          goal = fmax(row.p * (row.k > 0 ? (double)sum : b.sum * kUnit), 0.5);
        }
        uint32_t prefix = 0;
        uint64_t ahead = 0;
        for (int shift = 24; shift >= 0; shift -= 8) {
          __syncthreads();
          if (tid < 256) mass[tid] = 0, counts[tid] = 0;
          __syncthreads();
          for (int v = tid; v < a.V; v += kPickThreads) {
            const uint32_t key = key_of(clean(logit_value(logits[v])));
            if (shift < 24 && key >> (shift + 8) != prefix >> (shift + 8)) continue;
            if (key < edge) continue;
            if (by_mass)
              atomicAdd((unsigned long long *)&mass[key >> shift & 255],
                        (unsigned long long)units(weight_of(key)));
            atomicAdd(&counts[key >> shift & 255], 1u);
          }
          __syncthreads();
          if (tid == 0) {
            uint64_t run = ahead;
            int i = 255;
            for (; i > 0; --i) {
              const uint64_t next = run + (by_mass ? mass[i] : (uint64_t)counts[i]);
              if (by_mass ? !((double)next < goal) : next >= (uint64_t)row.k) break;
              run = next;
            }
            s_key = prefix | (uint32_t)i << shift;
            s_sum = run;
            s_ties = counts[i];
          }
          __syncthreads();
          prefix = s_key;
          ahead = s_sum;
        }
        uint64_t r = (uint64_t)row.k - ahead;
        if (by_mass) {
          r = ties_in(goal, ahead, units(weight_of(prefix)), s_ties);
          if (prefix == edge && r > ties) r = ties;
        }
        edge = prefix;
        ties = r;
        __syncthreads();
      }
      // each chunk's elements at the edge, then what it keeps, a wave a chunk
      for (int c = tid / kWave; c < a.chunks; c += kPickThreads / kWave) {
        uint32_t equal = 0;
        const int end = min(a.V, (c + 1) * chunk_len);
        for (int v = c * chunk_len + tid % kWave; v < end; v += kWave)
          equal += key_of(clean(logit_value(logits[v]))) == edge;
        equal = wave_reduce(equal, [](uint32_t x, uint32_t y) { return x + y; });
        if (tid % kWave == 0) ties_of[c] = equal;
      }
      __syncthreads();
      for (int c = tid / kWave; c < a.chunks; c += kPickThreads / kWave) {
        uint64_t ahead = 0, sum = 0;
        for (int i = 0; i < c; ++i) ahead += ties_of[i];
        const int end = min(a.V, (c + 1) * chunk_len);
        for (int v = c * chunk_len + tid % kWave; v < end; v += kWave) {
          const uint32_t key = key_of(clean(logit_value(logits[v])));
          const double e = weight_of(key);
          if (key > edge && e >= row.m) sum += units(e);
        }
        sum = wave_reduce(sum, [](uint64_t x, uint64_t y) { return x + y; });
        const uint64_t left = ties > ahead ? ties - ahead : 0;
        if (tid % kWave == 0) {
          const double e = weight_of(edge);
          kept_of[c] = sum + (e >= row.m ? (left < ties_of[c] ? left : ties_of[c]) * units(e) : 0);
        }
      }
      b.lo = -1;                                     // the bins say nothing
    }
    __syncthreads();
    // the chunk of the draw
    const uint64_t x = tid < a.chunks ? kept_of[tid] : 0;
    uint64_t sum;
    const uint64_t before = group_scan<kPickThreads>(x, sum, mpart);
    total = (double)sum;
    const double goal = (double)u * total;
    if (tid == 0) s_chunk = -1;
    __syncthreads();
    if (x > 0 && (double)before <= goal) atomicMax(&s_chunk, tid);
    __syncthreads();
    if (tid == s_chunk) s_mass = before;
    __syncthreads();
  }

  // the draw within the chunk: neighbouring elements a thread
  const int c = s_chunk, per = chunk_len / kPickThreads;
  const double goal = (double)u * total;
  const int v0 = c * chunk_len + tid * per;
  uint64_t tie0 = 0;
  if (ties != ~0ull) {
    uint64_t equal = 0, unused;
    for (int i = 0; i < per; ++i)
      equal += v0 + i < a.V && key_of(clean(logit_value(logits[v0 + i]))) == edge;
    tie0 = group_scan<kPickThreads>(equal, unused, mpart);
    for (int i = 0; i < c; ++i) tie0 += ties_of[i];
  }
  auto weight_at = [&](int v, uint64_t &seen, double &x) -> double {
    const float z = clean(logit_value(logits[v]));
    x = scaled(z, top, row.inv_t);
    if (row.filtered()) {
      const uint32_t key = key_of(z);
      const bool tied = key == edge && (ties == ~0ull ? (uint32_t)v <= tie_index : seen++ < ties);
      const bool sure = b.lo >= 0 && (!row.binned() || bin_of(x, b.bin_scale) < b.lo);
      if (!(key > edge || tied || sure)) return 0.0;
    }
    const double e = weight_exp(x);
    if (e < row.m) return 0.0;
    return row.filtered() ? (double)units(e) : e;
  };
  double own = 0.0, x, unused;
  uint64_t seen = tie0;
  for (int i = 0; i < per; ++i)
    if (v0 + i < a.V) own += weight_at(v0 + i, seen, x);
  const double start = row.filtered() ? (double)s_mass : s_before;
  const double before = start + group_scan<kPickThreads>(own, unused, dpart);
  if (tid == 0) s_token = -1;
  __syncthreads();
  // the first element whose running sum passes the goal; should rounding leave none, the
  // last that weighs anything
  int token = -1;
  bool past = false;
  double run = before;
  seen = tie0;
  for (int i = 0; i < per && !past; ++i) {
    if (v0 + i >= a.V) break;
    const double w = weight_at(v0 + i, seen, x);
    run += w;
    if (w > 0.0) token = v0 + i;
    past = w > 0.0 && run > goal;
  }
  if (token >= 0 && before <= goal) atomicMax(&s_token, token);
  __syncthreads();
  if (tid == 0) {
    const int t = s_token;
    a.tokens[n] = t;
    if (a.logprob)
      a.logprob[n] = (float)(scaled(clean(logit_value(logits[t])), top, row.inv_t) -
                             log(row.filtered() ? total / kUnit : total));
  }
}

// Elements a thread holds of a chunk: 32 (chunks of 8,192); 8 where the call has too few
// chunks of that size to fill the GPU, the rows still fit kMaxChunks and a load is one.
int32_t sample_per(int32_t N, int32_t V) {
  const int64_t chunks = ((int64_t)V + kThreads * 32 - 1) / (kThreads * 32) * N;
  return chunks < 512 ? 8 : 32;
}

struct SampleLayout {
  int32_t per, chunks;
  size_t c_top, c_low, c_first, c_sum, bin_mass, bin_count, c_kept, c_listed, c_keys, list, border;
  size_t bytes;
};
SampleLayout sample_layout(int32_t N, int32_t V) {
  SampleLayout l;
  l.per = sample_per(N, V);
  l.chunks = (V + kThreads * l.per - 1) / (kThreads * l.per);
  const size_t parts = (size_t)N * l.chunks;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  l.c_top = take(parts * 4);
  l.c_low = take(parts * 4);
  l.c_first = take(parts * 4);
  l.c_sum = take(parts * 8);
  l.bin_mass = take((size_t)N * kBins * 8);
  l.bin_count = take((size_t)N * kBins * 4);
  l.c_kept = take(parts * 8);
  l.c_listed = take(parts * 4);
  l.c_keys = take(parts * 8);
  l.list = take(parts * list_cap(l.per) * 8);
  l.border = take((size_t)N * sizeof(Border));
  l.bytes = at;
  return l;
}

template <typename T, int kPer>
void launch_passes(const SampleArgs &a, hipStream_t stream) {
  const dim3 grid((unsigned)a.N * (unsigned)a.chunks);
  const bool bins = a.top_k || a.top_p;
  hipLaunchKernelGGL((sample_stats_kernel<T, kPer>), grid, dim3(kThreads), 0, stream, a);
  if (bins) hipLaunchKernelGGL((sample_bins_kernel<T, kPer>), grid, dim3(kThreads), 0, stream, a);
  if (bins || a.min_p)
    hipLaunchKernelGGL((sample_border_kernel<T, kPer>), grid, dim3(kThreads), 0, stream, a);
  hipLaunchKernelGGL(sample_pick_kernel<T>, dim3(a.N), dim3(kPickThreads), 0, stream, a);
}

}  // namespace

size_t sample_workspace_bytes(int32_t N, int32_t V) { return sample_layout(N, V).bytes; }

hipError_t launch_sample(const void *logits, bool bf16, int32_t N, int32_t V, int64_t row_stride,
                         const float *temperature, const int32_t *top_k, const float *top_p,
                         const float *min_p, const float *uniform, int32_t *tokens,
                         float *logprob, void *workspace, hipStream_t stream) {
  const SampleLayout l = sample_layout(N, V);
  char *ws = static_cast<char *>(workspace);
  SampleArgs a;
  a.logits = logits;
  a.temperature = temperature;
  a.top_k = top_k;
  a.top_p = top_p;
  a.min_p = min_p;
  a.uniform = uniform;
  a.tokens = tokens;
  a.logprob = logprob;
  a.row_stride = row_stride;
  a.N = N;
  a.V = V;
  a.chunks = l.chunks;
  a.per = l.per;
  a.c_top = reinterpret_cast<float *>(ws + l.c_top);
  a.c_low = reinterpret_cast<float *>(ws + l.c_low);
  a.c_first = reinterpret_cast<uint32_t *>(ws + l.c_first);
  a.c_sum = reinterpret_cast<double *>(ws + l.c_sum);
  a.bin_mass = reinterpret_cast<uint64_t *>(ws + l.bin_mass);
  a.bin_count = reinterpret_cast<uint32_t *>(ws + l.bin_count);
  a.c_kept = reinterpret_cast<uint64_t *>(ws + l.c_kept);
  a.c_listed = reinterpret_cast<uint32_t *>(ws + l.c_listed);
  a.c_keys = reinterpret_cast<uint32_t *>(ws + l.c_keys);
  a.list = reinterpret_cast<uint64_t *>(ws + l.list);
  a.border = reinterpret_cast<Border *>(ws + l.border);
  if (bf16) {
    if (l.per == 8)
      launch_passes<uint16_t, 8>(a, stream);
    else
      launch_passes<uint16_t, 32>(a, stream);
  } else {
    if (l.per == 8)
      launch_passes<float, 8>(a, stream);
    else
      launch_passes<float, 32>(a, stream);
  }
  return hipGetLastError();
}

}  // namespace ra
