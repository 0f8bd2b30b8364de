// Drawing a token from a row of logits (token_sample): temperature, top-k, top-p and min-p
// filters, then the inverse of the cumulative distribution at a given uniform number.
//
// With M the row's largest logit, an element's weight is e = exp((z - M) / T) in 64-bit
// floating point. Where weights are added up by atomics or in no fixed order they are whole
// numbers of 2^-44 (0 below half a unit, 31.2 below M), so that no order changes a sum:
// a sum of V weights is off by at most V half units, and a row's is at most 2^63 for V <= 2^19
// (2^19 equal logits): sums are unsigned. The other sums are taken in a fixed order.
//
// All filters keep a prefix of the order (logit descending, index ascending), so what is
// sought is where it ends. Rows are cut into chunks, a wave each, and the call runs:
//   stats   each chunk's and each of its lanes' largest logit, the chunk's smallest, and its
//           sum of weights (rows without filters, or with top-p alone)
//   range   a workgroup a row: how far below M the end can lie. Top-k: the k-th of the
//           largest logits of parts of the row is no larger than the k-th logit. Top-p:
//           elements below (1 - p) sum / V weigh less than (1 - p) sum together.
//   bins    counts and weights of the elements in the range, in 512 bins of it
//   border  the bin or bins that hold the end. What lies above is kept: each chunk sums it;
//           the elements in them are listed
//   pick    a workgroup a row: the listed elements binned again and the few in question
//           sorted, the end found, the chunk of the drawn token from the chunks' sums, the
//           token from the chunk's elements
// Without filters stats and pick are the whole call; with min-p alone there are no bins.
// Bins and border read only what the lanes' largest logits put into the range: of 156 MB of
// logits (512 rows of 151,936 bf16) 47 and 61. Measured there, all filters: stats 38 us (4.1
// TB/s), range 6, bins 31, border 42, pick 19, the call 136-139; 64 rows of them with top-p 13,
// 4, 13, 15, 17 and 63; 64 rows of fp32 without filters 12, 7 and 18 (39 MB); a row of 32,000
// 3, 4, 5, 6, 8 and 25. The first pass is bound by its read and, where sums are wanted, by 64-bit
// arithmetic; the others by the round trips of a workgroup that does little.
#include <type_traits>

#include "ra_device.h"
#include "ra_internal.h"
#include "ra_wave.h"

namespace ra {
namespace {

constexpr int kThreads = 256;           // four chunks
constexpr int kGroup = kThreads / kWave;
constexpr int kRowThreads = 512;        // of a row's range
constexpr int kBins = 512;
constexpr int kMaxChunks = 256;         // of a row
constexpr int kListed = 256;            // elements that a chunk can list
constexpr int kMaxSorted = 2048;        // of them, that the pick sorts
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
// Its whole units: in the low bits of the sum with 2^52.
__device__ __forceinline__ uint64_t units(double e) {
  return __builtin_bit_cast(uint64_t, __builtin_fma(e, kUnit, 0x1p52)) & 0xfffffffffffffull;
}

// The same for many elements: exp(d inv_t), d <= 0, as 2^(j / 128) by table times the rest of
// the exponent, at most ln 2 / 256, by the Taylor series to r^4, whose next term is below
// 2^-49. No branch: NaN and what lies below -64 count as 2^-92. The constants are held in
// scalar registers, where an addend costs no move.
constexpr int kExpTable = 128;
constexpr double kStep = 0.6931471805599453 / kExpTable;
struct Pow2Table {
  double at[kExpTable];
  constexpr Pow2Table() : at() {
    for (int j = 0; j < kExpTable; ++j) {
      double sum = 0.0;                              // the Taylor series from its small end
      for (int i = 20; i > 0; --i) sum = (sum + 1.0) * (j * kStep) / i;
      at[j] = 1.0 + sum;
    }
  }
};
__constant__ Pow2Table kPow2 = Pow2Table();

struct TableExp {
  const double *table;
  double scale, low, round, c1, c2, c3, c4;
  __device__ __forceinline__ TableExp(const double *t, double inv_t)
      : table(t), scale(inv_t * (1.4426950408889634 * kExpTable)),
        low(-64.0 * (1.4426950408889634 * kExpTable)), round(0x1.8p52), c1(kStep),
        c2(kStep * kStep / 2.0), c3(kStep * kStep * kStep / 6.0),
        c4(kStep * kStep * kStep * kStep / 24.0) {
    asm volatile("" : "+s"(low), "+s"(round), "+s"(c1), "+s"(c2), "+s"(c3), "+v"(c4));
  }
  __device__ __forceinline__ double operator()(double d) const {
    // adding `round` rounds to whole numbers, in the low bits
    const double y = fmax(d * scale, low), t = y + round, f = y - (t - round);
    const int n = (int)(uint32_t)__builtin_bit_cast(uint64_t, t);
    double p = __builtin_fma(c4, f, c3);
    p = __builtin_fma(p, f, c2);
    p = __builtin_fma(p, f, c1);
    const uint64_t pow2 = __builtin_bit_cast(uint64_t, table[n & (kExpTable - 1)]);
    const uint32_t high = (uint32_t)(pow2 >> 32) + ((uint32_t)(n >> 7) << 20);   // times 2^(n / 128)
    const double e = __builtin_bit_cast(double, (uint64_t)high << 32 | (uint32_t)pow2);
    return __builtin_fma(e, p * f, e);
  }
};

// What a workgroup has of its chunks, for the next launches: a cache line each, written as a
// whole.
struct alignas(128) Stats {
  float top[kGroup], low[kGroup];       // largest and smallest finite logit
  double sum[kGroup];                   // of weights against top
  uint32_t first[kGroup];               // lowest index of the largest one
};
struct alignas(128) Kept {
  uint64_t mass[kGroup];                // weight kept for certain
  uint32_t listed[kGroup];              // elements in the border's bins
  uint32_t high[kGroup], low[kGroup];   // their largest and smallest key
};
// By the first lanes of a wave, from LDS.
template <typename Line>
__device__ __forceinline__ void write_line(Line *to, const Line *lds) {
  static_assert(sizeof(Line) == 128, "a line");
  const int lane = threadIdx.x % kWave;
  if (lane < 32) reinterpret_cast<uint32_t *>(to)[lane] = reinterpret_cast<const uint32_t *>(lds)[lane];
}

struct SampleArgs {
  const void *logits;
  const float *temperature;
  const int32_t *top_k;
  const float *top_p, *min_p, *uniform;
  int32_t *tokens;
  float *logprob;
  int64_t row_stride;
  int32_t N, V, chunks, groups;         // groups: of kGroup chunks
  // workspace
  Stats *stats;                         // [N][groups]
  float *l_top;                         // [N][chunks][kWave] largest of a lane's
  uint64_t *bin_mass;                   // [N][kBins]
  uint32_t *bin_count;                  // [N][kBins]
  Kept *kept;                           // [N][groups]
  uint64_t *list;                       // [N][chunks][kListed] key << 32 | ~index
  struct BorderLine *border, *ends;     // [N] with the range; with the end's bins too
};

// What a row asks for. The four loads go out together: a parameter that is not given is read
// from kNotGiven instead of being branched around.
struct NotGiven {
  float temperature, top_p, min_p;
  int32_t top_k;
};
__constant__ NotGiven kNotGiven = {1.f, 1.f, 0.f, 0};
struct Row {
  double inv_t, p, m;                   // p < 1: top-p, m > 0: min-p
  int k;                                // 0: no top-k
  bool greedy;
  __device__ __forceinline__ Row(const SampleArgs &a, int n) {
    const float t = *(a.temperature ? a.temperature + n : &kNotGiven.temperature);
    const float tp = *(a.top_p ? a.top_p + n : &kNotGiven.top_p);
    const float mp = *(a.min_p ? a.min_p + n : &kNotGiven.min_p);
    k = *(a.top_k ? a.top_k + n : &kNotGiven.top_k);
    greedy = !(t > 0.f);
    inv_t = 1.0 / (double)t;
    if (k < 0 || k >= a.V) k = 0;
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
  double sum;                           // of the weights (top-p alone)
  float top, rate;                      // largest logit; bins two units of logit
  int lo, hi, bin_k;                    // kBins: none
  uint32_t count_lo, count_k;           // elements before bin lo, bin_k
  uint64_t mass_lo, mass_k;             // weights before them
};

struct alignas(128) BorderLine {
  Border b;
};

// The bin of a logit, `below` under the largest one: non-decreasing in it. kBins: beyond.
__device__ __forceinline__ int bin_of(float below, float rate) {
  const float b = below * rate;
  return b < kBins ? (int)b : kBins;
}
// Half the distance: a whole one can pass the largest fp32 number.
__device__ __forceinline__ float below(float top, float z) {
  return z == top ? 0.f : fmaf(-0.5f, z, 0.5f * top);
}
// Bins two units of logit, for a range of (M - z) / T. The slack takes in what rounds past it.
__device__ __forceinline__ float rate_of(double range, double inv_t) {
  return (float)fmin(inv_t * (2 * kBins / (fmax(range, 1e-30) * (1.0 + 1e-6))), 0x1.fp127);
}

// ---- reductions, in a fixed order ----
template <typename V, typename Op>
__device__ __forceinline__ V wave_reduce(V x, Op op) {
  x = op(x, lane_pattern<kSwapOnes, 0xf>(x));
  x = op(x, lane_pattern<kSwapTwos, 0xf>(x));
  x = op(x, lane_pattern<kMirrorHalf, 0xf>(x));
  x = op(x, lane_pattern<kMirrorRow, 0xf>(x));
  return op(op(of_lane(x, 0), of_lane(x, 16)), op(of_lane(x, 32), of_lane(x, 48)));
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
  const V s = wave_sums(x);
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

// Sums over the lanes before this one, and over all.
template <typename V>
__device__ __forceinline__ V wave_scan(V x, V &total) {
  const V s = wave_sums(x);
  total = of_lane(s, kWave - 1);
  return s - x;
}

__device__ __forceinline__ float max_of(float a, float b) { return fmaxf(a, b); }
__device__ __forceinline__ float min_of(float a, float b) { return fminf(a, b); }

// Chunk c's logits of a lane: vectors lane, lane + kWave, ...; -inf past the row. NaN stays:
// no comparison takes it in.
template <typename T, int kPer>
__device__ __forceinline__ void load_chunk(const SampleArgs &a, int n, int c, float (&z)[kPer]) {
  constexpr int kVec = kVector<T>;
  const int lane = threadIdx.x % kWave;
  const T *row = static_cast<const T *>(a.logits) + n * a.row_stride;
  u32x4_any w[kPer / kVec];
  if ((c + 1) * kWave * kPer <= a.V) {
#pragma unroll
    for (int j = 0; j < kPer / kVec; ++j)
      w[j] = *reinterpret_cast<const u32x4_any *>(row + c * kWave * kPer + (j * kWave + lane) * kVec);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      if constexpr (sizeof(T) == 4)
        z[i] = __uint_as_float(w[i / kVec][i % kVec]);
      else
        z[i] = __uint_as_float(i % 2 ? w[i / kVec][i % kVec / 2] & 0xffff0000u
                                     : w[i / kVec][i % kVec / 2] << 16);
    }
  } else {
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int v = c * kWave * kPer + (i / kVec * kWave + lane) * kVec + i % kVec;
      z[i] = v < a.V ? logit_value(row[v]) : -__builtin_inff();
    }
  }
}
// Where logits are weighed from: the largest, or 0 once those at +inf are at 0 and the rest
// at -inf.
template <int kPer>
__device__ __forceinline__ float flatten(float (&z)[kPer], float top) {
  if (top < __builtin_inff()) return top;
#pragma unroll
  for (int i = 0; i < kPer; ++i) z[i] = z[i] == top ? 0.f : -__builtin_inff();
  return 0.f;
}

// The index of a lane's i-th logit.
template <typename T, int kPer>
__device__ __forceinline__ int index_of(int c, int i) {
  constexpr int kVec = kVector<T>;
  return c * kWave * kPer + (i / kVec * kWave + (int)(threadIdx.x % kWave)) * kVec + i % kVec;
}

// 2^(j / kExpTable) for TableExp; there by the next barrier.
__device__ __forceinline__ void fill_table(double *table) {
  if (threadIdx.x < kExpTable) table[threadIdx.x] = kPow2.at[threadIdx.x];
}

template <typename T, int kPer>
__global__ __launch_bounds__(kThreads) void sample_stats_kernel(SampleArgs a) {
  const int n = blockIdx.x / a.groups, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int c = blockIdx.x % a.groups * kGroup + wave;
  __shared__ double table[kExpTable];
  __shared__ Stats own;
  const Row row(a, n);
  if (row.needs_sums()) {
    fill_table(table);
    __syncthreads();
  }
  float z[kPer], top = -__builtin_inff(), low = __builtin_inff();
  int first = a.V;
  double sum = 0.0;
  if (c < a.chunks) {
    load_chunk<T, kPer>(a, n, c, z);
    float mine = -__builtin_inff();
#pragma unroll
    for (int i = 0; i < kPer; ++i) mine = fmaxf(mine, z[i]);
    top = wave_reduce(mine, max_of);
    if (row.greedy) {
#pragma unroll
      for (int i = kPer - 1; i >= 0; --i) first = z[i] == top ? index_of<T, kPer>(c, i) : first;
      first = wave_reduce(first, [](int x, int y) { return min(x, y); });
    } else {
      if (row.filtered()) a.l_top[((int64_t)n * a.chunks + c) * kWave + lane] = mine;
      if (row.binned()) {
#pragma unroll
        for (int i = 0; i < kPer; ++i) low = z[i] > -__builtin_inff() ? fminf(low, z[i]) : low;
        low = wave_reduce(low, min_of);
      }
      if (row.needs_sums()) {
        if (top > -__builtin_inff()) {
          const TableExp weight(table, row.inv_t);
          const double from = flatten(z, top);
#pragma unroll
          for (int i = 0; i < kPer; ++i) sum += weight((double)z[i] - from);
        }
        sum = wave_reduce(sum, [](double x, double y) { return x + y; });
      }
    }
  }
  if (lane == 0) own.top[wave] = top, own.low[wave] = low, own.sum[wave] = sum, own.first[wave] = first;
  __syncthreads();
  if (wave == 0) write_line(a.stats + blockIdx.x, &own);
}

// A lane holds the four chunks of the group of its number, every wave all of them. Their
// lines are read whether there is such a group or not (the last one instead) and whatever
// the row asks for, and awaited together: each load behind a branch is another round trip to
// memory, 0.7 us for a row by itself and 7 us among 512.
static_assert(kMaxChunks == kGroup * kWave && kGroup == 4, "a group a lane");
template <typename Line>
__device__ __forceinline__ const Line &line_of(const Line *lines, int n, int groups) {
  return lines[(int64_t)n * groups + min((int)(threadIdx.x % kWave), groups - 1)];
}
template <typename V>
__device__ __forceinline__ void load_four(const V (&of_group)[kGroup], V (&x)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = of_group[i];
}
// Loads before are issued, and awaited, by here.
template <typename V>
__device__ __forceinline__ void here(V (&x)[4]) {
  asm volatile("" : "+v"(x[0]), "+v"(x[1]), "+v"(x[2]), "+v"(x[3]));
}
template <typename V>
__device__ __forceinline__ void mask_four(int groups, V none, V (&x)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) x[i] = (int)(threadIdx.x % kWave) < groups ? x[i] : none;
}
__device__ __forceinline__ float top_of(const float (&c_top)[4]) {
  return wave_reduce(fmaxf(fmaxf(c_top[0], c_top[1]), fmaxf(c_top[2], c_top[3])), max_of);
}

// Ranges of rows with filters; their bins start at zero.
__global__ __launch_bounds__(kRowThreads) void sample_range_kernel(SampleArgs a) {
  const int n = blockIdx.x, tid = threadIdx.x, lane = tid % kWave;
  const Row row(a, n);
  __shared__ uint32_t count[kBins];
  __shared__ BorderLine own;
  const int64_t at = (int64_t)n * a.chunks;
  const Stats &of = line_of(a.stats, n, a.groups);
  float c_top[4], c_low[4];
  double c_sum[4];
  load_four(of.top, c_top);
  load_four(of.low, c_low);
  load_four(of.sum, c_sum);
  here(c_top);
  here(c_low);
  here(c_sum);
  if (!row.filtered()) return;
  mask_four(a.groups, -__builtin_inff(), c_top);
  mask_four(a.groups, __builtin_inff(), c_low);
  mask_four(a.groups, 0.0, c_sum);
  const float top = top_of(c_top);
  double sum = 0.0;
  double range = kRange;
  if (row.binned()) {
    static_assert(kRowThreads == kBins, "a bin a thread");
    a.bin_mass[(int64_t)n * kBins + tid] = 0;
    a.bin_count[(int64_t)n * kBins + tid] = 0;
    const float low = wave_reduce(fminf(fminf(c_low[0], c_low[1]), fminf(c_low[2], c_low[3])), min_of);
    range = fmin(range, -scaled(fminf(low, top), top, row.inv_t));
    if (row.k > 0) {
      // the k-th of the largest logits of chunks, of four lanes or of lanes, of the coarsest
      // that are twice as many: the k-th of any k elements will do. As far as a bin tells.
      count[tid] = 0;
      __syncthreads();
      const float rate = rate_of(range, row.inv_t);
      auto put = [&](float z) {
        const int bin = bin_of(below(top, z), rate);
        if (bin < kBins) atomicAdd(&count[bin], 1u);
      };
      const int parts = a.chunks * kWave / 4;
      if (2 * row.k <= a.chunks) {
        if (tid < kWave)
#pragma unroll
          for (int i = 0; i < 4; ++i) put(c_top[i]);
      } else {
        const f32x4 *l_top = reinterpret_cast<const f32x4 *>(a.l_top + at * kWave);
#pragma unroll 4
        for (int i = tid; i < parts; i += kRowThreads) {
          const f32x4 z = l_top[i];
          if (2 * row.k <= parts) {
            put(fmaxf(fmaxf(z[0], z[1]), fmaxf(z[2], z[3])));
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) put(z[e]);
          }
        }
      }
      __syncthreads();
      constexpr int kOwn = kBins / kWave;
      uint32_t own = 0, all, c[kOwn];
#pragma unroll
      for (int i = 0; i < kOwn; ++i) own += c[i] = count[kOwn * lane + i];
      uint32_t before = wave_scan(own, all);
      int bin = kBins;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        if (before < (uint32_t)row.k && before + c[i] >= (uint32_t)row.k) bin = kOwn * lane + i;
        before += c[i];
      }
      bin = wave_reduce(bin, [](int x, int y) { return min(x, y); });
      if (bin < kBins) range = fmin(range, 2 * (bin + 1) / (double)rate * row.inv_t * (1.0 + 1e-6));
    } else {
      double x = 0.0;
#pragma unroll
      for (int i = 0; i < 4; ++i) x += c_sum[i] * weight_exp(scaled(c_top[i], top, row.inv_t));
      sum = wave_reduce(x, [](double u, double v) { return u + v; });
      if (row.p > 0.0) range = fmin(range, log((double)a.V / ((1.0 - row.p) * sum)) + 1e-3);
    }
  } else {
    range = fmin(range, -log(row.m) + 1e-12);
  }
  // member by member: a struct copied here is kept in memory, in LDS by the number of the
  // thread, for which the launch's packet is read from the host: 5 us, 15 us of 512 workgroups
  if (tid == 0) own.b.sum = sum, own.b.top = top, own.b.rate = rate_of(range, row.inv_t);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  if (tid < kWave) write_line(a.border + n, &own);
}

// The weight of a logit in a row with filters: by this wherever one is taken, so that sums and
// what they are compared with agree to the last unit.
struct Weigh {
  TableExp exp;
  double top;
  bool infinite;
  __device__ __forceinline__ Weigh(const double *table, double inv_t, float t)
      : exp(table, inv_t), top((double)t), infinite(t == __builtin_inff()) {}
  __device__ __forceinline__ double operator()(float z) const {
    return infinite ? (z == __builtin_inff() ? 1.0 : 0.0) : exp((double)z - top);
  }
};

// Whether a logit is in the row's range.
__device__ __forceinline__ bool in_range(const Border &b, float z) {
  return bin_of(below(b.top, z), b.rate) < kBins;
}

template <typename T, int kPer>
__global__ __launch_bounds__(kThreads) void sample_bins_kernel(SampleArgs a) {
  const int n = blockIdx.x / a.groups, tid = threadIdx.x, lane = tid % kWave;
  const int c0 = blockIdx.x % a.groups * kGroup, c = c0 + tid / kWave;
  const Border b = a.border[n].b;
  float c_top[kGroup];
#pragma unroll
  for (int i = 0; i < kGroup; ++i) c_top[i] = a.stats[blockIdx.x].top[i];
  const float l_top = c < a.chunks ? a.l_top[((int64_t)n * a.chunks + c) * kWave + lane] : 0.f;
  const Row row(a, n);
  if (!row.binned() || b.top == -__builtin_inff()) return;
  bool any = false, mine = false;
#pragma unroll
  for (int i = 0; i < kGroup; ++i) {
    const bool in = in_range(b, c_top[i]);
    any |= in;
    mine = c == c0 + i ? in : mine;
  }
  if (!any) return;
  __shared__ uint64_t mass[kBins];
  __shared__ uint32_t count[kBins];
  __shared__ double table[kExpTable];
  for (int i = tid; i < kBins; i += kThreads) mass[i] = 0, count[i] = 0;
  if (row.p < 1.0) fill_table(table);
  __syncthreads();
  if (mine && in_range(b, l_top)) {
    float z[kPer];
    load_chunk<T, kPer>(a, n, c, z);
    const Weigh weigh(table, row.inv_t, b.top);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      const int bin = bin_of(below(b.top, z[i]), b.rate);
      if (bin < kBins) {
        if (row.k > 0) atomicAdd(&count[bin], 1u);
        if (row.p < 1.0)
          atomicAdd((unsigned long long *)&mass[bin], (unsigned long long)units(weigh(z[i])));
      }
    }
  }
  __syncthreads();
  for (int i = tid; i < kBins; i += kThreads) {
    if (count[i]) atomicAdd(&a.bin_count[(int64_t)n * kBins + i], count[i]);
    if (mass[i])
      atomicAdd((unsigned long long *)&a.bin_mass[(int64_t)n * kBins + i], (unsigned long long)mass[i]);
  }
}

// The end's bins, from weights and counts of eight neighbouring bins a lane, by one wave.
// `mass0` and `count0` are ahead of the first bin; by_k: top-k may end in a bin; `all`: what
// top-p takes its share of if it does not.
constexpr int kOwnBins = kBins / kWave;
__device__ __forceinline__ void locate(const uint64_t (&m)[kOwnBins], const uint32_t (&c)[kOwnBins],
                                       uint64_t mass0, uint32_t count0, bool by_k, uint32_t k,
                                       double p, double all, Border &b) {
  const int lane = threadIdx.x % kWave;
  uint64_t m_own = 0, m_all;
  uint32_t c_own = 0, c_all;
#pragma unroll
  for (int i = 0; i < kOwnBins; ++i) m_own += m[i], c_own += c[i];
  const uint64_t m_before = mass0 + wave_scan(m_own, m_all);
  const uint32_t c_before = count0 + wave_scan(c_own, c_all);
  b.lo = b.hi = b.bin_k = kBins;
  b.count_lo = b.count_k = count0;
  b.mass_lo = b.mass_k = mass0 + m_all;
  uint64_t of_bin_k = 0;
  if (by_k) {
    // where the count reaches k
    int bin = kBins;
    uint32_t count = c_before, c_at = 0;
    uint64_t mass = m_before, m_at = 0, m_in = 0;
#pragma unroll
    for (int i = 0; i < kOwnBins; ++i) {
      if (count < k && count + c[i] >= k)
        bin = kOwnBins * lane + i, c_at = count, m_at = mass, m_in = m[i];
      count += c[i];
      mass += m[i];
    }
    const uint64_t found = __ballot(bin < kBins);
    if (found) {
      const int from = __ffsll((unsigned long long)found) - 1;
      b.lo = b.hi = b.bin_k = of_lane(bin, from);
      b.count_lo = b.count_k = of_lane(c_at, from);
      b.mass_lo = b.mass_k = of_lane(m_at, from);
      of_bin_k = of_lane(m_in, from);
      all = (double)b.mass_k;
    }
  }
  if (p < 1.0) {
    // lo, hi: where the weight reaches p of the least and of the most that top-k can keep; by
    // rounding alone it might not by bin_k, which then is the end's
    const double least = fmax(p * all, 0.5), most = fmax(p * (all + (double)of_bin_k), 0.5);
    int lo = kBins, hi = kBins;
    uint32_t count = c_before, c_at = 0;
    uint64_t mass = m_before, m_at = 0;
#pragma unroll
    for (int i = 0; i < kOwnBins; ++i) {
      const int bin = kOwnBins * lane + i;
      const uint64_t after = mass + m[i];
      if (bin <= b.bin_k) {
        if ((double)mass < least && !((double)after < least)) lo = bin, c_at = count, m_at = mass;
        if ((double)mass < most && !((double)after < most)) hi = bin;
      }
      mass = after;
      count += c[i];
    }
    const uint64_t has_lo = __ballot(lo < kBins), has_hi = __ballot(hi < kBins);
    b.hi = has_hi ? of_lane(hi, __ffsll((unsigned long long)has_hi) - 1) : b.bin_k;
    if (has_lo) {
      const int from = __ffsll((unsigned long long)has_lo) - 1;
      b.lo = of_lane(lo, from);
      b.count_lo = of_lane(c_at, from);
      b.mass_lo = of_lane(m_at, from);
    }
  }
}

// From the row's bins.
__device__ __forceinline__ void find_border(const SampleArgs &a, int n, const Row &row, Border &b) {
  const int64_t at = (int64_t)n * kBins + kOwnBins * (threadIdx.x % kWave);
  uint64_t m[kOwnBins], sum = 0;
  uint32_t c[kOwnBins];
#pragma unroll
  for (int i = 0; i < kOwnBins; ++i) {
    m[i] = row.p < 1.0 ? a.bin_mass[at + i] : 0;
    c[i] = row.k > 0 ? a.bin_count[at + i] : 0;
    sum += m[i];
  }
  double all = b.sum * kUnit;
  if (row.k > 0) all = (double)wave_reduce(sum, [](uint64_t x, uint64_t y) { return x + y; });
  locate(m, c, 0, 0, row.k > 0, (uint32_t)row.k, row.p, all, b);
}

template <typename T, int kPer>
__global__ __launch_bounds__(kThreads) void sample_border_kernel(SampleArgs a) {
  const int n = blockIdx.x / a.groups, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int c0 = blockIdx.x % a.groups * kGroup, c = c0 + wave;
  const int64_t at = (int64_t)n * a.chunks + c;
  Border b = a.border[n].b;
  const float c_top = a.stats[blockIdx.x].top[wave];
  const float l_top = c < a.chunks ? a.l_top[at * kWave + lane] : -__builtin_inff();
  const Row row(a, n);
  if (!row.filtered() || b.top == -__builtin_inff()) return;
  __shared__ double table[kExpTable];
  __shared__ uint64_t list[kGroup][kListed];
  __shared__ Kept own;
  __shared__ BorderLine found;
  const bool mine = in_range(b, c_top);
  if (lane == 0)
    own.mass[wave] = 0, own.listed[wave] = 0, own.high[wave] = 0, own.low[wave] = 0xffffffffu;
  if (!__syncthreads_or(mine)) {
    if (wave == 0) write_line(a.kept + blockIdx.x, &own);
    return;
  }
  fill_table(table);
  if (wave == 0) {                        // 6 KB of bins: read by one of the waves
    if (row.binned())
      find_border(a, n, row, b);
    else
      b.lo = b.hi = b.bin_k = kBins;
    if (lane == 0) found.b = b;
  }
  __syncthreads();
  b = found.b;
  if (mine) {
    uint64_t kept = 0;
    uint32_t high = 0, low = 0xffffffffu;
    if (in_range(b, l_top)) {
      float z[kPer];
      load_chunk<T, kPer>(a, n, c, z);
      const Weigh weigh(table, row.inv_t, b.top);
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        const int bin = bin_of(below(b.top, z[i]), b.rate);
        if (bin < b.lo) {
          const double e = weigh(z[i]);
          if (e >= row.m) kept += units(e);
        } else if (bin < kBins && (bin <= b.hi || bin == b.bin_k)) {
          const uint32_t slot = atomicAdd(&own.listed[wave], 1u), key = key_of(z[i]);
          if (slot < (uint32_t)kListed)
            list[wave][slot] = (uint64_t)key << 32 | (uint32_t)~index_of<T, kPer>(c, i);
          high = key > high ? key : high;
          low = key < low ? key : low;
        }
      }
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    const int listed = min(of_lane((int)own.listed[wave], 0), kListed);
    for (int i = lane; i < (listed + 15) / 16 * 16; i += kWave)   // whole lines
      a.list[at * kListed + i] = list[wave][i];
    kept = wave_reduce(kept, [](uint64_t x, uint64_t y) { return x + y; });
    if (listed) {
      high = wave_reduce(high, [](uint32_t x, uint32_t y) { return x > y ? x : y; });
      low = wave_reduce(low, [](uint32_t x, uint32_t y) { return x < y ? x : y; });
    }
    if (lane == 0) own.mass[wave] = kept, own.high[wave] = high, own.low[wave] = low;
    // one of the chunks that hold the largest: all write the same
    if (c_top == b.top) write_line(a.ends + n, &found);
  }
  __syncthreads();
  if (wave == 0) write_line(a.kept + blockIdx.x, &own);
}

// ---- pick -----------------------------------------------------------------------------
// Neighbouring logits of a thread from index v0 on; -inf past the row.
template <typename T, int kOwn>
__device__ __forceinline__ void load_neighbours(const T *row, int v0, int V, float (&z)[kOwn]) {
  constexpr int kVec = kVector<T>;
  if (kOwn % kVec == 0 && v0 + kOwn <= V) {
#pragma unroll
    for (int j = 0; j < kOwn / kVec; ++j) {
      const u32x4_any w = *reinterpret_cast<const u32x4_any *>(row + v0 + j * kVec);
#pragma unroll
      for (int e = 0; e < kVec; ++e) {
        if constexpr (sizeof(T) == 4)
          z[j * kVec + e] = __uint_as_float(w[e]);
        else
          z[j * kVec + e] = __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < kOwn; ++e) z[e] = v0 + e < V ? logit_value(row[v0 + e]) : -__builtin_inff();
  }
#pragma unroll
  for (int e = 0; e < kOwn; ++e) z[e] = clean(z[e]);
}

// What the pick's waves share; kN: its threads.
template <int kN>
struct PickLds {
  uint64_t sorted[kMaxSorted];          // listed elements
  uint64_t mass[kBins];                 // finer bins
  uint32_t counts[kBins];
  uint64_t kept_of[kMaxChunks];         // weight kept of each chunk
  uint32_t ties_of[kMaxChunks];         // of each chunk: elements at the edge
  uint32_t first_of[kMaxChunks];        // and where its listed elements start
  uint64_t mpart[kN / kWave];
  double dpart[kN / kWave];
  double table[kExpTable];
  uint64_t sum;
  uint32_t key, count, ties, high, low;
  int token;
};

// The end of the kept prefix: keys above `key`, and of those at it the first `ties` of the
// row or, with ties = kByIndex, those up to `index`.
constexpr uint64_t kByIndex = ~0ull;
struct Edge {
  uint32_t key, index;
  uint64_t ties;
};

// Sums as functions of what is listed.
struct Goals {
  const Row &row;
  const Border &b;
  const Weigh &weigh;
  double all;                           // what top-p takes its share of if top-k keeps all
  uint32_t high;                        // key of the first of finer bins,
  int shift;                            // and their width; < 0: the row's bins
  __device__ __forceinline__ int bin(uint32_t key) const {
    if (shift >= 0) return (int)((high - key) >> shift);
    return bin_of(below(b.top, value_of(key)), b.rate);
  }
  __device__ __forceinline__ double weight(uint32_t key) const {
    return weigh(value_of(key));
  }
  __device__ __forceinline__ bool ends_in_k() const { return row.k > 0 && b.bin_k < kBins; }
  // the weight at which top-p ends, given what top-k keeps of bin_k
  __device__ __forceinline__ double goal(uint64_t of_bin_k) const {
    return fmax(row.p * (ends_in_k() ? (double)(b.mass_k + of_bin_k) : all), 0.5);
  }
  // how many of `avail` elements of weight w, `before` ahead of them, the goal lets in
  __device__ __forceinline__ uint64_t let_in(double goal, uint64_t before, uint64_t w,
                                             uint64_t avail) const {
    if (!((double)before < goal)) return 0;
    if (w == 0) return avail;
    const double r = __builtin_ceil((goal - (double)before) / (double)w);
    return r < 1.0 ? 1 : r >= (double)avail ? avail : (uint64_t)r;
  }
  // the rank in the row of the i-th listed element, n_p of them in bins lo .. hi
  __device__ __forceinline__ uint64_t rank(uint64_t i, int bin, uint64_t n_p) const {
    return bin == b.bin_k && b.bin_k > b.hi ? b.count_k + (i - n_p) : b.count_lo + i;
  }
  __device__ __forceinline__ bool keeps(uint64_t rank, int bin, uint64_t before, double goal) const {
    return bin <= b.hi && !(ends_in_k() && rank >= (uint64_t)row.k) &&
           !(row.p < 1.0 && !((double)before < goal));
  }
};

// Up to 64 listed elements, by one wave: lane i has one of them in `x` (0: none); adds what
// is kept to the chunks' sums.
template <int kN>
__device__ __forceinline__ Edge end_in_a_wave(uint64_t x, const Goals &g, int chunk_len, PickLds<kN> &lds) {
  const int lane = threadIdx.x % kWave;
  // each goes where as many larger ones are; the elements differ
  const uint64_t some = __ballot(x != 0);
  int place = x ? 0 : __popcll(some) + __popcll(~some & ((1ull << lane) - 1));
#pragma unroll
  for (int i = 0; i < kWave; ++i) place += x && of_lane(x, i) > x;
  const u32x2 halves = __builtin_bit_cast(u32x2, x);
  u32x2 sorted;
  sorted[0] = __builtin_amdgcn_ds_permute(4 * place, halves[0]);
  sorted[1] = __builtin_amdgcn_ds_permute(4 * place, halves[1]);
  x = __builtin_bit_cast(uint64_t, sorted);
  uint64_t w = 0, all;
  double e = 0.0;
  int bin = kBins << 10;
  if (x) {
    e = g.weight((uint32_t)(x >> 32));
    w = units(e);
    bin = g.bin((uint32_t)(x >> 32));
  }
  const uint64_t before = wave_scan(w, all);
  const uint64_t n_p = __popcll(__ballot(x && bin <= g.b.hi)), rank = g.rank(lane, bin, n_p);
  const bool of_k = g.ends_in_k() && x && bin == g.b.bin_k && rank < (uint64_t)g.row.k;
  const uint64_t mass_k = wave_reduce(of_k ? w : (uint64_t)0, [](uint64_t u, uint64_t v) { return u + v; });
  const double goal = g.row.p < 1.0 ? g.goal(mass_k) : 0.0;
  const bool kept = x && g.keeps(rank, bin, g.b.mass_lo + before, goal);
  const uint64_t mask = __ballot(kept);
  const uint32_t v = ~(uint32_t)x;
  if (kept && e >= g.row.m)
    atomicAdd((unsigned long long *)&lds.kept_of[v / chunk_len], (unsigned long long)w);
  if (!mask) return {0xffffffffu, 0, kByIndex};
  const uint64_t last = of_lane(x, __popcll(mask) - 1);
  return {(uint32_t)(last >> 32), ~(uint32_t)last, kByIndex};
}

// Up to kMaxSorted listed elements, in lds.sorted.
template <int kN>
__device__ __forceinline__ Edge end_by_sorting(int count, const Goals &g, int chunk_len, PickLds<kN> &lds) {
  const int tid = threadIdx.x;
  int size = 64;
  while (size < count) size *= 2;
  for (int i = count + tid; i < size; i += kN) lds.sorted[i] = 0;
  __syncthreads();
  for (int len = 2; len <= size; len *= 2)
    for (int step = len / 2; step > 0; step /= 2) {
      for (int i = tid; i < size / 2; i += kN) {
        const int lo = i / step * 2 * step + i % step, hi = lo + step;
        const uint64_t x = lds.sorted[lo], y = lds.sorted[hi];
        if ((x < y) == ((lo & len) == 0)) lds.sorted[lo] = y, lds.sorted[hi] = x;
      }
      __syncthreads();
    }
  // neighbouring elements a thread: their weights, and the sums before them
  constexpr int kOwn = kMaxSorted / kN;
  auto add = [](uint64_t x, uint64_t y) { return x + y; };
  uint64_t w[kOwn], own = 0, of_k = 0, in_p = 0, all;
  int bin[kOwn];
#pragma unroll
  for (int j = 0; j < kOwn; ++j) {
    const int i = tid * kOwn + j;
    w[j] = 0, bin[j] = kBins << 10;
    if (i < count) {
      w[j] = units(g.weight((uint32_t)(lds.sorted[i] >> 32)));
      bin[j] = g.bin((uint32_t)(lds.sorted[i] >> 32));
      in_p += bin[j] <= g.b.hi;
    }
    own += w[j];
  }
  uint64_t run = group_scan<kN>(own, all, lds.mpart);
  const uint64_t n_p = group_reduce<kN>(in_p, add, lds.mpart);
  if (g.ends_in_k() && g.row.p < 1.0) {
#pragma unroll
    for (int j = 0; j < kOwn; ++j)
      if (bin[j] == g.b.bin_k && g.rank(tid * kOwn + j, bin[j], n_p) < (uint64_t)g.row.k) of_k += w[j];
    of_k = group_reduce<kN>(of_k, add, lds.mpart);
  }
  const double goal = g.row.p < 1.0 ? g.goal(of_k) : 0.0;
  if (tid == 0) lds.count = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kOwn; ++j) {
    const int i = tid * kOwn + j;
    if (i < count && g.keeps(g.rank(i, bin[j], n_p), bin[j], g.b.mass_lo + run, goal)) {
      atomicMax(&lds.count, (uint32_t)i + 1);         // kept: a prefix of the sorted elements
      const uint32_t v = ~(uint32_t)lds.sorted[i];
      if (g.weight((uint32_t)(lds.sorted[i] >> 32)) >= g.row.m)
        atomicAdd((unsigned long long *)&lds.kept_of[v / chunk_len], (unsigned long long)w[j]);
    }
    run += w[j];
  }
  __syncthreads();
  if (lds.count == 0) return {0xffffffffu, 0, kByIndex};
  const uint64_t last = lds.sorted[lds.count - 1];
  return {(uint32_t)(last >> 32), ~(uint32_t)last, kByIndex};
}

// Any number: the edge by eight bits of the key a pass over the row, first that of top-k,
// then that of top-p among what top-k keeps. The chunks' sums are those of the whole prefix.
// Up to eleven passes over the row by one workgroup: 0.6-1.0 ms for 64 rows of 151,936 bf16,
// 0.2-0.35 ms for a row of 32,000.
template <typename T, int kN>
__device__ __forceinline__ Edge end_by_passes(const T *logits, int V, const Goals &g, int chunks,
                                           int chunk_len, PickLds<kN> &lds) {
  const int tid = threadIdx.x;
  uint64_t *mass = lds.mass;
  uint32_t *counts = lds.counts;
  auto add = [](uint64_t x, uint64_t y) { return x + y; };
  auto key_at = [&](int v) { return key_of(clean(logit_value(logits[v]))); };
  Edge end = {0, 0, ~0ull >> 1};
  for (int round = 0; round < 2; ++round) {
    const bool by_mass = round == 1;
    if (by_mass ? !(g.row.p < 1.0) : !(g.row.k > 0)) continue;
    double goal = 0.0;
    if (by_mass) {
      // the weight that top-k keeps
      uint64_t sum = 0, equal = 0;
      for (int v = tid; v < V; v += kN) {
        const uint32_t key = key_at(v);
        if (key > end.key) sum += units(g.weight(key));
        equal += key == end.key;
      }
      sum = group_reduce<kN>(sum, add, lds.mpart);
      equal = group_reduce<kN>(equal, add, lds.mpart);
      if (end.key) sum += (equal < end.ties ? equal : end.ties) * units(g.weight(end.key));
      goal = fmax(g.row.p * (g.row.k > 0 ? (double)sum : g.all), 0.5);
    }
    uint32_t prefix = 0;
    uint64_t ahead = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      __syncthreads();
      if (tid < 256) mass[tid] = 0, counts[tid] = 0;
      __syncthreads();
      for (int v = tid; v < V; v += kN) {
        const uint32_t key = key_at(v);
        if (shift < 24 && key >> (shift + 8) != prefix >> (shift + 8)) continue;
        if (key < end.key) continue;
        if (by_mass)
          atomicAdd((unsigned long long *)&mass[key >> shift & 255],
                    (unsigned long long)units(g.weight(key)));
        atomicAdd(&counts[key >> shift & 255], 1u);
      }
      __syncthreads();
      if (tid == 0) {
        uint64_t run = ahead;
        int i = 255;
        for (; i > 0; --i) {
          const uint64_t next = run + (by_mass ? mass[i] : (uint64_t)counts[i]);
          if (by_mass ? !((double)next < goal) : next >= (uint64_t)g.row.k) break;
          run = next;
        }
        lds.key = prefix | (uint32_t)i << shift;
        lds.sum = run;
        lds.ties = counts[i];
      }
      __syncthreads();
      prefix = lds.key;
      ahead = lds.sum;
    }
    uint64_t r = (uint64_t)g.row.k - ahead;
    if (by_mass) {
      r = g.let_in(goal, ahead, units(g.weight(prefix)), lds.ties);
      if (prefix == end.key && r > end.ties) r = end.ties;
    }
    end = {prefix, 0, r};
    __syncthreads();
  }
  // each chunk's elements at the edge, then what it keeps, a wave a chunk
  const int lane = tid % kWave;
  for (int c = tid / kWave; c < chunks; c += kN / kWave) {
    uint32_t equal = 0;
    const int last = min(V, (c + 1) * chunk_len);
    for (int v = c * chunk_len + lane; v < last; v += kWave) equal += key_at(v) == end.key;
    equal = wave_reduce(equal, [](uint32_t x, uint32_t y) { return x + y; });
    if (lane == 0) lds.ties_of[c] = equal;
  }
  __syncthreads();
  for (int c = tid / kWave; c < chunks; c += kN / kWave) {
    uint64_t ahead = 0, sum = 0;
    for (int i = 0; i < c; ++i) ahead += lds.ties_of[i];
    const int last = min(V, (c + 1) * chunk_len);
    for (int v = c * chunk_len + lane; v < last; v += kWave) {
      const uint32_t key = key_at(v);
      const double e = g.weight(key);
      if (key > end.key && e >= g.row.m) sum += units(e);
    }
    sum = wave_reduce(sum, add);
    const uint64_t left = end.ties > ahead ? end.ties - ahead : 0;
    if (lane == 0) {
      const double e = g.weight(end.key);
      lds.kept_of[c] =
          sum + (e >= g.row.m ? (left < lds.ties_of[c] ? left : lds.ties_of[c]) * units(e) : 0);
    }
  }
  return end;
}

// The last chunk whose sums begin at or before u of the whole and that weighs anything, from
// the four chunks a lane holds: found by every wave by itself.
struct Drawn {
  int chunk;
  double before, total;
};
template <typename V>
__device__ __forceinline__ Drawn draw_chunk(const V (&x)[4], float u) {
  const int lane = threadIdx.x % kWave;
  V total, run = wave_scan(x[0] + x[1] + x[2] + x[3], total);
  const double goal = (double)u * (double)total;
  int chunk = -1;
  V before = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (x[i] > (V)0 && (double)run <= goal) chunk = 4 * lane + i, before = run;
    run += x[i];
  }
  const uint64_t found = __ballot(chunk >= 0);       // never empty: the first that weighs is in
  const int from = kWave - 1 - __clzll((long long)found);
  return {of_lane(chunk, from), (double)of_lane(before, from), (double)total};
}

// The chunk of the i-th listed element; first_of: where each chunk's start.
__device__ __forceinline__ int chunk_of(const uint32_t *first_of, uint32_t i) {
  int c = 0;                              // the last chunk that starts at or before i
#pragma unroll
  for (int step = kMaxChunks / 2; step > 0; step /= 2)
    if (first_of[c + step] <= i) c += step;
  return c;
}
// Calls take(chunk, entry) for the listed elements from `from` on.
template <int kN, typename Take>
__device__ __forceinline__ void for_listed(const SampleArgs &a, int n, uint32_t from, uint32_t count,
                                           const uint32_t *first_of, Take take) {
  for (uint32_t i = from + threadIdx.x; i < count; i += kN) {
    const int c = chunk_of(first_of, i);
    take(c, a.list[((int64_t)n * a.chunks + c) * kListed + (i - first_of[c])]);
  }
}

// kN threads: 256, or 512 for filters in a call of some size, where more is listed: 64 rows of
// 151,936 with top-p 20 and 17 us, without filters 6.7 and 7.6, 7 rows with all 9.3 and 10.3.
template <typename T, int kPer, int kN>
__global__ __launch_bounds__(kN) void sample_pick_kernel(SampleArgs a) {
  const int n = blockIdx.x, tid = threadIdx.x, lane = tid % kWave;
  const T *logits = static_cast<const T *>(a.logits) + n * a.row_stride;
  __shared__ PickLds<kN> lds;
  constexpr int chunk_len = kWave * kPer;

  const Row row(a, n);
  const int mine = a.chunks - 4 * lane;               // of the lane's four chunks: how many are
  const Stats &of = line_of(a.stats, n, a.groups);
  float c_top[4];
  double c_sum[4];
  uint32_t listed[4], key_high[4], key_low[4];
  uint64_t kept[4];
  const Kept &sure = line_of(a.kept, n, a.groups);
  load_four(of.top, c_top);
  load_four(of.sum, c_sum);
  load_four(sure.listed, listed);
  load_four(sure.high, key_high);
  load_four(sure.low, key_low);
  load_four(sure.mass, kept);
  Border b = a.ends[n].b;
  float u = a.uniform[n];
  here(c_top);
  here(c_sum);
  here(listed);
  here(key_high);
  here(key_low);
  here(kept);
  mask_four(a.groups, -__builtin_inff(), c_top);
  mask_four(a.groups, 0.0, c_sum);
  mask_four(a.groups, 0u, listed);
  mask_four(a.groups, (uint64_t)0, kept);
  if (row.filtered()) {
    fill_table(lds.table);
    __syncthreads();
  }
  const float top = top_of(c_top);
  u = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
  if (top == -__builtin_inff() || row.greedy) {
    int first = a.V;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (row.greedy && i < mine && c_top[i] == top) first = min(first, (int)of.first[i]);
    first = wave_reduce(first, [](int x, int y) { return min(x, y); });
    if (tid == 0) {
      const bool none = top == -__builtin_inff();
      a.tokens[n] = none ? -1 : first;
      if (a.logprob) a.logprob[n] = none ? __builtin_nanf("") : 0.f;
    }
    return;
  }

  const Weigh weigh(lds.table, row.inv_t, top);
  Edge end = {0, 0, kByIndex};                        // everything
  Drawn drawn;
  if (!row.filtered()) {
#pragma unroll
    for (int i = 0; i < 4; ++i) c_sum[i] *= weight_exp(scaled(c_top[i], top, row.inv_t));
    drawn = draw_chunk(c_sum, u);
  } else {
    uint32_t first[4], count, longest = 0, high = 0, low = 0xffffffffu;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (listed[i]) {                                // only then are there keys
        high = key_high[i] > high ? key_high[i] : high;
        low = key_low[i] < low ? key_low[i] : low;
        longest = listed[i] > longest ? listed[i] : longest;
      }
    }
    auto umax = [](uint32_t x, uint32_t y) { return x > y ? x : y; };
    high = wave_reduce(high, umax);
    low = wave_reduce(low, [](uint32_t x, uint32_t y) { return x < y ? x : y; });
    longest = wave_reduce(longest, umax);
    first[0] = wave_scan(listed[0] + listed[1] + listed[2] + listed[3], count);
#pragma unroll
    for (int i = 1; i < 4; ++i) first[i] = first[i - 1] + listed[i - 1];
    Border fine = b;                                  // of what is still in question
    const double all = row.k > 0 ? (double)b.mass_k : b.sum * kUnit;
    const Goals rough = {row, b, weigh, all, 0, -1};
    Goals g = {row, fine, weigh, all, high, -1};
    // `ties` of the equal elements `key`, listed[] and first[] of them in the chunks
    auto split_ties = [&](uint32_t key, uint32_t of_them) {
      const double e = g.weight(key);
      const uint64_t w = units(e);
      uint64_t ties = of_them;
      if (g.ends_in_k()) {
        const uint64_t of_k = (uint64_t)row.k - fine.count_k;
        ties = of_k < ties ? of_k : ties;
      }
      if (row.p < 1.0) ties = g.let_in(g.goal(g.ends_in_k() ? ties * w : 0), fine.mass_lo, w, ties);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint64_t left = ties > first[i] ? ties - first[i] : 0;
        if (e >= row.m) kept[i] += (left < listed[i] ? left : listed[i]) * w;
      }
      end = {key, 0, ties};
    };
    const bool apart = rough.ends_in_k() && b.bin_k > b.hi;   // bin_k behind the others
    if (count == 0) {
      // everything in the bins is kept (min-p alone: everything)
      if (row.binned()) end.key = 0xffffffffu;
    } else if (high == low) {
      // equal elements, however many
      split_ties(high, count);
      if (tid < kWave)
#pragma unroll
        for (int i = 0; i < 4; ++i) lds.ties_of[4 * lane + i] = listed[i];
      __syncthreads();
    } else if (longest > (uint32_t)kListed || (apart && count > (uint32_t)kMaxSorted)) {
      end = end_by_passes(logits, a.V, rough, a.chunks, chunk_len, lds);
      b.lo = -1;                                      // the bins say nothing
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) kept[i] = i < mine ? lds.kept_of[4 * lane + i] : 0;
    } else {
      if (tid < kWave)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          lds.kept_of[4 * lane + i] = kept[i], lds.first_of[4 * lane + i] = first[i];
      const uint32_t listed_all = count;
      if (tid == 0) lds.count = 0, lds.high = 0, lds.low = 0xffffffffu;
      uint32_t below = 0xffffffffu;                   // keys above it are kept if none listed is
      if (count <= kWave || apart) {
        __syncthreads();
        for_listed<kN>(a, n, 0, listed_all, lds.first_of,
                   [&](int, uint64_t x) { lds.sorted[atomicAdd(&lds.count, 1u)] = x; });
        __syncthreads();
      } else {
        // 512 bins of the listed keys' range, and the end's among them. The first elements of
        // a thread, mostly all, stay in registers from one pass to the next.
        const uint32_t span = high - low;
        g.shift = span < (uint32_t)kBins ? 0 : 32 - __clz(span / kBins);
        for (int i = tid; i < kBins; i += kN) lds.mass[i] = 0, lds.counts[i] = 0;
        constexpr int kHeld = 2048 / kN;
        uint64_t held[kHeld], weight[kHeld];
        int of_chunk[kHeld];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kHeld; ++j) {
          const uint32_t i = tid + j * kN;
          of_chunk[j] = chunk_of(lds.first_of, i);
          held[j] = i < listed_all ? a.list[((int64_t)n * a.chunks + of_chunk[j]) * kListed +
                                            (i - lds.first_of[of_chunk[j]])]
                                   : 0;
        }
        auto put = [&](uint64_t x, uint64_t w) {
          const int bin = g.bin((uint32_t)(x >> 32));
          atomicAdd(&lds.counts[bin], 1u);
          atomicAdd((unsigned long long *)&lds.mass[bin], (unsigned long long)w);
        };
        auto units_of = [&](uint64_t x) { return units(g.weight((uint32_t)(x >> 32))); };
#pragma unroll
        for (int j = 0; j < kHeld; ++j)
          if (held[j]) put(held[j], weight[j] = units_of(held[j]));
        for_listed<kN>(a, n, kHeld * kN, listed_all, lds.first_of,
                   [&](int, uint64_t x) { put(x, units_of(x)); });
        __syncthreads();
        uint64_t m[kOwnBins];
        uint32_t c[kOwnBins];
#pragma unroll
        for (int i = 0; i < kOwnBins; ++i)
          m[i] = lds.mass[kOwnBins * lane + i], c[i] = lds.counts[kOwnBins * lane + i];
        locate(m, c, b.mass_lo, b.count_lo, rough.ends_in_k(), (uint32_t)row.k, row.p, all, fine);
        if (fine.lo > 0) below = high - ((uint32_t)fine.lo << g.shift);
        auto settle = [&](int chunk, uint64_t x, uint64_t w) {
          const uint32_t key = (uint32_t)(x >> 32);
          const int bin = g.bin(key);
          if (bin < fine.lo) {
            if (row.m == 0.0 || g.weight(key) >= row.m)
              atomicAdd((unsigned long long *)&lds.kept_of[chunk], (unsigned long long)w);
          } else if (bin <= fine.hi || bin == fine.bin_k) {
            const uint32_t slot = atomicAdd(&lds.count, 1u);
            if (slot < (uint32_t)kMaxSorted) lds.sorted[slot] = x;
            atomicMax(&lds.high, key);
            atomicMin(&lds.low, key);
          }
        };
#pragma unroll
        for (int j = 0; j < kHeld; ++j)
          if (held[j]) settle(of_chunk[j], held[j], weight[j]);
        for_listed<kN>(a, n, kHeld * kN, listed_all, lds.first_of,
                   [&](int chunk, uint64_t x) { settle(chunk, x, units_of(x)); });
        __syncthreads();
        count = lds.count;
        high = lds.high;
        low = lds.low;
      }
      if (count > 0 && high == low) {
        if (tid < kMaxChunks) lds.ties_of[tid] = 0;
        __syncthreads();
        for_listed<kN>(a, n, 0, listed_all, lds.first_of, [&](int chunk, uint64_t x) {
          if ((uint32_t)(x >> 32) == high) atomicAdd(&lds.ties_of[chunk], 1u);
        });
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          listed[i] = lds.ties_of[4 * lane + i];
          kept[i] = lds.kept_of[4 * lane + i];
        }
        first[0] = wave_scan(listed[0] + listed[1] + listed[2] + listed[3], count);
#pragma unroll
        for (int i = 1; i < 4; ++i) first[i] = first[i - 1] + listed[i - 1];
        split_ties(high, count);
      } else if (count > (uint32_t)kMaxSorted) {
        end = end_by_passes(logits, a.V, rough, a.chunks, chunk_len, lds);
        b.lo = -1;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 4; ++i) kept[i] = i < mine ? lds.kept_of[4 * lane + i] : 0;
      } else {
        if (count <= kWave) {
          if (tid < kWave) {
            end = end_in_a_wave((uint32_t)lane < count ? lds.sorted[lane] : 0, g, chunk_len, lds);
            if (lane == 0) lds.key = end.key, lds.ties = end.index;
          }
          __syncthreads();
          end.key = lds.key, end.index = lds.ties;
        } else {
          end = end_by_sorting(count, g, chunk_len, lds);
        }
        if (end.key == 0xffffffffu) end = {below, 0, below == 0xffffffffu ? kByIndex : 0};
#pragma unroll
        for (int i = 0; i < 4; ++i) kept[i] = lds.kept_of[4 * lane + i];
      }
    }
    drawn = draw_chunk(kept, u);
  }

  // the draw within the chunk: neighbouring elements a thread
  constexpr int kOwn = chunk_len / kN;
  const int v0 = drawn.chunk * chunk_len + tid * kOwn;
  const double goal = (double)u * drawn.total;
  float z[kOwn];
  load_neighbours<T, kOwn>(logits, v0, a.V, z);
  uint64_t seen = 0;
  if (end.ties != kByIndex) {
    uint64_t equal = 0, all;
#pragma unroll
    for (int i = 0; i < kOwn; ++i) equal += v0 + i < a.V && key_of(z[i]) == end.key;
    seen = group_scan<kN>(equal, all, lds.mpart);
    if (end.ties > 0)
      for (int c = 0; c < drawn.chunk; ++c) seen += lds.ties_of[c];
  }
  double w[kOwn], own = 0.0, all;
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    double e = 0.0;
    if (row.filtered()) {
      const uint32_t key = key_of(z[i]);
      const bool tied = key == end.key && (end.ties == kByIndex ? (uint32_t)(v0 + i) <= end.index
                                                                : seen++ < end.ties);
      const bool sure = b.lo >= 0 && (!row.binned() || bin_of(below(top, z[i]), b.rate) < b.lo);
      if (key > end.key || tied || sure) e = weigh(z[i]);
    } else {
      e = weight_exp(scaled(z[i], top, row.inv_t));
    }
    w[i] = e < row.m ? 0.0 : row.filtered() ? (double)units(e) : e;
    own += w[i];
  }
  if (tid == 0) lds.token = -1;
  const double before = drawn.before + group_scan<kN>(own, all, lds.dpart);
  // the first element whose running sum passes the goal; should rounding leave none, the
  // last that weighs anything
  int token = -1;
  double run = before;
#pragma unroll
  for (int i = 0; i < kOwn; ++i) {
    const bool past = run > goal;                     // an element before did
    run += w[i];
    if (w[i] > 0.0 && !past) token = v0 + i;
  }
  if (token >= 0 && before <= goal) atomicMax(&lds.token, token);
  __syncthreads();
  if (token >= 0 && token == lds.token) {
    a.tokens[n] = token;
    if (a.logprob) {
      float zt = 0.f;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) zt = v0 + i == token ? z[i] : zt;
      a.logprob[n] = (float)(scaled(zt, top, row.inv_t) -
                             log(row.filtered() ? drawn.total / kUnit : drawn.total));
    }
  }
}

// Elements a lane holds of a chunk: 32 (chunks of 2,048), and fewer where the call would have
// few workgroups and the row's chunks still fit. Measured, bf16 with top-p, by 8 / 16 / 32: a
// row of 32,000 24 / 27 / 38 us, 32 of 128,000 41 / 37 / 40, 128 of 32,000 39 / 36 / 42; by
// 16 / 32: 64 of 100,000 47 / 52, 64 of 151,936 equal, 256 of them 146 / 139.
int32_t sample_per(int32_t N, int32_t V) {
  auto chunks = [&](int32_t per) { return ((int64_t)V + kWave * per - 1) / (kWave * per); };
  if (chunks(16) > kMaxChunks || N * chunks(32) > 8 * kGroup * 256) return 32;
  if (chunks(8) > kMaxChunks || N * chunks(16) >= 2 * kGroup * 256) return 16;
  return 8;
}

struct SampleLayout {
  int32_t per, chunks;
  size_t stats, l_top, bin_mass, bin_count, kept, list, border, ends;
  size_t bytes;
};
SampleLayout sample_layout(int32_t N, int32_t V) {
  SampleLayout l;
  l.per = sample_per(N, V);
  l.chunks = (V + kWave * l.per - 1) / (kWave * l.per);
  const size_t parts = (size_t)N * l.chunks, groups = (size_t)N * ((l.chunks + kGroup - 1) / kGroup);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t here = at;
    at += (bytes + 255) / 256 * 256;
    return here;
  };
  l.stats = take(groups * sizeof(Stats));
  l.l_top = take(parts * kWave * 4);
  l.bin_mass = take((size_t)N * kBins * 8);
  l.bin_count = take((size_t)N * kBins * 4);
  l.kept = take(groups * sizeof(Kept));
  l.list = take(parts * kListed * 8);
  l.border = take((size_t)N * sizeof(BorderLine));
  l.ends = take((size_t)N * sizeof(BorderLine));
  l.bytes = at + sizeof(Stats);         // to a line's start
  return l;
}

template <typename T, int kPer>
void launch_passes(const SampleArgs &a, hipStream_t stream) {
  const dim3 grid((unsigned)a.N * (unsigned)a.groups);
  const bool bins = a.top_k || a.top_p;
  hipLaunchKernelGGL((sample_stats_kernel<T, kPer>), grid, dim3(kThreads), 0, stream, a);
  if (bins || a.min_p)
    hipLaunchKernelGGL(sample_range_kernel, dim3(a.N), dim3(kRowThreads), 0, stream, a);
  if (bins) hipLaunchKernelGGL((sample_bins_kernel<T, kPer>), grid, dim3(kThreads), 0, stream, a);
  if (bins || a.min_p)
    hipLaunchKernelGGL((sample_border_kernel<T, kPer>), grid, dim3(kThreads), 0, stream, a);
  constexpr int kMany = kPer > 8 ? 512 : 256;
  if (bins)
    hipLaunchKernelGGL((sample_pick_kernel<T, kPer, kMany>), dim3(a.N), dim3(kMany), 0, stream, a);
  else
    hipLaunchKernelGGL((sample_pick_kernel<T, kPer, 256>), dim3(a.N), dim3(256), 0, stream, a);
}

}  // namespace

size_t sample_workspace_bytes(int32_t N, int32_t V) { return sample_layout(N, V).bytes; }

hipError_t launch_sample(const void *logits, bool bf16, int32_t N, int32_t V, int64_t row_stride,
                         const float *temperature, const int32_t *top_k, const float *top_p,
                         const float *min_p, const float *uniform, int32_t *tokens,
                         float *logprob, void *workspace, hipStream_t stream) {
  const SampleLayout l = sample_layout(N, V);
  char *ws = reinterpret_cast<char *>((reinterpret_cast<uintptr_t>(workspace) + sizeof(Stats) - 1) /
                                      sizeof(Stats) * sizeof(Stats));
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
  a.groups = (l.chunks + kGroup - 1) / kGroup;
  a.stats = reinterpret_cast<Stats *>(ws + l.stats);
  a.bin_mass = reinterpret_cast<uint64_t *>(ws + l.bin_mass);
  a.bin_count = reinterpret_cast<uint32_t *>(ws + l.bin_count);
  a.kept = reinterpret_cast<Kept *>(ws + l.kept);
  a.list = reinterpret_cast<uint64_t *>(ws + l.list);
  a.l_top = reinterpret_cast<float *>(ws + l.l_top);
  a.border = reinterpret_cast<BorderLine *>(ws + l.border);
  a.ends = reinterpret_cast<BorderLine *>(ws + l.ends);
  auto launch = [&](auto per) {
    constexpr int kPer = decltype(per)::value;
    if (bf16)
      launch_passes<uint16_t, kPer>(a, stream);
    else
      launch_passes<float, kPer>(a, stream);
  };
  if (l.per == 8)
    launch(std::integral_constant<int, 8>());
  else if (l.per == 16)
    launch(std::integral_constant<int, 16>());
  else
    launch(std::integral_constant<int, 32>());
  return hipGetLastError();
}

}  // namespace ra
