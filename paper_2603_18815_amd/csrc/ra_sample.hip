// Drawing a token from a row of logits (token_sample): temperature, top-k, top-p and min-p
// filters, then the inverse of the cumulative distribution at a given uniform number.
//
// With M the row's largest logit, an element's weight is e = exp((z - M) / T), held as a
// whole number of units of 2^-44 (0 below half a unit, 31.2 below M). Sums of whole numbers
// do not depend on their order, so every sum here is exact whichever threads add it up, and
// a draw falls on the token that sums in 64-bit floating point give: a sum of V weights is
// off by at most V half units, 2^-45 of the largest weight each. V <= 2^19 keeps a row's
// sum below 2^63.
//
// All filters keep a prefix of the order (logit descending, index ascending). A prefix is a
// logit and how many of the elements equal to it are in: those of the lowest indices. The
// weights of equal elements are equal, so neither filter needs the indices.
#include "ra_device.h"
#include "ra_internal.h"

namespace ra {
namespace {

constexpr int kThreads = 1024;
constexpr double kUnit = 0x1p44;


__device__ __forceinline__ float load_logit(const float *p) { return *p; }
__device__ __forceinline__ float load_logit(const uint16_t *p) {
  return __uint_as_float((uint32_t)*p << 16);
}

// Order of fp32 values as that of whole numbers; NaN counts as -inf, -0 as 0.
__device__ __forceinline__ uint32_t key_of(float z) {
  z = z != z ? -__builtin_inff() : z + 0.f;
  const uint32_t u = __float_as_uint(z);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float value_of(uint32_t key) {
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
constexpr uint32_t kKeyNone = 0x007fffffu;   // -inf

// exp(x) for x <= 0 (0 below -31.5 and for NaN): exp(x) = 2^n exp(r), |r| <= ln 2 / 2, and
// the Taylor series of exp(r) to r^13, whose next term is below 2^-57.
__device__ __forceinline__ double weight_exp(double x) {
  const double n = __builtin_rint(x * 1.4426950408889634);
  // ln 2 in two parts, the first of 38 bits: its products with n are exact
  const double r = __builtin_fma(n, -0x1.cf79abc9e3b3ap-40, __builtin_fma(n, -0x1.62e42fefap-1, x));
  double p = 1.0 / 6227020800.0;
  p = __builtin_fma(p, r, 1.0 / 479001600.0);
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
  return x >= -31.5 ? __builtin_ldexp(p, (int)n) : 0.0;
}

__device__ __forceinline__ double scaled(float z, float top, double inv_t) {
  return z == top ? 0.0 : ((double)z - (double)top) * inv_t;
}
__device__ __forceinline__ uint64_t units(double e) { return (uint64_t)(e * kUnit + 0.5); }

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_row_kernel(
    const T *logits, int64_t row_stride, int32_t V, const float *temperature,
    const int32_t *top_k, const float *top_p, const float *min_p, const float *uniform,
    int32_t *tokens, float *logprob) {
  const int n = blockIdx.x, tid = threadIdx.x;
  const T *row = logits + n * row_stride;
  __shared__ uint64_t s_mass[kThreads];
  __shared__ uint32_t s_count[kThreads];
  __shared__ uint64_t s_best;
  __shared__ uint32_t s_key;
  __shared__ uint64_t s_above;
  __shared__ uint32_t s_ties;

  // largest logit, at its lowest index
  if (tid == 0) s_best = 0;
  __syncthreads();
  uint64_t best = 0;
  for (int v = tid; v < V; v += kThreads) {
    const uint64_t c = (uint64_t)key_of(load_logit(row + v)) << 32 | (uint32_t)~v;
    best = c > best ? c : best;
  }
  atomicMax((unsigned long long *)&s_best, (unsigned long long)best);
  __syncthreads();
  const uint32_t top_key = (uint32_t)(s_best >> 32);
  const float top = value_of(top_key);
  const float temp = temperature ? temperature[n] : 1.f;
  if (top_key == kKeyNone || !(temp > 0.f)) {
    if (tid == 0) {
      tokens[n] = top_key == kKeyNone ? -1 : (int)~(uint32_t)s_best;
      if (logprob) logprob[n] = top_key == kKeyNone ? __builtin_nanf("") : 0.f;
    }
    return;
  }
  const double inv_t = 1.0 / (double)temp;
  const int k = top_k ? top_k[n] : 0;
  const double p = top_p ? (double)top_p[n] : 1.0;
  const double m = min_p ? (double)min_p[n] : 0.0;

  // the prefix: keys above `edge`, and `ties` elements at it
  uint32_t edge = kKeyNone, ties = 0xffffffffu;
  for (int round = 0; round < 2; ++round) {
    const bool by_mass = round == 1;
    if (by_mass ? !(p < 1.0) : !(k > 0 && k < V)) continue;
    uint64_t want = 0;
    double goal = 0.0;
    if (by_mass) {
      // mass of the elements that top-k keeps
      if (tid == 0) s_above = 0, s_ties = 0;
      __syncthreads();
      uint64_t mass = 0;
      uint32_t at = 0;
      for (int v = tid; v < V; v += kThreads) {
        const float z = load_logit(row + v);
        const uint32_t key = key_of(z);
        if (key > edge) mass += units(weight_exp(scaled(value_of(key), top, inv_t)));
        at += key == edge;
      }
      atomicAdd((unsigned long long *)&s_above, (unsigned long long)mass);
      atomicAdd(&s_ties, at);
      __syncthreads();
      const uint64_t e = units(weight_exp(scaled(value_of(edge), top, inv_t)));
      // at least half a unit: the first element is always kept
      goal = fmax(p * (double)(s_above + (uint64_t)min(s_ties, ties) * e), 0.5);
      __syncthreads();
    } else {
      want = k;
    }
    // the edge's key, eight bits a pass from the top: the first bin, from the largest
    // key down, at which the count reaches k or the mass the goal
    uint32_t prefix = 0;
    uint64_t sum = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) s_mass[tid] = 0, s_count[tid] = 0;
      __syncthreads();
      for (int v = tid; v < V; v += kThreads) {
        const uint32_t key = key_of(load_logit(row + v));
        if (shift < 24 && (key >> (shift + 8)) != (prefix >> (shift + 8))) continue;
        if (key < edge) continue;
        if (by_mass)
          atomicAdd((unsigned long long *)&s_mass[(key >> shift) & 255],
                    (unsigned long long)units(weight_exp(scaled(value_of(key), top, inv_t))));
        atomicAdd(&s_count[(key >> shift) & 255], 1u);
      }
      __syncthreads();
      if (tid == 0) {
        uint64_t run = sum;
        int bin = 255;
        for (; bin > 0; --bin) {
          const uint64_t next = run + (by_mass ? s_mass[bin] : (uint64_t)s_count[bin]);
          if (by_mass ? !((double)next < goal) : next >= want) break;
          run = next;
        }
        s_key = prefix | (uint32_t)bin << shift;
        s_above = run;
        s_ties = s_count[bin];
      }
      __syncthreads();
      prefix = s_key;
      sum = s_above;
      __syncthreads();
    }
    if (by_mass) {
      const uint64_t e = units(weight_exp(scaled(value_of(prefix), top, inv_t)));
      uint64_t r = s_ties;
      if (e > 0) {
        const double more = (goal - (double)sum) / (double)e;
        r = more <= 1.0 ? 1 : more >= (double)s_ties ? s_ties : (uint64_t)__builtin_ceil(more);
      }
      if (prefix == edge && r > ties) r = ties;
      edge = prefix;
      ties = (uint32_t)r;
    } else {
      edge = prefix;
      ties = (uint32_t)(want - sum);
    }
    __syncthreads();
  }

  // each thread's stretch of the row: its ties, then the mass it keeps, then the draw
  const int len = (V + kThreads - 1) / kThreads;
  const int v0 = min(V, tid * len), v1 = min(V, v0 + len);
  uint32_t at = 0;
  for (int v = v0; v < v1; ++v) at += key_of(load_logit(row + v)) == edge;
  s_count[tid] = at;
  __syncthreads();
  uint64_t tie0 = 0;
  for (int t = 0; t < tid; ++t) tie0 += s_count[t];
  const double floor_e = m > 0.0 ? (m < 1.0 ? m : 1.0) : 0.0;
  auto kept = [&](int v, uint64_t &seen) -> uint64_t {
    const uint32_t key = key_of(load_logit(row + v));
    if (key < edge) return 0;
    if (key == edge && seen++ >= ties) return 0;
    const double e = weight_exp(scaled(value_of(key), top, inv_t));
    return e >= floor_e ? units(e) : 0;
  };
  uint64_t mass = 0, seen = tie0;
  for (int v = v0; v < v1; ++v) mass += kept(v, seen);
  s_mass[tid] = mass;
  __syncthreads();
  uint64_t before = 0, total = 0;
  for (int t = 0; t < kThreads; ++t) {
    if (t == tid) before = total;
    total += s_mass[t];
  }
  float u = uniform[n];
  u = u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f;
  const double goal = (double)u * (double)total;
  if ((double)before <= goal && (double)(before + mass) > goal) {
    uint64_t run = before;
    seen = tie0;
    for (int v = v0; v < v1; ++v) {
      run += kept(v, seen);
      if ((double)run > goal) {
        tokens[n] = v;
        if (logprob)
          logprob[n] = (float)(scaled(value_of(key_of(load_logit(row + v))), top, inv_t) -
                               log((double)total / kUnit));
        break;
      }
    }
  }
}

}  // namespace

size_t sample_workspace_bytes(int32_t N, int32_t V) { return (size_t)0 * N * V; }

hipError_t launch_sample(const void *logits, bool bf16, int32_t N, int32_t V, int64_t row_stride,
                         const float *temperature, const int32_t *top_k, const float *top_p,
                         const float *min_p, const float *uniform, int32_t *tokens,
                         float *logprob, void *workspace, hipStream_t stream) {
  if (bf16)
    hipLaunchKernelGGL(sample_row_kernel<uint16_t>, dim3(N), dim3(kThreads), 0, stream,
                       static_cast<const uint16_t *>(logits), row_stride, V, temperature, top_k,
                       top_p, min_p, uniform, tokens, logprob);
  else
    hipLaunchKernelGGL(sample_row_kernel<float>, dim3(N), dim3(kThreads), 0, stream,
                       static_cast<const float *>(logits), row_stride, V, temperature, top_k,
                       top_p, min_p, uniform, tokens, logprob);
  return hipGetLastError();
}

}  // namespace ra
