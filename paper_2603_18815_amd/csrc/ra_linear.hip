// Linear attention with a decay for each KV head: rollout_linear_attn_decode (one token a
// row) and rollout_linear_attn_append (new tokens after a row's earlier ones). A row's
// history is a state of fixed size in place of pages:
//   S_t = l S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t,   l = exp(log_decay) per KV head.
#include "ra_device.h"
#include "ra_internal.h"

namespace ra {
namespace {

constexpr int kThreads = 256;

// The recurrence itself, a workgroup per (row, KV head), token by token. Thread t holds
// column t % 128 of the state, the 64 key dims of half t / 128, in registers.
__global__ __launch_bounds__(kThreads) void linear_recurrent_kernel(
    const uint16_t *q, const uint16_t *k, const uint16_t *v, const int32_t *cu_q,
    const int32_t *lens, float *states, const int32_t *slots, int32_t num_slots,
    const float *log_decay, int32_t hq, int32_t hkv, int32_t total_q, float scale,
    uint16_t *out) {
  const int b = blockIdx.y, g = blockIdx.x, tid = threadIdx.x;
  const int col = tid % kHeadDim, half = tid / kHeadDim, group = hq / hkv;
  const int slot = slots[b];
  // decode (no cu_q): one token, lens counts it; append: lens are the tokens before
  int t0 = b, t1 = b + 1;
  bool fresh;
  bool live = slot >= 0 && slot < num_slots;
  if (cu_q) {
    t0 = min(max(cu_q[b], 0), total_q);
    t1 = min(max(cu_q[b + 1], t0), total_q);
    fresh = lens[b] <= 0;
  } else {
    live = live && lens[b] > 0;
    fresh = lens[b] <= 1;
  }
  __shared__ float sk[kHeadDim], sq[kHeadDim], part[kHeadDim];
  if (!live) {
    for (int t = t0; t < t1; ++t)
      for (int i = tid; i < group * kHeadDim; i += kThreads)
        out[((int64_t)t * hq + g * group) * kHeadDim + i] = 0;
    return;
  }
  if (t0 == t1) return;
  float *state = states + ((int64_t)slot * hkv + g) * kHeadDim * kHeadDim;
  // the decay in two parts: its rounding to fp32 alone would be felt after 2^24 / t of t steps
  const double decay = exp((double)fminf(log_decay[g], 0.f));
  const float l = (float)decay, l_low = (float)(decay - (double)l);
  float s[64];
#pragma unroll
  for (int i = 0; i < 64; ++i)
    s[i] = fresh ? 0.f : state[(half * 64 + i) * kHeadDim + col];
  for (int t = t0; t < t1; ++t) {
    __syncthreads();
    if (tid < kHeadDim)
      sk[tid] = __uint_as_float((uint32_t)k[((int64_t)t * hkv + g) * kHeadDim + tid] << 16);
    const float vc = __uint_as_float((uint32_t)v[((int64_t)t * hkv + g) * kHeadDim + col] << 16);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 64; ++i) s[i] = fmaf(l, s[i], fmaf(l_low, s[i], sk[half * 64 + i] * vc));
    for (int h = 0; h < group; ++h) {
      const int64_t at = ((int64_t)t * hq + g * group + h) * kHeadDim;
      __syncthreads();
      if (tid < kHeadDim) sq[tid] = __uint_as_float((uint32_t)q[at + tid] << 16);
      __syncthreads();
      float o = 0.f;
#pragma unroll
      for (int i = 0; i < 64; ++i) o = fmaf(sq[half * 64 + i], s[i], o);
      if (half) part[col] = o;
      __syncthreads();
      if (!half) out[at + col] = __builtin_bit_cast(uint16_t, (__bf16)(scale * (o + part[col])));
    }
  }
#pragma unroll
  for (int i = 0; i < 64; ++i) state[(half * 64 + i) * kHeadDim + col] = s[i];
}

}  // namespace

size_t linear_append_workspace_bytes(int32_t B, int32_t hq, int32_t hkv, int32_t total_q,
                                     int32_t max_q_len) {
  return 0;
}

hipError_t launch_linear_decode(const uint16_t *q, const uint16_t *k, const uint16_t *v,
                                float *states, const int32_t *slots, int32_t num_slots,
                                const int32_t *kv_lens, const float *log_decay, int32_t B,
                                int32_t hq, int32_t hkv, float scale, uint16_t *out,
                                hipStream_t stream) {
  hipLaunchKernelGGL(linear_recurrent_kernel, dim3(hkv, B), dim3(kThreads), 0, stream, q, k, v,
                     nullptr, kv_lens, states, slots, num_slots, log_decay, hq, hkv, B, scale, out);
  return hipGetLastError();
}

hipError_t launch_linear_append(const uint16_t *q, const uint16_t *k, const uint16_t *v,
                                const int32_t *cu_q, const int32_t *ctx_lens, float *states,
                                const int32_t *slots, int32_t num_slots, const float *log_decay,
                                int32_t B, int32_t hq, int32_t hkv, int32_t total_q,
                                int32_t max_q_len, float scale, uint16_t *out, void *workspace,
                                hipStream_t stream) {
  hipLaunchKernelGGL(linear_recurrent_kernel, dim3(hkv, B), dim3(kThreads), 0, stream, q, k, v,
                     cu_q, ctx_lens, states, slots, num_slots, log_decay, hq, hkv, total_q, scale,
                     out);
  return hipGetLastError();
}

}  // namespace ra
