// Linear attention with a decay for each KV head: rollout_linear_attn_decode (one token a
// row) and rollout_linear_attn_append (new tokens after a row's earlier ones). A row's
// history is a state of fixed size in place of pages:
//   S_t = l S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t,   l = exp(log_decay) per KV head.
//
// Decode reads and writes the state, 128 KiB a (row, KV head), and is bound by that.
//
// Append takes chunks of 64 tokens on the matrix cores. With i, j a chunk's tokens, S the
// state before it and n its length:
//   o_i = scale (l^(i+1) S^T q_i + sum_{j <= i} l^(i-j) <q_i, k_j> v_j)
//   S'  = l^n S + sum_j k_j (l^(n-1-j) v_j)^T
// A row's chunks follow one another; with too few (row, KV head) pairs to fill the GPU the
// row is cut into stretches: their own contributions to the state first (states pass), then
// the state before each (scan), then the outputs (outputs pass).
#include "ra_device.h"
#include "ra_internal.h"

namespace ra {
namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kChunk = 64;              // tokens of a chunk
constexpr int kStateSize = kHeadDim * kHeadDim;

struct LinearArgs {
  const uint16_t *q, *k, *v;
  const int32_t *cu_q, *ctx_lens;
  float *states;
  const int32_t *slots;
  const float *log_decay;
  uint16_t *out;
  float *carry;                         // [B][Hkv][segments] states (cut rows only)
  int32_t num_slots, B, hq, hkv, total_q, max_q_len;
  int32_t segments, segment_len;        // stretches a row has at most, tokens of each
  int32_t head_splits;                  // workgroups that share a group's query heads
  float scale;
};

__device__ __forceinline__ double log_decay_of(const float *log_decay, int g) {
  const float x = log_decay[g];
  return x < 0.f ? fmax((double)x, -1e30) : 0.0;   // NaN and larger values: no decay
}

// ---- decode ---------------------------------------------------------------------------
// A workgroup per (row, KV head). Thread t holds column t % 128 of the state, the 64 key
// dims of half t / 128, in registers.
__global__ __launch_bounds__(kThreads) void linear_decode_kernel(
    const uint16_t *q, const uint16_t *k, const uint16_t *v, const int32_t *kv_lens,
    float *states, const int32_t *slots, int32_t num_slots, const float *log_decay, int32_t hq,
    int32_t hkv, float scale, uint16_t *out) {
  const int b = blockIdx.y, g = blockIdx.x, tid = threadIdx.x;
  const int col = tid % kHeadDim, half = tid / kHeadDim, group = hq / hkv;
  const int slot = slots[b], len = kv_lens[b];
  uint16_t *o_row = out + ((int64_t)b * hq + g * group) * kHeadDim;
  if (slot < 0 || slot >= num_slots || len <= 0) {
    for (int i = tid; i < group * kHeadDim; i += kThreads) o_row[i] = 0;
    return;
  }
  __shared__ float sk[kHeadDim], sq[kHeadDim], part[kHeadDim];
  float *state = states + ((int64_t)slot * hkv + g) * kStateSize;
  // the decay in two parts: its rounding to fp32 alone would be felt after 2^24 / t of t steps
  const double decay = exp(log_decay_of(log_decay, g));
  const float l = (float)decay, l_low = (float)(decay - (double)l);
  if (tid < kHeadDim)
    sk[tid] = __uint_as_float((uint32_t)k[((int64_t)b * hkv + g) * kHeadDim + tid] << 16);
  const float vc = __uint_as_float((uint32_t)v[((int64_t)b * hkv + g) * kHeadDim + col] << 16);
  __syncthreads();
  float s[64];
#pragma unroll
  for (int i = 0; i < 64; ++i)
    s[i] = len == 1 ? 0.f : state[(half * 64 + i) * kHeadDim + col];
#pragma unroll
  for (int i = 0; i < 64; ++i) {
    s[i] = fmaf(l, s[i], fmaf(l_low, s[i], sk[half * 64 + i] * vc));
    state[(half * 64 + i) * kHeadDim + col] = s[i];
  }
  for (int h = 0; h < group; ++h) {
    __syncthreads();
    if (tid < kHeadDim)
      sq[tid] = __uint_as_float((uint32_t)q[((int64_t)b * hq + g * group + h) * kHeadDim + tid] << 16);
    __syncthreads();
    float o = 0.f;
#pragma unroll
    for (int i = 0; i < 64; ++i) o = fmaf(sq[half * 64 + i], s[i], o);
    if (half) part[col] = o;
    __syncthreads();
    if (!half)
      o_row[h * kHeadDim + col] = __builtin_bit_cast(uint16_t, (__bf16)(scale * (o + part[col])));
  }
}

// ---- append: LDS tiles ----------------------------------------------------------------
// A tile holds 64 tokens of 128 bf16 in 16-byte units, unit u of row r at u ^ swizzle(r):
// 16 rows at one unit, and 4 rows at two neighbouring units, fall on different banks, so
// that the reads along a token and the transposing reads along a dim are both spread.
__device__ __forceinline__ int swizzle(int row) { return (row & 7) << 1 | (row >> 3 & 1); }
__device__ __forceinline__ int tile_at(int row, int dim) {     // in elements; dim % 4 == 0
  return row * kHeadDim + (((dim >> 3) ^ swizzle(row)) << 3) + (dim & 4);
}
__device__ __forceinline__ int score_at(int row, int col) {    // [64][64] scores, col % 4 == 0
  return row * kChunk + (((col >> 3) ^ (row >> 1 & 7)) << 3) + (col & 4);
}

__device__ __forceinline__ bf16x8 join(bf16x4 a, bf16x4 b) {
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// Operands of 32 contraction slots: lane l's eight are 4 (l / 16) + 0..3 and 16 more, the
// order in which two accumulator tiles hold their rows.
__device__ __forceinline__ bf16x8 read_rows(const uint16_t *tile, int row, int dim) {
  return join(*reinterpret_cast<const bf16x4 *>(tile + tile_at(row, dim)),
              *reinterpret_cast<const bf16x4 *>(tile + tile_at(row, dim + 16)));
}

// ds_read_b64_tr_b16: of 16 lanes, lane i supplies the address of row i / 4's four columns
// at i % 4 and receives column i of the four rows.
__device__ __forceinline__ bf16x4 read_transposed(const uint16_t *at) {
  typedef __attribute__((address_space(3))) s16x4 lds_t;
  return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                                        (lds_t *)const_cast<uint16_t *>(at)));
}

// The bf16 rounding of x, taken off x.
__device__ __forceinline__ bf16x8 take_bf16(f32x8 &x) {
  const bf16x8 h = to_bf16x8(x);
  x -= to_f32x8(h);
  return h;
}

enum { kWhole, kStates, kOutputs };

// 16 bytes a lane from global memory to LDS, lane l's at `lds` + 16 l (lds and lane 0's
// address are the wave's). In assembly: behind the builtin the compiler waits for all such
// loads before any LDS read; here await_loads() does, before the barrier that hands the
// tile over.
__device__ __forceinline__ void load_to_lds(const uint16_t *g, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, off"
      :
      : "s"(lds), "v"(g)
      : "memory", "m0");
}
__device__ __forceinline__ void await_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
__device__ __forceinline__ uint32_t lds_address(const uint16_t *p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p;
}

// One stretch of a (row, KV head): chunks in order, the state in the accumulators. Wave w
// holds the 32 value dims from 32 w, all 128 key dims: tile (t, u), t < 8, u < 2, has key
// dims 16 t + 0..15 as its rows and value dims 32 w + 8 (c / 4) + 4 u + c % 4 as its
// columns c, so that a lane's accumulators of two result tiles are eight neighbouring
// value dims of a token. An accumulator tile of the state is the matrix operand of
// S^T Q^T as it stands, rounded to bf16. Scores go through LDS: wave w computes those of
// tokens 16 w .. 16 w + 15, all waves use all of them.
//
// A step is a chunk and a query head of the group, with two barriers: the step's tiles are
// there (scores, then with the chunk's last head the state's update); the scores are there
// (outputs, while the next chunk's K and V load; V's tile is free once the first head
// has its operands, K's after the update). Q has two tiles. 72 KB of LDS: two workgroups
// per CU, whose steps overlap.
template <int kMode>
__global__ __launch_bounds__(kThreads, 2) void linear_chunk_kernel(LinearArgs a) {
  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int r = lane % 16, quad = lane / 16;
  int unit = blockIdx.x;
  const int split = kMode == kStates ? 0 : unit % a.head_splits;
  if (kMode != kStates) unit /= a.head_splits;
  const int seg = kMode == kWhole ? 0 : unit % a.segments;
  if (kMode != kWhole) unit /= a.segments;
  const int g = unit % a.hkv, b = unit / a.hkv, group = a.hq / a.hkv;

  const int row0 = min(max(a.cu_q[b], 0), a.total_q);
  const int T = min(min(max(a.cu_q[b + 1], row0), a.total_q) - row0, a.max_q_len);
  const int from = kMode == kWhole ? 0 : seg * a.segment_len;
  if (from >= T) return;
  const int len = kMode == kWhole ? T : min(T - from, a.segment_len);
  const int h0 = group * split / a.head_splits, h1 = group * (split + 1) / a.head_splits;
  const int64_t tok0 = row0 + from;
  const int slot = a.slots[b];
  if (slot < 0 || slot >= a.num_slots) {
    if (kMode != kStates)
      for (int t = 0; t < len; ++t)
        for (int i = tid; i < (h1 - h0) * kHeadDim; i += kThreads)
          a.out[((tok0 + t) * a.hq + g * group + h0) * kHeadDim + i] = 0;
    return;
  }

  constexpr int kTile = kChunk * kHeadDim;
  constexpr int kVTiles = kMode == kStates ? 2 : 1, kKTiles = kMode == kStates ? 2 : 1;
  __shared__ __align__(1024) uint16_t sk[kKTiles * kTile], sv[kVTiles * kTile];
  __shared__ __align__(1024) uint16_t sq[kMode == kStates ? 8 : 2 * kTile];
  __shared__ __align__(1024) uint16_t sp[kMode == kStates ? 8 : kChunk * kChunk];
  __shared__ float power[kChunk + 1], power_low[kChunk + 1];   // l^n and what fp32 leaves out
  const double ld = log_decay_of(a.log_decay, g);
  const float l2 = (float)(ld * 1.4426950408889634);
  if (tid <= kChunk) {
    const double p = exp(ld * tid);
    power[tid] = (float)p;
    power_low[tid] = (float)(p - (double)(float)p);
  }

  // loads: wave w takes rows 16 w .. 16 w + 15 of a tile, four rows an instruction, lane l
  // the unit of row l / 16 that belongs at l % 16; rows past the end repeat the last one
  const uint32_t lds_k = lds_address(sk) + wave * 4096, lds_v = lds_address(sv) + wave * 4096;
  const uint32_t lds_q = lds_address(sq) + wave * 4096;
  const int ld_unit = (lane % 16) ^ (lane / 16 << 1);
  auto load = [&](uint32_t lds, const uint16_t *src, int c, int heads, int head) {
#pragma unroll
    for (int m = 0; m < 4; ++m) {
      const int t = min(c * kChunk + 16 * wave + 4 * m + lane / 16, len - 1);
      load_to_lds(src + ((tok0 + t) * heads + head) * kHeadDim +
                      ((ld_unit ^ ((m & 1) << 3 | m >> 1)) << 3),
                  lds + 1024 * m);
    }
  };
  const int chunks = (len + kChunk - 1) / kChunk;
  load(lds_k, a.k, 0, a.hkv, g);
  load(lds_v, a.v, 0, a.hkv, g);
  if (kMode != kStates) load(lds_q, a.q, 0, a.hq, g * group + h0);

  // state tile (t, u), register i: key dim 16 t + 4 quad + i, value dim `dv` + 4 u
  const int dv = 32 * wave + 8 * (r >> 2) + (r & 3);
  f32x4 s[8][2];
  float *pool = a.states + ((int64_t)slot * a.hkv + g) * kStateSize;
  float *carry = kMode == kWhole ? pool
                                 : a.carry + (((int64_t)b * a.hkv + g) * a.segments + seg) * kStateSize;
  const bool zero = kMode == kStates || (kMode == kWhole && a.ctx_lens[b] <= 0);
#pragma unroll
  for (int t = 0; t < 8; ++t)
#pragma unroll
    for (int u = 0; u < 2; ++u) s[t][u] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (!zero) {
    const float *at = carry + 4 * quad * kHeadDim + dv;
#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[t][u][i] = at[(16 * t + i) * kHeadDim + 4 * u];
  }

  const int tr_row = 4 * quad + (r >> 2);               // transposing reads: this lane's row
  // V^T of a chunk, rows the wave's value dims: [u][32 tokens x]
  auto read_v = [&](bf16x8(&vf)[2][2], const uint16_t *tile) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        const int d = 32 * wave + 8 * (r & 3) + 4 * u, row = 32 * x + tr_row;
        vf[u][x] = join(read_transposed(tile + tile_at(row, d)),
                        read_transposed(tile + tile_at(row + 16, d)));
      }
  };
  // S' = l^n S + K^T (l^(n-1-j) V): the decayed values in three bf16 parts, which hold all
  // 24 bits (the outputs pass needs the state as bf16 operands only: one part)
  auto update = [&](const bf16x8(&vf)[2][2], const uint16_t *tile, int n) {
    const float dh = power[n], dl = power_low[n];
#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[t][u][i] = fmaf(s[t][u][i], dh, s[t][u][i] * dl);
    constexpr int kParts = kMode == kOutputs ? 1 : 3;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      bf16x8 part[2][kParts];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        f32x8 y = to_f32x8(vf[u][x]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int j = 32 * x + 4 * quad + (e & 3) + (e & 4) * 4;
          y[e] = j < n ? y[e] * power[max(n - 1 - j, 0)] : 0.f;
        }
#pragma unroll
        for (int m = 0; m < kParts; ++m) part[u][m] = take_bf16(y);
      }
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const int row = 32 * x + tr_row, d = 16 * t + 4 * (r & 3);
        const bf16x8 kf = join(read_transposed(tile + tile_at(row, d)),
                               read_transposed(tile + tile_at(row + 16, d)));
#pragma unroll
        for (int m = 0; m < kParts; ++m)
#pragma unroll
          for (int u = 0; u < 2; ++u) s[t][u] = mfma16x16x32(kf, part[u][m], s[t][u]);
      }
    }
  };

  int buf = 0;
  for (int c = 0; c < chunks; ++c) {
    const int n = min(len - c * kChunk, kChunk);
    bf16x8 vf[2][2];
    if constexpr (kMode == kStates) {
      await_loads();
      __syncthreads();
      if (c + 1 < chunks) {
        load(lds_k + (buf ^ 1) * kTile * 2, a.k, c + 1, a.hkv, g);
        load(lds_v + (buf ^ 1) * kTile * 2, a.v, c + 1, a.hkv, g);
      }
      read_v(vf, sv + buf * kTile);
      update(vf, sk + buf * kTile, n);
      buf ^= 1;
    } else {
      bf16x8 sb[2][4];                                  // the state before the chunk, in bf16
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          sb[u][x] = to_bf16x8(__builtin_shufflevector(s[2 * x][u], s[2 * x + 1][u], 0, 1, 2, 3, 4,
                                                       5, 6, 7));
      for (int h = h0; h < h1; ++h) {
        const uint16_t *tq = sq + buf * kTile;
        const bool last = h + 1 == h1;
        await_loads();
        __syncthreads();
        buf ^= 1;
        if (!last || c + 1 < chunks)
          load(lds_q + buf * kTile * 2, a.q, last ? c + 1 : c, a.hq, g * group + (last ? h0 : h + 1));
        // scores of tokens 16 wave + r against tokens 16 jt + 4 quad + 0..3
        {
          bf16x8 qf[4];
#pragma unroll
          for (int x = 0; x < 4; ++x) qf[x] = read_rows(tq, 16 * wave + r, 32 * x + 4 * quad);
          for (int jt = 0; jt <= (wave | 1); ++jt) {
            f32x4 p = {0.f, 0.f, 0.f, 0.f};
            if (jt <= wave) {
#pragma unroll
              for (int x = 0; x < 4; ++x)
                p = mfma16x16x32(read_rows(sk, 16 * jt + r, 32 * x + 4 * quad), qf[x], p);
            }
            bf16x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int d = 16 * (wave - jt) + r - 4 * quad - i;
              w[i] = (__bf16)(d >= 0 ? p[i] * __builtin_amdgcn_exp2f(l2 * (float)d) : 0.f);
            }
            *reinterpret_cast<bf16x4 *>(sp + score_at(16 * wave + r, 16 * jt + 4 * quad)) = w;
          }
        }
        if (h == h0) read_v(vf, sv);
        if (last && (kMode == kWhole || c + 1 < chunks)) update(vf, sk, n);
        __syncthreads();
        if (c + 1 < chunks) {
          if (h == h0) load(lds_v, a.v, c + 1, a.hkv, g);
          if (last) load(lds_k, a.k, c + 1, a.hkv, g);
        }
#pragma unroll
        for (int it = 0; it < 4; ++it) {
          if (16 * it >= n) break;
          f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const bf16x8 qf = read_rows(tq, 16 * it + r, 32 * x + 4 * quad);
#pragma unroll
            for (int u = 0; u < 2; ++u) acc[u] = mfma16x16x32(sb[u][x], qf, acc[u]);
          }
          const float w = power[16 * it + r + 1];
#pragma unroll
          for (int u = 0; u < 2; ++u) acc[u] *= w;
#pragma unroll
          for (int x = 0; x <= it / 2; ++x) {
            const int row = 16 * it + r;
            const bf16x8 pf = join(
                *reinterpret_cast<const bf16x4 *>(sp + score_at(row, 32 * x + 4 * quad)),
                *reinterpret_cast<const bf16x4 *>(sp + score_at(row, 32 * x + 16 + 4 * quad)));
#pragma unroll
            for (int u = 0; u < 2; ++u) acc[u] = mfma16x16x32(vf[u][x], pf, acc[u]);
          }
          if (16 * it + r < n) {
            const f32x8 o = __builtin_shufflevector(acc[0], acc[1], 0, 1, 2, 3, 4, 5, 6, 7) * a.scale;
            const int64_t t = tok0 + c * kChunk + 16 * it + r;
            store_u32x4(a.out + (t * a.hq + g * group + h) * kHeadDim + 32 * wave + 8 * quad,
                        __builtin_bit_cast(u32x4, to_bf16x8(o)));
          }
        }
      }
    }
  }
  if (kMode != kOutputs) {
    float *at = carry + 4 * quad * kHeadDim + dv;
#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) at[(16 * t + i) * kHeadDim + 4 * u] = s[t][u][i];
  }
}

// The state before each stretch of a row in place of the stretch's own contribution, and
// the state after the last one in the pool. A thread takes four elements.
__global__ __launch_bounds__(kThreads) void linear_scan_kernel(LinearArgs a) {
  const int g = blockIdx.y % a.hkv, b = blockIdx.y / a.hkv;
  const int row0 = min(max(a.cu_q[b], 0), a.total_q);
  const int T = min(min(max(a.cu_q[b + 1], row0), a.total_q) - row0, a.max_q_len);
  const int slot = a.slots[b];
  if (T == 0 || slot < 0 || slot >= a.num_slots) return;
  const int at = (blockIdx.x * kThreads + threadIdx.x) * 4;
  float *pool = a.states + ((int64_t)slot * a.hkv + g) * kStateSize + at;
  float *carry = a.carry + ((int64_t)b * a.hkv + g) * a.segments * kStateSize + at;
  const double ld = log_decay_of(a.log_decay, g);
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (a.ctx_lens[b] > 0) s = *reinterpret_cast<const f32x4 *>(pool);
  for (int from = 0; from < T; from += a.segment_len) {
    const double p = exp(ld * min(T - from, a.segment_len));
    const float dh = (float)p, dl = (float)(p - (double)dh);
    const f32x4 own = *reinterpret_cast<const f32x4 *>(carry);
    *reinterpret_cast<f32x4 *>(carry) = s;
#pragma unroll
    for (int i = 0; i < 4; ++i) s[i] = fmaf(s[i], dh, fmaf(s[i], dl, own[i]));
    carry += kStateSize;
  }
  *reinterpret_cast<f32x4 *>(pool) = s;
}

// How an append call is cut.
struct LinearPlan {
  int32_t segments, segment_len, head_splits;
};
LinearPlan linear_plan(int32_t B, int32_t hq, int32_t hkv, int32_t total_q, int32_t max_q_len) {
  LinearPlan p = {1, max_q_len, 1};
  const int64_t pairs = (int64_t)B * hkv;
  const int32_t chunks = (max_q_len + kChunk - 1) / kChunk;
  if (pairs < 512 && chunks >= 8) {
    const int32_t want = (int32_t)((512 + pairs - 1) / pairs);
    int32_t per = (chunks + want - 1) / want;
    if (per < 4) per = 4;
    p.segment_len = per * kChunk;
    p.segments = (chunks + per - 1) / per;
  }
  return p;
}

}  // namespace

size_t linear_append_workspace_bytes(int32_t B, int32_t hq, int32_t hkv, int32_t total_q,
                                     int32_t max_q_len) {
  const LinearPlan p = linear_plan(B, hq, hkv, total_q, max_q_len);
  return p.segments > 1 ? (size_t)B * hkv * p.segments * kStateSize * sizeof(float) : 0;
}

hipError_t launch_linear_decode(const uint16_t *q, const uint16_t *k, const uint16_t *v,
                                float *states, const int32_t *slots, int32_t num_slots,
                                const int32_t *kv_lens, const float *log_decay, int32_t B,
                                int32_t hq, int32_t hkv, float scale, uint16_t *out,
                                hipStream_t stream) {
  hipLaunchKernelGGL(linear_decode_kernel, dim3(hkv, B), dim3(kThreads), 0, stream, q, k, v,
                     kv_lens, states, slots, num_slots, log_decay, hq, hkv, scale, out);
  return hipGetLastError();
}

hipError_t launch_linear_append(const uint16_t *q, const uint16_t *k, const uint16_t *v,
                                const int32_t *cu_q, const int32_t *ctx_lens, float *states,
                                const int32_t *slots, int32_t num_slots, const float *log_decay,
                                int32_t B, int32_t hq, int32_t hkv, int32_t total_q,
                                int32_t max_q_len, float scale, uint16_t *out, void *workspace,
                                hipStream_t stream) {
  const LinearPlan p = linear_plan(B, hq, hkv, total_q, max_q_len);
  LinearArgs a = {q, k, v, cu_q, ctx_lens, states, slots, log_decay, out,
                  static_cast<float *>(workspace), num_slots, B, hq, hkv, total_q, max_q_len,
                  p.segments, p.segment_len, p.head_splits, scale};
  const unsigned pairs = (unsigned)B * (unsigned)hkv;
  if (p.segments == 1) {
    hipLaunchKernelGGL(linear_chunk_kernel<kWhole>, dim3(pairs), dim3(kThreads), 0, stream, a);
  } else {
    hipLaunchKernelGGL(linear_chunk_kernel<kStates>, dim3(pairs * p.segments), dim3(kThreads), 0,
                       stream, a);
    hipLaunchKernelGGL(linear_scan_kernel, dim3(kStateSize / (4 * kThreads), pairs),
                       dim3(kThreads), 0, stream, a);
    hipLaunchKernelGGL(linear_chunk_kernel<kOutputs>, dim3(pairs * p.segments * p.head_splits),
                       dim3(kThreads), 0, stream, a);
  }
  return hipGetLastError();
}

}  // namespace ra
