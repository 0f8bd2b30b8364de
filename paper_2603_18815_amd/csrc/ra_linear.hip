// Linear attention with a decay for each KV head: rollout_linear_attn_decode (one token a
// row) and rollout_linear_attn_append (new tokens after a row's earlier ones). A row's
// history is a state of fixed size in place of pages:
//   S_t = l S_{t-1} + k_t v_t^T,   o_t = scale S_t^T q_t,   l = exp(log_decay) per KV head.
//
// Decode reads and writes the state, 128 KiB a (row, KV head), and is bound by that: 256
// rows of 32 KV heads, 1.08 GB, take 216-219 us, 5.0 TB/s (a large copy: 4.75).
//
// Append takes chunks of 64 tokens on the matrix cores. With i, j a chunk's tokens, S the
// state before it and n its length:
//   o_i = scale (l^(i+1) S^T q_i + sum_{j <= i} l^(i-j) <q_i, k_j> v_j)
//   S'  = l^n S + sum_j k_j (l^(n-1-j) v_j)^T
// A row's chunks follow one another, so that the longest row decides. Where compute units are
// idle behind it, workgroups share its query heads, each with the state for itself, or rows
// are cut into stretches: their own contributions to the state first (states pass), then the
// state before each (scan), then the outputs (outputs pass).
// The products are of bf16: what has more bits, the state, the scores and the decayed values,
// goes into them in two or three parts, so that the result's own rounding is the largest. One
// part each of the state and the scores took 15 to 20 % less time, and was off by 2^-9 of
// |S| |q|, however little of that a result keeps.
// Measured: 32 rows of 120 to 2,038 tokens, 32 heads on 8, 744 MB, 230-240 us (shared by
// two); a row of 16,384 with 32 heads each, 541 MB of which K and V are read twice, 218-224
// us (cut into 8 stretches of 32 chunks: states 65, scan 8, outputs 149); 905 tokens in 2
// rows 25 us (cut).
#include "ra_device.h"
#include "ra_internal.h"

namespace ra {
namespace {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kChunk = 64;              // tokens of a chunk
constexpr int kComputeUnits = 256;
constexpr int kStateSize = kHeadDim * kHeadDim;

struct LinearArgs {
  const uint16_t *q, *k, *v;
  const int32_t *cu_q, *ctx_lens;
  float *states;
  const int32_t *slots;
  const float *log_decay;
  uint16_t *out;
  float *carry;                         // cut rows: [Hkv][carry_slots] states before stretches
                                        // parts > 1: [B][Hkv] states after the call
  int32_t num_slots, B, hq, hkv, total_q, max_q_len;
  int32_t segment_len;                  // tokens of a stretch; longer rows are cut
  int32_t carry_slots;                  // 0: no row is cut
  int32_t parts;                        // workgroups that share a whole row's query heads
  bool by_row;
  float scale;
};

__device__ __forceinline__ double log_decay_of(const float *log_decay, int g) {
  const float x = log_decay[g];
  return x < 0.f ? fmax((double)x, -1e30) : 0.0;   // NaN and larger values: no decay
}

// ---- decode ---------------------------------------------------------------------------
// A workgroup takes kCols value dims of a (row, KV head)'s state, all 128 key dims: a thread
// four neighbouring columns of every kGroups-th row, so that a wave's load is contiguous and
// all loads of the state are in flight before anything waits. The products with q over the
// rows are joined in the wave, then between the waves through LDS. Quarters of the columns
// (kCols = 32) where whole states are too few to fill the GPU.
constexpr int kHeadsAtOnce = 4;
template <int kCols>
__global__ __launch_bounds__(kThreads) void linear_decode_kernel(
    const uint16_t *q, const uint16_t *k, const uint16_t *v, const int32_t *kv_lens,
    float *states, const int32_t *slots, int32_t num_slots, const float *log_decay, int32_t hq,
    int32_t hkv, float scale, uint16_t *out) {
  constexpr int kLanes = kCols / 4, kGroups = kThreads / kLanes, kRows = kHeadDim / kGroups;
  constexpr int kWaves = kThreads / kWave;
  const int b = blockIdx.y, tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int g = blockIdx.x / (kHeadDim / kCols), col0 = blockIdx.x % (kHeadDim / kCols) * kCols;
  const int group = hq / hkv, col = tid % kLanes * 4, row = tid / kLanes;
  const int slot = slots[b], len = kv_lens[b];
  const int64_t head0 = (int64_t)b * hq + g * group;
  if (slot < 0 || slot >= num_slots || len <= 0) {
    for (int i = tid; i < group * kCols; i += kThreads)
      out[(head0 + i / kCols) * kHeadDim + col0 + i % kCols] = 0;
    return;
  }
  __shared__ float sk[kHeadDim], sq[kHeadsAtOnce][kHeadDim], part[kWaves][kHeadsAtOnce][kCols];
  float *state = states + ((int64_t)slot * hkv + g) * kStateSize + row * kHeadDim + col0 + col;
  f32x4 s[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i)
    s[i] = len > 1 ? *reinterpret_cast<const f32x4 *>(state + i * kGroups * kHeadDim)
                   : f32x4{0.f, 0.f, 0.f, 0.f};
  const uint16_t *kv_row = k + ((int64_t)b * hkv + g) * kHeadDim;
  if (tid < kHeadDim) sk[tid] = __uint_as_float((uint32_t)kv_row[tid] << 16);
  const bf16x4 vb =
      *reinterpret_cast<const bf16x4 *>(v + ((int64_t)b * hkv + g) * kHeadDim + col0 + col);
  const f32x4 vc = __builtin_convertvector(vb, f32x4);
  // the decay in two parts: its rounding to fp32 alone would be felt after 2^24 / t of t steps
  const double decay = exp(log_decay_of(log_decay, g));
  const float l = (float)decay, l_low = (float)(decay - (double)l);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const float kr = sk[row + i * kGroups];
#pragma unroll
    for (int e = 0; e < 4; ++e) s[i][e] = fmaf(l, s[i][e], fmaf(l_low, s[i][e], kr * vc[e]));
    *reinterpret_cast<f32x4 *>(state + i * kGroups * kHeadDim) = s[i];
  }
  for (int h0 = 0; h0 < group; h0 += kHeadsAtOnce) {
    const int heads = min(group - h0, kHeadsAtOnce);
    if (h0 > 0) __syncthreads();                      // part and sq are read no more
    for (int i = tid; i < heads * kHeadDim; i += kThreads)
      sq[i / kHeadDim][i % kHeadDim] = __uint_as_float((uint32_t)q[(head0 + h0) * kHeadDim + i] << 16);
    __syncthreads();
    for (int h = 0; h < heads; ++h) {
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const float qr = sq[h][row + i * kGroups];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = fmaf(qr, s[i][e], o[e]);
      }
#pragma unroll
      for (int d = kLanes; d < kWave; d *= 2)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], d);
      if (lane < kLanes) *reinterpret_cast<f32x4 *>(&part[wave][h][col]) = o;
    }
    __syncthreads();
    for (int i = tid; i < heads * kCols; i += kThreads) {
      float o = 0.f;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) o += part[w][i / kCols][i % kCols];
      out[(head0 + h0 + i / kCols) * kHeadDim + col0 + i % kCols] =
          __builtin_bit_cast(uint16_t, (__bf16)(scale * o));
    }
  }
}

// ---- append: LDS tiles ----------------------------------------------------------------
constexpr int kAppendThreads = 512;
constexpr int kTile = kChunk * kHeadDim;

// A tile holds 64 tokens of 128 bf16 in 16-byte units, unit u of row x at u ^ swizzle(x):
// 16 rows at one unit, and four neighbouring rows at four neighbouring units, fall on
// different banks, so that the reads along a token and the transposing reads along a dim
// are both spread.
__device__ __forceinline__ int swizzle(int row) {
  return (row & 3) << 2 | ((row >> 2 ^ row >> 3) & 1) << 1 | (row >> 3 & 1);
}
constexpr int kRowBytes = 2 * kHeadDim, kScoreRowBytes = 2 * kChunk;
// Scores of a head: 64 rows of 64 bf16, of which tokens 0..31 fill the first half only. Their
// second parts lie in their rows' second half, those of tokens 32..63 in 32 rows behind.
constexpr int kScores = (kChunk + kChunk / 2) * kChunk;

__device__ __forceinline__ bf16x8 lds_bf16x8(const uint16_t *tile, int byte) {
  return *reinterpret_cast<const bf16x8 *>(reinterpret_cast<const char *>(tile) + byte);
}

// ds_read_b64_tr_b16: of 16 lanes, lane i supplies the address of row i / 4's four columns
// at i % 4 and receives column i of the four rows. Two of them: eight rows (the second
// four's swizzle differs in bit 1).
__device__ __forceinline__ bf16x8 read_transposed(const uint16_t *tile, int byte) {
  typedef __attribute__((address_space(3))) s16x4 lds_t;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (lds_t *)(const_cast<char *>(reinterpret_cast<const char *>(tile)) + byte));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (lds_t *)(const_cast<char *>(reinterpret_cast<const char *>(tile + 4 * kHeadDim)) +
                (byte ^ 32)));
  return __builtin_shufflevector(__builtin_bit_cast(bf16x4, a), __builtin_bit_cast(bf16x4, b), 0,
                                 1, 2, 3, 4, 5, 6, 7);
}

// x's upper 16 bits as bf16, taken off x: three times, and the parts hold all 24 bits.
__device__ __forceinline__ bf16x8 take_bf16(f32x8 &x) {
  u32x4 packed;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t lo = __float_as_uint(x[2 * i]), hi = __float_as_uint(x[2 * i + 1]);
    packed[i] = __builtin_amdgcn_perm(hi, lo, 0x07060302);
    x[2 * i] -= __uint_as_float(lo & 0xffff0000u);
    x[2 * i + 1] -= __uint_as_float(hi & 0xffff0000u);
  }
  return __builtin_bit_cast(bf16x8, packed);
}

// x as the sum of two bf16, off by 2^-17 of it at most (2^-9 of a rest that is 2^-8 of it).
__device__ __forceinline__ void two_parts(f32x8 x, bf16x8 &high, bf16x8 &low) {
  high = to_bf16x8(x);
  low = to_bf16x8(x - to_f32x8(high));
}

// 16 bytes a lane from global memory (base + the lane's byte offset) to LDS, lane l's at
// `lds` + 16 l; base and lds are the wave's. In assembly: behind the builtin the compiler
// waits for all such loads before any LDS read; here await_loads() does, before the
// barrier that hands the tile over.
__device__ __forceinline__ void load_to_lds(const uint16_t *base, uint32_t offset, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %0\n\t"
      "s_nop 0\n\t"
      "global_load_lds_dwordx4 %1, %2"
      :
      : "s"(lds), "v"(offset), "s"(base)
      : "memory", "m0");
}
__device__ __forceinline__ void await_loads() { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); }
// The same for loads with kStores stores issued behind them (counted in order): the stores
// may still be on their way.
template <int kStores>
__device__ __forceinline__ void await_loads_before() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kStores) : "memory");
}
__device__ __forceinline__ uint32_t lds_address(const uint16_t *p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void *)p;
}

// Nothing moves across: reads placed before a group of products are issued before it.
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0); }

// x, as a value the compiler computes from anew: what follows from it is not kept in
// registers around a loop, of which the state leaves few.
__device__ __forceinline__ int fresh(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Where stretches are, without a pass that counts them. With L a stretch's tokens, the
// stretches of row b can have the places from floor((cu_q[b] - b) / L) + b on: ceil(T / L)
// of them end by the next row's. Cut rows alone can have those from 2 cu_q[b] / L on, as
// T > L: of these there are no more with more rows. The carry takes the fewer.
__device__ __forceinline__ int start_of(const LinearArgs &a, int b) {
  return min(max(a.cu_q[b], 0), a.total_q);
}
__device__ __forceinline__ int place_of(const LinearArgs &a, int start, int b, bool by_row) {
  if (!by_row) return (int)(2u * (uint32_t)start / (uint32_t)a.segment_len);
  const int behind = start - b, len = a.segment_len;
  return b + (behind >= 0 ? behind / len : -((len - 1 - behind) / len));
}
// The row of that rank, the longest first: of up to 64.
__device__ __forceinline__ int longest_row(const LinearArgs &a, int rank) {
  const int lane = threadIdx.x % kWave;
  const int mine = lane < a.B ? start_of(a, lane + 1) - start_of(a, lane) : -1;
  int ahead = 0;
  for (int i = 0; i < a.B; ++i) {
    const int other = __builtin_amdgcn_readlane(mine, i);
    ahead += other > mine || (other == mine && i < lane);
  }
  return __ffsll((unsigned long long)__ballot(lane < a.B && ahead == rank)) - 1;
}

// The states before a cut row's stretches.
__device__ __forceinline__ float *carry_of(const LinearArgs &a, int start, int b, int g) {
  return a.carry + ((int64_t)g * a.carry_slots + place_of(a, start, b, a.by_row)) * kStateSize;
}

// One stretch of a (row, KV head): chunks in order, the state in the accumulators. Wave w
// of 8 holds the 16 value dims from 16 w, all 128 key dims: tile t = 2 x + y has key dims
// 32 x + 8 (m / 4) + 4 y + m % 4 as its rows m, so that two accumulator tiles, in two bf16
// parts, are the operands of S^T Q^T for the 32 key dims from 32 x as they stand (a lane's
// eight contraction slots: 8 (l / 16) + 0..7), and a lane's results are four neighbouring
// value dims of a token. Scores go through LDS: a wave computes two of the 16 tiles, all
// waves use all of them.
//
// A step is a chunk and kHeads query heads of the group, with three barriers: the step's
// tiles are there (scores, the state's part of the results, and with the chunk's last heads
// the state's update); the scores are there (their part of the results, which go into Q's
// tiles); the results are there (they leave as whole rows). K and V have two stages, the next
// chunk's loads go out during the first heads' step; Q has two buffers of kHeads tiles. 112 KB
// of LDS (157 KB with two heads) and up to 256 registers: one workgroup per CU.
template <bool kStates, int kHeads, bool kCut>
__global__ __launch_bounds__(kAppendThreads, kStates ? 4 : 2) void linear_chunk_kernel(LinearArgs a) {
  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int r = lane % 16, quad = lane / 16;
  // the outputs pass starts with what the states pass read last, and may still be cached
  const int unit = !kCut || kStates ? blockIdx.x : gridDim.x - 1 - blockIdx.x;
  const int items = gridDim.x / a.hkv, group = a.hq / a.hkv / a.parts;
  int g = unit % a.hkv, b = unit / a.hkv / a.parts, seg = 0;
  const int part = unit / a.hkv % a.parts;
  if (!kCut) {
    if (a.B <= kWave) b = longest_row(a, b);
  } else {
    const bool by_row = !kStates || a.by_row;
    const int item = unit % items;
    g = unit / items;
    b = wave_search(a.B, item, [&](int i) { return place_of(a, start_of(a, i), i, by_row); });
    seg = max(item - place_of(a, start_of(a, b), b, by_row), 0);
  }
  const int row0 = start_of(a, b);
  const int T = min(min(max(a.cu_q[b + 1], row0), a.total_q) - row0, a.max_q_len);
  if (seg >= (T + a.segment_len - 1) / a.segment_len) return;
  const int from = seg * a.segment_len;
  const int len = min(T - from, a.segment_len);
  const bool whole = !kCut || T <= a.segment_len;    // an uncut row keeps its own state
  if (kStates && whole) return;
  const int64_t tok0 = row0 + from;
  const int head0 = (g * a.parts + part) * group;
  const int slot = a.slots[b];
  if (slot < 0 || slot >= a.num_slots) {
    if (!kStates)
      for (int t = 0; t < len; ++t)
        for (int i = tid; i < group * kHeadDim; i += kAppendThreads)
          a.out[((tok0 + t) * a.hq + head0) * kHeadDim + i] = 0;
    return;
  }

  __shared__ __align__(1024) uint16_t sk[2 * kTile], sv[2 * kTile];
  __shared__ __align__(1024) uint16_t sq[kStates ? 8 : 2 * kHeads * kTile];
  __shared__ __align__(1024) uint16_t sp[kStates ? 8 : kHeads * kScores];
  // l^n; scale l^n; l^(63 - j), then zeros
  __shared__ float power[kChunk + 1], weight[2 * kChunk];
  __shared__ double decays[kChunk + 1];
  const double ld = log_decay_of(a.log_decay, g);
  const float l2 = (float)(ld * 1.4426950408889634);
  if (tid <= kChunk) {
    const double p = exp(ld * tid);
    decays[tid] = p;
    power[tid] = (float)(a.scale * p);
    if (tid < kChunk) {
      weight[kChunk - 1 - tid] = (float)p;
      weight[kChunk + tid] = 0.f;
    }
  }

  // loads: wave w takes rows 8 w .. 8 w + 7 of a tile, four rows an instruction, lane l the
  // unit of row l / 16 that belongs at l % 16; rows past the end repeat the last one
  const uint32_t lds_k = lds_address(sk) + wave * 2048, lds_v = lds_address(sv) + wave * 2048;
  const uint32_t lds_q = lds_address(sq) + wave * 2048;
  const int ld_unit = (lane % 16) ^ swizzle(8 * wave + lane / 16);
  const int q_stride = a.hq * kRowBytes, kv_stride = a.hkv * kRowBytes;
  const uint32_t q_off = __umul24(8 * wave + lane / 16, q_stride) + (ld_unit << 4);
  const uint32_t kv_off = __umul24(8 * wave + lane / 16, kv_stride) + (ld_unit << 4);
  // base: row 0 of the tile, left: rows behind it
  auto load = [&](uint32_t lds, const uint16_t *base, uint32_t off, int stride, int left) {
    if (left >= kChunk - 1) {
      load_to_lds(base, off, lds);
      load_to_lds(base, (off ^ 32) + 4 * stride, lds + 1024);
    } else {
#pragma unroll
      for (int m = 0; m < 2; ++m)
        load_to_lds(base,
                    __umul24(min(8 * wave + 4 * m + lane / 16, left), stride) + ((ld_unit ^ 2 * m) << 4),
                    lds + 1024 * m);
    }
  };
  const int chunks = (len + kChunk - 1) / kChunk;
  const size_t q_chunk = (size_t)kChunk * a.hq * kHeadDim, kv_chunk = (size_t)kChunk * a.hkv * kHeadDim;
  const size_t q_first = ((size_t)tok0 * a.hq + head0) * kHeadDim;
  const uint16_t *kp = a.k + ((size_t)tok0 * a.hkv + g) * kHeadDim;   // the chunk to load next
  const uint16_t *vp = a.v + ((size_t)tok0 * a.hkv + g) * kHeadDim;
  const uint16_t *qp = a.q + q_first;                                 // the chunk at hand
  uint16_t *op = a.out + q_first;
  load(lds_k, kp, kv_off, kv_stride, len - 1);
  load(lds_v, vp, kv_off, kv_stride, len - 1);
  auto load_q = [&](int buf, const uint16_t *base, int left) {
#pragma unroll
    for (int j = 0; j < kHeads; ++j)
      load(lds_q + (buf * kHeads + j) * kTile * 2, base + j * kHeadDim, q_off, q_stride, left);
  };
  if (!kStates) load_q(0, qp, len - 1);

  // state tile t = 2 x + y, register i: key dim 32 x + 8 quad + 4 y + i, value dim 16 wave + r
  f32x4 s[8];
  float *pool = a.states + ((int64_t)slot * a.hkv + g) * kStateSize;
  float *carry = whole ? pool : carry_of(a, row0, b, g) + (int64_t)seg * kStateSize;
  const bool zero = kStates || (whole && a.ctx_lens[b] <= 0);
  float *const s_at = carry + 8 * quad * kHeadDim + 16 * wave + r;
#pragma unroll
  for (int t = 0; t < 8; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
  if (!zero) {
#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        s[t][i] = s_at[(32 * (t / 2) + 4 * (t % 2) + i) * kHeadDim];
  }

  // byte addresses in the tiles: rows r at unit quad (32 dims on: ^ 64), and for the
  // transposing reads rows 8 quad + r / 4 at this lane's four dims of the first K tile, the
  // wave's of V
  const int at_row = r * kRowBytes + ((quad ^ swizzle(r)) << 4);
  const int tr_row = 8 * quad + (r >> 2), tr_swizzle = swizzle(tr_row);
  const int at_k = tr_row * kRowBytes + (((r & 3) ^ tr_swizzle) << 4);
  const int at_v = tr_row * kRowBytes + (((2 * wave + (r >> 1 & 1)) ^ tr_swizzle) << 4) + (r & 1) * 8;
  // results: rows r at the wave's four value dims of the quad
  const int at_o = r * kRowBytes + (((2 * wave + (quad >> 1)) ^ swizzle(r)) << 4) + (quad & 1) * 8;
  const int at_score = r * kScoreRowBytes + ((quad ^ (r >> 1)) << 4);

  // V^T of a chunk, rows the wave's value dims, slots the 32 tokens from 32 x
  auto read_v = [&](bf16x8(&vf)[2], const uint16_t *tile) {
#pragma unroll
    for (int x = 0; x < 2; ++x) vf[x] = read_transposed(tile + 32 * x * kHeadDim, at_v);
  };
  // An infinite or NaN value makes NaN of a score of zero: tokens before it would have it too.
  // A wave with such values multiplies with zeros in their place, and makes NaN of their dims
  // from their tokens on.
  auto not_finite = [](uint32_t bits) { return (bits & 0x7f80u) == 0x7f80u; };
  auto strange = [&](const bf16x8(&vf)[2]) {
    uint32_t any = 0;                                   // an exponent of ones carries into the sign
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const u32x4 w = __builtin_bit_cast(u32x4, vf[x]);
#pragma unroll
      for (int e = 0; e < 4; ++e) any |= (w[e] & 0x7f807f80u) + 0x00800080u;
    }
    return __ballot(any & 0x80008000u) != 0;
  };
  auto zero_strange = [&](bf16x8(&vf)[2]) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      u32x4 w = __builtin_bit_cast(u32x4, vf[x]);
#pragma unroll
      for (int e = 0; e < 4; ++e)
        w[e] &= (not_finite(w[e]) ? 0u : 0xffffu) | (not_finite(w[e] >> 16) ? 0u : 0xffff0000u);
      vf[x] = __builtin_bit_cast(bf16x8, w);
    }
  };
  auto fill_strange = [&](uint16_t *results, const uint16_t *tile, int n) {
    uint32_t bad = 0;
    const int l = fresh(lane), unit = 2 * wave + (l >> 5), half = (l >> 4 & 1) * 4;
#pragma unroll 1
    for (int t = 0; t < n; ++t) {
      const int at = t * kHeadDim + ((unit ^ swizzle(t)) << 3) + half;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        bad |= not_finite(tile[at + e]) << e;
        if (t % 16 == l % 16 && (bad >> e & 1)) results[at + e] = 0x7fc0;
      }
    }
  };
  // S' = decay S + K^T (after l^(n-1-j) V), n the chunk's tokens: the decayed values in
  // bf16 parts, of which three hold all 24 bits. The states pass has no state to decay: its
  // weights reach to the end of the stretch (after = l^tokens behind the chunk).
  auto update = [&](const bf16x8(&vf)[2], const uint16_t *tile, int n, float decay, float after) {
    const int at = fresh(at_k);
    if (!kStates) {
#pragma unroll
      for (int t = 0; t < 8; ++t) s[t] *= decay;
    }
    // K's operands are read a pair of tiles ahead of the products
    bf16x8 kf[2][2];
    auto read_pair = [&](int i) {
#pragma unroll
      for (int y = 0; y < 2; ++y)
        kf[i % 2][y] = read_transposed(tile + 32 * (i / 4) * kHeadDim + 4 * y, at ^ (i % 4 << 6));
    };
    read_pair(0);
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      bf16x8 part[3];
      f32x8 y = to_f32x8(vf[x]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float w = weight[kChunk - n + 32 * x + 8 * quad + e];
        y[e] *= kStates ? w * after : w;
      }
#pragma unroll
      for (int m = 0; m < 3; ++m) part[m] = take_bf16(y);
#pragma unroll
      for (int i = 4 * x; i < 4 * x + 4; ++i) {
        if (i + 1 < 8) read_pair(i + 1);
        keep_order();
#pragma unroll
        for (int m = 0; m < 3; ++m)
#pragma unroll
          for (int y = 0; y < 2; ++y)
            s[2 * (i % 4) + y] = mfma16x16x32(kf[i % 2][y], part[m], s[2 * (i % 4) + y]);
        keep_order();
      }
    }
  };

  // where the lane's scores of tokens 16 (wave % 4) + r against 16 (wave / 4) + 4 quad + 0..3 go
  const int at_p = (16 * (wave & 3) + r) * kScoreRowBytes +
                   (((2 * (wave >> 2) + (quad >> 1)) ^ (r >> 1)) << 4) + (quad & 1) * 8;
  // scores: this wave's two tiles' scale l^(i - j), zero above the diagonal; the lane's four
  // j are 4 quad + 0..3
  float mult[2][4];
#pragma unroll
  for (int jj = 0; jj < 2; ++jj)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int d = 16 * ((wave & 3) - (wave >> 2) - 2 * jj) + r - 4 * quad - i;
      mult[jj][i] = d >= 0 ? a.scale * __builtin_amdgcn_exp2f(l2 * (float)d) : 0.f;
    }

  int q_buf = 0;
  double drift = 1.0;
  for (int c = 0; c < chunks; ++c) {
    const int n = min(len - c * kChunk, kChunk);
    bf16x8 vf[2];
    bool odd = false;                                   // values that are infinite or NaN
    const int buf = c & 1;
    const bool more = c + 1 < chunks;
    const int left = len - 1 - (c + 1) * kChunk;        // rows behind the next chunk's first
    const uint16_t *const tk = sk + buf * kTile, *const tv = sv + buf * kTile;
    kp += kv_chunk;
    vp += kv_chunk;
    auto load_k = [&]() {
      if (more) load(lds_k + (buf ^ 1) * kTile * 2, kp, kv_off, kv_stride, left);
    };
    auto load_v = [&]() {
      if (more) load(lds_v + (buf ^ 1) * kTile * 2, vp, kv_off, kv_stride, left);
    };
    if constexpr (kStates) {
      await_loads();
      __syncthreads();
      load_k();
      load_v();
      read_v(vf, tv);
      update(vf, tk, n, 1.f, __builtin_amdgcn_exp2f(l2 * (float)(len - c * kChunk - n)));
    } else {
      bf16x8 sb[2][4];                                  // the state before the chunk, in two parts
#pragma unroll
      for (int x = 0; x < 4; ++x)
        two_parts(__builtin_shufflevector(s[2 * x], s[2 * x + 1], 0, 1, 2, 3, 4, 5, 6, 7), sb[0][x],
                  sb[1][x]);
      for (int h = 0; h < group; h += kHeads) {
        uint16_t *const tq = sq + q_buf * kHeads * kTile;
        const bool last = h + kHeads == group;
        // behind the tiles' loads: the step before's stores, two a head where its chunk was full
        if (n == kChunk && (c > 0 || h > 0)) {
          await_loads_before<2 * kHeads>();
        } else {
          await_loads();
        }
        __syncthreads();
        // K of the wave's two score tiles: those of tokens 16 it + r against 16 jt + 4 quad +
        // 0..3, jt = wave / 4 and 2 more. Above the diagonal they are zero, and needed where a
        // tile shares 32 slots with one on it.
        const int it_p = wave & 3, jt_p = wave >> 2, at = fresh(at_row), pt = fresh(at_p);
        bf16x8 kf[2][4];
#pragma unroll
        for (int x = 0; x < 4; ++x) kf[0][x] = lds_bf16x8(tk + 16 * jt_p * kHeadDim, at ^ (x << 6));
        if (it_p >= 2)
#pragma unroll
          for (int x = 0; x < 4; ++x)
            kf[1][x] = lds_bf16x8(tk + 16 * (jt_p + 2) * kHeadDim, at ^ (x << 6));
        if (h == 0) read_v(vf, tv);
        q_buf ^= 1;
        if (!last) {
          load_q(q_buf, qp + (h + kHeads) * kHeadDim, left + kChunk);
        } else if (more) {
          load_q(q_buf, qp + q_chunk, left);
        }
        f32x4 acc[kHeads][4];
#pragma unroll
        for (int j = 0; j < kHeads; ++j) {
          const uint16_t *const tj = tq + j * kTile;
          // Q of all tokens, and of those of the wave's scores, a quarter of the dims ahead of
          // the products
          bf16x8 qf[2][4], qs[2];
          auto read_q = [&](int x) {
            qs[x % 2] = lds_bf16x8(tj + 16 * it_p * kHeadDim, at ^ (x << 6));
#pragma unroll
            for (int it = 0; it < 4; ++it)
              qf[x % 2][it] = lds_bf16x8(tj + 16 * it * kHeadDim, at ^ (x << 6));
          };
          f32x4 p[2];
          p[0] = p[1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int it = 0; it < 4; ++it) acc[j][it] = f32x4{0.f, 0.f, 0.f, 0.f};
          read_q(0);
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            if (x + 1 < 4) read_q(x + 1);
            keep_order();
            p[0] = mfma16x16x32(kf[0][x], qs[x % 2], p[0]);
#pragma unroll
            for (int m = 0; m < 2; ++m)
#pragma unroll
              for (int it = 0; it < 4; ++it)
                acc[j][it] = mfma16x16x32(sb[m][x], qf[x % 2][it], acc[j][it]);
            if (it_p >= 2) p[1] = mfma16x16x32(kf[1][x], qs[x % 2], p[1]);
            keep_order();
          }
#pragma unroll
          for (int jj = 0; jj < 2; ++jj) {
            if (jj == 1 && it_p < 2) break;
            bf16x4 w, w2;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float x = mult[jj][i] == 0.f ? 0.f : p[jj][i] * mult[jj][i];
              w[i] = (__bf16)x;
              w2[i] = (__bf16)(x - (float)w[i]);
            }
            char *const scores = reinterpret_cast<char *>(sp + j * kScores);
            *reinterpret_cast<bf16x4 *>(scores + (pt ^ (jj << 6))) = w;
            *reinterpret_cast<bf16x4 *>(scores + (it_p < 2 ? 0 : kChunk / 2 * kScoreRowBytes) +
                                        (pt ^ ((it_p < 2 ? 1 : jj) << 6))) = w2;
          }
#pragma unroll
          for (int it = 0; it < 4; ++it) acc[j][it] *= power[16 * it + r + 1];
        }
        if (h == 0) load_k();
        if (odd && last) read_v(vf, tv);
        if (last && (more || (whole && part == 0))) {
          // the product of the chunks' decays as they were rounded is kept at l^tokens: what
          // one rounding adds, the next chunk's takes off
          const double exact = decays[n];
          const float decay = (float)(exact * drift);
          if (exact > 1e-30) drift = exact * drift / decay;
          update(vf, tk, n, decay, 1.f);
        }
        if (h == 0) odd = strange(vf);
        if (odd && (h == 0 || last)) zero_strange(vf);
        if (h == 0) load_v();
        __syncthreads();
        const int st = fresh(at_score);
#pragma unroll
        for (int j = 0; j < kHeads; ++j) {
          const uint16_t *const scores = sp + j * kScores;
#pragma unroll
          for (int m = 0; m < 2; ++m) {                 // the scores' two parts
            bf16x8 pf[4][2];
#pragma unroll
            for (int it = 0; it < 4; ++it)
#pragma unroll
              for (int x = 0; x <= it / 2; ++x)
                pf[it][x] = lds_bf16x8(scores + (16 * it + (it < 2 ? 0 : m * kChunk / 2)) * kChunk,
                                       st ^ ((it < 2 ? m : x) << 6));
#pragma unroll
            for (int x = 0; x < 2; ++x)
#pragma unroll
              for (int it = 2 * x; it < 4; ++it)
                acc[j][it] = mfma16x16x32(vf[x], pf[it][x], acc[j][it]);
          }
        }
        // the results through Q's tiles, which nothing reads any more: a wave has 32 bytes of
        // each token, whose stores alone took longer than the products; whole rows leave
        const int ot = fresh(at_o);
#pragma unroll
        for (int j = 0; j < kHeads; ++j)
#pragma unroll
          for (int it = 0; it < 4; ++it)
            *reinterpret_cast<bf16x4 *>(reinterpret_cast<char *>(tq + j * kTile + 16 * it * kHeadDim) +
                                        ot) = __builtin_convertvector(acc[j][it], bf16x4);
        if (odd)
          for (int j = 0; j < kHeads; ++j) fill_strange(tq + j * kTile, tv, n);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kHeads; ++j)
#pragma unroll
          for (int m = 0; m < 2; ++m) {
            const u32x4 w = load_u32x4(tq + j * kTile + (8 * wave + 4 * m) * kHeadDim + lane * 8);
            char *const o_row = reinterpret_cast<char *>(op + (h + j) * kHeadDim);
            if (n == kChunk || 8 * wave + 4 * m + lane / 16 < n)
              store_u32x4(reinterpret_cast<uint16_t *>(
                              o_row + (m ? (q_off ^ 32) + 4 * q_stride : q_off)), w);
          }
      }
      qp += q_chunk;
      op += q_chunk;
    }
  }
  if (kStates || (whole && part == 0)) {
    // the other parts may not have read the pool yet
    float *const to = !kCut && a.parts > 1
                          ? a.carry + ((int64_t)b * a.hkv + g) * kStateSize + (s_at - carry)
                          : s_at;
#pragma unroll
    for (int t = 0; t < 8; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        to[(32 * (t / 2) + 4 * (t % 2) + i) * kHeadDim] = s[t][i];
  }
}

// The state before each stretch of a row in place of the stretch's own contribution, and
// the state after the last one in the pool. A thread takes four elements.
__global__ __launch_bounds__(kThreads) void linear_scan_kernel(LinearArgs a) {
  const int g = blockIdx.y % a.hkv;
  int b = blockIdx.y / a.hkv;
  if (!a.by_row) {                      // cut rows differ in start / L
    const int x = b;
    b = wave_search(a.B, x, [&](int i) { return start_of(a, i) / a.segment_len; });
    if (start_of(a, b) / a.segment_len != x) return;
  }
  const int row0 = start_of(a, b);
  const int T = min(min(max(a.cu_q[b + 1], row0), a.total_q) - row0, a.max_q_len);
  const int slot = a.slots[b];
  if (T <= a.segment_len || slot < 0 || slot >= a.num_slots) return;
  const int at = (blockIdx.x * kThreads + threadIdx.x) * 4;
  float *pool = a.states + ((int64_t)slot * a.hkv + g) * kStateSize + at;
  float *carry = carry_of(a, row0, b, g) + at;
  const double ld = log_decay_of(a.log_decay, g);
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  if (a.ctx_lens[b] > 0) s = *reinterpret_cast<const f32x4 *>(pool);
  // eight stretches' loads at a time: one by one each waits for the store before it
  constexpr int kAhead = 8;
  const int stretches = (T + a.segment_len - 1) / a.segment_len;
  const double full = exp(ld * a.segment_len), last = exp(ld * (T - (stretches - 1) * a.segment_len));
  for (int first = 0; first < stretches; first += kAhead) {
    f32x4 own[kAhead];
#pragma unroll
    for (int j = 0; j < kAhead; ++j)
      own[j] = *reinterpret_cast<const f32x4 *>(carry + (int64_t)min(first + j, stretches - 1) * kStateSize);
#pragma unroll
    for (int j = 0; j < kAhead; ++j) {
      if (first + j >= stretches) break;
      const double p = first + j < stretches - 1 ? full : last;
      const float dh = (float)p, dl = (float)(p - (double)dh);
      *reinterpret_cast<f32x4 *>(carry + (int64_t)(first + j) * kStateSize) = s;
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i] = fmaf(s[i], dh, fmaf(s[i], dl, own[j][i]));
    }
  }
  *reinterpret_cast<f32x4 *>(pool) = s;
}

// The states after the call, where parts of a row's heads shared it, into the pool.
__global__ __launch_bounds__(kThreads) void linear_states_kernel(LinearArgs a) {
  const int g = blockIdx.y % a.hkv, b = blockIdx.y / a.hkv, slot = a.slots[b];
  if (start_of(a, b + 1) <= start_of(a, b) || slot < 0 || slot >= a.num_slots) return;
  const int at = (blockIdx.x * kThreads + threadIdx.x) * 4;
  *reinterpret_cast<f32x4 *>(a.states + ((int64_t)slot * a.hkv + g) * kStateSize + at) =
      *reinterpret_cast<const f32x4 *>(a.carry + (int64_t)blockIdx.y * kStateSize + at);
}

// How an append call is cut.
struct LinearPlan {
  int32_t segment_len, stretches, carry_slots, parts;
  bool by_row;
};
// A chunk's time by a workgroup that takes `heads` query heads of it, in ns (measured, alone
// on the GPU; an even number is taken two at once).
int64_t chunk_ns(int32_t heads) {
  return heads % 2 == 0 ? 1600 + 1560 * (int64_t)heads : 2000 + 1700 * (int64_t)heads;
}
LinearPlan linear_plan(int32_t B, int32_t hq, int32_t hkv, int32_t total_q, int32_t max_q_len) {
  const int32_t longest = max_q_len < total_q ? max_q_len : total_q, group = hq / hkv;
  const int64_t chunks = ((int64_t)longest + kChunk - 1) / kChunk;
  // a compute unit's even share of the call's chunks
  int64_t share = ((int64_t)total_q * hkv / kComputeUnits + kChunk - 1) / kChunk;
  share = share < 1 ? 1 : share;
  LinearPlan p = {longest, B, 0, 1, true};  // whole rows
  if (chunks <= share) return p;
  // Compute units are idle behind the longest row. Either they share whole rows by their
  // heads (each part keeps the state for itself, one writes it out, a launch behind sets it in
  // the pool), where there are that many more of them than of longest rows; or rows are cut.
  // Measured, 32 heads on 8, rows of 2,048: 16 rows 270 us as they are, 205-235 by two parts;
  // 8 rows 262, by four parts 140-147, cut 174; 4 rows 253, 127, 95; rows of 512: 8 rows 69,
  // 43, 59; 2 rows 67, 37, 28.
  while (group % (2 * p.parts) == 0 && 4 * (2 * p.parts) * share <= 5 * chunks &&
         (int64_t)B * hkv <= 2 * kComputeUnits)
    p.parts *= 2;
  // the parts read K and V again
  const int64_t whole_ns =
      p.parts > 1 ? chunks * chunk_ns(group / p.parts) * 108 / 100 + 8000 : chunks * chunk_ns(group) + 5000;
  LinearPlan c = p;
  c.parts = 1;
  c.segment_len = (int32_t)(share * kChunk);
  c.stretches = B + (total_q > B ? (total_q - B) / c.segment_len : 0);
  const int32_t of_cut = (int32_t)(2 * (int64_t)total_q / c.segment_len) + 1;
  c.by_row = c.stretches <= of_cut;
  c.carry_slots = c.by_row ? c.stretches : of_cut;
  // 2 us of the states pass, 3.5 us for the bandwidth that all units share, and the states of
  // the stretches written and read
  const int64_t cut_ns = share * (chunk_ns(group) + 5500) + 8000 + 85 * (int64_t)c.carry_slots * hkv;
  return cut_ns < whole_ns ? c : p;
}

}  // namespace

size_t linear_append_workspace_bytes(int32_t B, int32_t hq, int32_t hkv, int32_t total_q,
                                     int32_t max_q_len) {
  const LinearPlan p = linear_plan(B, hq, hkv, total_q, max_q_len);
  return (size_t)(p.parts > 1 ? B : p.carry_slots) * hkv * kStateSize * sizeof(float);
}

hipError_t launch_linear_decode(const uint16_t *q, const uint16_t *k, const uint16_t *v,
                                float *states, const int32_t *slots, int32_t num_slots,
                                const int32_t *kv_lens, const float *log_decay, int32_t B,
                                int32_t hq, int32_t hkv, float scale, uint16_t *out,
                                hipStream_t stream) {
  // whole states a workgroup, or quarters where those are fewer than one a compute unit: 64
  // pairs 6.4 us whole, 5.5 by quarters; 256 pairs 8.4 and 9.7; 1,024 pairs 24 and 27
  const bool quarters = (int64_t)B * hkv < kComputeUnits;
  if (quarters)
    hipLaunchKernelGGL(linear_decode_kernel<32>, dim3(hkv * 4, B), dim3(kThreads), 0, stream, q, k,
                       v, kv_lens, states, slots, num_slots, log_decay, hq, hkv, scale, out);
  else
    hipLaunchKernelGGL(linear_decode_kernel<128>, dim3(hkv, B), dim3(kThreads), 0, stream, q, k, v,
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
                  p.segment_len, p.carry_slots, p.parts, p.by_row, scale};
  const dim3 threads(kAppendThreads);
  const dim3 grid((unsigned)(p.stretches * p.parts) * (unsigned)hkv);
  if (p.carry_slots) {
    const unsigned rows = (unsigned)(p.by_row ? B : total_q / p.segment_len + 1);
    hipLaunchKernelGGL((linear_chunk_kernel<true, 1, true>), dim3((unsigned)p.carry_slots * (unsigned)hkv),
                       threads, 0, stream, a);
    hipLaunchKernelGGL(linear_scan_kernel,
                       dim3(kStateSize / (4 * kThreads), rows * (unsigned)hkv),
                       dim3(kThreads), 0, stream, a);
  }
  // two query heads a step share K's operands and the step's waits
  const bool pairs = hq / hkv / p.parts % 2 == 0, cut = p.carry_slots > 0;
  if (pairs && cut)
    hipLaunchKernelGGL((linear_chunk_kernel<false, 2, true>), grid, threads, 0, stream, a);
  else if (pairs)
    hipLaunchKernelGGL((linear_chunk_kernel<false, 2, false>), grid, threads, 0, stream, a);
  else if (cut)
    hipLaunchKernelGGL((linear_chunk_kernel<false, 1, true>), grid, threads, 0, stream, a);
  else
    hipLaunchKernelGGL((linear_chunk_kernel<false, 1, false>), grid, threads, 0, stream, a);
  if (p.parts > 1)
    hipLaunchKernelGGL(linear_states_kernel, dim3(kStateSize / (4 * kThreads), (unsigned)B * (unsigned)hkv),
                       dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace ra
