// Attention of a tree of drafted tokens over the paged cache (rollout_attn_decode_tree).
//
// Row b's T nodes lie behind its ctx cached tokens. The query rows of a KV head are its G =
// Hq / Hkv query heads of all nodes, taken as columns of the matrix products as in decode
// (ra_decode_split.h), 16 kTiles of them a workgroup: node r / G, head r % G for query row r.
// All see the context; which of the nodes a node sees is in its bit mask. Keys are cut into
// splits, whose partial results a second launch joins.
#include "ra_device.h"
#include "ra_internal.h"

namespace ra {
namespace {

constexpr int kSplitWaves = 4;
constexpr int kPair = 2 * kPage;
constexpr int kOPitch = kHeadDim + 4;

struct TreeArgs {
  const uint16_t *q;
  const int32_t *cu_q, *ctx_lens;
  const uint64_t *mask;
  const uint16_t *k_pool, *v_pool;
  const int32_t *block_table;
  float *ws_o, *ws_m, *ws_l;   // [total_q][Hq][slots][128], [total_q][Hq][slots] twice
  float *out, *lse;
  int32_t B, hq, hkv, group, words, bt_stride, num_pages, total_q, max_q_len, max_kv_len;
  int32_t split_tokens, slots, tiles;
  float scale_log2, v_scale;
};

struct TreeRow {
  int first, T, ctx;
};
__device__ __forceinline__ TreeRow tree_row(const TreeArgs &a, int b) {
  TreeRow r;
  r.first = min(max(a.cu_q[b], 0), a.total_q);
  r.T = min(min(max(a.cu_q[b + 1] - r.first, 0), a.max_q_len), a.total_q - r.first);
  r.T = min(r.T, a.max_kv_len);
  r.ctx = min(max(a.ctx_lens[b], 0), a.max_kv_len - r.T);
  return r;
}

// Of a pair of bf16 values: all ones in the place of each that is infinite or NaN.
__device__ __forceinline__ uint32_t not_finite(uint32_t w) {
  return ((w & 0x7f80u) == 0x7f80u ? 0xffffu : 0u) |
         ((w & 0x7f800000u) == 0x7f800000u ? 0xffff0000u : 0u);
}

// The lower n (0, 1, or 2 and more) of a pair of bf16 values.
__device__ __forceinline__ uint32_t low_keys(int n) {
  return (n > 0 ? 0xffffu : 0u) | (n > 1 ? 0xffff0000u : 0u);
}

// A value that is infinite or NaN must not meet the zero weights of nodes that do not see it:
// past the context the products run with zeros in the place of such values, and where there was
// one this writes NaN into the results (row c's at o_row(c)) that it reaches. Keys [t0, t1).
template <bool kFp8, int kThreads, typename Row>
__device__ __forceinline__ void reach_odd(const TreeArgs &a, const TreeRow &row, const int32_t *bt,
                                          int g, int t0, int t1, int r0, int rows, Row o_row) {
  const int from = max(t0, row.ctx);
  for (int x = threadIdx.x; x < (t1 - from) * kHeadDim; x += kThreads) {
    const int pos = from + x / kHeadDim, d = x % kHeadDim, j = pos - row.ctx;
    const size_t at = (((size_t)clamp_page(bt[pos / kPage], a.num_pages) * a.hkv + g) * kHeadDim + d) *
                          kPage + pos % kPage;
    const bool odd = kFp8 ? (reinterpret_cast<const uint8_t *>(a.v_pool)[at] & 0x7f) == 0x7f
                          : (a.v_pool[at] & 0x7f80) == 0x7f80;
    if (!odd) continue;
    for (int c = 0; c < rows; ++c) {
      const size_t t = row.first + (r0 + c) / a.group;
      if (a.mask[t * a.words + (j >> 6)] >> (j & 63) & 1) o_row(c)[d] = NAN;
    }
  }
}

template <int kTiles>
struct TreeLds {
  float m[kSplitWaves][16 * kTiles];
  float l[kSplitWaves][16 * kTiles];
  float o[kSplitWaves][16 * kTiles][kOPitch];
};

template <int kTiles, bool kFp8>
__global__ __launch_bounds__(kSplitWaves * kWave, 2) void tree_split_kernel(TreeArgs a) {
  __shared__ TreeLds<kTiles> lds;
  int id = blockIdx.x;
  const int g = id % a.hkv;
  id /= a.hkv;
  const int tile = id % a.tiles;
  id /= a.tiles;
  const int split = id % a.slots, b = id / a.slots;
  const TreeRow row = tree_row(a, b);
  const int G = a.group, rows = row.T * G, r0 = tile * 16 * kTiles;
  const int end = row.ctx + row.T;
  const int t0 = split * a.split_tokens, t1 = min(end, t0 + a.split_tokens);
  if (r0 >= rows || t0 >= t1) return;
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int npairs = (t1 - t0 + kPair - 1) / kPair;
  const int row_pages = (t1 + kPage - 1) / kPage;
  const int32_t *bt = a.block_table + (size_t)b * a.bt_stride;
  const int col = lane & 15, kgrp = lane >> 4;

  bf16x8 qop[kTiles][4];
  const uint64_t *mask[kTiles];
#pragma unroll
  for (int nt = 0; nt < kTiles; ++nt) {
    const int r = min(r0 + 16 * nt + col, rows - 1), node = r / G;
    const size_t t = row.first + node;
    mask[nt] = a.mask + t * a.words;
    const uint16_t *qrow = a.q + (t * a.hq + (size_t)g * G + (r - node * G)) * kHeadDim;
#pragma unroll
    for (int kk = 0; kk < 4; ++kk)
      qop[nt][kk] = kFp8 ? load_bf16x8(qrow + 64 * (kk >> 1) + 16 * kgrp + 8 * (kk & 1))
                         : load_bf16x8(qrow + 32 * kk + 8 * kgrp);
  }
  const int ka_sel = col >> 3, ka_slot = 8 * ((col >> 2) & 1) + (col & 3);
  const int sv_sel = lane >> 5, sv_slot = 8 * ((lane >> 4) & 1);

  f32x4 o[kTiles][8];
  float m_run[kTiles], l_run[kTiles];
#pragma unroll
  for (int nt = 0; nt < kTiles; ++nt) {
#pragma unroll
    for (int mt = 0; mt < 8; ++mt) o[nt][mt] = f32x4{0.f, 0.f, 0.f, 0.f};
    m_run[nt] = -INFINITY;
    l_run[nt] = 0.f;
  }
  uint32_t odd = 0;                         // infinite or NaN values of nodes
  const size_t head_stride = (size_t)kPage * kHeadDim;
  for (int pr = wave; pr < npairs; pr += kSplitWaves) {
    const int tok = t0 + pr * kPair, pg = tok / kPage;
    const int id0 = clamp_page(bt[pg], a.num_pages);
    const int id1 = pg + 1 < row_pages ? clamp_page(bt[pg + 1], a.num_pages) : id0;
    const size_t kbase = ((size_t)(ka_sel ? id1 : id0) * a.hkv + g) * head_stride;
    const size_t vbase = ((size_t)(sv_sel ? id1 : id0) * a.hkv + g) * head_stride;
    bf16x8 ka[2][4], va[8];
    if constexpr (kFp8) {
      const uint8_t *kb = reinterpret_cast<const uint8_t *>(a.k_pool) + kbase;
      const uint8_t *vb = reinterpret_cast<const uint8_t *>(a.v_pool) + vbase;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const u32x4 w = *reinterpret_cast<const u32x4 *>(kb + (ka_slot + 4 * t) * kHeadDim +
                                                           64 * h + 16 * kgrp);
          ka[t][2 * h] = fp8x8_to_bf16x8(u32x2{w[0], w[1]});
          ka[t][2 * h + 1] = fp8x8_to_bf16x8(u32x2{w[2], w[3]});
        }
#pragma unroll
      for (int mt = 0; mt < 8; ++mt)
        va[mt] = fp8x8_to_bf16x8(
            *reinterpret_cast<const u32x2 *>(vb + (16 * mt + col) * kPage + sv_slot));
    } else {
      const uint16_t *kb = a.k_pool + kbase, *vb = a.v_pool + vbase;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          ka[t][kk] = load_bf16x8(kb + (ka_slot + 4 * t) * kHeadDim + 32 * kk + 8 * kgrp);
#pragma unroll
      for (int mt = 0; mt < 8; ++mt) va[mt] = load_bf16x8(vb + (16 * mt + col) * kPage + sv_slot);
    }
    // Pairs that reach past the context: keys at or past the row's end are not attended (their
    // values replaced by zeros), the nodes' keys by those whose masks name them.
    const bool tail = tok + kPair > min(row.ctx, t1);
    const int first = tok + sv_sel * kPage + sv_slot;
    if (tail) {
      const int alive = t1 - first, context = row.ctx - first;   // of the lane's eight keys
#pragma unroll
      for (int mt = 0; mt < 8; ++mt) {
        u32x4 w = __builtin_bit_cast(u32x4, va[mt]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          w[e] &= low_keys(alive - 2 * e);
          const uint32_t bad = not_finite(w[e]) & ~low_keys(context - 2 * e);
          odd |= bad;
          w[e] &= ~bad;
        }
        va[mt] = __builtin_bit_cast(bf16x8, w);
      }
    }
#pragma unroll
    for (int nt = 0; nt < kTiles; ++nt) {
      f32x4 st[2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        st[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) st[t] = mfma16x16x32(ka[t][kk], qop[nt][kk], st[t]);
      }
      float sc[8];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[4 * t + r] = st[t][r] * a.scale_log2;
      if (tail) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int j = first + e - row.ctx;
          const bool sees = j < 0 || (first + e < t1 && (mask[nt][j >> 6] >> (j & 63) & 1));
          sc[e] = sees ? sc[e] : -INFINITY;
        }
      }
      float mx = sc[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) mx = fmaxf(mx, sc[e]);
      mx = col_max4(mx);
      const float m_new = fmaxf(m_run[nt], mx);
      const float m_use = m_new == -INFINITY ? 0.f : m_new;
      const float alpha = fast_exp2(m_run[nt] - m_use);
      f32x8 p;
      float psum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = fast_exp2(sc[e] - m_use);
        psum += p[e];
      }
      l_run[nt] = l_run[nt] * alpha + psum;
      m_run[nt] = m_new;
      const bf16x8 p_hi = to_bf16x8(p);
      const bf16x8 p_lo = to_bf16x8(p - to_f32x8(p_hi));
#pragma unroll
      for (int mt = 0; mt < 8; ++mt) {
        o[nt][mt] *= alpha;
        o[nt][mt] = mfma16x16x32(va[mt], p_hi, o[nt][mt]);
        o[nt][mt] = mfma16x16x32(va[mt], p_lo, o[nt][mt]);
      }
    }
  }

  // join the waves
#pragma unroll
  for (int nt = 0; nt < kTiles; ++nt) {
    const float l_sum = col_sum4(l_run[nt]);
    if (kgrp == 0) {
      lds.m[wave][16 * nt + col] = m_run[nt];
      lds.l[wave][16 * nt + col] = l_sum;
    }
#pragma unroll
    for (int mt = 0; mt < 8; ++mt)
      *reinterpret_cast<f32x4 *>(&lds.o[wave][16 * nt + col][16 * mt + 4 * kgrp]) = o[nt][mt];
  }
  const int ncols = min(rows - r0, 16 * kTiles);
  if (__syncthreads_or(odd != 0)) {
    reach_odd<kFp8, kSplitWaves * kWave>(a, row, bt, g, t0, t1, r0, ncols,
                                         [&](int c) { return &lds.o[0][c][0]; });
    __syncthreads();
  }
  for (int idx = tid; idx < ncols * kHeadDim; idx += kSplitWaves * kWave) {
    const int c = idx / kHeadDim, d = idx % kHeadDim;
    float M = lds.m[0][c];
#pragma unroll
    for (int w = 1; w < kSplitWaves; ++w) M = fmaxf(M, lds.m[w][c]);
    const float M_use = M == -INFINITY ? 0.f : M;
    float acc = 0.f, lsum = 0.f;
#pragma unroll
    for (int w = 0; w < kSplitWaves; ++w) {
      const float f = fast_exp2(lds.m[w][c] - M_use);
      acc += f * lds.o[w][c][d];
      lsum += f * lds.l[w][c];
    }
    const int r = r0 + c, node = r / G;
    const size_t head = (size_t)(row.first + node) * a.hq + (size_t)g * G + (r - node * G);
    if (a.slots == 1) {
      a.out[head * kHeadDim + d] = lsum == 0.f ? 0.f : acc / lsum * a.v_scale;
      if (a.lse && d == 0) a.lse[head] = (M + __log2f(lsum)) * kLn2;
    } else {
      const size_t part = head * a.slots + split;
      a.ws_o[part * kHeadDim + d] = acc;
      if (d == 0) {
        a.ws_m[part] = M;
        a.ws_l[part] = lsum;
      }
    }
  }
}

// ---- wide tiles ----
// 256 query rows of one KV head, by eight waves of 32 rows each: the columns of 32 x 32 matrix
// tiles, their queries in registers. Blocks of 128 keys are loaded into registers one block
// ahead and stored to one of two LDS buffers, one barrier a block:
//   S^T[key][row] = K[key][:] . Q^T[:][row]       (8 products of 32 x 32 x 16 for 32 keys)
//   O^T[d][row]  += V^T[d][key] . P^T[key][row]   (8, twice: the weights' two bf16 parts)
// Keys are ordered inside a pair of pages so that the 16 scores of a lane are the weights it
// supplies to the second product. Tiles with fewer live rows split the pairs of a block over
// the waves that have none of their own, and join them at the end. The running maximum moves
// only when a score passes it by 8 (in powers of two), so that O is rescaled rarely; weights
// are at most 2^8 then.
typedef float f32x16 __attribute__((ext_vector_type(16)));
constexpr int kWideWaves = 8, kWideThreads = kWideWaves * kWave;
constexpr int kWideRows = 32 * kWideWaves;
constexpr int kWideKeys = 128, kWidePages = kWideKeys / kPage, kWidePairs = kWideKeys / kPair;
constexpr int kWKPitch = kHeadDim + 8;                    // of a key's row in LDS (elements)
constexpr int kWKElems = kWideKeys * kWKPitch, kWVElems = kWideKeys * kHeadDim;
constexpr float kSlack = 8.f;

struct WideLds {
  union {
    struct {
      __attribute__((aligned(16))) uint16_t k[2][kWKElems];
      __attribute__((aligned(16))) uint16_t v[2][kWVElems];
    } in;
    __attribute__((aligned(16))) float o[kWideWaves][32][kOPitch];
  };
  float m[kWideWaves][32], l[kWideWaves][32];
};
static_assert(sizeof(WideLds) <= 160 * 1024, "LDS of a compute unit");

__device__ __forceinline__ f32x16 mfma32x32x16(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ bf16x8 lds_bf16x8(const uint16_t *p) {
  return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(p));
}
// The two 8-slot halves of V row d change places where bit 3 of d is set: rows 8 apart would
// meet in the same banks.
__device__ __forceinline__ int wide_v(int page, int d, int half) {
  return (page * kHeadDim + d) * kPage + ((half ^ ((d >> 3) & 1)) * 8);
}
// Of the two lanes of a column.
__device__ __forceinline__ float pair_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <bool kFp8>
__global__ __launch_bounds__(kWideThreads) void tree_wide_kernel(TreeArgs a) {
  __shared__ WideLds lds;
  int id = blockIdx.x;
  const int g = id % a.hkv;
  id /= a.hkv;
  const int tile = id % a.tiles;
  id /= a.tiles;
  const int split = id % a.slots, b = id / a.slots;
  const TreeRow row = tree_row(a, b);
  const int G = a.group, r0 = tile * kWideRows, rows = min(row.T * G - r0, kWideRows);
  const int end = row.ctx + row.T;
  const int t0 = split * a.split_tokens, t1 = min(end, t0 + a.split_tokens);
  if (rows <= 0 || t0 >= t1) return;
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int col = lane & 31, grp = lane >> 5;
  const int nblocks = (t1 - t0 + kWideKeys - 1) / kWideKeys;
  const int row_pages = (t1 + kPage - 1) / kPage;
  const int32_t *bt = a.block_table + (size_t)b * a.bt_stride;
  const size_t head_stride = (size_t)kPage * kHeadDim;

  // which rows and which pairs of a block are this wave's
  const int parts = (rows + 31) / 32;
  const int lanes_log = parts <= 1 ? 0 : parts <= 2 ? 1 : parts <= 4 ? 2 : 3;
  const int share = wave >> lanes_log, shares = min(kWideWaves >> lanes_log, kWidePairs);
  const int part = wave & ((1 << lanes_log) - 1);
  const bool live = part < parts && share < shares;

  const int r = r0 + min(32 * part + col, rows - 1), node = r / G;
  const size_t t = row.first + node;
  const uint64_t *mask = a.mask + t * a.words;
  bf16x8 q[8];
  {
    const uint16_t *qrow = a.q + (t * a.hq + (size_t)g * G + (r - node * G)) * kHeadDim + 8 * grp;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) q[kk] = load_bf16x8(qrow + 16 * kk);
  }

  uint32_t odd = 0;                             // infinite or NaN values of nodes

  // ---- staging: a wave a page of the block, 16 bytes a lane and load
  u32x4 kreg[4], vreg[4];
  auto page_id = [&](int blk) {
    const int pg = t0 / kPage + blk * kWidePages + wave;
    return clamp_page(bt[pg < row_pages ? pg : row_pages - 1], a.num_pages);
  };
  int next_id = page_id(0);
  auto load = [&](int blk) __attribute__((always_inline)) {
    const size_t base = ((size_t)next_id * a.hkv + g) * head_stride;
    if (blk + 1 < nblocks) next_id = page_id(blk + 1);
    constexpr int kLoads = kFp8 ? 2 : 4;
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      if constexpr (kFp8) {
        kreg[i] = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const uint8_t *>(a.k_pool) +
                                                   base + (i * kWave + lane) * 16);
        vreg[i] = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const uint8_t *>(a.v_pool) +
                                                   base + (i * kWave + lane) * 16);
      } else {
        kreg[i] = load_u32x4(a.k_pool + base + (i * kWave + lane) * 8);
        vreg[i] = load_u32x4(a.v_pool + base + (i * kWave + lane) * 8);
      }
    }
  };
  auto store = [&](int blk) __attribute__((always_inline)) {
    uint16_t *sk = lds.in.k[blk & 1], *sv = lds.in.v[blk & 1];
    const int pos = t0 + blk * kWideKeys + wave * kPage;   // the page's first key
    const bool tail = pos + kPage > row.ctx;
    // values past the row's end, and those of nodes that are infinite or NaN, become zeros
    auto alive = [&](u32x4 w, int first) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        w[e] &= low_keys(end - first - 2 * e);
        const uint32_t bad = not_finite(w[e]) & ~low_keys(row.ctx - first - 2 * e);
        odd |= bad;
        w[e] &= ~bad;
      }
      return w;
    };
    if constexpr (kFp8) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int c = i * kWave + lane;
        uint16_t *kd = sk + (wave * kPage + (c >> 3)) * kWKPitch + (c & 7) * 16;
        *reinterpret_cast<bf16x8 *>(kd) = fp8x8_to_bf16x8(u32x2{kreg[i][0], kreg[i][1]});
        *reinterpret_cast<bf16x8 *>(kd + 8) = fp8x8_to_bf16x8(u32x2{kreg[i][2], kreg[i][3]});
        u32x4 v0 = __builtin_bit_cast(u32x4, fp8x8_to_bf16x8(u32x2{vreg[i][0], vreg[i][1]}));
        u32x4 v1 = __builtin_bit_cast(u32x4, fp8x8_to_bf16x8(u32x2{vreg[i][2], vreg[i][3]}));
        if (tail) v0 = alive(v0, pos), v1 = alive(v1, pos + 8);
        *reinterpret_cast<u32x4 *>(sv + wide_v(wave, c, 0)) = v0;
        *reinterpret_cast<u32x4 *>(sv + wide_v(wave, c, 1)) = v1;
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = i * kWave + lane;
        *reinterpret_cast<u32x4 *>(sk + (wave * kPage + (c >> 4)) * kWKPitch + (c & 15) * 8) = kreg[i];
        u32x4 w = vreg[i];
        if (tail) w = alive(w, pos + (c & 1) * 8);
        *reinterpret_cast<u32x4 *>(sv + wide_v(wave, c >> 1, c & 1)) = w;
      }
    }
  };

  f32x16 o[4];
#pragma unroll
  for (int mt = 0; mt < 4; ++mt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[mt][i] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  // row i of a tile of scores is key i with bits 2 and 3 exchanged
  const int key = (col & ~12) | ((col & 4) << 1) | ((col & 8) >> 1);

  auto pair = [&](int blk, int pp) __attribute__((always_inline)) {
    const int tok = t0 + blk * kWideKeys + pp * kPair;
    if (tok >= t1) return;
    const uint16_t *sk = lds.in.k[blk & 1] + (pp * kPair + key) * kWKPitch + 8 * grp;
    const uint16_t *sv = lds.in.v[blk & 1];
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) s = mfma32x32x16(lds_bf16x8(sk + 16 * kk), q[kk], s);
    const bool tail = tok + kPair > row.ctx;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] *= a.scale_log2;
    if (tail) {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int pos = tok + 16 * (i >> 3) + 8 * grp + (i & 7), j = pos - row.ctx;
        const bool sees = j < 0 || (pos < end && (mask[j >> 6] >> (j & 63) & 1));
        s[i] = sees ? s[i] : -INFINITY;
      }
    }
    float mx = s[0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[i]);
    mx = pair_max(mx);
    const bool grows = mx > m_run + kSlack;     // (each row by itself: no row's bits depend on others)
    if (__any(grows)) {
      const float alpha = grows ? fast_exp2(m_run - mx) : 1.f;
      m_run = grows ? mx : m_run;
      l_run *= alpha;
#pragma unroll
      for (int mt = 0; mt < 4; ++mt) o[mt] *= alpha;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
    bf16x8 hi[2], lo[2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      f32x8 p;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        p[e] = fast_exp2(s[8 * h + e] - m_use);
        l_run += p[e];
      }
      hi[h] = to_bf16x8(p);
      lo[h] = to_bf16x8(p - to_f32x8(hi[h]));
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int mt = 0; mt < 4; ++mt) {
        const bf16x8 v = lds_bf16x8(sv + wide_v(2 * pp + h, 32 * mt + col, grp));
        o[mt] = mfma32x32x16(v, hi[h], o[mt]);
        o[mt] = mfma32x32x16(v, lo[h], o[mt]);
      }
  };

  load(0);
  store(0);
  for (int blk = 0; blk < nblocks; ++blk) {
    if (blk + 1 < nblocks) load(blk + 1);
    __syncthreads();
    if (live)
      for (int pp = share; pp < kWidePairs; pp += shares) pair(blk, pp);
    if (blk + 1 < nblocks) store(blk + 1);
  }
  __syncthreads();

  // whole rows through LDS, joining the waves that shared them
  if (live) {
    const auto l = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run),
                                                    false, false);
    if (grp == 0) {
      lds.m[wave][col] = m_run;
      lds.l[wave][col] = __uint_as_float(l[0]) + __uint_as_float(l[1]);
    }
#pragma unroll
    for (int mt = 0; mt < 4; ++mt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4 *>(&lds.o[wave][col][32 * mt + 8 * i + 4 * grp]) =
            f32x4{o[mt][4 * i], o[mt][4 * i + 1], o[mt][4 * i + 2], o[mt][4 * i + 3]};
  }
  if (__syncthreads_or(odd != 0)) {
    reach_odd<kFp8, kWideThreads>(a, row, bt, g, t0, t1, r0, rows,
                                  [&](int c) { return &lds.o[c >> 5][c & 31][0]; });
    __syncthreads();
  }
  for (int idx = tid; idx < rows * (kHeadDim / 4); idx += kWideThreads) {
    const int c = idx / (kHeadDim / 4), d = idx % (kHeadDim / 4) * 4;
    float M = -INFINITY, lsum = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < shares; ++w) M = fmaxf(M, lds.m[(w << lanes_log) + (c >> 5)][c & 31]);
    const float M_use = M == -INFINITY ? 0.f : M;
    for (int w = 0; w < shares; ++w) {
      const int from = (w << lanes_log) + (c >> 5);
      const float f = fast_exp2(lds.m[from][c & 31] - M_use);
      acc += f * *reinterpret_cast<const f32x4 *>(&lds.o[from][c & 31][d]);
      lsum += f * lds.l[from][c & 31];
    }
    const int rr = r0 + c, n = rr / G;
    const size_t head = (size_t)(row.first + n) * a.hq + (size_t)g * G + (rr - n * G);
    if (a.slots == 1) {
      const float inv = a.v_scale / lsum;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = lsum == 0.f ? 0.f : acc[e] * inv;
      *reinterpret_cast<f32x4 *>(a.out + head * kHeadDim + d) = acc;
      if (a.lse && d == 0) a.lse[head] = (M + __log2f(lsum)) * kLn2;
    } else {
      const size_t at = head * a.slots + split;
      *reinterpret_cast<f32x4 *>(a.ws_o + at * kHeadDim + d) = acc;
      if (d == 0) {
        a.ws_m[at] = M;
        a.ws_l[at] = lsum;
      }
    }
  }
}

// Joins the splits of one node's heads, a wave a head.
constexpr int kJoinWaves = 4;
__global__ __launch_bounds__(kJoinWaves * kWave) void tree_join_kernel(TreeArgs a) {
  const int t = blockIdx.x, lane = threadIdx.x & (kWave - 1);
  const int b = wave_search(a.B, t, [&](int i) { return a.cu_q[i]; });
  const TreeRow row = tree_row(a, b);
  if (t < row.first || t >= row.first + row.T) return;
  const int n = (row.ctx + row.T + a.split_tokens - 1) / a.split_tokens;
  for (int h = threadIdx.x / kWave; h < a.hq; h += kJoinWaves) {
    const size_t head = (size_t)t * a.hq + h, part = head * a.slots;
    float M = -INFINITY;
    for (int s = 0; s < n; ++s) M = fmaxf(M, a.ws_m[part + s]);
    const float M_use = M == -INFINITY ? 0.f : M;
    float x = 0.f, y = 0.f, lsum = 0.f;
    for (int s = 0; s < n; ++s) {
      const float f = fast_exp2(a.ws_m[part + s] - M_use);
      const float2 v = *reinterpret_cast<const float2 *>(a.ws_o + (part + s) * kHeadDim + 2 * lane);
      x += f * v.x;
      y += f * v.y;
      lsum += f * a.ws_l[part + s];
    }
    const float inv = a.v_scale / lsum;
    float2 v = {lsum == 0.f ? 0.f : x * inv, lsum == 0.f ? 0.f : y * inv};
    *reinterpret_cast<float2 *>(a.out + head * kHeadDim + 2 * lane) = v;
    if (a.lse && lane == 0) a.lse[head] = (M + __log2f(lsum)) * kLn2;
  }
}

}  // namespace

TreePlan tree_plan(int32_t B, int32_t hq, int32_t hkv, int32_t max_q_len, int32_t max_kv_len) {
  const int64_t rows = (int64_t)max_q_len * (hq / hkv);
  TreePlan p;
  p.rows = rows <= 16 ? 16 : rows <= 32 ? 32 : kWideRows;
  p.tiles = (rows + p.rows - 1) / p.rows;
  const int64_t units = (int64_t)B * hkv * p.tiles;
  int64_t split = 512;
  if (p.rows == kWideRows)
    while (split < 8192 && units * max_kv_len / split > 2048) split *= 2;
  else
    while (split < 4096 && units * max_kv_len / split > 8192) split *= 2;
  p.split_tokens = (int32_t)split;
  p.slots = (int32_t)((max_kv_len + split - 1) / split);
  if (p.slots < 1) p.slots = 1;
  p.groups = units * p.slots;
  return p;
}

size_t tree_workspace_bytes(int32_t total_q, int32_t hq, const TreePlan &p) {
  return p.slots == 1 ? 0 : (size_t)total_q * hq * p.slots * (kHeadDim + 2) * sizeof(float);
}

hipError_t launch_tree(const uint16_t *q, const int32_t *cu_q, const int32_t *ctx_lens,
                       const uint64_t *mask, int32_t words, const PagedKV &kv, int32_t B,
                       int32_t hq, int32_t total_q, int32_t max_q_len, int32_t max_kv_len,
                       float scale, float *out, float *lse, void *workspace, const TreePlan &p,
                       hipStream_t stream) {
  const size_t parts = (size_t)total_q * hq * p.slots;
  TreeArgs a;
  a.q = q;
  a.cu_q = cu_q;
  a.ctx_lens = ctx_lens;
  a.mask = mask;
  a.k_pool = kv.k_pool;
  a.v_pool = kv.v_pool;
  a.block_table = kv.block_table;
  a.ws_o = static_cast<float *>(workspace);
  a.ws_m = p.slots == 1 ? nullptr : a.ws_o + parts * kHeadDim;
  a.ws_l = p.slots == 1 ? nullptr : a.ws_m + parts;
  a.out = out;
  a.lse = lse;
  a.B = B;
  a.hq = hq;
  a.hkv = kv.hkv;
  a.group = hq / kv.hkv;
  a.words = words;
  a.bt_stride = kv.bt_stride;
  a.num_pages = kv.num_pages;
  a.total_q = total_q;
  a.max_q_len = max_q_len;
  a.max_kv_len = max_kv_len;
  a.split_tokens = p.split_tokens;
  a.slots = p.slots;
  a.tiles = (int32_t)p.tiles;
  a.scale_log2 = scale * kLog2e * kv.k_scale;
  a.v_scale = kv.v_scale;
  const dim3 grid((unsigned)p.groups), block(kSplitWaves * kWave);
  if (p.rows == kWideRows && kv.fp8)
    tree_wide_kernel<true><<<grid, kWideThreads, 0, stream>>>(a);
  else if (p.rows == kWideRows)
    tree_wide_kernel<false><<<grid, kWideThreads, 0, stream>>>(a);
  else if (p.rows == 32 && kv.fp8)
    tree_split_kernel<2, true><<<grid, block, 0, stream>>>(a);
  else if (p.rows == 32)
    tree_split_kernel<2, false><<<grid, block, 0, stream>>>(a);
  else if (kv.fp8)
    tree_split_kernel<1, true><<<grid, block, 0, stream>>>(a);
  else
    tree_split_kernel<1, false><<<grid, block, 0, stream>>>(a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.slots == 1) return e;
  tree_join_kernel<<<total_q, kJoinWaves * kWave, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace ra
