// Attention of a tree of drafted tokens over the paged cache (rollout_attn_decode_tree).
//
// Row b's T nodes lie behind its ctx cached tokens. The query rows of a KV head are its G =
// Hq / Hkv query heads of all nodes, node r / G and head r % G for query row r, in tiles of 16,
// 32, 128 or 256 that are columns of the matrix products, so that a key is read once for a tile.
// All nodes see the context; which of the nodes a node sees is in its bit mask:
//   out = sum_j p_j v_j / sum_j p_j,  p_j = 2^(c q.k_j - max),  j of the keys that the node sees.
//
// Softmax is the online form in fp32, base 2. Weights meet the values in two bf16 parts, off by
// 2^-16 of a weight: one part would be off by 2^-8. (Narrow tiles over bf16 pools take a third
// part, which is free there. In wide tiles it costs what the matrix cores do not have: 32 rows
// of 64 nodes over 2k to 24k keys 666 -> 813 us.) The later parts of a weight can be 0 or negative, so
// that an infinite value of the context gives NaN where the formula has an infinity.
//
// Read: every row's keys and values once a tile, 512 bytes a key and KV head in bf16. Computed:
// 512 flops a key and query row, 768 with the weights' second part. Bound by HBM up to about 60
// rows a tile and by the matrix cores, softmax beside them, from about 100. Measured, Hq 32 on 8:
// 64 rows of 8 nodes over 4k to 32k keys (5.08 GB) 807 us, 6.3 TB/s, as decode of one token
// (795); of 16 nodes 915-930; 32 rows of 16 to 64 nodes over 2k to 24k 501-535 us (249 GFLOP, 374
// with the parts: 0.70-0.75 PFLOP/s); 1 row of 4 nodes over 16,000 keys 26 us, of 32 nodes 47.
//
// The work of a call is a line: its tiles in the order of rows, tiles and KV heads, each as long
// as its blocks of keys, weighted by what a block costs with the tile's rows. Every workgroup
// takes an equal share of the line, so that rows of different lengths and trees of different
// sizes end together, and a tile is cut only where a share ends: a cut tile's pieces go to the
// workspace and a second launch joins them. (Splits of a fixed length, a workgroup each, left
// the compute units idle for 13 to 29 % of the time, and wrote 2 to 8 times the partial
// results.) Calls of short rows (kDirectKeys) take a workgroup a tile and one launch: there is
// no join, and no tile begins twice.
#include <algorithm>
#include <type_traits>

#include "ra_device.h"
#include "ra_internal.h"
#include "ra_lds.h"
#include "ra_wave.h"

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
  float *out, *lse;
  // workspace: the share's length, where the rows begin on the line, and of each workgroup two
  // pieces' results: unnormalised O, (maximum, sum)
  int64_t *share, *start;      // [1], [B]
  float *ws_o;                 // [2 groups][piece_rows][128]
  float2 *ws_ml;               // [2 groups][piece_rows]
  int64_t min_share;
  int32_t B, hq, hkv, group, words, bt_stride, num_pages, total_q, max_q_len, max_kv_len;
  int32_t piece_rows, tiles, direct;
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

// What a block of keys costs with a tile's rows, by parts of 32 rows: tiles of up to 128 rows
// wait for their keys, larger ones for their products.
template <int kRows>
__device__ __forceinline__ int block_cost(int rows) {
  if constexpr (kRows < 256) return 1;
  const int parts = (rows + 31) / 32;
  return parts <= 3 ? 8 : parts == 4 ? 9 : parts <= 6 ? 12 : 16;
}
template <int kRows>
__host__ __device__ constexpr int block_keys() { return kRows <= 32 ? 128 : 64; }

// A row's tiles on the line: all but the last have kRows query rows.
template <int kRows>
struct RowLine {
  int blocks, tiles, last_cost;
  __device__ __forceinline__ RowLine(const TreeRow &r, int G) {
    blocks = r.T > 0 ? (r.ctx + r.T + block_keys<kRows>() - 1) / block_keys<kRows>() : 0;
    tiles = r.T > 0 ? (r.T * G + kRows - 1) / kRows : 0;
    last_cost = block_cost<kRows>(r.T * G - (tiles - 1) * kRows);
  }
  __device__ __forceinline__ int cost(int tile) const {
    return tile + 1 < tiles ? block_cost<kRows>(kRows) : last_cost;
  }
  __device__ __forceinline__ int64_t before(int tile, int g, int hkv) const {
    return ((int64_t)tile * hkv * block_cost<kRows>(kRows) + (int64_t)g * cost(tile)) * blocks;
  }
  __device__ __forceinline__ int64_t length(int hkv) const {
    return tiles > 0 ? before(tiles - 1, hkv, hkv) : 0;
  }
};

template <int kThreads>
struct WalkLds {
  int64_t begin[kThreads + 1];       // of rows on the line
  int64_t part[kThreads / kWave];
};

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  const u32x2 w = __builtin_bit_cast(u32x2, x);
  u32x2 r;
  r[0] = __builtin_amdgcn_readfirstlane(w[0]);
  r[1] = __builtin_amdgcn_readfirstlane(w[1]);
  return __builtin_bit_cast(int64_t, r);
}

// x / y of numbers that are not negative: by 32 bits where both have no more.
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t y) {
  return ((x | y) >> 32) == 0 ? (int64_t)((uint32_t)x / (uint32_t)y) : x / y;
}

__device__ __forceinline__ TreeRow uniform_row(const TreeArgs &a, int b) {
  TreeRow r = tree_row(a, b);
  r.first = uniform(r.first);
  r.T = uniform(r.T);
  r.ctx = uniform(r.ctx);
  return r;
}

// Calls piece(b, row, tile, g, first block, behind the last one, place of the result) for all that
// is this workgroup's; place -1: a whole tile, whose result is final.
template <int kRows, int kThreads, typename Piece>
__device__ __forceinline__ void walk(const TreeArgs &a, WalkLds<kThreads> &lds, Piece piece) {
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  const int s = blockIdx.x;
  if (a.direct) {
    const int g = s % a.hkv, at = s / a.hkv, tile = at % a.tiles, b = at / a.tiles;
    const TreeRow row = uniform_row(a, b);
    const RowLine<kRows> line(row, a.group);
    if (tile < line.tiles) piece(b, row, tile, g, 0, line.blocks, -1);
    return;
  }
  // the rows' places, kThreads rows at a time; of up to 64 rows every wave works them all out
  // (and writes the same to LDS), so that none waits for another
  const bool few = a.B <= kWave;
  auto place = [&](int c0) {
    const int i = few ? lane : tid;
    int64_t mine = 0;
    if (c0 + i < a.B) mine = RowLine<kRows>(tree_row(a, c0 + i), a.group).length(a.hkv);
    const int64_t sum = wave_sums(mine);
    int64_t before = 0, all = of_lane(sum, kWave - 1);
    if (!few) {
      __syncthreads();
      if (lane == kWave - 1) lds.part[wave] = sum;
      __syncthreads();
      all = 0;
      for (int w = 0; w < kThreads / kWave; ++w) {
        if (w == wave) before = all;
        all += lds.part[w];
      }
    }
    if (i == 0) lds.begin[0] = 0;
    lds.begin[i + 1] = before + sum;
    if (!few) __syncthreads();
    return uniform(all);
  };
  int64_t all = 0;
  for (int c0 = 0; c0 < a.B; c0 += kThreads) {
    const int64_t n = place(c0);
    if (s == 0 && c0 + tid < a.B) a.start[c0 + tid] = all + lds.begin[tid];
    all += n;
  }
  const int64_t even = quotient(all + gridDim.x - 1, gridDim.x);
  const int64_t share = even > a.min_share ? even : a.min_share;
  if (s == 0 && tid == 0) *a.share = share;
  const int64_t s0 = uniform(s * share), s1 = uniform(min(all, s0 + share));
  int64_t base = 0;
  for (int c0 = 0; c0 < a.B && base < s1; c0 += kThreads) {
    const int rows = min(kThreads, a.B - c0);
    if (a.B > kThreads) place(c0);
    const int64_t n = uniform(lds.begin[rows]);
    if (base + n > s0) {
      // the last row that begins at or before s0, then those behind it
      int lo = 0, hi = rows - 1;
      while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (base + uniform(lds.begin[mid]) <= s0) lo = mid; else hi = mid - 1;
      }
      for (int i = lo; i < rows; ++i) {
        const int64_t begin = base + uniform(lds.begin[i]);
        if (begin >= s1) break;
        const int b = c0 + i;
        const TreeRow row = uniform_row(a, b);
        const RowLine<kRows> line(row, a.group);
        if (line.tiles == 0) continue;
        // its first tile and KV head that end behind s0
        const int64_t off = s0 > begin ? s0 - begin : 0;
        const int64_t full = line.before(1, 0, a.hkv);       // of a tile that is not the last
        int tile = uniform(line.tiles > 1 ? (int)min((int64_t)line.tiles - 1, quotient(off, full)) : 0);
        int g = uniform((int)quotient(off - line.before(tile, 0, a.hkv), (int64_t)line.cost(tile) * line.blocks));
        for (; tile < line.tiles; ++tile, g = 0)
          for (; g < a.hkv; ++g) {
            const int64_t at = begin + line.before(tile, g, a.hkv);
            if (at >= s1) return;
            const int cost = line.cost(tile);
            const int b0 = uniform(at >= s0 ? 0 : (int)quotient(s0 - at + cost - 1, cost));
            const int b1 = uniform((int)min((int64_t)line.blocks, quotient(s1 - at + cost - 1, cost)));
            if (b0 >= b1) continue;
            piece(b, row, tile, g, b0, b1, b0 == 0 && b1 == line.blocks ? -1 : 2 * s + (b0 == 0));
          }
      }
    }
    base += n;
  }
}

// Page ids by the scalar unit: vector loads of them would wait for all that are on their way.
__device__ __forceinline__ int page_at(const int32_t *bt, int i, int num_pages) {
  return clamp_page(((const __attribute__((address_space(4))) int32_t *)(uintptr_t)bt)[i], num_pages);
}

// Which of the 32 keys from position pos on node `mask` sees: those of the context, and the
// nodes below T that its mask names.
__device__ __forceinline__ uint32_t seen_keys(const uint64_t *mask, int pos, int ctx, int T) {
  const int j0 = pos - ctx, j = max(j0, 0);
  uint64_t bits = mask[min(j, T - 1) >> 6] >> (j & 63);
  if ((j & 63) > 32 && ((j + 31) >> 6) <= (T - 1) >> 6) bits |= mask[(j >> 6) + 1] << (64 - (j & 63));
  const int nodes = T - j;                   // bits of nodes that there are
  uint32_t w = nodes >= 32 ? (uint32_t)bits : nodes <= 0 ? 0u : (uint32_t)bits & ((1u << nodes) - 1);
  if (j0 < 0) w = j0 <= -32 ? ~0u : (w << -j0) | ((1u << -j0) - 1);
  return w;
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

// ---- narrow tiles ----
// 16 kTiles query rows by four waves, each of which takes every fourth pair of pages (32 keys)
// of the piece straight from HBM into its registers:
//   S^T[key][row] = K[key][:] . Q^T[:][row]       (4 products of 16 x 16 x 32 for 16 keys and rows)
//   O^T[d][row]  += V^T[d][key] . P^T[key][row]   (8 for 32 keys, once for each of the weights' parts)
// Bound by HBM: nothing of a key is used by two waves, so LDS would be a detour; the waves are
// joined through it at the end of a piece. 64 rows of 8 nodes over 4k to 32k keys: 802 us where
// decode's kernel takes 790, and 9 of the join.
template <int kTiles>
struct TreeLds {
  WalkLds<kSplitWaves * kWave> walk;
  float m[kSplitWaves][16 * kTiles];
  float l[kSplitWaves][16 * kTiles];
  float o[kSplitWaves][16 * kTiles][kOPitch];
};

template <int kTiles, bool kFp8>
__device__ __forceinline__ void narrow_piece(const TreeArgs &a, TreeLds<kTiles> &lds, int b,
                                             const TreeRow &row, int tile, int g, int blk0,
                                             int blk1, int place) {
  const int G = a.group, rows = row.T * G, r0 = tile * 16 * kTiles;
  const int end = row.ctx + row.T;
  const int t0 = blk0 * block_keys<16>(), t1 = min(end, blk1 * block_keys<16>());
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));             // (what follows from it is not kept from piece to piece)
  const int lane = tid & (kWave - 1);
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
  // arrived before the loop: a wait for them in it would wait for the keys and values as well
#pragma unroll
  for (int nt = 0; nt < kTiles; ++nt)
#pragma unroll
    for (int kk = 0; kk < 4; ++kk) asm volatile("" : "+v"(qop[nt][kk]));
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
  // A pair's keys are loaded while the pair before meets its values, its values while it meets
  // its own keys.
  size_t kbase = 0, vbase = 0;
  int id0 = 0, id1 = 0;                     // of the pair whose loads come next
  auto ids = [&](int pr) __attribute__((always_inline)) {
    const int pg = t0 / kPage + 2 * pr;
    id0 = page_at(bt, min(pg, row_pages - 1), a.num_pages);
    id1 = page_at(bt, min(pg + 1, row_pages - 1), a.num_pages);
  };
  auto pages = [&]() __attribute__((always_inline)) {
    kbase = ((size_t)(ka_sel ? id1 : id0) * a.hkv + g) * head_stride;
    vbase = ((size_t)(sv_sel ? id1 : id0) * a.hkv + g) * head_stride;
  };
  constexpr int kRaw = kFp8 ? 4 : 8;
  u32x4 kraw[kRaw];
  u32x4 vraw[kFp8 ? 4 : 8];
  auto load_k = [&]() __attribute__((always_inline)) {
    if constexpr (kFp8) {
      const uint8_t *kb = reinterpret_cast<const uint8_t *>(a.k_pool) + kbase;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int h = 0; h < 2; ++h)
          kraw[2 * t + h] = *reinterpret_cast<const u32x4 *>(kb + (ka_slot + 4 * t) * kHeadDim +
                                                             64 * h + 16 * kgrp);
    } else {
      const uint16_t *kb = a.k_pool + kbase;
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)
          kraw[4 * t + kk] = load_u32x4(kb + (ka_slot + 4 * t) * kHeadDim + 32 * kk + 8 * kgrp);
    }
  };
  // (values are read once, in whole lines: marked so that they do not displace the keys' lines,
  // of which two loads take a half each)
  auto load_v = [&]() __attribute__((always_inline)) {
    if constexpr (kFp8) {
      // whole 16-slot rows: lane l loads row 16 (2 j + l / 16 % 2) + col of its page
      const uint8_t *vb = reinterpret_cast<const uint8_t *>(a.v_pool) + vbase;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        vraw[j] = load_stream_u32x4(vb + (16 * (2 * j + (kgrp & 1)) + col) * kPage);
    } else {
      const uint16_t *vb = a.v_pool + vbase;
#pragma unroll
      for (int mt = 0; mt < 8; ++mt) vraw[mt] = load_stream_u32x4(vb + (16 * mt + col) * kPage + sv_slot);
    }
  };
  if (wave < npairs) {
    ids(wave);
    pages();
    load_k();
    load_v();
    ids(wave + kSplitWaves);
  }
  // kMore: another pair follows (a load under a condition would make the waits of what is not
  // under it wait for it too)
  auto step = [&](int pr, auto kMore) __attribute__((always_inline)) {
    const int tok = t0 + pr * kPair;
    bf16x8 ka[2][4], va[8];
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int h = 0; h < 2; ++h)
        if constexpr (kFp8) {
          ka[t][2 * h] = fp8x8_to_bf16x8(u32x2{kraw[2 * t + h][0], kraw[2 * t + h][1]});
          ka[t][2 * h + 1] = fp8x8_to_bf16x8(u32x2{kraw[2 * t + h][2], kraw[2 * t + h][3]});
        } else {
          ka[t][2 * h] = __builtin_bit_cast(bf16x8, kraw[4 * t + 2 * h]);
          ka[t][2 * h + 1] = __builtin_bit_cast(bf16x8, kraw[4 * t + 2 * h + 1]);
        }
    f32x4 st[kTiles][2];
#pragma unroll
    for (int nt = 0; nt < kTiles; ++nt)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        st[nt][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) st[nt][t] = mfma16x16x32(ka[t][kk], qop[nt][kk], st[nt][t]);
      }
    keep_order();
    if constexpr (kMore) {
      pages();
      load_k();
      ids(pr + 2 * kSplitWaves);
    }
    keep_order();
    if constexpr (kFp8) {
      // lanes l and l ^ 16 hold rows 2 j and 2 j + 1 of one page: exchanged, each has the slots
      // that it supplies of both
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const auto s0 = __builtin_amdgcn_permlane16_swap(vraw[j][0], vraw[j][2], false, false);
        const auto s1 = __builtin_amdgcn_permlane16_swap(vraw[j][1], vraw[j][3], false, false);
        va[2 * j] = fp8x8_to_bf16x8(u32x2{s0[0], s1[0]});
        va[2 * j + 1] = fp8x8_to_bf16x8(u32x2{s0[1], s1[1]});
      }
    } else {
#pragma unroll
      for (int mt = 0; mt < 8; ++mt) va[mt] = __builtin_bit_cast(bf16x8, vraw[mt]);
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
      float sc[8];
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int r = 0; r < 4; ++r) sc[4 * t + r] = st[nt][t][r] * a.scale_log2;
      if (tail) {
        const uint32_t sees = seen_keys(mask[nt], tok, row.ctx, row.T) >> (first - tok);
#pragma unroll
        for (int e = 0; e < 8; ++e) sc[e] = sees >> e & 1 ? sc[e] : -INFINITY;
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
      const f32x8 rest = p - to_f32x8(p_hi);
      const bf16x8 p_lo = to_bf16x8(rest);
      // a third part of the weights, to fp32, where it is free (64 rows of 8 nodes over 4k to 32k
      // keys: bf16 pools 807 us with two parts and 808 with three, codes 452 and 487)
      bf16x8 p_last = {};
      if constexpr (!kFp8) p_last = to_bf16x8(rest - to_f32x8(p_lo));
#pragma unroll
      for (int mt = 0; mt < 8; ++mt) {
        o[nt][mt] *= alpha;
        o[nt][mt] = mfma16x16x32(va[mt], p_hi, o[nt][mt]);
        o[nt][mt] = mfma16x16x32(va[mt], p_lo, o[nt][mt]);
        if constexpr (!kFp8) o[nt][mt] = mfma16x16x32(va[mt], p_last, o[nt][mt]);
      }
    }
    keep_order();
    if constexpr (kMore) load_v();
    keep_order();
  };
  int pr = wave;
  for (; pr + kSplitWaves < npairs; pr += kSplitWaves) step(pr, std::true_type{});
  if (pr < npairs) step(pr, std::false_type{});

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
  // (four dims a thread: with one, 4 rows of up to 256 keys, 8 nodes took 12.0 us in place of 9.0)
  if (__syncthreads_or(odd != 0)) {
    reach_odd<kFp8, kSplitWaves * kWave>(a, row, bt, g, t0, t1, r0, ncols,
                                         [&](int c) { return &lds.o[0][c][0]; });
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < 16 * kTiles * kHeadDim / (4 * kSplitWaves * kWave); ++i) {
    const int idx = i * kSplitWaves * kWave + tid, c = idx / (kHeadDim / 4), d = idx % (kHeadDim / 4) * 4;
    if (c >= ncols) break;
    float M = lds.m[0][c];
#pragma unroll
    for (int w = 1; w < kSplitWaves; ++w) M = fmaxf(M, lds.m[w][c]);
    const float M_use = M == -INFINITY ? 0.f : M;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float lsum = 0.f;
#pragma unroll
    for (int w = 0; w < kSplitWaves; ++w) {
      const float f = fast_exp2(lds.m[w][c] - M_use);
      acc += f * *reinterpret_cast<const f32x4 *>(&lds.o[w][c][d]);
      lsum += f * lds.l[w][c];
    }
    if (place < 0) {
      const int r = r0 + c, node = r / G;
      const size_t head = (size_t)(row.first + node) * a.hq + (size_t)g * G + (r - node * G);
      const float inv = a.v_scale / lsum;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = lsum == 0.f ? 0.f : acc[e] * inv;
      *reinterpret_cast<f32x4 *>(a.out + head * kHeadDim + d) = acc;
      if (a.lse && d == 0) a.lse[head] = (M + __log2f(lsum)) * kLn2;
    } else {
      const size_t part = (size_t)place * a.piece_rows + c;
      *reinterpret_cast<f32x4 *>(a.ws_o + part * kHeadDim + d) = acc;
      if (d == 0) a.ws_ml[part] = float2{M, lsum};
    }
  }
  __syncthreads();                          // the next piece writes there
}

template <int kTiles, bool kFp8>
__global__ __launch_bounds__(kSplitWaves * kWave, 2) void tree_narrow_kernel(TreeArgs a) {
  __shared__ TreeLds<kTiles> lds;
  walk<16 * kTiles>(a, lds.walk,
                    [&](int b, const TreeRow &row, int tile, int g, int blk0, int blk1, int place)
                        __attribute__((always_inline)) {
                          narrow_piece<kTiles, kFp8>(a, lds, b, row, tile, g, blk0, blk1, place);
                        });
}

// ---- wide tiles ----
// 32 kW query rows of one KV head, by kW waves of 32 rows each: the columns of 32 x 32 matrix
// tiles, their queries in registers. Blocks of 64 keys are loaded straight into a ring of LDS
// buffers, one barrier a block:
//   S^T[key][row] = K[key][:] . Q^T[:][row]       (8 products of 32 x 32 x 16 for 32 keys)
//   O^T[d][row]  += V^T[d][key] . P^T[key][row]   (8, twice: the weights' two bf16 parts)
// Keys are ordered inside a pair of pages so that the 16 scores of a lane are the weights it
// supplies to the second product. Tiles with fewer live rows split the pairs of keys over the
// waves that have none of their own, and join them at the end. The running maximum moves
// only when a score passes it by 8 (in powers of two), so that O is rescaled rarely; weights
// are at most 2^8 then.
// kW is 4 for trees of up to 128 query rows, two workgroups a compute unit, each of which works
// while the other waits, and 8 (a ring of four, three blocks ahead) for larger ones. (64 rows
// of 16 nodes, 64 query rows: 915-930 us, with kW 8 948; over fp8 pools 643-680 and 791. 32 rows of
// 16 to 64 nodes over 2k to 24k keys in codes 493-512, of 32 nodes 386-397. Codes fill half of a
// ring's slots, whose size is that of bf16 pages.) With
// few query rows bound by the loads: those of 64 rows of 16 nodes alone take 912 of 956 us
// (5.6 TB/s); with many by the products and the softmax beside them, which a wave issues in
// turn: 32 rows of 64 nodes 751 us with a pair of keys a wave at a time, 683 with a block's two
// pairs by one wave, the second's weights beside the first's products.
typedef float f32x16 __attribute__((ext_vector_type(16)));
constexpr int kWideKeys = 64, kWidePages = kWideKeys / kPage, kWidePairs = kWideKeys / kPair;
constexpr int kPageElems = kPage * kHeadDim;
constexpr float kSlack = 8.f;               // (powers of two that a weight may pass 1 by)
constexpr int kBeside = 10;                 // vector instructions beside a product

template <int kW>
struct WideLds {
  static constexpr int kRing = kW == 8 ? 4 : 2;
  union {
    __attribute__((aligned(16))) uint16_t in[kRing][2 * kWidePages][kPageElems];   // K, then V
    __attribute__((aligned(16))) float o[kW][32][kOPitch];
  };
  float m[kW][32], l[kW][32];
  WalkLds<kW * kWave> walk;
};
static_assert(sizeof(WideLds<8>) <= 160 * 1024 && sizeof(WideLds<4>) <= 80 * 1024,
              "LDS of a compute unit, for one workgroup and for two");

// LDS places. Unit c (16 bytes) of key `slot` of a page is at 16 slot + (c ^ slot), half h of value
// row d at 2 d + (h ^ bit 3 of d): 16 lanes that read together meet no bank twice. Codes (fp8): 8
// units a key, unit c at 8 slot + (c ^ slot / 2), one unit a value row.
__device__ __forceinline__ u32x4 read_lds(uint32_t at) {
  return *(const __attribute__((address_space(3))) u32x4 *)(uintptr_t)at;
}

__device__ __forceinline__ f32x16 mfma32x32x16(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
// Of the two lanes of a column.
__device__ __forceinline__ float pair_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

template <int kW, bool kFp8>
__device__ __forceinline__ void wide_piece(const TreeArgs &a, WideLds<kW> &lds, int b,
                                           const TreeRow &row, int tile, int g, int blk0, int blk1,
                                           int place) {
  constexpr int kWideRows = 32 * kW, kThreads = kW * kWave, kRing = WideLds<kW>::kRing;
  const int G = a.group, r0 = tile * kWideRows, rows = min(row.T * G - r0, kWideRows);
  const int end = row.ctx + row.T;
  const int t0 = blk0 * kWideKeys, t1 = min(end, blk1 * kWideKeys), nblocks = blk1 - blk0;
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));                 // (what follows from it is not kept from piece to piece)
  const int lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int col = lane & 31, grp = lane >> 5;
  const int row_pages = (t1 + kPage - 1) / kPage;
  const int32_t *bt = a.block_table + (size_t)b * a.bt_stride;

  // Which rows and which pairs of a block are this wave's: kW / parts waves share a part, or one
  // more; the parts with fewer have the first waves, which do more and lie on different SIMDs.
  const int parts = (rows + 31) / 32, base = kW / parts, extra = kW % parts;
  const int few = parts - extra, heavy = few * base;
  const bool first_waves = wave < heavy;
  const int part = first_waves ? extra + wave % few : (wave - heavy) % extra;
  const int share = first_waves ? wave / few : (wave - heavy) / extra;
  const int shares = first_waves ? base : base + 1;

  const int r = r0 + min(32 * part + col, rows - 1), node = r / G;
  const size_t t = row.first + node;
  const uint64_t *mask = a.mask + t * a.words;
  bf16x8 q[8];                                  // dims 16 kk + 8 grp .. (fp8: see read_k)
  {
    const uint16_t *qrow = a.q + (t * a.hq + (size_t)g * G + (r - node * G)) * kHeadDim;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk)
      q[kk] = load_bf16x8(qrow + (kFp8 ? 32 * (kk >> 1) + 16 * grp + 8 * (kk & 1) : 16 * kk + 8 * grp));
    // arrived before the loads to LDS begin: a wait for them later would wait for those too
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) asm volatile("" : "+v"(q[kk]));
    if (a.scale_log2 < 0.f)                     // the scale's sign, so that c below has none
#pragma unroll
      for (int kk = 0; kk < 8; ++kk)
        q[kk] = __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, q[kk]) ^ 0x80008000u);
  }
  const float c = fabsf(a.scale_log2);
  // ---- loads: a wave the keys or the values of one page of the block (of four waves both), 1 KB
  // an instruction, each lane the unit that belongs to its place in LDS
  constexpr int kLoads = kFp8 ? 2 : 4;          // of a page's keys or values
  constexpr int kBoth = kW == 8 ? 1 : 2;
  const int my_page = kW == 8 ? wave >> 1 : wave, my_kind = kW == 8 ? wave & 1 : 0;
  // the unit in the i-th KB at this lane's place: of values the same in each, of keys xor 4 i
  const uint32_t k_unit = lane ^ (lane >> 4), v_unit = kFp8 ? lane : lane ^ (lane >> 4 & 1);
  const uint32_t ring = lds_address(lds.in[0][0]);
  constexpr uint32_t kPageBytes = 2 * kPageElems, kBlockBytes = 2 * kWidePages * kPageBytes;
  auto page_id = [&](int blk) {
    return page_at(bt, min(t0 / kPage + blk * kWidePages + my_page, row_pages - 1), a.num_pages);
  };
  int next_id = page_id(0);
  auto load = [&](int blk) __attribute__((always_inline)) {
    const size_t at = ((size_t)next_id * a.hkv + g) * kPageElems;
#pragma unroll
    for (int j = 0; j < kBoth; ++j) {
      const int is_v = kBoth == 2 ? j : my_kind;
      const uint32_t unit = is_v ? v_unit : k_unit, turn = is_v ? 0 : 64;
      const uint16_t *base = (is_v ? a.v_pool : a.k_pool) + (kFp8 ? at / 2 : at);
      const uint32_t to = __builtin_amdgcn_readfirstlane(
          ring + blk % kRing * kBlockBytes + (is_v * kWidePages + my_page) * kPageBytes);
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        load_to_lds(base, (16 * unit ^ turn * i) + 1024 * i, to + i * 1024);
    }
  };
#pragma unroll
  for (int i = 0; i < kRing - 1; ++i)
    if (i < nblocks) {
      load(i);
      next_id = page_id(i + 1);
    }

  uint32_t odd = 0;                             // infinite or NaN values of nodes

  f32x16 o[4];
#pragma unroll
  for (int mt = 0; mt < 4; ++mt)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[mt][i] = 0.f;
  float m_run = -INFINITY, l_run = 0.f;
  // row i of a tile of scores is key i with bits 2 and 3 exchanged
  const int key = (col & ~12) | ((col & 4) << 1) | ((col & 8) >> 1);

  constexpr int kKReads = kFp8 ? 4 : 8;
  const int slot = key & 15;
  const uint32_t k_at = (key >> 4) * kPageBytes + 16 * (kFp8 ? slot * 8 + (grp ^ (slot >> 1)) : slot * 16 + (grp ^ slot));
  const uint32_t v_at = kWidePages * kPageBytes + 16 * (kFp8 ? 32 * grp + col : 2 * col + (grp ^ (col >> 3 & 1)));
  struct Keys {
    u32x4 raw[kKReads];
  };
  auto read_k = [&](int blk, int pp, Keys &k) __attribute__((always_inline)) {
    const uint32_t at = ring + blk % kRing * kBlockBytes + 2 * pp * kPageBytes + k_at;
#pragma unroll
    for (int i = 0; i < kKReads; ++i) k.raw[i] = read_lds(at ^ (32 * i));   // unit 2 i + grp
  };
  // Reads are issued a phase ahead: the values before the scores' products, the next pair's keys
  // behind them.
  auto pair = [&](int blk, int pp, bool more, Keys &keys) __attribute__((always_inline)) {
    const int tok = t0 + blk * kWideKeys + pp * kPair;
    const bool tail = tok + kPair > row.ctx;
    u32x4 vraw[kFp8 ? 4 : 8];
    const uint32_t from = ring + blk % kRing * kBlockBytes + 2 * pp * kPageBytes + v_at;
#pragma unroll
    for (int h = 0; h < 2; ++h)
      if constexpr (kFp8) {
        // lane groups 0 and 1 read rows 32 apart, whole; see below
#pragma unroll
        for (int j = 0; j < 2; ++j) vraw[2 * h + j] = read_lds(from + h * kPageBytes + j * 1024);
      } else {
#pragma unroll
        for (int mt = 0; mt < 4; ++mt) vraw[4 * h + mt] = read_lds(from + h * kPageBytes + mt * 1024);
      }
    keep_order();
    f32x16 s;
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] = 0.f;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      bf16x8 k;
      if constexpr (kFp8)
        k = fp8x8_to_bf16x8(u32x2{keys.raw[kk >> 1][2 * (kk & 1)], keys.raw[kk >> 1][2 * (kk & 1) + 1]});
      else
        k = __builtin_bit_cast(bf16x8, keys.raw[kk]);
      s = mfma32x32x16(k, q[kk], s);
    }
    keep_order();
    if (more) read_k(blk, pp + 1, keys);       // (shares is 1)
    keep_order();
#pragma unroll
    for (int i = 0; i < 16; ++i) s[i] *= c;
    if (tail) {
      const uint32_t sees = seen_keys(mask, tok, row.ctx, row.T) >> (8 * grp);
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i] = sees >> (16 * (i >> 3) + (i & 7)) & 1 ? s[i] : -INFINITY;
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
      for (int e = 0; e < 8; ++e) p[e] = fast_exp2(s[8 * h + e] - m_use);
      l_run += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
      hi[h] = to_bf16x8(p);
      lo[h] = to_bf16x8(p - to_f32x8(hi[h]));
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      bf16x8 v[4];
      if constexpr (kFp8) {
        // lanes l and l ^ 32 hold rows d and d + 32, all slots: exchanged, each has the slots
        // that it supplies of both
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const u32x4 w = vraw[2 * h + j];
          const auto s0 = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
          const auto s1 = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
          v[2 * j] = fp8x8_to_bf16x8(u32x2{s0[0], s1[0]});
          v[2 * j + 1] = fp8x8_to_bf16x8(u32x2{s0[1], s1[1]});
        }
      } else {
#pragma unroll
        for (int mt = 0; mt < 4; ++mt) v[mt] = __builtin_bit_cast(bf16x8, vraw[4 * h + mt]);
      }
      if (tail) {
        // values past the row's end, and those of nodes that are not finite, become zeros
        const int first = tok + 16 * h + 8 * grp, alive = end - first, context = row.ctx - first;
#pragma unroll
        for (int mt = 0; mt < 4; ++mt) {
          u32x4 w = __builtin_bit_cast(u32x4, v[mt]);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            w[e] &= low_keys(alive - 2 * e);
            const uint32_t bad = not_finite(w[e]) & ~low_keys(context - 2 * e);
            odd |= bad;
            w[e] &= ~bad;
          }
          v[mt] = __builtin_bit_cast(bf16x8, w);
        }
      }
#pragma unroll
      for (int mt = 0; mt < 4; ++mt) o[mt] = mfma32x32x16(v[mt], hi[h], o[mt]);
#pragma unroll
      for (int mt = 0; mt < 4; ++mt) o[mt] = mfma32x32x16(v[mt], lo[h], o[mt]);
    }
  };

  // Both pairs of a block of context by one wave: their scores' products side by side, one check of
  // the maximum, and the second pair's weights worked out while the first pair's meet its values.
  auto block = [&](int blk) __attribute__((always_inline)) {
    const uint32_t at = ring + blk % kRing * kBlockBytes;
    f32x16 s[2];
#pragma unroll
    for (int i = 0; i < 16; ++i) s[0][i] = s[1][i] = 0.f;
    auto operand = [&](u32x4 w, int kk) __attribute__((always_inline)) {
      if constexpr (kFp8) return fp8x8_to_bf16x8(u32x2{w[2 * (kk & 1)], w[2 * (kk & 1) + 1]});
      else return __builtin_bit_cast(bf16x8, w);
    };
    constexpr int kStep = kFp8 ? 2 : 4;         // reads of each pair at a time: half of a key
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      u32x4 k[2][kStep];
#pragma unroll
      for (int i = 0; i < kStep; ++i)
#pragma unroll
        for (int p = 0; p < 2; ++p)
          k[p][i] = read_lds((at + 2 * p * kPageBytes + k_at) ^ (32 * (h * kStep + i)));
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int p = 0; p < 2; ++p)
          s[p] = mfma32x32x16(operand(k[p][kFp8 ? i >> 1 : i], i), q[4 * h + i], s[p]);
    }
    u32x4 vraw[kFp8 ? 4 : 8];
    auto read_v = [&](int p) __attribute__((always_inline)) {
      const uint32_t from = at + 2 * p * kPageBytes + v_at;
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < (kFp8 ? 2 : 4); ++i)
          vraw[(kFp8 ? 2 : 4) * h + i] = read_lds(from + h * kPageBytes + i * 1024);
    };
    read_v(0);
    keep_order();
    float mx = s[0][0];
#pragma unroll
    for (int i = 1; i < 16; ++i) mx = fmaxf(mx, s[0][i]);
#pragma unroll
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, s[1][i]);
    mx = pair_max(mx) * c;
    const bool grows = mx > m_run + kSlack;
    if (__any(grows)) {
      const float alpha = grows ? fast_exp2(m_run - mx) : 1.f;
      m_run = grows ? mx : m_run;
      l_run *= alpha;
#pragma unroll
      for (int mt = 0; mt < 4; ++mt) o[mt] *= alpha;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
    bf16x8 hi[2][2], lo[2][2];
    auto weights = [&](int p) __attribute__((always_inline)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        f32x8 w;
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = fast_exp2(__builtin_fmaf(s[p][8 * h + e], c, -m_use));
        l_run += ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7]));
        hi[p][h] = to_bf16x8(w);
        lo[p][h] = to_bf16x8(w - to_f32x8(hi[p][h]));
      }
    };
    auto values = [&](int p) __attribute__((always_inline)) {
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        bf16x8 v[4];
        if constexpr (kFp8) {
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const u32x4 w = vraw[2 * h + j];
            const auto s0 = __builtin_amdgcn_permlane32_swap(w[0], w[2], false, false);
            const auto s1 = __builtin_amdgcn_permlane32_swap(w[1], w[3], false, false);
            v[2 * j] = fp8x8_to_bf16x8(u32x2{s0[0], s1[0]});
            v[2 * j + 1] = fp8x8_to_bf16x8(u32x2{s0[1], s1[1]});
          }
        } else {
#pragma unroll
          for (int mt = 0; mt < 4; ++mt) v[mt] = __builtin_bit_cast(bf16x8, vraw[4 * h + mt]);
        }
#pragma unroll
        for (int mt = 0; mt < 4; ++mt) o[mt] = mfma32x32x16(v[mt], hi[p][h], o[mt]);
#pragma unroll
        for (int mt = 0; mt < 4; ++mt) o[mt] = mfma32x32x16(v[mt], lo[p][h], o[mt]);
      }
    };
    weights(0);
    keep_order();
    values(0);
    weights(1);
    // a product, then some of the vector instructions beside it
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, kBeside, 0);
    }
    keep_order();
    read_v(1);
    values(1);
  };

  // this block's loads are done (of those behind them kLoads a block may be on their way), all
  // waves', and the block before is consumed
  auto arrive = [&](int blk) __attribute__((always_inline)) {
    const int behind = min(kRing - 2, nblocks - 1 - blk);
    if (behind >= 2)
      await_loads_before<2 * kLoads>();
    else if (behind == 1)
      await_loads_before<kLoads>();
    else
      await_loads();
    __syncthreads();
    if (blk + kRing - 1 < nblocks) load(blk + kRing - 1);
    next_id = page_id(blk + kRing);
  };
  int blk = 0;
  if (shares == 1) {
    const int full = min(nblocks, max(0, row.ctx - t0) / kWideKeys);
    for (; blk < full; ++blk) {
      arrive(blk);
      block(blk);
    }
  }
  int mine = shares == 1 ? kWidePairs * blk : share;
  for (; blk < nblocks; ++blk) {
    arrive(blk);
    const int pairs = min(kWidePairs, (t1 - t0 - blk * kWideKeys + kPair - 1) / kPair);
    // the wave's next pair of all, `shares` behind its last one
    int pp = mine - kWidePairs * blk;
    if (pp < pairs) {
      Keys keys;
      read_k(blk, pp, keys);
      for (; pp < pairs; pp += shares, mine += shares) pair(blk, pp, pp + shares < pairs, keys);
    }
  }
  __syncthreads();

  // whole rows through LDS, joining the waves that shared them
  {
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
  auto first_wave = [&](int p) { return p >= extra ? p - extra : heavy + p; };
  if (__syncthreads_or(odd != 0)) {
    reach_odd<kFp8, kThreads>(a, row, bt, g, t0, t1, r0, rows,
                                  [&](int c) { return &lds.o[first_wave(c >> 5)][c & 31][0]; });
    __syncthreads();
  }
  for (int idx = tid; idx < rows * (kHeadDim / 4); idx += kThreads) {
    const int c = idx / (kHeadDim / 4), d = idx % (kHeadDim / 4) * 4;
    const bool of_first = c >> 5 >= extra;     // the part's waves
    const int w0 = first_wave(c >> 5), step = of_first ? few : extra;
    const int n_waves = of_first ? base : base + 1;
    float M = -INFINITY, lsum = 0.f;
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int w = 0; w < n_waves; ++w) M = fmaxf(M, lds.m[w0 + w * step][c & 31]);
    const float M_use = M == -INFINITY ? 0.f : M;
    for (int w = 0; w < n_waves; ++w) {
      const int from = w0 + w * step;
      const float f = fast_exp2(lds.m[from][c & 31] - M_use);
      acc += f * *reinterpret_cast<const f32x4 *>(&lds.o[from][c & 31][d]);
      lsum += f * lds.l[from][c & 31];
    }
    if (place < 0) {
      const int rr = r0 + c, n = rr / G;
      const size_t head = (size_t)(row.first + n) * a.hq + (size_t)g * G + (rr - n * G);
      const float inv = a.v_scale / lsum;
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[e] = lsum == 0.f ? 0.f : acc[e] * inv;
      *reinterpret_cast<f32x4 *>(a.out + head * kHeadDim + d) = acc;
      if (a.lse && d == 0) a.lse[head] = (M + __log2f(lsum)) * kLn2;
    } else {
      const size_t at = (size_t)place * a.piece_rows + c;
      *reinterpret_cast<f32x4 *>(a.ws_o + at * kHeadDim + d) = acc;
      if (d == 0) a.ws_ml[at] = float2{M, lsum};
    }
  }
  __syncthreads();                              // the next piece's loads go there
}

template <int kW, bool kFp8>
__global__ __launch_bounds__(kW * kWave, 2) void tree_wide_kernel(TreeArgs a) {
  __shared__ __attribute__((aligned(1024))) WideLds<kW> lds;
  walk<32 * kW>(a, lds.walk,
                [&](int b, const TreeRow &row, int tile, int g, int blk0, int blk1, int place)
                    __attribute__((always_inline)) {
                      wide_piece<kW, kFp8>(a, lds, b, row, tile, g, blk0, blk1, place);
                    });
}

constexpr int kJoinWaves = 4;
// Joins the pieces of one node and head, a wave each: the weights of up to 64 pieces are worked
// out one a lane, the partial results taken four dims a lane by half a wave a piece, four pieces
// of each half in flight. For calls of few nodes, whose rows are in many pieces.
template <int kRows>
__global__ __launch_bounds__(kJoinWaves * kWave) void tree_join_head_kernel(TreeArgs a) {
  const int lane = threadIdx.x & (kWave - 1), half = lane >> 5;
  const int64_t at = (int64_t)blockIdx.x * kJoinWaves + threadIdx.x / kWave;
  const int t = (int)(at / a.hq), h = (int)(at - (int64_t)t * a.hq);
  if (t >= a.total_q) return;
  const int b = wave_search(a.B, t, [&](int i) { return a.cu_q[i]; });
  const TreeRow row = tree_row(a, b);
  if (t < row.first || t >= row.first + row.T) return;
  const RowLine<kRows> line(row, a.group);
  const int g = h / a.group, r = (t - row.first) * a.group + h - g * a.group, tile = r / kRows;
  const int64_t share = *a.share, begin = a.start[b] + line.before(tile, g, a.hkv);
  const int64_t first = quotient(begin, share);
  const int n = (int)(quotient(begin + (int64_t)(line.blocks - 1) * line.cost(tile), share) - first) + 1;
  if (n == 1) return;
  // piece i's result, query row r of its tile: the first piece is the last of its share
  auto piece = [&](int i) { return (size_t)(2 * (first + i) + (i == 0)) * a.piece_rows + (r - tile * kRows); };
  float M = -INFINITY;
  for (int s = lane; s < n; s += kWave) M = fmaxf(M, a.ws_ml[piece(s)].x);
#pragma unroll
  for (int off = 1; off < kWave; off *= 2) M = fmaxf(M, __shfl_xor(M, off));
  const float M_use = M == -INFINITY ? 0.f : M;
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float lsum = 0.f;
  for (int s0 = 0; s0 < n; s0 += kWave) {
    const int m = min(n - s0, kWave);
    float f = 0.f;
    if (lane < m) {
      const float2 ml = a.ws_ml[piece(s0 + lane)];
      f = fast_exp2(ml.x - M_use);
      lsum += f * ml.y;
    }
    for (int s = 0; s < m; s += 8) {
      f32x4 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int k = min(s + 2 * i + half, m - 1);
        v[i] = *reinterpret_cast<const f32x4 *>(a.ws_o + piece(s0 + k) * kHeadDim + 4 * (lane & 31));
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int k = s + 2 * i + half;
        const float fk = __shfl(f, min(k, m - 1));
        if (k < m) acc += fk * v[i];
      }
    }
  }
#pragma unroll
  for (int off = 1; off < kWave; off *= 2) lsum += __shfl_xor(lsum, off);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    acc[e] += __shfl_xor(acc[e], 32);
    acc[e] = lsum == 0.f ? 0.f : acc[e] * (a.v_scale / lsum);
  }
  if (half == 0) *reinterpret_cast<f32x4 *>(a.out + at * kHeadDim + 4 * lane) = acc;
  if (a.lse && lane == 0) a.lse[at] = (M + __log2f(lsum)) * kLn2;
}

// Joins the pieces of one node's heads on one KV head, a wave each: four heads at a time and, of
// each, up to 16 pieces, whose weights are worked out one a lane; the partial results are taken
// four dims a lane by half a wave a head. Nodes of uncut tiles are final already. Bound by round
// trips (the node's row, its place on the line, the weights, the results) and by the partial
// results' bytes.
constexpr int kJoinHeads = 4, kJoinPieces = 16;
template <int kRows>
__global__ __launch_bounds__(kJoinWaves * kWave) void tree_join_kernel(TreeArgs a) {
  const int lane = threadIdx.x & (kWave - 1), half = lane >> 5;
  const int64_t at = (int64_t)blockIdx.x * kJoinWaves + threadIdx.x / kWave;
  const int t = (int)(at / a.hkv), g = (int)(at - (int64_t)t * a.hkv);
  if (t >= a.total_q) return;
  const int b = uniform(wave_search(a.B, t, [&](int i) { return a.cu_q[i]; }));
  const TreeRow row = uniform_row(a, b);
  if (t < row.first || t >= row.first + row.T) return;
  const RowLine<kRows> line(row, a.group);
  const int64_t share = uniform(*a.share), start = uniform(a.start[b]);
  for (int h0 = 0; h0 < a.group; h0 += kJoinHeads) {
    // the heads' query rows lie in one tile or two
    const int r = (t - row.first) * a.group + h0 + lane / kJoinPieces;   // this lane's of the weights
    const int last = min(h0 + kJoinHeads, a.group) - 1 - h0;
    const int tile0 = ((t - row.first) * a.group + h0) / kRows;
    const int tile1 = ((t - row.first) * a.group + h0 + last) / kRows;
    for (int tile = tile0; tile <= tile1; ++tile) {
      const int64_t begin = start + line.before(tile, g, a.hkv);
      const int first = (int)quotient(begin, share);
      const int n =
          (int)quotient(begin + (int64_t)(line.blocks - 1) * line.cost(tile), share) - first + 1;
      if (n == 1) continue;
      // piece i's result of query row r: the first piece is the last of its share
      auto piece = [&](int i, int r) {
        return (size_t)(2 * (first + i) + (i == 0)) * a.piece_rows + (r - tile * kRows);
      };
      const bool mine = lane / kJoinPieces <= last && r / kRows == tile;
      float M = -INFINITY;
      for (int s = lane % kJoinPieces; s < n; s += kJoinPieces)
        if (mine) M = fmaxf(M, a.ws_ml[piece(s, r)].x);
#pragma unroll
      for (int off = 1; off < kJoinPieces; off *= 2) M = fmaxf(M, __shfl_xor(M, off));
      const float M_use = M == -INFINITY ? 0.f : M;
      f32x4 acc[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};       // heads half, half + 2
      float lsum = 0.f;
      for (int s0 = 0; s0 < n; s0 += kJoinPieces) {
        const int m = min(n - s0, kJoinPieces), s = lane % kJoinPieces;
        float f = 0.f;
        if (mine && s < m) {
          const float2 ml = a.ws_ml[piece(s0 + s, r)];
          f = fast_exp2(ml.x - M_use);
          lsum += f * ml.y;
        }
        for (int i0 = 0; i0 < m; i0 += 4) {
          f32x4 v[2][4];
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const int h = min(2 * j + half, last), rr = (t - row.first) * a.group + h0 + h;
            const int safe = min(max(rr, tile * kRows), tile * kRows + kRows - 1);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              v[j][i] = *reinterpret_cast<const f32x4 *>(
                  a.ws_o + piece(s0 + min(i0 + i, m - 1), safe) * kHeadDim + 4 * (lane & 31));
          }
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float w = __shfl(f, (2 * j + half) * kJoinPieces + min(i0 + i, m - 1));
              if (i0 + i < m) acc[j] += w * v[j][i];
            }
        }
      }
#pragma unroll
      for (int off = 1; off < kJoinPieces; off *= 2) lsum += __shfl_xor(lsum, off);
      const size_t head = (size_t)t * a.hq + (size_t)g * a.group + h0;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int h = 2 * j + half;
        const float l = __shfl(lsum, h * kJoinPieces);
        const bool here = h <= last && ((t - row.first) * a.group + h0 + h) / kRows == tile;
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][e] = l == 0.f ? 0.f : acc[j][e] * (a.v_scale / l);
        if (here) *reinterpret_cast<f32x4 *>(a.out + (head + h) * kHeadDim + 4 * (lane & 31)) = acc[j];
      }
      if (a.lse && mine && lane % kJoinPieces == 0)
        a.lse[head + lane / kJoinPieces] = (M + __log2f(lsum)) * kLn2;
    }
  }
}

// Workgroups of a call that is cut: as many as are on the GPU together, or a block each. Half of
// them: 64 rows of 4k to 32k keys (4.6 GB), 8 nodes 732 us for 732, fp8 498 for 425, 16 nodes over
// fp8 713 for 620, but 4 rows of 8,000 39 for 42; twice as many: 747, 32 rows of 16 to 64 nodes over
// 2k to 24k 551 for 535.
int64_t line_groups(int32_t tile_rows, int64_t units, int32_t max_kv_len) {
  const int keys = tile_rows <= 32 ? block_keys<32>() : block_keys<128>();
  return std::min(units * ((max_kv_len + keys - 1) / keys), (int64_t)(tile_rows == 256 ? 256 : 512));
}

// The query rows of a call's tiles.
int32_t tile_rows(int64_t rows) { return rows <= 16 ? 16 : rows <= 32 ? 32 : rows <= 128 ? 128 : 256; }

}  // namespace

// Rows of up to kDirectKeys keys are not cut, nor are those of up to kDirectUnitKeys for each
// tile and KV head of the call, as far as kDirectMost. Uncut and cut (us, 32 heads on 8, rows
// from an eighth of the longest on): 1 row of 500, 8 nodes 14.7 and 17.0; 64 rows of up to 400,
// 8 nodes 24.6 and 48.8, 32 nodes 40 and 83; 8 rows of 900 21.0 and 20.4; 16 rows of up to
// 1,900 28.4 and 32.7 (32 nodes 55.7 and 53.6); 16 of 3,900 46 and 41 (97 and 70); 64 of
// 1,900 61 and 95 (102 and 147); 64 of 3,900 122 and 137 (181 and 194); 64 of 8,000 231 and 228
// (337 and 319); 256 of 3,900 443 and 484 (622 and 683).
constexpr int kDirectKeys = 512, kDirectUnitKeys = 16, kDirectMost = 4096;
// The least that a workgroup takes of a tile. Twice as much and half: 4 rows of 1,000 keys, 64
// nodes 51.5, 40.0 and 40.0 us; 1 of 2,000, 32 nodes 25.2, 23.8 and 25.0; 2 of 2,000, 16 nodes
// 20.7, 20.9 and 24.3.
constexpr int kMinShareKeys = 128;
// (node, head) pairs up to which each has a wave in the join. Call times, a wave a pair and a wave
// a node and KV head: 4 nodes over 16,000 keys, 32 heads on 8: 25.9 and 35.6 us; 32 nodes 46.4 and
// 56.3; 64 nodes over 8,000 51.6 and 54.8; 64 rows of 16 nodes (32,768 pairs) 922 and 915; 32 rows
// of 64 nodes (65,536) 660 and 643.
constexpr int64_t kFewHeads = 4096;

TreePlan tree_plan(int32_t B, int32_t hq, int32_t hkv, int32_t max_q_len, int32_t max_kv_len) {
  const int64_t rows = (int64_t)max_q_len * (hq / hkv);
  TreePlan p;
  p.rows = tile_rows(rows);
  p.tiles = (rows + p.rows - 1) / p.rows;
  p.piece_rows = (int32_t)(rows < p.rows ? rows : p.rows);
  const int64_t units = (int64_t)B * hkv * p.tiles;
  p.direct = max_kv_len <= kDirectKeys ||
             (max_kv_len <= kDirectMost && max_kv_len <= units * kDirectUnitKeys);
  p.groups = p.direct ? units : line_groups(p.rows, units, max_kv_len);
  return p;
}

static bool join_by_head(int32_t total_q, int32_t hq) { return (int64_t)total_q * hq <= kFewHeads; }

int64_t tree_threads(const TreePlan &p, int32_t total_q, int32_t hq, int32_t hkv) {
  const int64_t tiles = p.groups * (p.rows == 256 ? 8 : kSplitWaves) * kWave;
  if (p.direct) return tiles;
  const int64_t joins = (int64_t)total_q * (join_by_head(total_q, hq) ? hq : hkv);
  const int64_t join = (joins + kJoinWaves - 1) / kJoinWaves * (kJoinWaves * kWave);
  return tiles > join ? tiles : join;
}

namespace {
size_t up256(size_t n) { return (n + 255) / 256 * 256; }
}  // namespace

size_t tree_workspace_bytes(int32_t B, const TreePlan &p) {
  if (p.direct) return 0;
  return up256(((size_t)B + 1) * sizeof(int64_t)) +
         (size_t)2 * p.groups * p.piece_rows * (kHeadDim + 2) * sizeof(float);
}

// More keys are cut sooner and into no fewer pieces, so the most keys need most; of each size of
// tile, the largest tree that has it, and as many tiles and KV heads as are still cut.
size_t tree_most_workspace_bytes(int32_t B, int32_t hq, int32_t hkv, int32_t max_q_len,
                                 int32_t max_kv_len) {
  const int64_t cut = max_kv_len <= kDirectMost ? (max_kv_len - 1) / kDirectUnitKeys : INT64_MAX;
  if (max_kv_len <= kDirectKeys || cut < hkv) return 0;
  const int64_t group = hq / hkv;
  size_t most = 0;
  for (const int32_t rows : {16, 32, 128, 256}) {
    const int64_t nodes = rows == 256 ? max_q_len : std::min<int64_t>(max_q_len, rows / group);
    if (nodes == 0 || tile_rows(nodes * group) != rows) continue;
    const int64_t tiles = (nodes * group + rows - 1) / rows;
    const int64_t units = std::min((int64_t)B * hkv * tiles, cut / hkv * hkv);
    const TreePlan p = {rows, (int32_t)std::min<int64_t>(nodes * group, rows), false, tiles,
                        line_groups(rows, units, max_kv_len)};
    most = std::max(most, tree_workspace_bytes(B, p));
  }
  return most;
}

hipError_t launch_tree(const uint16_t *q, const int32_t *cu_q, const int32_t *ctx_lens,
                       const uint64_t *mask, int32_t words, const PagedKV &kv, int32_t B,
                       int32_t hq, int32_t total_q, int32_t max_q_len, int32_t max_kv_len,
                       float scale, float *out, float *lse, void *workspace, const TreePlan &p,
                       hipStream_t stream) {
  TreeArgs a;
  a.q = q;
  a.cu_q = cu_q;
  a.ctx_lens = ctx_lens;
  a.mask = mask;
  a.k_pool = kv.k_pool;
  a.v_pool = kv.v_pool;
  a.block_table = kv.block_table;
  a.out = out;
  a.lse = lse;
  a.share = nullptr;
  a.start = nullptr;
  a.ws_o = nullptr;
  a.ws_ml = nullptr;
  if (!p.direct) {
    a.share = static_cast<int64_t *>(workspace);
    a.start = a.share + 1;
    a.ws_o = reinterpret_cast<float *>(static_cast<char *>(workspace) +
                                       up256(((size_t)B + 1) * sizeof(int64_t)));
    a.ws_ml = reinterpret_cast<float2 *>(a.ws_o + (size_t)2 * p.groups * p.piece_rows * kHeadDim);
  }
  a.min_share = p.rows == 256   ? kMinShareKeys / kWideKeys * 16
                : p.rows == 128 ? kMinShareKeys / kWideKeys
                                : kMinShareKeys / block_keys<16>();
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
  a.piece_rows = p.piece_rows;
  a.tiles = (int32_t)p.tiles;
  a.direct = p.direct;
  a.scale_log2 = scale * kLog2e * kv.k_scale;
  a.v_scale = kv.v_scale;
  const dim3 grid((unsigned)p.groups);
  const bool by_head = join_by_head(total_q, hq);
  const int64_t joins = (int64_t)total_q * (by_head ? hq : kv.hkv);
  const dim3 join_grid((unsigned)((joins + kJoinWaves - 1) / kJoinWaves)), join(kJoinWaves * kWave);
  auto launch = [&](auto rows) {
    constexpr int kRows = decltype(rows)::value;
    if constexpr (kRows > 32) {
      constexpr int kW = kRows / 32;
      if (kv.fp8)
        tree_wide_kernel<kW, true><<<grid, kW * kWave, 0, stream>>>(a);
      else
        tree_wide_kernel<kW, false><<<grid, kW * kWave, 0, stream>>>(a);
    } else {
      if (kv.fp8)
        tree_narrow_kernel<kRows / 16, true><<<grid, kSplitWaves * kWave, 0, stream>>>(a);
      else
        tree_narrow_kernel<kRows / 16, false><<<grid, kSplitWaves * kWave, 0, stream>>>(a);
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.direct) return e;
    if (by_head)
      tree_join_head_kernel<kRows><<<join_grid, join, 0, stream>>>(a);
    else
      tree_join_kernel<kRows><<<join_grid, join, 0, stream>>>(a);
    return hipGetLastError();
  };
  switch (p.rows) {
    case 16: return launch(std::integral_constant<int, 16>{});
    case 32: return launch(std::integral_constant<int, 32>{});
    case 128: return launch(std::integral_constant<int, 128>{});
    default: return launch(std::integral_constant<int, 256>{});
  }
}

}  // namespace ra
