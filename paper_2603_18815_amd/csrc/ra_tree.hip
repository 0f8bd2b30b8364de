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

template <int kTiles>
struct TreeLds {
  float m[kSplitWaves][16 * kTiles];
  float l[kSplitWaves][16 * kTiles];
  float o[kSplitWaves][16 * kTiles][kOPitch];
};

template <int kTiles, bool kFp8>
__global__ __launch_bounds__(kSplitWaves * kWave) void tree_split_kernel(TreeArgs a) {
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
    bool odd = false;                       // an infinite or NaN value among these
    bf16x8 vodd[8];
    if (tail) {
      const int alive = t1 - first;         // of the lane's eight keys
      uint32_t any = 0;
#pragma unroll
      for (int mt = 0; mt < 8; ++mt) {
        u32x4 w = __builtin_bit_cast(u32x4, va[mt]), m;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          w[e] &= (2 * e < alive ? 0xffffu : 0u) | (2 * e + 1 < alive ? 0xffff0000u : 0u);
          m[e] = not_finite(w[e]);
          any |= m[e];
          w[e] &= ~m[e];
        }
        va[mt] = __builtin_bit_cast(bf16x8, w);
        vodd[mt] = __builtin_bit_cast(bf16x8, m & 0x3f803f80u);
      }
      // a value that some nodes do not see must not meet their zero weights: the products run
      // without it, and a second one says which results it reaches
      odd = __any(any != 0);
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
      bool sees[8];
      if (tail) {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int j = first + e - row.ctx;
          sees[e] = j < 0 || (first + e < t1 && (mask[nt][j >> 6] >> (j & 63) & 1));
          sc[e] = sees[e] ? sc[e] : -INFINITY;
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
      if (tail && odd) {
        u32x4 m;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          m[e] = (sees[2 * e] ? 0x3f80u : 0u) | (sees[2 * e + 1] ? 0x3f800000u : 0u);
        const bf16x8 met = __builtin_bit_cast(bf16x8, m);
#pragma unroll
        for (int mt = 0; mt < 8; ++mt) {
          const f32x4 reached = mfma16x16x32(vodd[mt], met, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
          for (int r = 0; r < 4; ++r) o[nt][mt][r] = reached[r] > 0.f ? NAN : o[nt][mt][r];
        }
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
  __syncthreads();
  const int ncols = min(rows - r0, 16 * kTiles);
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
  p.wide = rows > 16;
  const int64_t per = p.wide ? 32 : 16;
  p.tiles = (rows + per - 1) / per;
  int64_t split = 512;
  while (split < 4096 && (int64_t)B * hkv * max_kv_len / split > 8192) split *= 2;
  if (max_kv_len <= 512) split = 512;
  p.split_tokens = (int32_t)split;
  p.slots = (int32_t)((max_kv_len + split - 1) / split);
  if (p.slots < 1) p.slots = 1;
  p.groups = p.tiles * p.slots * B * hkv;
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
  if (p.wide && kv.fp8)
    tree_split_kernel<2, true><<<grid, block, 0, stream>>>(a);
  else if (p.wide)
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
