// Block tables from lengths: kv_block_table_extend reserves the pages of a step's new
// tokens off a free list, kv_block_table_release gives pages back.
//
// With held_b = ceil(start_b / 16) pages in hand and need_b = ceil((start_b + n_b) / 16) -
// held_b more to take, row b's j-th new page is the free list's entry count - 1 - (P_b + j),
// P the exclusive sums of need. A page that is taken begins with a new token (its first
// position 16 j is not below start_b), so one pass over the new tokens writes the table
// (the tokens at slot 0) and the slot map.
//
// Bound by latency: some bytes a row, 8 a token. Every workgroup reads all rows, twice where
// they are more than its threads (the totals decide whether the call is refused, the running
// sums place its share of the tokens), which takes the place of a second launch and a
// workspace: 5.0 us for 64 rows of one token, 10.8 for 512 rows and 4.7 MB of slots, releases
// 5.5 and 6.6. Only the free list's length cannot change while other workgroups read it: one
// workgroup sets it itself, several leave it to a launch of one thread behind them.
#include "ra_device.h"
#include "ra_internal.h"
#include "ra_wave.h"

namespace ra {
namespace {

constexpr int kThreads = 1024;          // rows a scan step takes, and token slots of a pass
constexpr int kWaves = kThreads / kWave;
constexpr int kTokensPerGroup = 4096;   // more tokens than this are shared by workgroups

// Inclusive sums of two counts over the workgroup's threads; all threads get the totals.
__device__ __forceinline__ void group_scan(int64_t &a, int64_t &b, int64_t &total_a,
                                           int64_t &total_b, int64_t (*part)[2]) {
  const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
  a = wave_sums(a);
  b = wave_sums(b);
  __syncthreads();                      // part may still be read by the scan before
  if (lane == kWave - 1) part[wave][0] = a, part[wave][1] = b;
  __syncthreads();
  int64_t before_a = 0, before_b = 0;
  total_a = total_b = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w == wave) before_a = total_a, before_b = total_b;
    total_a += part[w][0];
    total_b += part[w][1];
  }
  a += before_a;
  b += before_b;
}

__device__ __forceinline__ int64_t pages_of(int64_t tokens) { return (tokens + kPage - 1) / kPage; }

// Row `i` of a scan step as the scan left it in LDS: the first i with first[i + 1] > t.
__device__ __forceinline__ int row_of(const int *first, int rows, int t) {
  int lo = 0, hi = rows - 1;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (first[mid + 1] > t) hi = mid; else lo = mid + 1;
  }
  return lo;
}

__global__ __launch_bounds__(kThreads) void extend_kernel(
    const int32_t *start_pos, const int32_t *num_new, const int32_t *free_pages,
    int32_t *free_count, int32_t capacity, int32_t *block_table, int32_t B, int32_t bt_stride,
    int32_t total_new, int32_t *cu_new, int32_t *kv_lens, int64_t *slot_map, int32_t *taken) {
  __shared__ int64_t part[kWaves][2];
  __shared__ int first[kThreads + 1], page0[kThreads], start[kThreads];
  __shared__ int bad;
  const int tid = threadIdx.x;
  if (tid == 0) bad = 0;
  __syncthreads();
  const int64_t limit = (int64_t)bt_stride * kPage;
  int64_t tokens = 0, pages = 0, total_n = 0, total_need = 0, after = 0, page_after = 0;
  for (int base = 0; base < B; base += kThreads) {
    int64_t n = 0, need = 0;
    if (base + tid < B) {
      const int64_t s = start_pos[base + tid];
      n = num_new[base + tid];
      if (s < 0 || n < 0 || s + n > limit) bad = 1;
      need = pages_of(s + n) - pages_of(s);
    }
    group_scan(n, need, total_n, total_need, part);
    tokens += total_n;
    pages += total_need;
    after = n, page_after = need;
  }
  __syncthreads();
  const int32_t count = *free_count;
  const bool ok = !bad && tokens <= total_new && count >= 0 && count <= capacity && pages <= count;

  // this workgroup's share of the tokens, and of the slots behind the last one
  const int64_t share = ((int64_t)total_new + gridDim.x - 1) / gridDim.x;
  const int64_t t0 = blockIdx.x * share;
  const int64_t t1 = t0 + share < total_new ? t0 + share : total_new;
  const int64_t end = ok ? tokens : 0;
  if (slot_map)
    for (int64_t t = (t0 > end ? t0 : end) + tid; t < t1; t += kThreads) slot_map[t] = -1;

  int64_t token_base = 0, page_base = 0;
  for (int base = 0; base < B; base += kThreads) {
    const int b = base + tid, rows = B - base < kThreads ? B - base : kThreads;
    int64_t s = 0, n = 0, need = 0;
    if (b < B) {
      s = start_pos[b];
      if (ok) {
        n = num_new[b];
        need = pages_of(s + n) - pages_of(s);
      }
    }
    if (B > kThreads) {                   // else the sums of the pass before are at hand
      after = n, page_after = need;
      group_scan(after, page_after, total_n, total_need, part);   // also: LDS is free again
    } else if (!ok) {
      after = page_after = total_n = total_need = 0;
    }
    if (b < B) {
      first[tid] = (int)(token_base + after - n);
      page0[tid] = (int)(page_base + page_after - need);
      start[tid] = (int)s;
      if (tid == rows - 1) first[rows] = (int)(token_base + after);
      if (blockIdx.x == 0) {
        cu_new[b] = (int)(token_base + after - n);
        kv_lens[b] = (int)(s + n);
      }
    }
    __syncthreads();
    const int64_t from = t0 > token_base ? t0 : token_base;
    const int64_t to = t1 < token_base + total_n ? t1 : token_base + total_n;
    for (int64_t t = from + tid; t < to; t += kThreads) {
      const int r = row_of(first, rows, (int)t);
      const int pos = start[r] + ((int)t - first[r]);
      const int held = (start[r] + kPage - 1) / kPage, j = pos / kPage;
      int32_t *entry = block_table + (int64_t)(base + r) * bt_stride + j;
      int page;
      if (j >= held) {
        page = free_pages[count - 1 - (page0[r] + j - held)];
        if (pos % kPage == 0) *entry = page;
      } else {
        page = *entry;
      }
      if (slot_map) slot_map[t] = (int64_t)page * kPage + pos % kPage;
    }
    token_base += total_n;
    page_base += total_need;
  }
  if (blockIdx.x == 0 && tid == 0) {
    cu_new[B] = (int)end;
    *taken = ok ? (int)pages : -1;
    if (gridDim.x == 1 && ok) *free_count = count - (int)pages;
  }
}

__global__ __launch_bounds__(kThreads) void release_kernel(
    const int32_t *lens, const int32_t *keep_lens, const int32_t *block_table, int32_t B,
    int32_t bt_stride, int32_t *free_pages, int32_t *free_count, int32_t capacity,
    int32_t *released) {
  __shared__ int64_t part[kWaves][2];
  __shared__ int first[kThreads + 1], page0[kThreads];
  __shared__ int bad;
  const int tid = threadIdx.x;
  if (tid == 0) bad = 0;
  __syncthreads();
  const int64_t limit = (int64_t)bt_stride * kPage;
  int64_t pages = 0;
  for (int base = 0; base < B; base += kThreads) {
    int64_t n = 0, unused = 0;
    if (base + tid < B) {
      const int64_t len = lens[base + tid], keep = keep_lens[base + tid];
      if (keep < 0 || keep > len || len > limit) bad = 1;
      n = pages_of(len) - pages_of(keep);
    }
    int64_t total, total_unused;
    group_scan(n, unused, total, total_unused, part);
    pages += total;
  }
  __syncthreads();
  const int32_t count = *free_count;
  const bool ok = !bad && count >= 0 && count <= capacity && pages <= capacity - count;
  if (ok) {
    const int64_t share = (pages + gridDim.x - 1) / gridDim.x;
    const int64_t p0 = blockIdx.x * share, p1 = p0 + share < pages ? p0 + share : pages;
    int64_t page_base = 0;
    for (int base = 0; base < B; base += kThreads) {
      const int b = base + tid, rows = B - base < kThreads ? B - base : kThreads;
      int64_t kept = 0, n = 0;
      if (b < B) {
        kept = pages_of(keep_lens[b]);
        n = pages_of(lens[b]) - kept;
      }
      int64_t after = n, unused = 0, total, total_unused;
      group_scan(after, unused, total, total_unused, part);
      if (b < B) {
        first[tid] = (int)(page_base + after - n);
        page0[tid] = (int)kept;
        if (tid == rows - 1) first[rows] = (int)(page_base + after);
      }
      __syncthreads();
      const int64_t from = p0 > page_base ? p0 : page_base;
      const int64_t to = p1 < page_base + total ? p1 : page_base + total;
      for (int64_t p = from + tid; p < to; p += kThreads) {
        const int r = row_of(first, rows, (int)p);
        const int j = page0[r] + ((int)p - first[r]);
        free_pages[count + pages - 1 - p] = block_table[(int64_t)(base + r) * bt_stride + j];
      }
      page_base += total;
    }
  }
  if (blockIdx.x == 0 && tid == 0) {
    *released = ok ? (int)pages : -1;
    if (gridDim.x == 1 && ok) *free_count = count + (int)pages;
  }
}

// The free list's new length, behind a launch of several workgroups.
__global__ void count_kernel(int32_t *free_count, const int32_t *moved, int32_t sign) {
  if (*moved > 0) *free_count += sign * *moved;
}

int32_t groups_for(int64_t items) {
  const int64_t g = (items + kTokensPerGroup - 1) / kTokensPerGroup;
  return (int32_t)(g < 1 ? 1 : g > 256 ? 256 : g);
}

}  // namespace

hipError_t launch_table_extend(const int32_t *start_pos, const int32_t *num_new,
                               const int32_t *free_pages, int32_t *free_count, int32_t capacity,
                               int32_t *block_table, int32_t B, int32_t bt_stride,
                               int32_t total_new, int32_t *cu_new, int32_t *kv_lens,
                               int64_t *slot_map, int32_t *taken, hipStream_t stream) {
  const int32_t groups = groups_for(total_new);
  extend_kernel<<<groups, kThreads, 0, stream>>>(start_pos, num_new, free_pages, free_count,
                                                 capacity, block_table, B, bt_stride, total_new,
                                                 cu_new, kv_lens, slot_map, taken);
  if (groups > 1) count_kernel<<<1, 1, 0, stream>>>(free_count, taken, -1);
  return hipGetLastError();
}

hipError_t launch_table_release(const int32_t *lens, const int32_t *keep_lens,
                                const int32_t *block_table, int32_t B, int32_t bt_stride,
                                int32_t *free_pages, int32_t *free_count, int32_t capacity,
                                int32_t max_pages, int32_t *released, hipStream_t stream) {
  const int32_t groups = groups_for(max_pages);
  release_kernel<<<groups, kThreads, 0, stream>>>(lens, keep_lens, block_table, B, bt_stride,
                                                  free_pages, free_count, capacity, released);
  if (groups > 1) count_kernel<<<1, 1, 0, stream>>>(free_count, released, 1);
  return hipGetLastError();
}

}  // namespace ra
