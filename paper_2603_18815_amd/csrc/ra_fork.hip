// Rows that share pages: kv_block_table_fork gives a row the pages of another row's tokens,
// kv_page_copy copies the last, partly filled page that they cannot share, and
// kv_block_table_release_shared gives pages back once no row is left that holds them.
// kv_page_compact moves the kept tokens of a row's end together.
//
// shares[p] counts the rows that hold page p beyond the first. A release takes one off for
// every table entry it covers; a page is free if that leaves less than none. Which entry of
// such a page counts must not depend on the order of atomics: the last one in the order of rows
// and entries does, found by an atomic minimum of codes that fall as the entry's place rises
// and lie below what any count can reach.
#include "ra_device.h"
#include "ra_internal.h"
#include "ra_wave.h"

namespace ra {
namespace {

constexpr int kForkThreads = 256;
constexpr int kMaxRows = 65536;            // rows a block table can have
// Calls that one workgroup does, up to 8 forks and tables of up to 4,096 entries: a launch is 2-3
// us of the GPU's time and 4-5 of the host's. A fork of one row, its copy and its release 29 us
// in place of 39 (in a graph 16 and 21); 7 forks of 7,000 tokens 30 and 43 (20 and 25.5); at
// 8,192 entries the two are even, at 16,384 one workgroup takes 2.5 times as long.
constexpr int kSmallForks = 8, kSmallThreads = 128, kSmallEntries = 4096;
constexpr int kCode = 1 << 30;             // codes of entries: -(kCode + 1 + place), place < kCode

__device__ __forceinline__ bool page_ok(int id, int num_pages) { return (unsigned)id < (unsigned)num_pages; }

// A workgroup a fork, or one for all of a small call (kOne: 128 threads a fork), which then sets
// the list's length itself. Every workgroup looks at all forks: whether the call holds decides
// what each does, and the forks before it say which page is its own. Bound by latency and, for
// long prompts, by the atomics on the shared pages' counts: one fork of 130 tokens 2.6 us, 448 forks of
// 64 prompts of 2k to 8k tokens (147,000 entries) 11.6 us.
template <bool kOne>
__global__ __launch_bounds__(kOne ? kSmallForks * kSmallThreads : kForkThreads) void fork_kernel(
    const int32_t *src_rows, const int32_t *dst_rows, const int32_t *lens, int32_t n,
    int32_t *block_table, int32_t B, int32_t bt_stride, int32_t *shares, int32_t num_pages,
    const int32_t *free_pages, int32_t *free_count, int32_t capacity, int32_t *copy_src,
    int32_t *copy_dst, int32_t *taken) {
  __shared__ uint32_t is_dst[kMaxRows / 32];
  __shared__ int bad, need, before[kOne ? kSmallForks : 1];
  const int tid = threadIdx.x, threads = blockDim.x;
  const int f = kOne ? tid / kSmallThreads : blockIdx.x;                // this thread's fork
  const int t0 = kOne ? tid % kSmallThreads : tid, step = kOne ? kSmallThreads : kForkThreads;
  const int count = *free_count;
  for (int i = tid; i < (B + 31) / 32; i += threads) is_dst[i] = 0;
  if (tid == 0) bad = need = 0;
  if (t0 == 0) before[kOne ? f : 0] = 0;
  __syncthreads();
  const int64_t limit = (int64_t)bt_stride * kPage;
  for (int i = tid; i < n; i += threads) {
    const int s = src_rows[i], d = dst_rows[i], len = lens[i];
    if (s < 0 || s >= B || d < 0 || d >= B || len < 0 || len > limit) {
      bad = 1;
      continue;
    }
    const uint32_t bit = 1u << (d & 31);
    if (atomicOr(&is_dst[d >> 5], bit) & bit) bad = 1;   // two forks into one row
    if (len % kPage) {
      atomicAdd(&need, 1);
      if constexpr (kOne) {
        for (int j = i + 1; j < n; ++j) atomicAdd(&before[j], 1);
      } else {
        if (i < f) atomicAdd(&before[0], 1);
      }
    }
  }
  __syncthreads();
  for (int i = tid; i < n; i += threads) {               // a row forked from is not forked into
    const int s = src_rows[i];
    if (s >= 0 && s < B && (is_dst[s >> 5] >> (s & 31) & 1)) bad = 1;
  }
  __syncthreads();
  const bool ok = !bad && count >= 0 && count <= capacity && need <= count;
  if (f < n) {
    int from = -1, to = -1;
    if (ok) {
      const int64_t src = (int64_t)src_rows[f] * bt_stride, dst = (int64_t)dst_rows[f] * bt_stride;
      const int len = lens[f], full = len / kPage;
      if (t0 == 0 && len % kPage) {
        from = block_table[src + full];
        to = free_pages[count - 1 - before[kOne ? f : 0]];
        block_table[dst + full] = to;
      }
      for (int j = t0; j < full; j += step) {
        const int page = block_table[src + j];
        block_table[dst + j] = page;
        if (page_ok(page, num_pages)) atomicAdd(&shares[page], 1);
      }
    }
    if (t0 == 0) {
      copy_src[f] = from;
      copy_dst[f] = to;
    }
  }
  if (blockIdx.x == 0 && tid == 0) {
    *taken = ok ? need : -1;
    if (gridDim.x == 1 && ok) *free_count = count - need;
  }
}

// The free list's new length, behind a launch of several workgroups.
__global__ void fork_count_kernel(int32_t *free_count, const int32_t *taken) {
  if (*taken > 0) *free_count -= *taken;
}

constexpr int kRowThreads = 256;

// What a release keeps in its workspace: whether it goes ahead, the free list's length before
// it, and the pages that each row frees.
struct SharedRelease {
  const int32_t *lens, *keep_lens, *block_table;
  int32_t B, bt_stride, num_pages, capacity;
  int32_t *shares, *free_pages, *free_count, *released;
  int32_t *head;      // [2]: goes ahead, length
  int32_t *freed;     // [B]
};

__device__ __forceinline__ int64_t pages_of(int64_t tokens) { return (tokens + kPage - 1) / kPage; }

// The release of a large table, each step a launch because atomics of all rows have to be there
// before the next. Of 448 rows' 147,000 entries, in a table of 512: 9.3 + 4.0 + 3.3 + 8.9 us, bound by
// the atomics on shared counts and by round trips.
//
// Takes an owner off every entry that is given up.
__global__ __launch_bounds__(kRowThreads) void shared_sub_kernel(SharedRelease r) {
  __shared__ int bad;
  const int tid = threadIdx.x, b = blockIdx.x;
  if (tid == 0) bad = 0;
  __syncthreads();
  const int64_t limit = (int64_t)r.bt_stride * kPage;
  for (int i = tid; i < r.B; i += kRowThreads) {
    const int64_t len = r.lens[i], keep = r.keep_lens[i];
    if (keep < 0 || keep > len || len > limit) bad = 1;
  }
  __syncthreads();
  const int count = *r.free_count;
  const bool ok = !bad && count >= 0 && count <= r.capacity;
  if (b == 0 && tid == 0) {
    r.head[0] = ok;
    r.head[1] = count;
    if (!ok) *r.released = -1;
  }
  if (!ok) return;
  const int32_t *row = r.block_table + (int64_t)b * r.bt_stride;
  const int end = (int)pages_of(r.lens[b]);
  for (int j = (int)pages_of(r.keep_lens[b]) + tid; j < end; j += kRowThreads) {
    const int page = row[j];
    if (page_ok(page, r.num_pages)) atomicSub(&r.shares[page], 1);
  }
}

// Names the last entry of every page that nobody holds any more.
__global__ __launch_bounds__(kRowThreads) void shared_last_kernel(SharedRelease r) {
  if (!r.head[0]) return;
  const int tid = threadIdx.x, b = blockIdx.x;
  const int32_t *row = r.block_table + (int64_t)b * r.bt_stride;
  const int end = (int)pages_of(r.lens[b]);
  for (int j = (int)pages_of(r.keep_lens[b]) + tid; j < end; j += kRowThreads) {
    const int page = row[j];
    if (page_ok(page, r.num_pages) && r.shares[page] < 0)
      atomicMin(&r.shares[page], -(kCode + 1) - (b * r.bt_stride + j));
  }
}

__device__ __forceinline__ bool frees(const SharedRelease &r, int b, int j, int &page) {
  page = r.block_table[(int64_t)b * r.bt_stride + j];
  return page_ok(page, r.num_pages) && r.shares[page] == -(kCode + 1) - (b * r.bt_stride + j);
}

// How many pages each row frees.
__global__ __launch_bounds__(kRowThreads) void shared_count_kernel(SharedRelease r) {
  __shared__ int sum;
  if (!r.head[0]) return;
  const int tid = threadIdx.x, b = blockIdx.x;
  if (tid == 0) sum = 0;
  __syncthreads();
  const int end = (int)pages_of(r.lens[b]);
  int mine = 0, page;
  for (int j = (int)pages_of(r.keep_lens[b]) + tid; j < end; j += kRowThreads)
    mine += frees(r, b, j, page);
  if (mine) atomicAdd(&sum, mine);
  __syncthreads();
  if (tid == 0) r.freed[b] = sum;
}

// Puts them on the list: entry rank of the freed ones, in the order of rows and entries, goes
// to place count + all - 1 - rank, as kv_block_table_release does with every entry.
__global__ __launch_bounds__(kRowThreads) void shared_put_kernel(SharedRelease r) {
  __shared__ int all, before, wave_sum[kRowThreads / kWave];
  if (!r.head[0]) return;
  const int tid = threadIdx.x, b = blockIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  if (tid == 0) all = before = 0;
  __syncthreads();
  int a = 0, f = 0;
  for (int i = tid; i < r.B; i += kRowThreads) {
    const int n = r.freed[i];
    a += n;
    if (i < b) f += n;
  }
  if (a) atomicAdd(&all, a);
  if (f) atomicAdd(&before, f);
  __syncthreads();
  const int count = r.head[1];
  if (b == 0 && tid == 0) {
    *r.released = all;
    *r.free_count = min(count + all, r.capacity);
  }
  const int first = (int)pages_of(r.keep_lens[b]), end = (int)pages_of(r.lens[b]);
  int rank = before;
  for (int j0 = first; j0 < end; j0 += kRowThreads) {
    const int j = j0 + tid;
    int page = 0;
    const bool mine = j < end && frees(r, b, j, page);
    const uint64_t votes = __ballot(mine);
    if (lane == 0) wave_sum[wave] = (int)__popcll(votes);
    __syncthreads();
    int at = rank + (int)__popcll(votes & ((1ull << lane) - 1));
    int step = 0;
    for (int w = 0; w < kRowThreads / kWave; ++w) {
      if (w < wave) at += wave_sum[w];
      step += wave_sum[w];
    }
    if (mine) {
      const int64_t to = (int64_t)count + all - 1 - at;
      if (to < r.capacity) r.free_pages[to] = page;
      r.shares[page] = 0;   // (no other entry's code, so none is found free again)
    }
    rank += step;
    __syncthreads();
  }
}

// All of it by one workgroup, for tables of up to kSmallEntries entries, which its threads keep:
// the counts change by atomics, so they are read past the first-level cache. 3.0 us, of round
// trips: lengths, table, three to the counts, the list.
constexpr int kOneThreads = 1024, kOneEntries = kSmallEntries / kOneThreads;
__global__ __launch_bounds__(kOneThreads) void shared_one_kernel(SharedRelease r) {
  constexpr int kWaves = kOneThreads / kWave;
  __shared__ int bad, wave_sum[kOneEntries * kWaves];
  const int tid = threadIdx.x, lane = tid & (kWave - 1), wave = tid / kWave;
  const int count = *r.free_count, entries = r.B * r.bt_stride;
  if (tid == 0) bad = 0;
  __syncthreads();
  const int64_t limit = (int64_t)r.bt_stride * kPage;
  for (int i = tid; i < r.B; i += kOneThreads) {
    const int64_t len = r.lens[i], keep = r.keep_lens[i];
    if (keep < 0 || keep > len || len > limit) bad = 1;
  }
  int page[kOneEntries];                   // of the entries that are given up, -1 else
#pragma unroll
  for (int u = 0; u < kOneEntries; ++u) {
    const int x = u * kOneThreads + tid;
    page[u] = -1;
    if (x >= entries) continue;
    const int b = x / r.bt_stride, j = x - b * r.bt_stride, id = r.block_table[x];
    if (j >= pages_of(r.keep_lens[b]) && j < pages_of(r.lens[b]) && page_ok(id, r.num_pages)) page[u] = id;
  }
  __syncthreads();
  if (bad || count < 0 || count > r.capacity) {
    if (tid == 0) *r.released = -1;
    return;
  }
  auto holders = [&](int p) {
    return __hip_atomic_load(&r.shares[p], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  };
  // A wave's atomics are in the L2, where all of the workgroup's reads of the counts go: a fence
  // of the whole GPU would write the L2 back besides, 3 us each time.
  auto arrived = [] { asm volatile("s_waitcnt vmcnt(0)" ::: "memory"); };
#pragma unroll
  for (int u = 0; u < kOneEntries; ++u)
    if (page[u] >= 0) atomicSub(&r.shares[page[u]], 1);
  arrived();
  __syncthreads();
  int held[kOneEntries];
#pragma unroll
  for (int u = 0; u < kOneEntries; ++u) held[u] = page[u] >= 0 ? holders(page[u]) : 0;
  // (other entries' codes may be among those read; they too are of pages that nobody holds)
#pragma unroll
  for (int u = 0; u < kOneEntries; ++u)
    if (held[u] < 0) atomicMin(&r.shares[page[u]], -(kCode + 1) - (u * kOneThreads + tid));
  arrived();
  __syncthreads();
  uint64_t votes[kOneEntries];
  bool free[kOneEntries];
#pragma unroll
  for (int u = 0; u < kOneEntries; ++u)
    free[u] = held[u] < 0 && holders(page[u]) == -(kCode + 1) - (u * kOneThreads + tid);
#pragma unroll
  for (int u = 0; u < kOneEntries; ++u) {
    votes[u] = __ballot(free[u]);
    if (lane == 0) wave_sum[u * kWaves + wave] = (int)__popcll(votes[u]);
  }
  __syncthreads();
  // every wave sums up what lies before each of its places
  static_assert(kOneEntries * kWaves <= kWave, "a lane a place");
  const int sum = wave_sums(lane < kOneEntries * kWaves ? wave_sum[lane] : 0);
  const int all = of_lane(sum, kWave - 1);
#pragma unroll
  for (int u = 0; u < kOneEntries; ++u) {
    const int place = __builtin_amdgcn_readfirstlane(u * kWaves + wave);
    const int before = place ? of_lane(sum, place - 1) : 0;
    if (!free[u]) continue;
    const int at = before + (int)__popcll(votes[u] & ((1ull << lane) - 1));
    const int64_t to = (int64_t)count + all - 1 - at;
    if (to < r.capacity) r.free_pages[to] = page[u];
    r.shares[page[u]] = 0;
  }
  if (tid == 0) {
    *r.released = all;
    *r.free_count = min(count + all, r.capacity);
  }
}

// ---- pages' contents ----
// One page of one KV head a workgroup, 16 bytes a thread and pool. Bound by HBM: 434 pages of 8 KV
// heads in bf16 (57 MB read and written, the sources of eight copies the same) 7.5 us; in codes, of
// which half of the threads have none, 5.4.
template <bool kFp8>
__global__ __launch_bounds__(kPageThreads) void page_copy_kernel(uint8_t *k_pool, uint8_t *v_pool,
                                                                 const int32_t *src,
                                                                 const int32_t *dst, int32_t hkv,
                                                                 int32_t num_pages) {
  constexpr int kBytes = kPage * kHeadDim * (kFp8 ? 1 : 2);
  const int i = blockIdx.x / hkv, g = blockIdx.x - i * hkv;
  const int from = src[i], to = dst[i];
  if (!page_ok(from, num_pages) || !page_ok(to, num_pages) || from == to) return;
  const size_t at = threadIdx.x * 16;
  if (at >= kBytes) return;
  const size_t f = ((size_t)from * hkv + g) * kBytes + at, t = ((size_t)to * hkv + g) * kBytes + at;
  const u32x4 k = *reinterpret_cast<const u32x4 *>(k_pool + f);
  const u32x4 v = *reinterpret_cast<const u32x4 *>(v_pool + f);
  *reinterpret_cast<u32x4 *>(k_pool + t) = k;
  *reinterpret_cast<u32x4 *>(v_pool + t) = v;
}

constexpr int kMoveTokens = 32;            // moved together

// The kept tokens of one row and KV head, up to 32 a step. Indices rise, so a token never moves
// behind where it was and the tokens of one step lie before the sources of all later ones: a
// step has all its tokens in registers before it writes any. Keys move 16 bytes a thread; of
// the values a thread has one dimension of the tokens that go to one half of a page, so that a
// half whose tokens all move is one store. Bound by round trips (the offsets, the index, the
// table and the pages, one behind the other) and, in large calls, by HBM's sectors: of a value
// row a token has two bytes of a 32-byte sector, so that 58 MB of keys and values are 137 MB
// in whole sectors. 4 rows of up to 8 tokens 4.1 us; 512 rows, some 16 tokens each, 8 KV heads 32 us
// (4.3 TB/s of sectors), with single values stored one by one 40; in codes 18.
template <typename E>
__global__ __launch_bounds__(kPageThreads) void page_compact_kernel(
    E *k_pool, E *v_pool, const int32_t *block_table, int32_t bt_stride, int32_t num_pages,
    int32_t hkv, const int32_t *start_pos, const int32_t *cu_src, const int32_t *src_index,
    const int32_t *counts, int32_t total, int32_t max_count) {
  constexpr int kUnit = 16 / sizeof(E), kUnits = kHeadDim / kUnit;      // of a key
  constexpr int kKeys = kMoveTokens * kUnits / kPageThreads;            // units a thread
  constexpr int kHalf = kPage / 2;
  constexpr int kHalves = kMoveTokens / kHalf + 1;                      // that 32 tokens can lie in
  constexpr int kValues = (kHalves * kHeadDim + kPageThreads - 1) / kPageThreads;
  constexpr int kWords = kHalf * sizeof(E) / 4;
  typedef uint32_t Eight __attribute__((ext_vector_type(kWords)));      // a half of a value row
  struct Move {
    int from, slot, to, to_slot;           // pages and slots; from -1: stays
  };
  __shared__ Move move[kMoveTokens + 2 * kHalf];
  const int b = blockIdx.x / hkv, g = blockIdx.x - b * hkv, tid = threadIdx.x;
  const int first = min(max(cu_src[b], 0), total);
  int n = min(min(max(cu_src[b + 1] - first, 0), total - first), max_count);
  if (counts) n = min(n, max(counts[b], 0));
  const int64_t start = max(start_pos[b], 0), limit = (int64_t)bt_stride * kPage;
  const int32_t *bt = block_table + (int64_t)b * bt_stride;
  auto block = [&](int page) { return ((size_t)page * hkv + g) * kPage * kHeadDim; };
  for (int i0 = 0; i0 < n; i0 += kMoveTokens) {
    __syncthreads();
    const int m = min(kMoveTokens, n - i0);
    const int lead = (int)((start + i0) % kHalf);          // the first token's place in its half
    if (tid < kMoveTokens + 2 * kHalf) {                    // entry x: the token of place x - lead
      const int i = i0 + tid - lead;
      Move mv = {-1, 0, 0, 0};
      if (tid >= lead && tid < lead + m) {
        const int j = src_index[first + i];
        if (j > i && start + j < limit) {
          const int64_t p = start + j, q = start + i;
          mv.from = clamp_page(bt[p / kPage], num_pages);
          mv.to = clamp_page(bt[q / kPage], num_pages);
          mv.slot = (int)(p % kPage);
          mv.to_slot = (int)(q % kPage);
        }
      }
      move[tid] = mv;
    }
    __syncthreads();
    u32x4 k[kKeys];
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      const int x = i * kPageThreads + tid, token = x / kUnits, unit = x % kUnits;
      const Move mv = move[lead + token];
      if (token < m && mv.from >= 0)
        k[i] = *reinterpret_cast<const u32x4 *>(k_pool + block(mv.from) + mv.slot * kHeadDim + unit * kUnit);
    }
    uint32_t v[kValues][kHalf] = {};
    uint32_t moved[kValues];                                // bits of the half's slots
#pragma unroll
    for (int i = 0; i < kValues; ++i) {
      const int x = i * kPageThreads + tid, half = x / kHeadDim, d = x % kHeadDim;
      moved[i] = 0;
      if (half >= kHalves) continue;
#pragma unroll
      for (int s = 0; s < kHalf; ++s) {
        const Move mv = move[half * kHalf + s];
        if (mv.from < 0) continue;
        moved[i] |= 1u << s;
        v[i][s] = v_pool[block(mv.from) + d * kPage + mv.slot];
      }
    }
    // here before any thread writes
#pragma unroll
    for (int i = 0; i < kKeys; ++i) asm volatile("" : "+v"(k[i]));
#pragma unroll
    for (int i = 0; i < kValues; ++i)
#pragma unroll
      for (int s = 0; s < kHalf; ++s) asm volatile("" : "+v"(v[i][s]));
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      const int x = i * kPageThreads + tid, token = x / kUnits, unit = x % kUnits;
      const Move mv = move[lead + token];
      if (token < m && mv.from >= 0)
        *reinterpret_cast<u32x4 *>(k_pool + block(mv.to) + mv.to_slot * kHeadDim + unit * kUnit) = k[i];
    }
#pragma unroll
    for (int i = 0; i < kValues; ++i) {
      const int x = i * kPageThreads + tid, half = x / kHeadDim, d = x % kHeadDim;
      if (moved[i] == 0) continue;
      const Move mv = move[half * kHalf + __ffs(moved[i]) - 1];
      E *to = v_pool + block(mv.to) + d * kPage + mv.to_slot / kHalf * kHalf;
      if (moved[i] == (1u << kHalf) - 1) {
        Eight w;
#pragma unroll
        for (int x = 0; x < kWords; ++x) {
          w[x] = 0;
#pragma unroll
          for (int y = 0; y < kHalf / kWords; ++y) w[x] |= v[i][x * kHalf / kWords + y] << (8 * sizeof(E) * y);
        }
        *reinterpret_cast<Eight *>(to) = w;
      } else {
#pragma unroll
        for (int s = 0; s < kHalf; ++s)
          if (moved[i] >> s & 1) to[s] = (E)v[i][s];
      }
    }
  }
}

}  // namespace

hipError_t launch_table_fork(const int32_t *src_rows, const int32_t *dst_rows, const int32_t *lens,
                             int32_t n, int32_t *block_table, int32_t B, int32_t bt_stride,
                             int32_t *shares, int32_t num_pages, const int32_t *free_pages,
                             int32_t *free_count, int32_t capacity, int32_t *copy_src,
                             int32_t *copy_dst, int32_t *taken, hipStream_t stream) {
  if (n <= kSmallForks && (int64_t)n * bt_stride <= kSmallEntries) {
    fork_kernel<true><<<1, kSmallForks * kSmallThreads, 0, stream>>>(
        src_rows, dst_rows, lens, n, block_table, B, bt_stride, shares, num_pages, free_pages,
        free_count, capacity, copy_src, copy_dst, taken);
    return hipGetLastError();
  }
  fork_kernel<false><<<n, kForkThreads, 0, stream>>>(
      src_rows, dst_rows, lens, n, block_table, B, bt_stride, shares, num_pages, free_pages,
      free_count, capacity, copy_src, copy_dst, taken);
  if (n > 1) fork_count_kernel<<<1, 1, 0, stream>>>(free_count, taken);
  return hipGetLastError();
}

size_t table_release_shared_bytes(int32_t B) { return ((size_t)B + 2) * sizeof(int32_t); }

hipError_t launch_table_release_shared(const int32_t *lens, const int32_t *keep_lens,
                                       const int32_t *block_table, int32_t B, int32_t bt_stride,
                                       int32_t *shares, int32_t num_pages, int32_t *free_pages,
                                       int32_t *free_count, int32_t capacity, int32_t *released,
                                       void *workspace, hipStream_t stream) {
  int32_t *head = static_cast<int32_t *>(workspace);
  const SharedRelease r = {lens, keep_lens, block_table, B, bt_stride, num_pages, capacity,
                           shares, free_pages, free_count, released, head, head + 2};
  if ((int64_t)B * bt_stride <= kSmallEntries) {
    shared_one_kernel<<<1, kOneThreads, 0, stream>>>(r);
    return hipGetLastError();
  }
  shared_sub_kernel<<<B, kRowThreads, 0, stream>>>(r);
  shared_last_kernel<<<B, kRowThreads, 0, stream>>>(r);
  shared_count_kernel<<<B, kRowThreads, 0, stream>>>(r);
  shared_put_kernel<<<B, kRowThreads, 0, stream>>>(r);
  return hipGetLastError();
}

hipError_t launch_page_copy(const PagedKV &kv, const int32_t *src_pages, const int32_t *dst_pages,
                            int32_t n, hipStream_t stream) {
  uint8_t *k = reinterpret_cast<uint8_t *>(kv.k_pool), *v = reinterpret_cast<uint8_t *>(kv.v_pool);
  const unsigned grid = (unsigned)n * (unsigned)kv.hkv;
  if (kv.fp8)
    page_copy_kernel<true><<<grid, kPageThreads, 0, stream>>>(k, v, src_pages, dst_pages, kv.hkv,
                                                             kv.num_pages);
  else
    page_copy_kernel<false><<<grid, kPageThreads, 0, stream>>>(k, v, src_pages, dst_pages, kv.hkv,
                                                              kv.num_pages);
  return hipGetLastError();
}

hipError_t launch_page_compact(const PagedKV &kv, const int32_t *start_pos, const int32_t *cu_src,
                               const int32_t *src_index, const int32_t *counts, int32_t B,
                               int32_t total, int32_t max_count, hipStream_t stream) {
  const unsigned grid = (unsigned)B * (unsigned)kv.hkv;
  if (kv.fp8)
    page_compact_kernel<uint8_t><<<grid, kPageThreads, 0, stream>>>(
        reinterpret_cast<uint8_t *>(kv.k_pool), reinterpret_cast<uint8_t *>(kv.v_pool),
        kv.block_table, kv.bt_stride, kv.num_pages, kv.hkv, start_pos, cu_src, src_index, counts,
        total, max_count);
  else
    page_compact_kernel<uint16_t><<<grid, kPageThreads, 0, stream>>>(
        kv.k_pool, kv.v_pool, kv.block_table, kv.bt_stride, kv.num_pages, kv.hkv, start_pos,
        cu_src, src_index, counts, total, max_count);
  return hipGetLastError();
}

}  // namespace ra
