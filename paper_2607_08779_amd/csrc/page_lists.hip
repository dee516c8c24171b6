// What a paged cache's tables and pools need between steps: requests that continue others (fork), the pages
// that nobody holds (collect), held pages brought to the front (compact), and copies of pages
// (see include/ssq_cache.h).
//
// Fork, collect and compact move a few bytes for each table entry and page, so that launches and latency
// bound them.  Fork is one launch: every workgroup finds for itself how many pages the rows before its
// own take, as page_tables.hip does (64 rows 3.9 us, 1024 rows of 512 pages 5.7).  Collect and compact mark held
// pages, count them and write lists whose places follow from the counts (64 requests, 9000 pages 8.7 us;
// compacting 98000 pages of 512 requests 13.7, 140000 pages 31.8).  A copy is bound by the pages' bytes, read and written (939 MB 167 us,
// 5.6 TB/s).  Nothing depends on the order in which workgroups or atomics run.
#include "page_lists.h"

namespace ssq {
namespace {

constexpr int kThreads = 256;

// --- fork ------------------------------------------------------------------------------------

constexpr int kForkThreads = 1024, kForkRows = kForkThreads / 64;     // a wavefront a row

__device__ __forceinline__ uint32_t pages_of(int len, int shift) { return ((uint32_t)max(len, 0) + (1u << shift) - 1u) >> shift; }

__global__ __launch_bounds__(kForkThreads) void page_fork_kernel(const PageFork a) {
  extern __shared__ int first[];                           // of every row that is continued, its first continuation
  __shared__ int sums[kForkRows];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, rows = (int)a.rows, requests = (int)a.requests;
  for (int i = tid; i < rows; i += kForkThreads) first[i] = 0x7fffffff;
  __syncthreads();
  for (int i = tid; i < requests; i += kForkThreads) {
    const int parent = a.parents[i];
    if (parent >= 0 && parent < rows) atomicMin(&first[parent], i);
  }
  __syncthreads();
  // The entry of row i that a new page replaces, or -1: the last page of a continuation that is not its
  // parent's first, where tokens will still be added to it.
  auto shared_last = [&](int i) {
    const int parent = a.parents[i];
    if (parent < 0 || parent >= rows || first[parent] == i) return -1;
    const int len = a.lens[parent];
    const uint32_t n = pages_of(len, a.shift);
    if ((len & ((1 << a.shift) - 1)) == 0 || n == 0 || n > min(a.stride, a.stride_out)) return -1;
    return max(a.table[parent * a.stride + n - 1], -1);
  };
  const int row0 = (int)blockIdx.x * kForkRows;
  int before = 0;
  for (int i = tid; i < row0; i += kForkThreads) before += shared_last(i) >= 0;
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) before += __shfl_xor(before, d, 64);
  if (lane == 0) sums[wave] = before;
  __syncthreads();
  before = 0;
#pragma unroll
  for (int w = 0; w < kForkRows; ++w) before += sums[w];
  const bool mine = lane < kForkRows && row0 + lane < requests;
  const int last_of_lane = mine ? shared_last(row0 + lane) : -1;
  const uint64_t needs = __builtin_amdgcn_ballot_w64(last_of_lane >= 0);
  const int32_t taken = a.taken != nullptr ? *a.taken : 0;
  if (tid == 0 && row0 + kForkRows >= requests) *a.taken_after = (int32_t)((uint32_t)taken + (uint32_t)(before + __popcll(needs)));
  const int row = row0 + wave;
  if (row >= requests) return;
  const int last = __shfl(last_of_lane, wave, 64);
  int page = -1;
  if (last >= 0) {
    const int64_t at = (int64_t)(int32_t)((uint32_t)taken + (uint32_t)(before + __popcll(needs & ((1ull << wave) - 1ull))));
    page = at >= 0 && at < a.free_count ? max(a.free_pages[at], -1) : -1;
  }
  const int parent = a.parents[row];
  const bool there = parent >= 0 && parent < rows;
  const int len = there ? max(a.lens[parent], 0) : 0;
  const int64_t n = pages_of(len, a.shift);
  const int32_t* from = a.table + (there ? parent : 0) * a.stride;
  int32_t* to = a.table_out + row * a.stride_out;
#pragma unroll 4
  for (int64_t c = lane; c < a.stride_out; c += 64) {
    int32_t e = c < n && c < a.stride ? from[c] : -1;
    if (last >= 0 && c == n - 1) e = page;
    to[c] = e;
  }
  if (lane == 0) {
    a.lens_out[row] = len;
    a.src[row] = page >= 0 ? last : -1;
    a.dst[row] = page;
  }
}

// --- collect and compact ----------------------------------------------------------------------

constexpr int kBlockPages = 4096, kPerThread = kBlockPages / kThreads;      // pages of a workgroup and of a thread
constexpr int kHeld = 1, kPinned = 2;                                       // bits of a mark

struct Pools {
  uint8_t* marks;            // [pages, rounded up to blocks]
  uint2* counts;             // of each block: free pages, pinned pages
  int32_t* list;             // compact: the free pages before the moves
  int32_t* to;               // compact: where a page that moves goes
  int64_t blocks;
};

__global__ __launch_bounds__(kThreads) void clear_kernel(const PageCollect a, const Pools s) {
  const int64_t i0 = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * kPerThread;
  uint32_t w[kPerThread / 4];
#pragma unroll
  for (int j = 0; j < kPerThread; ++j) {
    const int64_t i = i0 + j;
    // past the end: held, so that nothing is free there, and not pinned
    const uint32_t mark = i >= a.pages ? kHeld : a.pinned != nullptr && a.pinned[i] != 0 ? kHeld | kPinned : 0u;
    w[j / 4] = (j % 4 == 0 ? 0u : w[j / 4]) | mark << (8 * (j % 4));
  }
  *reinterpret_cast<u32x4*>(s.marks + i0) = u32x4{w[0], w[1], w[2], w[3]};
}

__global__ __launch_bounds__(kThreads) void mark_kernel(const PageCollect a, const Pools s, int64_t row_groups) {
  const int64_t row = blockIdx.x / row_groups, c0 = blockIdx.x % row_groups * (4 * kThreads);
  const int64_t n = min((int64_t)pages_of(a.lens[row], a.shift), a.stride);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t c = c0 + j * kThreads + threadIdx.x;
    if (c >= n) continue;
    const int64_t page = a.table[row * a.stride + c];
    if (page < 0 || page >= a.pages) continue;
    if (a.pinned == nullptr || a.pinned[page] == 0) s.marks[page] = kHeld;
  }
}

__device__ __forceinline__ uint2 sum2(uint2 v, uint2* waves) {        // over the workgroup, in every thread
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) v.x += __shfl_xor(v.x, d, 64), v.y += __shfl_xor(v.y, d, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = v;
  __syncthreads();
  uint2 all = {0u, 0u};
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) all.x += waves[w].x, all.y += waves[w].y;
  return all;
}
// Sums of v over the threads before this one; *all: over every thread.
__device__ __forceinline__ uint32_t before_in_group(uint32_t v, uint32_t* waves, uint32_t* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t x = __shfl_up(s, o, 64);
    if (lane >= o) s += x;
  }
  __syncthreads();
  if (lane == 63) waves[wave] = s;
  __syncthreads();
  uint32_t before = s - v, sum = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    if (w < wave) before += waves[w];
    sum += waves[w];
  }
  *all = sum;
  return before;
}

// Marks of a thread's pages of a block.
struct Marks {
  u32x4 w;
  __device__ __forceinline__ Marks(const Pools& s, int64_t block) : w(*reinterpret_cast<const u32x4*>(s.marks + block * kBlockPages + threadIdx.x * kPerThread)) {}
  __device__ __forceinline__ int of(int j) const { return (int)(w[j / 4] >> (8 * (j % 4)) & 3u); }
};

__global__ __launch_bounds__(kThreads) void count_kernel(const PageCollect a, const Pools s) {
  __shared__ uint2 waves[kThreads / 64];
  const Marks m(s, blockIdx.x);
  uint2 n = {0u, 0u};
#pragma unroll
  for (int j = 0; j < kPerThread; ++j) n.x += m.of(j) == 0, n.y += m.of(j) >> 1;
  n = sum2(n, waves);
  if (threadIdx.x == 0) s.counts[blockIdx.x] = n;
}

// Counts of blocks [0, before) and of all.
__device__ __forceinline__ uint2 count_blocks(const Pools& s, int64_t before, uint2* all, uint2* waves) {
  uint2 first = {0u, 0u}, sum = {0u, 0u};
  for (int64_t b = threadIdx.x; b < s.blocks; b += kThreads) {
    const uint2 c = s.counts[b];
    sum.x += c.x, sum.y += c.y;
    if (b < before) first.x += c.x, first.y += c.y;
  }
  *all = sum2(sum, waves);
  return sum2(first, waves);
}

// The free pages, ascending, then -1.
__global__ __launch_bounds__(kThreads) void list_kernel(const PageCollect a, const Pools s, int32_t* list, bool last) {
  __shared__ uint2 waves[kThreads / 64];
  __shared__ uint32_t wave_sums[kThreads / 64];
  uint2 all;
  const uint2 before = count_blocks(s, blockIdx.x, &all, waves);
  const Marks m(s, blockIdx.x);
  uint32_t n = 0, in_block;
#pragma unroll
  for (int j = 0; j < kPerThread; ++j) n += m.of(j) == 0;
  uint32_t at = before.x + before_in_group(n, wave_sums, &in_block);
  const int64_t i0 = blockIdx.x * (int64_t)kBlockPages + threadIdx.x * kPerThread;
#pragma unroll
  for (int j = 0; j < kPerThread; ++j)
    if (m.of(j) == 0) list[at++] = (int32_t)(i0 + j);
  if (!last) return;
  // the entries behind them: this block's share of the list's length
  for (int64_t i = blockIdx.x * (int64_t)kBlockPages + threadIdx.x; i < min((blockIdx.x + (int64_t)1) * kBlockPages, a.pages); i += kThreads)
    if (i >= all.x) list[i] = -1;
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.count = (int32_t)all.x;
}

// What lies below and above `used`, the number of held pages: holes are the free pages below it; as many
// pages above are held, of which those that are not pinned move into the first holes.
struct Split {
  int64_t used;
  uint32_t holes, moves;
};
__device__ __forceinline__ Split split_of(const PageCollect& a, const Pools& s, uint2* waves) {
  uint2 all;
  Split r;
  count_blocks(s, 0, &all, waves);
  r.used = a.pages - all.x;
  const int64_t block = min(r.used / kBlockPages, s.blocks - 1);
  uint2 none;
  const uint2 below = count_blocks(s, block, &none, waves);
  const Marks m(s, block);
  uint2 n = {0u, 0u};
#pragma unroll
  for (int j = 0; j < kPerThread; ++j)
    if (block * kBlockPages + threadIdx.x * kPerThread + j < r.used) n.x += m.of(j) == 0, n.y += m.of(j) >> 1;
  n = sum2(n, waves);
  r.holes = below.x + n.x;
  r.moves = r.holes - (all.y - below.y - n.y);
  return r;
}
// Of this block's pages from `used` on, the sums of `is` before this thread's, those of the blocks before included.
template <typename Is>
__device__ __forceinline__ uint32_t above_before(const PageCollect& a, const Pools& s, int64_t used, bool pinned, const Marks& m, Is is, uint2* waves, uint32_t* wave_sums) {
  // blocks wholly above, from their counts; the block that `used` lies in, from its marks
  const int64_t block = used / kBlockPages, here = blockIdx.x;
  uint32_t base = 0, all;
  if (here > block) {
    const Marks edge(s, block);
    uint2 n = {0u, 0u};
#pragma unroll
    for (int j = 0; j < kPerThread; ++j)
      if (block * kBlockPages + threadIdx.x * kPerThread + j >= used) n.x += is(edge.of(j));
    for (int64_t b = block + 1 + threadIdx.x; b < here; b += kThreads) n.x += pinned ? s.counts[b].y : kBlockPages - s.counts[b].x - s.counts[b].y;
    base = sum2(n, waves).x;
  }
  uint32_t n = 0;
  const int64_t i0 = here * kBlockPages + threadIdx.x * kPerThread;
#pragma unroll
  for (int j = 0; j < kPerThread; ++j)
    if (i0 + j >= used) n += is(m.of(j));
  return base + before_in_group(n, wave_sums, &all);
}

__global__ __launch_bounds__(kThreads) void move_kernel(const PageCollect a, const Pools s) {
  __shared__ uint2 waves[kThreads / 64];
  __shared__ uint32_t wave_sums[kThreads / 64];
  const Split split = split_of(a, s, waves);
  const Marks m(s, blockIdx.x);
  const int64_t i0 = blockIdx.x * (int64_t)kBlockPages + threadIdx.x * kPerThread;
  uint32_t at = above_before(a, s, split.used, false, m, [](int mark) { return mark == kHeld ? 1u : 0u; }, waves, wave_sums);
#pragma unroll
  for (int j = 0; j < kPerThread; ++j) {
    const int64_t i = i0 + j;
    if (i < split.used || i >= a.pages || m.of(j) != kHeld) continue;
    const int32_t hole = s.list[at];
    a.src[at] = (int32_t)i;
    a.dst[at] = hole;
    s.to[i] = hole;
    ++at;
  }
  for (int64_t i = blockIdx.x * (int64_t)kBlockPages + threadIdx.x; i < min((blockIdx.x + (int64_t)1) * kBlockPages, a.pages / 2); i += kThreads)
    if (i >= split.moves) a.src[i] = a.dst[i] = -1;
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    *a.count = (int32_t)(a.pages - split.used);
    *a.moved = (int32_t)split.moves;
  }
}

// The free pages after the moves: holes that are left, then what is not pinned above.
__global__ __launch_bounds__(kThreads) void free_after_kernel(const PageCollect a, const Pools s) {
  __shared__ uint2 waves[kThreads / 64];
  __shared__ uint32_t wave_sums[kThreads / 64];
  const Split split = split_of(a, s, waves);
  const Marks m(s, blockIdx.x);
  const int64_t i0 = blockIdx.x * (int64_t)kBlockPages + threadIdx.x * kPerThread, left = split.holes - split.moves, count = a.pages - split.used;
  uint32_t pinned = above_before(a, s, split.used, true, m, [](int mark) { return (uint32_t)mark >> 1; }, waves, wave_sums);
#pragma unroll
  for (int j = 0; j < kPerThread; ++j) {
    const int64_t i = i0 + j;
    if (i < split.used || i >= a.pages) continue;
    if (m.of(j) >> 1) ++pinned;
    else a.free_pages[left + (i - split.used) - pinned] = (int32_t)i;
  }
  for (int64_t i = blockIdx.x * (int64_t)kBlockPages + threadIdx.x; i < min((blockIdx.x + (int64_t)1) * kBlockPages, a.pages); i += kThreads) {
    if (i < left) a.free_pages[i] = s.list[split.moves + i];
    else if (i >= count) a.free_pages[i] = -1;
  }
}

__global__ __launch_bounds__(kThreads) void rename_kernel(const PageCollect a, const Pools s, int64_t row_groups) {
  __shared__ uint2 waves[kThreads / 64];
  uint2 all;
  count_blocks(s, 0, &all, waves);
  const int64_t used = a.pages - all.x;
  const int64_t row = blockIdx.x / row_groups, c0 = blockIdx.x % row_groups * (4 * kThreads);
  const int64_t n = min((int64_t)pages_of(a.lens[row], a.shift), a.stride);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t c = c0 + j * kThreads + threadIdx.x;
    if (c >= a.stride) continue;
    const int32_t page = a.table[row * a.stride + c];
    const bool moves = c < n && page >= used && page < a.pages && s.marks[page] == kHeld;
    a.table_out[row * a.stride + c] = moves ? s.to[page] : page;
  }
}

// Pools of up to 131072 pages and 2048 requests: every workgroup has all marks, in bits in LDS, and counts them for itself; then each takes
// its share of the lists and rows.  The marks of a small table every workgroup makes for itself, in the only launch
// (64 requests, 9000 pages: 10.4 us in the launches above, 8.6 so).  Where the table is larger, atomics on LDS at
// random places would take longer than marking in memory in launches of its own (compacting 98000 pages of 512
// requests: 31 us in the launches above, 46 in one, 13.6 in three).
constexpr int kOneThreads = 1024, kOneWaves = kOneThreads / 64;
constexpr int kOnePages = 1 << 17, kOneWords = kOnePages / 32, kOneRows = 2048;
constexpr int64_t kOneEntries = 1 << 14;          // of a table that every workgroup marks for itself
constexpr int kOneShare = 512, kOneGroups = 256;  // pages of a workgroup, where so many workgroups suffice
constexpr int kOneAhead = 16;                     // table entries that a lane has under way

struct OneLds {
  uint32_t held[kOneWords], pinned[kOneWords];
  uint32_t free_before[kOneWords], pinned_before[kOneWords];      // of each word, in all words before it
  uint32_t row_pages[kOneRows];
  uint32_t waves[2][kOneWaves];
};

// A stretch of a row, and steps from one to another without a division each.
struct Stretch {
  int row, column;
  __device__ __forceinline__ Stretch(int t, int stretches) : row(stretches > 0 ? t / stretches : 0), column(stretches > 0 ? t - row * stretches : 0) {}
  __device__ __forceinline__ void move(const Stretch& by, int stretches) {
    row += by.row;
    column += by.column;
    if (column >= stretches) column -= stretches, ++row;
  }
};

// Sums of v over the threads before this one; *all: over every thread.
__device__ __forceinline__ uint32_t before_in_one(uint32_t v, uint32_t (&waves)[kOneWaves], uint32_t* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t x = __shfl_up(s, o, 64);
    if (lane >= o) s += x;
  }
  if (lane == 63) waves[wave] = s;
  __syncthreads();
  uint32_t before = s - v, sum = 0;
#pragma unroll
  for (int w = 0; w < kOneWaves; ++w) {
    if (w < wave) before += waves[w];
    sum += waves[w];
  }
  *all = sum;
  return before;
}

template <bool COMPACT, bool MARKED>
__global__ __launch_bounds__(kOneThreads) void pool_kernel(const PageCollect a, const uint8_t* marks, int share) {
  __shared__ OneLds lds;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int pages = (int)a.pages, words = (pages + 31) / 32, rows = (int)a.requests, stride = (int)a.stride;
  const int stretches = (int)((a.stride + 63) / 64), tasks = rows * stretches;
  for (int r = tid; r < rows; r += kOneThreads) lds.row_pages[r] = min(pages_of(a.lens[r], a.shift), (uint32_t)stride);
  if constexpr (MARKED) {
    // 16 marks of a byte each to two bits; what lies behind the pages is marked as held
    auto four = [](uint32_t x) { return ((x & 0x01010101u) * 0x10204080u) >> 28; };
    constexpr int kLoads = 8;
    for (int i0 = tid; i0 < 2 * words; i0 += kOneThreads * kLoads) {
      u32x4 m[kLoads];
#pragma unroll
      for (int k = 0; k < kLoads; ++k) m[k] = *reinterpret_cast<const u32x4*>(marks + 16 * min(i0 + kOneThreads * k, 2 * words - 1));
#pragma unroll
      for (int k = 0; k < kLoads; ++k) {
        const int i = i0 + kOneThreads * k;
        uint32_t held = 0, pinned = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) held |= four(m[k][j]) << (4 * j), pinned |= four(m[k][j] >> 1) << (4 * j);
        if (i < 2 * words) {
          reinterpret_cast<uint16_t*>(lds.held)[i] = (uint16_t)held;
          reinterpret_cast<uint16_t*>(lds.pinned)[i] = (uint16_t)pinned;
        }
      }
    }
    __syncthreads();
  } else {
    for (int w = tid; w < words; w += kOneThreads) lds.held[w] = lds.pinned[w] = 0;
    __syncthreads();
    if (a.pinned != nullptr) {
      constexpr int kPins = 8;                   // 64 pages each, two words of the wavefront's own
      for (int i0 = 64 * wave; i0 < pages; i0 += kOneThreads * kPins) {
        uint8_t pin[kPins];
#pragma unroll
        for (int j = 0; j < kPins; ++j) pin[j] = a.pinned[min(i0 + kOneThreads * j + lane, pages - 1)];
#pragma unroll
        for (int j = 0; j < kPins; ++j) {
          const int i = i0 + kOneThreads * j;
          const uint64_t bits = __builtin_amdgcn_ballot_w64(i + lane < pages && pin[j] != 0);
          if (lane < 2 && i / 32 + lane < words) lds.held[i / 32 + lane] = lds.pinned[i / 32 + lane] = (uint32_t)(bits >> (32 * lane));
        }
      }
      __syncthreads();
    }
    // Stretches of 64 entries of a row, in turn for each wavefront.  Loads wait for nothing: what lies behind the last
    // stretch or a row's pages is the table's last entry or the row's, and looked at afterwards.
    Stretch at(wave, stretches);
    const Stretch by(kOneWaves, stretches);
    for (int t0 = wave; t0 < tasks; t0 += kOneWaves * kOneAhead) {
      int32_t page[kOneAhead];
      const Stretch first = at;
#pragma unroll
      for (int j = 0; j < kOneAhead; ++j) {
        page[j] = a.table[(int64_t)min(at.row, rows - 1) * stride + min(64 * at.column + lane, stride - 1)];
        at.move(by, stretches);
      }
      at = first;
#pragma unroll
      for (int j = 0; j < kOneAhead; ++j) {
        const bool held = at.row < rows && 64 * at.column + lane < (int)lds.row_pages[min(at.row, rows - 1)] && (uint32_t)page[j] < (uint32_t)pages;
        if (held) atomicOr(&lds.held[page[j] / 32], 1u << (page[j] % 32));
        at.move(by, stretches);
      }
    }
    __syncthreads();
  }
  // Pages past the end are no free ones.
  if (tid == 0 && pages % 32 != 0) lds.held[words - 1] |= ~0u << (pages % 32);
  __syncthreads();
  // Running counts; a thread has consecutive words.
  constexpr int kEach = kOneWords / kOneThreads;
  const int w0 = tid * kEach;
  uint32_t free_here = 0, pinned_here = 0, free_all, pinned_all;
#pragma unroll
  for (int k = 0; k < kEach; ++k)
    if (w0 + k < words) free_here += __popc(~lds.held[w0 + k]), pinned_here += __popc(lds.pinned[w0 + k]);
  uint32_t f = before_in_one(free_here, lds.waves[0], &free_all), p = before_in_one(pinned_here, lds.waves[1], &pinned_all);
#pragma unroll
  for (int k = 0; k < kEach; ++k)
    if (w0 + k < words) {
      lds.free_before[w0 + k] = f;
      lds.pinned_before[w0 + k] = p;
      f += __popc(~lds.held[w0 + k]);
      p += __popc(lds.pinned[w0 + k]);
    }
  __syncthreads();
  auto below = [](uint32_t bits, int i) { return (uint32_t)__popc(bits & ((1u << (i % 32)) - 1u)); };
  auto free_to = [&](int i) { return i < pages ? lds.free_before[i / 32] + below(~lds.held[i / 32], i) : free_all; };       // free pages below page i
  auto pinned_to = [&](int i) { return i < pages ? lds.pinned_before[i / 32] + below(lds.pinned[i / 32], i) : pinned_all; };
  const int used = pages - (int)free_all;
  const uint32_t holes = COMPACT ? free_to(used) : 0, pinned_below = COMPACT ? pinned_to(used) : 0, moves = holes - (pinned_all - pinned_below);

  // This workgroup's pages.
  const int end = min(pages, ((int)blockIdx.x + 1) * share);
  for (int i = (int)blockIdx.x * share + tid; i < end; i += kOneThreads) {
    const bool held = lds.held[i / 32] >> (i % 32) & 1u;
    const uint32_t at = free_to(i);
    if (!COMPACT) {
      if (!held) a.free_pages[at] = i;
    } else if (i < used) {                      // a hole is filled, or stays free
      if (held) continue;
      if (at < moves) a.dst[at] = i;
      else a.free_pages[at - moves] = i;
    } else if (!(lds.pinned[i / 32] >> (i % 32) & 1u)) {
      const uint32_t pins = pinned_to(i) - pinned_below;
      if (held) a.src[i - used - (at - holes) - pins] = i;          // behind the held pages above that move before it
      a.free_pages[(holes - moves) + (i - used) - pins] = i;
    }
  }
  // The entries behind the lists.
  for (int i = (int)blockIdx.x * share + tid; i < end; i += kOneThreads) {
    if (i >= (int)free_all) a.free_pages[i] = -1;
    if (COMPACT && i < pages / 2 && i >= (int)moves) a.src[i] = a.dst[i] = -1;
  }
  if (blockIdx.x == 0 && tid == 0) {
    *a.count = (int32_t)free_all;
    if (COMPACT) *a.moved = (int32_t)moves;
  }
  if (!COMPACT) return;
  // The rows, a stretch for a wavefront of the grid in turn.
  for (int t = (int)blockIdx.x * kOneWaves + wave; t < tasks; t += (int)gridDim.x * kOneWaves) {
    const int row = t / stretches, c = (t - row * stretches) * 64 + lane;
    if (c >= stride) continue;
    int32_t page = a.table[(int64_t)row * stride + c];
    if (c < (int)lds.row_pages[row] && page >= used && page < pages && !(lds.pinned[page / 32] >> (page % 32) & 1u)) {
      const uint32_t k = page - used - (free_to(page) - holes) - (pinned_to(page) - pinned_below);
      int lo = 0, hi = words - 1;               // the word that hole k lies in: the last with at most k free pages before it
      while (lo < hi) {
        const int mid = (lo + hi + 1) / 2;
        if (lds.free_before[mid] <= k) lo = mid;
        else hi = mid - 1;
      }
      uint32_t bits = ~lds.held[lo];
      for (uint32_t n = k - lds.free_before[lo]; n != 0; --n) bits &= bits - 1;
      page = 32 * lo + __builtin_ctz(bits);
    }
    a.table_out[(int64_t)row * stride + c] = page;
  }
}

Pools pools_in(void* workspace, int64_t pages, bool compact, size_t* bytes) {
  Pools s = {};
  s.blocks = max((pages + kBlockPages - 1) / kBlockPages, (int64_t)1);        // one where there is no page: the count is still written
  uint8_t* p = static_cast<uint8_t*>(workspace);
  size_t at = 0;
  auto take = [&](size_t n) {
    uint8_t* q = p != nullptr ? p + at : nullptr;
    at += (n + 255) / 256 * 256;
    return q;
  };
  s.marks = take((size_t)s.blocks * kBlockPages);
  s.counts = reinterpret_cast<uint2*>(take((size_t)s.blocks * sizeof(uint2)));
  if (compact) {
    s.list = reinterpret_cast<int32_t*>(take((size_t)pages * 4));
    s.to = reinterpret_cast<int32_t*>(take((size_t)pages * 4));
  }
  *bytes = at;
  return s;
}

// --- copy --------------------------------------------------------------------------------------

constexpr int kPieces = 2, kChunk = 16 * kThreads * kPieces;      // bytes of a page that a workgroup takes at a time
constexpr int64_t kCopyGroups = 1 << 16;

struct Arrays {
  uint8_t* p[kCopyArrays];
};

// A row of the grid is an array.  Streaming loads and stores of small chunks: 199 pages of 74 KB in 32 arrays (939 MB read and
// written) 167 us, 180 with cached ones, 168 to 171 and 181 in chunks of 16 KB.
__global__ __launch_bounds__(kThreads) void page_copy_kernel(const Arrays arrays, const int32_t* src, const int32_t* dst, int64_t entries,
                                                             int64_t pages, int64_t page_bytes, uint32_t chunks) {
  const uint32_t first = blockIdx.x / chunks, chunk = blockIdx.x - first * chunks;
  const int64_t at = (int64_t)chunk * kChunk + 16 * threadIdx.x, step = gridDim.x / chunks;
  uint8_t* base = arrays.p[blockIdx.y] + at;
  for (int64_t entry = first; entry < entries; entry += step) {
    const int64_t from = src[entry], to = dst[entry];
    if (from < 0 || to < 0 || from >= pages || to >= pages || from == to) continue;
    u32x4 d[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      if (at + 16 * kThreads * i < page_bytes) d[i] = load_stream16(base + from * page_bytes + 16 * kThreads * i);
#pragma unroll
    for (int i = 0; i < kPieces; ++i)
      if (at + 16 * kThreads * i < page_bytes) __builtin_nontemporal_store(d[i], reinterpret_cast<u32x4*>(base + to * page_bytes + 16 * kThreads * i));
  }
}

}  // namespace

hipError_t launch_page_fork(const PageFork& a, hipStream_t stream) {
  const int64_t groups = max((int64_t)1, (a.requests + kForkRows - 1) / kForkRows);
  page_fork_kernel<<<dim3((unsigned)groups), kForkThreads, (size_t)(4 * a.rows), stream>>>(a);
  return hipGetLastError();
}

size_t page_collect_workspace_bytes(int64_t pages, bool compact) {
  size_t bytes;
  pools_in(nullptr, pages, compact, &bytes);
  return bytes;
}

hipError_t launch_page_collect(const PageCollect& a, bool compact, void* workspace, hipStream_t stream) {
  size_t bytes;
  const Pools s = pools_in(workspace, a.pages, compact, &bytes);
  const dim3 blocks((unsigned)s.blocks);
  const int64_t row_groups = (a.stride + 4 * kThreads - 1) / (4 * kThreads);
  const dim3 rows((unsigned)(a.requests * row_groups));
  const int share = (int)max((int64_t)kOneShare, (a.pages + kOneGroups - 1) / kOneGroups);
  const dim3 groups((unsigned)max((a.pages + share - 1) / share, (int64_t)1));
  const bool few = a.pages <= kOnePages && a.requests <= kOneRows;
  // in place, rows would be renamed while other workgroups still mark
  if (few && a.requests * a.stride <= kOneEntries && !(compact && a.table_out == a.table && a.stride > 0)) {
    if (compact) pool_kernel<true, false><<<groups, kOneThreads, 0, stream>>>(a, nullptr, share);
    else pool_kernel<false, false><<<groups, kOneThreads, 0, stream>>>(a, nullptr, share);
    return hipGetLastError();
  }
  clear_kernel<<<blocks, kThreads, 0, stream>>>(a, s);
  if (rows.x > 0) mark_kernel<<<rows, kThreads, 0, stream>>>(a, s, row_groups);
  if (few) {
    if (compact) pool_kernel<true, true><<<groups, kOneThreads, 0, stream>>>(a, s.marks, share);
    else pool_kernel<false, true><<<groups, kOneThreads, 0, stream>>>(a, s.marks, share);
    return hipGetLastError();
  }
  count_kernel<<<blocks, kThreads, 0, stream>>>(a, s);
  if (!compact) {
    list_kernel<<<blocks, kThreads, 0, stream>>>(a, s, a.free_pages, true);
    return hipGetLastError();
  }
  list_kernel<<<blocks, kThreads, 0, stream>>>(a, s, s.list, false);
  move_kernel<<<blocks, kThreads, 0, stream>>>(a, s);
  free_after_kernel<<<blocks, kThreads, 0, stream>>>(a, s);
  if (rows.x > 0) rename_kernel<<<rows, kThreads, 0, stream>>>(a, s, row_groups);
  return hipGetLastError();
}

hipError_t launch_page_copy(uint8_t* const* arrays, int count, const int32_t* src, const int32_t* dst, int64_t entries, int64_t pages,
                            int64_t page_bytes, hipStream_t stream) {
  const int64_t chunks = (page_bytes + kChunk - 1) / kChunk;
  for (int first = 0; first < count; first += kCopyArrays) {
    Arrays some = {};
    const int n = min(count - first, kCopyArrays);
    for (int i = 0; i < n; ++i) some.p[i] = arrays[first + i];
    const int64_t together = min(entries, max((int64_t)1, kCopyGroups / (chunks * n)));        // entries that have workgroups of their own
    page_copy_kernel<<<dim3((unsigned)(together * chunks), (unsigned)n), kThreads, 0, stream>>>(some, src, dst, entries, pages, page_bytes, (uint32_t)chunks);
  }
  return hipGetLastError();
}

}  // namespace ssq
