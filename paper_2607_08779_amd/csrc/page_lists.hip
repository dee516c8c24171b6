// What a paged cache's tables and pools need between steps: requests that continue others (fork), the pages
// that nobody holds (collect), held pages brought to the front (compact), and copies of pages
// (see include/ssq_cache.h).
//
// Fork, collect and compact move a few bytes for each table entry and page, so that launches and latency
// bound them.  Fork is one launch: every workgroup finds for itself how many pages the rows before its
// own take, as page_tables.hip does.  Collect and compact mark held pages with plain byte stores
// (any order gives the same marks), count them for each block of pages, and write lists whose
// places follow from the counts.  A copy is bound by the pages' bytes, read and written.
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

constexpr int kChunk = 16 * kThreads * 4;                  // bytes of a page that a workgroup takes at a time
constexpr int64_t kCopyGroups = 1 << 16;

struct Arrays {
  uint8_t* p[kCopyArrays];
};

__global__ __launch_bounds__(kThreads) void page_copy_kernel(const Arrays arrays, int count, const int32_t* src, const int32_t* dst,
                                                             int64_t entries, int64_t pages, int64_t page_bytes, int64_t chunks) {
  const int64_t work = entries * count * chunks;
  for (int64_t w = blockIdx.x; w < work; w += gridDim.x) {
    const int64_t entry = w / (count * chunks), rest = w - entry * (count * chunks);
    const int64_t from = src[entry], to = dst[entry];
    if (from < 0 || to < 0 || from >= pages || to >= pages || from == to) continue;
    const int64_t array = rest / chunks, at = (rest - array * chunks) * kChunk;
    uint8_t* base = arrays.p[array];
    const int bytes = (int)min(page_bytes - at, (int64_t)kChunk);
    u32x4 d[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int o = 16 * (i * kThreads + (int)threadIdx.x);
      if (o < bytes) d[i] = *reinterpret_cast<const u32x4*>(base + from * page_bytes + at + o);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int o = 16 * (i * kThreads + (int)threadIdx.x);
      if (o < bytes) *reinterpret_cast<u32x4*>(base + to * page_bytes + at + o) = d[i];
    }
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
  clear_kernel<<<blocks, kThreads, 0, stream>>>(a, s);
  if (rows.x > 0) mark_kernel<<<rows, kThreads, 0, stream>>>(a, s, row_groups);
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
    const int64_t work = entries * n * chunks;
    page_copy_kernel<<<dim3((unsigned)min(work, kCopyGroups)), kThreads, 0, stream>>>(some, n, src, dst, entries, pages, page_bytes, chunks);
  }
  return hipGetLastError();
}

}  // namespace ssq
