// Page tables, slots and positions of one step's new tokens (see include/ssq_attention.h).
//
// Two running sums over the requests (tokens added, pages needed), and for each token and
// each new page the request it belongs to, found in those sums.  Nothing but a few bytes per
// token moves, so what bounds it is latency: one launch, in which every workgroup forms the
// sums for itself (1024 requests at a time, in LDS) instead of waiting for another's, then
// takes its share of the tokens and of the new pages and finds their requests by bisection.
// 64 requests of one token: 3.7 us of graph time, a launch by itself 2.7; 256 prompts of up to
// 2048 tokens: 8 us.
#include "attention_internal.h"

namespace ssq {
namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 4 * kThreads;        // requests summed at a time
constexpr int kTokens = 1024;               // tokens of a workgroup

struct Tables {
  const int32_t* held;
  const int32_t* added;
  const int32_t* free_pages;
  const int32_t* taken;
  int32_t* table;
  int32_t* starts;
  int32_t* lens;
  int32_t* positions;
  int32_t* slots;
  int32_t* taken_after;
  int64_t requests, free_count, table_stride, tokens;
  int shift;
};

// Sums of v over the workgroup's threads before this one; *all is the sum of every thread.
__device__ __forceinline__ uint2 sums_before(uint2 v, uint2* wave_sums, uint2* all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint2 s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t x = __shfl_up(s.x, o, 64), y = __shfl_up(s.y, o, 64);
    if (lane >= o) s.x += x, s.y += y;
  }
  if (lane == 63) wave_sums[wave] = s;
  __syncthreads();
  uint2 before = {s.x - v.x, s.y - v.y}, sum = {0u, 0u};
#pragma unroll
  for (int w = 0; w < kThreads / 64; ++w) {
    const uint2 t = wave_sums[w];
    if (w < wave) before.x += t.x, before.y += t.y;
    sum.x += t.x, sum.y += t.y;
  }
  *all = sum;
  return before;
}

// The last of a chunk's ascending sums that is at most x (sums[0] is).
__device__ __forceinline__ int last_at_most(const uint32_t* sums, int count, uint32_t x) {
  int lo = 0, hi = count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (sums[mid] <= x) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

__global__ __launch_bounds__(kThreads) void page_tables_kernel(const Tables a) {
  __shared__ uint32_t start[kChunk], first[kChunk], held_of[kChunk];
  __shared__ uint2 wave_sums[kThreads / 64];
  const int tid = threadIdx.x;
  const uint32_t round = (1u << a.shift) - 1u;
  const uint32_t taken = a.taken != nullptr ? (uint32_t)*a.taken : 0u;
  const uint32_t t_lo = (uint32_t)blockIdx.x * kTokens;
  const uint32_t t_hi = (uint32_t)min(a.tokens, (int64_t)t_lo + kTokens);
  uint2 base = {0u, 0u};                     // tokens and new pages of the chunks before

  auto new_page = [&](uint32_t x) {          // entry x of the pages needed, counted from *taken
    const int64_t i = (int64_t)(int32_t)(taken + x);
    return i >= 0 && i < a.free_count ? a.free_pages[i] : -1;
  };

  for (int64_t r0 = 0; r0 < a.requests || r0 == 0; r0 += kChunk) {
    const int count = (int)min(a.requests - r0, (int64_t)kChunk);
    uint32_t held[4], len[4];
    uint2 own = {0u, 0u}, part[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 4 * tid + i;
      const bool in = r < count;
      held[i] = in ? (uint32_t)max(a.held[r0 + r], 0) : 0u;
      len[i] = held[i] + (in ? (uint32_t)max(a.added[r0 + r], 0) : 0u);
      part[i] = own;
      own.x += len[i] - held[i];
      own.y += ((len[i] + round) >> a.shift) - ((held[i] + round) >> a.shift);
    }
    uint2 all;
    const uint2 before = sums_before(own, wave_sums, &all);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 4 * tid + i;
      start[r] = base.x + before.x + part[i].x;
      first[r] = base.y + before.y + part[i].y;
      held_of[r] = held[i];
      if (r < count && (uint32_t)(r0 / kChunk) % gridDim.x == blockIdx.x) {
        a.starts[r0 + r] = (int32_t)start[r];
        a.lens[r0 + r] = (int32_t)len[i];
      }
    }
    __syncthreads();
    // new pages of these requests, a stretch of kThreads for each workgroup in turn
    for (uint64_t x0 = (uint64_t)blockIdx.x * kThreads; x0 < all.y; x0 += (uint64_t)gridDim.x * kThreads) {
      const uint32_t x = base.y + (uint32_t)x0 + tid;
      if (x - base.y >= all.y) continue;
      const int r = last_at_most(first, count, x);
      const int64_t j = (int64_t)((held_of[r] + round) >> a.shift) + (x - first[r]);
      if (j < a.table_stride) a.table[(r0 + r) * a.table_stride + j] = new_page(x);
    }
    // tokens of these requests that are this workgroup's
    const uint32_t lo = max(t_lo, base.x), hi = min(t_hi, base.x + all.x);
    for (uint32_t t = lo + tid; t < hi; t += kThreads) {
      const int r = last_at_most(start, count, t);
      const uint32_t at = held_of[r] + (t - start[r]);
      const uint32_t have = (held_of[r] + round) >> a.shift, j = at >> a.shift;
      int32_t page = -1;
      if ((int64_t)j < a.table_stride)
        page = j < have ? a.table[(r0 + r) * a.table_stride + j] : new_page(first[r] + (j - have));
      const int64_t slot = ((int64_t)page << a.shift) + (at & round);
      a.positions[t] = (int32_t)at;
      a.slots[t] = page >= 0 && slot <= 0x7fffffff ? (int32_t)slot : -1;
    }
    base.x += all.x;
    base.y += all.y;
    __syncthreads();                         // the sums are overwritten next
  }
  for (uint32_t t = max(t_lo, base.x) + tid; t < t_hi; t += kThreads) {
    a.positions[t] = 0;
    a.slots[t] = -1;
  }
  if (blockIdx.x == 0 && tid == 0) {
    a.starts[a.requests] = (int32_t)base.x;
    *a.taken_after = (int32_t)(taken + base.y);
  }
}

}  // namespace

hipError_t launch_page_tables(const int32_t* held, const int32_t* added, int64_t requests, const int32_t* free_pages,
                              int64_t free_count, const int32_t* taken, int page_shift, int32_t* table,
                              int64_t table_stride, int64_t tokens, int32_t* starts, int32_t* lens, int32_t* positions,
                              int32_t* slots, int32_t* taken_after, hipStream_t stream) {
  const Tables a = {held, added, free_pages, taken, table, starts, lens, positions, slots, taken_after, requests, free_count, table_stride, tokens, page_shift};
  const int64_t groups = max((int64_t)1, (tokens + kTokens - 1) / kTokens);
  page_tables_kernel<<<dim3((unsigned)groups), kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace ssq
