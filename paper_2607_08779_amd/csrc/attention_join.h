// What the decode kernels share: where rows of the requests' new tokens lie, and the parts of a row that
// several workgroups leave, joined by a launch of their own.
//
// Parts leave O unnormalised in binary32 with its reference and sum, and are joined as
//   out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s,   M = max_s m_s.
#pragma once

#include <algorithm>
#include <type_traits>

#include "attention_tiles.h"

namespace ssq {
namespace attention {
namespace {

constexpr int kMaxParts = 64, kJoinThreads = 256;
constexpr int64_t kWaveJoinRows = 1536;               // rows of out from which a wavefront joins a row

inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct Parts {           // of every row: [part][row] and [part][row][D]
  float2* ml;            // null: one part, straight to out
  float* o;
};

// Rows of this wavefront: lane's column, where it goes and the last key it sees.
struct Row {
  bool present;
  int64_t line;          // row of q and out
  int column;            // head
  int last;
};

template <typename T>
__device__ __forceinline__ int request_len(const Decode<T>& a, int request) {
  const int64_t room = min(a.max_len, a.table_stride << a.cache.page_shift);
  return (int)min((int64_t)max(a.lens[request], 0), room);
}

// Four consecutive outputs of a row, of one part or of all.
template <typename T, int D>
__device__ __forceinline__ void put(const Decode<T>& a, int64_t line_rows, const Parts& parts, int part, const Row& row,
                                    int at, f32x4 o, float m, float l) {
  if (parts.ml == nullptr) {
    const float by = inverse_of(l);
    T* to = a.out.p + row.line * a.out.stride + row.column * D + at;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2*>(to) = u32x2{pack_bf16x2(o[0] * by, o[1] * by), pack_bf16x2(o[2] * by, o[3] * by)};
    else *reinterpret_cast<f32x4*>(to) = f32x4{o[0] * by, o[1] * by, o[2] * by, o[3] * by};
  } else {
    const int64_t r = part * line_rows + row.line * a.q_heads + row.column;
    *reinterpret_cast<f32x4*>(parts.o + r * D + at) = o;
    if (at == 0) parts.ml[r] = float2{m, l};
  }
}

// One row of out from its parts, by R lanes, a wavefront or a workgroup of them: D / 4 lanes hold the
// row, and the groups of so many lanes take the parts in turn, so that their loads are under way
// together.
template <typename T, int D, int R>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(const Decode<T> a, int64_t line_rows, int count, const Parts parts) {
  constexpr int kLanes = D / 4, kGroups = R / kLanes;
  const int lane = threadIdx.x & 63, at = (int)threadIdx.x % kLanes, group = (int)threadIdx.x % R / kLanes;
  const int64_t row = blockIdx.x * (int64_t)(kJoinThreads / R) + threadIdx.x / R;
  if (row >= line_rows) return;               // whole wavefronts; none where a workgroup holds a row
  const float* from = parts.o + row * D + 4 * at;
  constexpr int kAhead = R == 64 ? 8 : 4;
  f32x4 o[kAhead];
#pragma unroll
  for (int i = 0; i < kAhead; ++i) {
    const int s = group + i * kGroups;
    o[i] = s < count ? *reinterpret_cast<const f32x4*>(from + s * line_rows * D) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  // every wavefront forms the parts' weights, for itself
  const float2 x = lane < count ? parts.ml[lane * line_rows + row] : float2{-FLT_MAX, __uint_as_float(kSawNone)};
  const float m = wave_max(x.y != 0.0f ? x.x : -FLT_MAX);
  const float by = x.y != 0.0f ? __builtin_amdgcn_exp2f(x.x - m) : 0.0f;
  float l = wave_sum(by * x.y);
  if (l == 0.0f && __builtin_amdgcn_ballot_w64(__float_as_uint(x.y) != kSawNone) == 0) l = __uint_as_float(kSawNone);
  f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int i = 0; i < kMaxParts / kGroups; ++i) {
    const int s = group + i * kGroups;
    if (i * kGroups >= count) break;
    const float w = __shfl(by, s, 64);
    const f32x4 y = i < kAhead ? o[i] : s < count ? *reinterpret_cast<const f32x4*>(from + s * line_rows * D) : f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] = __builtin_fmaf(w, y[e], sum[e]);
  }
  if constexpr (R == 64) {
#pragma unroll
    for (int d = kLanes; d < 64; d <<= 1)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += __shfl_xor(sum[e], d, 64);
  } else {
    __shared__ f32x4 sums[kGroups][kLanes];
    sums[group][at] = sum;
    __syncthreads();
    if (group != 0) return;
#pragma unroll
    for (int g = 1; g < kGroups; ++g)
#pragma unroll
      for (int e = 0; e < 4; ++e) sum[e] += sums[g][at][e];
  }
  if (group != 0) return;
  const int64_t line = row / a.q_heads;
  const Row to = {true, line, (int)(row - line * a.q_heads), 0};
  put<T, D>(a, 0, Parts{nullptr, nullptr}, 0, to, 4 * at, sum, 0.0f, l);
}

// Bytes of `count` parts of every row, and their place in a workspace of as many.
size_t parts_bytes(int count, int64_t line_rows, int head_dim) {
  return count > 1 ? (size_t)count * (size_t)line_rows * (8 + 4 * (size_t)head_dim) : 0;
}
template <int D>
Parts place_parts(void* workspace, int count, int64_t line_rows) {
  float* o = static_cast<float*>(workspace);
  return {reinterpret_cast<float2*>(o + (size_t)count * line_rows * D), o};
}

// A wavefront a row where the rows fill the chip (2560 rows of 7 parts: a step of 20.3 us against
// 21.2 with a workgroup a row), a workgroup a row where they do not (32 rows of 32 parts: 18.9
// against 21.9; equal at about 1000 rows).
template <typename T, int D>
void launch_join(const Decode<T>& a, int64_t line_rows, int count, const Parts& parts, hipStream_t stream) {
  constexpr int kPerGroup = kJoinThreads / 64;
  if (line_rows >= kWaveJoinRows) join_kernel<T, D, 64><<<dim3((unsigned)((line_rows + kPerGroup - 1) / kPerGroup)), kJoinThreads, 0, stream>>>(a, line_rows, count, parts);
  else join_kernel<T, D, kJoinThreads><<<dim3((unsigned)line_rows), kJoinThreads, 0, stream>>>(a, line_rows, count, parts);
}

}  // namespace
}  // namespace attention
}  // namespace ssq
