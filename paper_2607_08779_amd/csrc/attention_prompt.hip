// Causal attention over whole prompts, packed, grouped heads (see
// include/ssq_attention.h).
//
// A workgroup of four wavefronts takes 128 query rows of one key/value head: the tokens of a
// stretch of one sequence times the heads of the group, token by token, so that the group's
// heads share every key and value that is loaded and the causal edge is one tile wide.  It
// walks the stretch's keys 64 at a time through two stages of LDS, the next tile on its way
// while this one is used.
#include "attention_tiles.h"

namespace ssq {
namespace attention {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves, kTileRows = 32 * kWaves, kTileKeys = 64;

// The sequence and its tile that stand at `rank` in the list of all tiles of all sequences;
// false past the end, with *rank what is left.
struct Place {
  int begin, end, tile, tiles;
};
__device__ __forceinline__ bool find_tile(const int32_t* starts, int requests, int tokens, int group, int* rank, Place* at) {
  const int lane = threadIdx.x & 63;
  for (int r0 = 0; r0 < requests; r0 += 64) {
    const int r = r0 + lane;
    int begin = 0, end = 0;
    if (r < requests) {
      begin = min(max(starts[r], 0), tokens);
      end = max(min(starts[r + 1], tokens), begin);
    }
    const int tiles = ((end - begin) * group + kTileRows - 1) / kTileRows;
    int sum = tiles;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(sum, o, 64);
      if (lane >= o) sum += x;
    }
    const uint64_t past = __builtin_amdgcn_ballot_w64(sum > *rank);
    if (past != 0) {
      const int found = __builtin_ctzll(past);
      at->begin = __builtin_amdgcn_readlane(begin, found);
      at->end = __builtin_amdgcn_readlane(end, found);
      at->tiles = __builtin_amdgcn_readlane(tiles, found);
      at->tile = *rank - (__builtin_amdgcn_readlane(sum, found) - at->tiles);
      return true;
    }
    *rank -= __builtin_amdgcn_readlane(sum, 63);
  }
  return false;
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void prompt_kernel(const Prompt<T> a, int group) {
  using S = Shape<T, D>;
  constexpr int kTile = kTileKeys * S::kRow;
  __shared__ __align__(1024) uint8_t k0[kTile], v0[kTile], k1[kTile], v1[kTile];
  __shared__ int spoiled;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = (int)blockIdx.x % a.kv_heads;
  int rank = (int)blockIdx.x / a.kv_heads;
  Place at;
  if (!find_tile(a.starts, (int)a.requests, (int)a.tokens, group, &rank, &at)) {
    // workgroups past the last tile clear the padding, tokens behind the last sequence
    const int last = a.requests > 0 ? min(max(a.starts[a.requests], 0), (int)a.tokens) : 0;
    const int rows = (int)(a.tokens - last) * group;
    for (int i = threadIdx.x; i < kTileRows * S::kChunks; i += kThreads) {
      const int row = rank * kTileRows + i / S::kChunks;
      if (row < rows)
        *reinterpret_cast<u32x4*>(a.out.p + (last + row / group) * a.out.stride + (head * group + row % group) * D + i % S::kChunks * (16 / (int)sizeof(T))) = u32x4{0u, 0u, 0u, 0u};
    }
    return;
  }
  // longest rows first: what is left at the end of the grid is short
  const int row0 = (at.tiles - 1 - at.tile) * kTileRows, rows = (at.end - at.begin) * group;
  const int row = row0 + 32 * wave + (lane & 31);
  const bool present = row < rows;
  const int token = row / group;                       // within the sequence: the last key that the row sees
  const int64_t line = at.begin + token, column = (head * group + row - token * group) * D;
  const int last = present ? token : -1;
  const int wave_row = row0 + 32 * wave;
  const int wave_first = wave_row / group;                                        // seen by every row
  const int wave_last = wave_row < rows ? (min(wave_row + 32, rows) - 1) / group : -1;
  const int keys = (min(row0 + kTileRows, rows) - 1) / group + 1;                 // that some row sees

  Rows32<T, D> r;
  r.load_query(a.q.p + line * a.q.stride + column, present, lane);
  const Loader<T, D> load_k(lane, (uint32_t)(sizeof(T) * a.k.stride)), load_v(lane, (uint32_t)(sizeof(T) * a.v.stride));
  const float scale = a.scale * kLog2e;

  auto fill = [&](int j, uint8_t* k, uint8_t* v) {        // keys j ... j + 63, 16 of them by each wavefront
    const int first = j + 16 * wave, count = min(keys - first, 16);
    const int64_t from = at.begin + first;
    const T *kp = a.k.p + from * a.k.stride + head * D, *vp = a.v.p + from * a.v.stride + head * D;
    load_k.keys(make_rsrc(kp, count > 0 ? (uint32_t)(sizeof(T) * ((count - 1) * a.k.stride + D)) : 0u), k + wave * S::kGroup);
    load_v.values(make_rsrc(vp, count > 0 ? (uint32_t)(sizeof(T) * ((count - 1) * a.v.stride + D)) : 0u), v + wave * S::kGroup);
  };
  auto tile = [&](int j, const uint8_t* k, const uint8_t* v, bool careful) {
    if (j > wave_last) return;
    r.template attend<2>(k, v, j + kTileKeys - 1 > wave_first, 0, last - j, 0u, scale, careful, lane);
  };
  if (threadIdx.x == 0) spoiled = 0;
  for (bool careful = false;; careful = true) {
    r.start(lane);
    fill(0, k0, v0);
    for (int j = 0; j < keys; j += 2 * kTileKeys) {
      wait_vmcnt<0>();
      lds_barrier();
      if (j + kTileKeys < keys) fill(j + kTileKeys, k1, v1);
      tile(j, k0, v0, careful);
      if (j + kTileKeys >= keys) break;
      wait_vmcnt<0>();
      lds_barrier();
      if (j + 2 * kTileKeys < keys) fill(j + 2 * kTileKeys, k0, v0);
      tile(j + kTileKeys, k1, v1, careful);
    }
    // An infinite or NaN value can have reached rows of its tile that do not see it: then
    // once more, edge tiles key by key.
    if (careful) break;
    if (present && r.spoiled()) spoiled = 1;
    __syncthreads();
    if (spoiled == 0) break;
  }
  const float l = sum_across(r.l);
  r.store(a.out.p + line * a.out.stride + column, present, l != 0.0f ? 1.0f / l : 0.0f, lane);
}

template <typename T>
hipError_t launch(const Prompt<T>& a, int head_dim, hipStream_t stream) {
  const int group = a.q_heads / a.kv_heads;
  const int64_t tiles = (a.tokens * group + kTileRows - 1) / kTileRows + a.requests;
  const dim3 grid((unsigned)(tiles * a.kv_heads));
  if (head_dim == 64) prompt_kernel<T, 64><<<grid, kThreads, 0, stream>>>(a, group);
  else prompt_kernel<T, 128><<<grid, kThreads, 0, stream>>>(a, group);
  return hipGetLastError();
}

}  // namespace
}  // namespace attention

hipError_t launch_attention_prompt(const Prompt<uint16_t>& a, int head_dim, hipStream_t stream) { return attention::launch(a, head_dim, stream); }
hipError_t launch_attention_prompt(const Prompt<float>& a, int head_dim, hipStream_t stream) { return attention::launch(a, head_dim, stream); }

}  // namespace ssq
