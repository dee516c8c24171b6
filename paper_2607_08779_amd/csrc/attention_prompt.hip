// Causal attention over whole prompts, packed, grouped heads (see
// include/ssq_attention.h).
//
// A workgroup of four wavefronts takes 128 query rows of one key/value head: the tokens of a
// stretch of one sequence times the heads of the group, token by token, so that the group's
// heads share every key and value that is loaded and the causal edge is one tile wide.  It
// walks the stretch's keys 64 at a time through two stages of LDS, the next tile on its way
// while this one is used.  Two workgroups share a CU, so that one's softmax runs beside the
// other's products.
//
// Bound by arithmetic.  One prompt of 16384 tokens (32/8 heads of 128) takes 1.95 to 2.0 ms by card,
// 1100 to 1130 TFLOP/s of the causal half, where a matrix product of 8192^3 random values reaches 1200: at both the
// card's power sets the clock (1.5 to 1.6 GHz here; the matrix cores are busy in 60 % of its cycles).
// Eight prompts of 300 to 2048 tokens (64/8 heads) take 250 us, 856 TFLOP/s: a workgroup's tiles
// take 1.57 us each, and looking up its place, its first loads, its edge and its end 6.8.
// Measured and not taken: wavefronts of 64 rows with half the reads of LDS (280 us: nothing
// beside a SIMD's one wavefront hides its start and end), the next tile's scores formed beside
// this one's weights (254), priorities of products or of the softmax (255).
#include <algorithm>
#include <type_traits>

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
template <int ROWS>
__device__ __forceinline__ bool find_tile(const int32_t* starts, int requests, int tokens, int group, int* rank, Place* at) {
  const int lane = threadIdx.x & 63;
  for (int r0 = 0; r0 < requests; r0 += 64) {
    const int r = r0 + lane;
    int begin = 0, end = 0;
    if (r < requests) {
      begin = min(max(starts[r], 0), tokens);
      end = max(min(starts[r + 1], tokens), begin);
    }
    const int tiles = ((end - begin) * group + ROWS - 1) / ROWS;
    int sum = tiles;                                   // with those of the lanes before it: DPP row shifts and broadcasts
    sum += __builtin_amdgcn_update_dpp(0, sum, 0x111, 0xF, 0xF, true);
    sum += __builtin_amdgcn_update_dpp(0, sum, 0x112, 0xF, 0xF, true);
    sum += __builtin_amdgcn_update_dpp(0, sum, 0x114, 0xF, 0xF, true);
    sum += __builtin_amdgcn_update_dpp(0, sum, 0x118, 0xF, 0xF, true);
    sum += __builtin_amdgcn_update_dpp(0, sum, 0x142, 0xA, 0xF, true);
    sum += __builtin_amdgcn_update_dpp(0, sum, 0x143, 0xC, 0xF, true);
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

// Workgroups past the last tile clear the padding, the tokens behind the last sequence.
template <typename T, int D, int ROWS>
__device__ __forceinline__ void clear_padding(const Prompt<T>& a, int group, int head, int rank) {
  constexpr int kChunks = Shape<T, D>::kChunks;
  const int last = a.requests > 0 ? min(max(a.starts[a.requests], 0), (int)a.tokens) : 0;
  const int rows = (int)(a.tokens - last) * group;
  for (int i = threadIdx.x; i < ROWS * kChunks; i += kThreads) {
    const int row = rank * ROWS + i / kChunks;
    if (row < rows)
      *reinterpret_cast<u32x4*>(a.out.p + (last + row / group) * a.out.stride + (head * group + row % group) * D + i % kChunks * (16 / (int)sizeof(T))) = u32x4{0u, 0u, 0u, 0u};
  }
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads, 2) void prompt_kernel(const Prompt<T> a, int group) {
  using S = Shape<T, D>;
  constexpr int kTile = kTileKeys * S::kRow;
  __shared__ __align__(1024) uint8_t lds[4 * kTile];
  __shared__ int spoiled;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = (int)blockIdx.x % a.kv_heads;
  int rank = (int)blockIdx.x / a.kv_heads;
  Place at;
  if (!find_tile<kTileRows>(a.starts, (int)a.requests, (int)a.tokens, group, &rank, &at)) return clear_padding<T, D, kTileRows>(a, group, head, rank);
  // longest rows first: what is left at the end of the grid is short
  const int row0 = (at.tiles - 1 - at.tile) * kTileRows, rows = (at.end - at.begin) * group;
  const int row = row0 + 32 * wave + (lane & 31);
  const bool present = row < rows;
  const int token = row / group;                       // within the sequence: the last key that the row sees
  const int64_t line = at.begin + token, column = (head * group + row - token * group) * D;
  const int last = present ? token : -1;
  const int wave_row = row0 + 32 * wave;
  const int wave_first = __builtin_amdgcn_readfirstlane(wave_row / group);                                        // seen by every row
  const int wave_last = __builtin_amdgcn_readfirstlane(wave_row < rows ? (min(wave_row + 32, rows) - 1) / group : -1);
  const int keys = __builtin_amdgcn_readfirstlane((min(row0 + kTileRows, rows) - 1) / group + 1);                 // that some row sees

  Rows32<T, D> r;
  r.load_query(a.q.p + line * a.q.stride + column, present, lane);
  const Loader<T, D> load_k(lane, (uint32_t)(sizeof(T) * a.k.stride)), load_v(lane, (uint32_t)(sizeof(T) * a.v.stride));
  const float scale = a.scale * kLog2e;

  auto walk = [&](auto careful) {
    int k_at = 16 * wave, v_at = k_at;                 // this wavefront's 16 keys of the next tile
    const T *kp = a.k.p + (at.begin + k_at) * a.k.stride + head * D, *vp = a.v.p + (at.begin + v_at) * a.v.stride + head * D;
    auto bytes = [&](int at, int64_t stride) { return at < keys ? (uint32_t)(sizeof(T) * ((min(keys - at, 16) - 1) * (uint32_t)stride + D)) : 0u; };
    walk_shared<decltype(careful)::value>(
        r, lds, (keys + kTileKeys - 1) / kTileKeys, wave_last < 0 ? 0 : wave_last / kTileKeys + 1, scale, lane, [](int) {},
        [&](uint8_t* to) {
          load_k.keys(describe(kp, bytes(k_at, a.k.stride)), to + wave * S::kGroup);
          kp += kTileKeys * a.k.stride;
          k_at += kTileKeys;
        },
        [&](uint8_t* to) {
          load_v.values(describe(vp, bytes(v_at, a.v.stride)), to + wave * S::kGroup);
          vp += kTileKeys * a.v.stride;
          v_at += kTileKeys;
        },
        [&](int t) { return kTileKeys * t + kTileKeys - 1 > wave_first; },
        [&](int t, f32x16 (&s)[2]) { return Rows32<T, D>::template mask<2>(s, 0, last - kTileKeys * t, 0u, lane); },
        [&](int t) { return last - kTileKeys * t; });
  };
  if (threadIdx.x == 0) spoiled = 0;
  walk(std::false_type{});
  // An infinite or NaN value can have reached rows of its tile that do not see it: then once
  // more, in edge tiles such values apart and key by key.
  if (present && r.spoiled()) spoiled = 1;
  __syncthreads();
  if (spoiled != 0) walk(std::true_type{});
  r.store(a.out.p + line * a.out.stride + column, present, inverse_of(sum_across(r.l)), lane);
}

// 32 rows a workgroup, whose wavefronts share out the keys.
template <typename T, int D>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void prompt_small_kernel(const Prompt<T> a, int group) {
  using S = Shape<T, D>;
  __shared__ __align__(1024) uint8_t lds[kWaves * 64 * S::kRow];
  __shared__ float2 ml[kWaves * 32];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int head = (int)blockIdx.x % a.kv_heads;
  int rank = (int)blockIdx.x / a.kv_heads;
  Place at;
  if (!find_tile<32>(a.starts, (int)a.requests, (int)a.tokens, group, &rank, &at)) return clear_padding<T, D, 32>(a, group, head, rank);
  const int row0 = (at.tiles - 1 - at.tile) * 32, rows = (at.end - at.begin) * group;
  const int row = row0 + (lane & 31), token = row / group;
  const bool present = row < rows;
  const int last = present ? token : -1;
  const int first = __builtin_amdgcn_readfirstlane(row0 / group);                           // seen by every row
  const int keys = __builtin_amdgcn_readfirstlane((min(row0 + 32, rows) - 1) / group + 1);  // that some row sees
  Rows32<T, D> r;
  r.load_query(a.q.p + (at.begin + token) * a.q.stride + (head * group + row - token * group) * D, present, lane);
  const Loader<T, D> load_k(lane, (uint32_t)(sizeof(T) * a.k.stride)), load_v(lane, (uint32_t)(sizeof(T) * a.v.stride));
  auto walk = [&](auto careful) {
    r.start(lane);
    walk_private<decltype(careful)::value>(r, lds, load_k, load_v, wave, kWaves, 0, keys, first, last, a.scale * kLog2e, lane, [&](int j) {
      const int count = min(keys - j, 16);
      auto bytes = [&](int64_t stride) { return count > 0 ? (uint32_t)(sizeof(T) * ((count - 1) * (uint32_t)stride + D)) : 0u; };
      return Group<T>{a.k.p + (at.begin + j) * a.k.stride + head * D, a.v.p + (at.begin + j) * a.v.stride + head * D, bytes(a.k.stride), bytes(a.v.stride), false};
    });
  };
  walk(std::false_type{});
  if (__builtin_amdgcn_ballot_w64(present && r.spoiled()) != 0) walk(std::true_type{});
  join_waves<kWaves>(r, lds, ml, min(rows - row0, 32), wave, lane, [&](int of, int d, f32x4 o, float, float l) {
    const float by = inverse_of(l);
    const int index = row0 + of, t = index / group;
    T* to = a.out.p + (at.begin + t) * a.out.stride + (head * group + index - t * group) * D + d;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2*>(to) = u32x2{pack_bf16x2(o[0] * by, o[1] * by), pack_bf16x2(o[2] * by, o[3] * by)};
    else *reinterpret_cast<f32x4*>(to) = f32x4{o[0] * by, o[1] * by, o[2] * by, o[3] * by};
  });
}

template <typename T>
int64_t small_groups(const Prompt<T>& a, int group) { return ((a.tokens * group + 31) / 32 + a.requests) * a.kv_heads; }
template <typename T, int D>
void launch_small(const Prompt<T>& a, int group, hipStream_t stream) {
  prompt_small_kernel<T, D><<<dim3((unsigned)small_groups(a, group)), kThreads, 0, stream>>>(a, group);
}

// Binary32 products take 16 times as long as bf16's, so that a workgroup of 128 rows is long and
// there are few: 32 rows a workgroup, its wavefronts sharing out the keys.
template <int D>
void launch_kernel(const Prompt<float>& a, int group, hipStream_t stream) {
  launch_small<float, D>(a, group, stream);
}

// In bf16 that form loads each key four times as often.  It pays where its workgroups are few and
// sequences are long for their number, as with the few key/value heads of a small model or of a
// shard: there a row tile's time is one walk over its keys, which the wavefronts then share.  The bound
// of 768 workgroups is between what was measured to gain and to lose, for both head sizes (of 128
// two are resident on a CU, of 64 four).  us, 128 rows -> 32 rows a workgroup, one sequence:
//   2 kv heads of 128, group 4: 400 tokens 10.7 -> 9.7, 1000 20.1 -> 13.5, 3000 49.8 -> 36.8
//   4 kv heads of 128, group 4: 1400 tokens (704 workgroups) 26.2 -> 24.5; 2000 (1004) 35.4 -> 36.7: not taken
//   8 kv heads of 128, group 4: 400 tokens 11.1 -> 11.5, 1000 21.4 -> 26.5: not taken
//   8 kv heads of 64, group 1: 100 tokens 5.5 -> 4.9, 1000 14.9 -> 9.6
//   8 kv heads of 64, group 4: 700 tokens (704) 11.6 -> 10.1; 1000 (1008) 15.3 -> 17.4: not taken
// and short sequences (16 of 47 tokens in the mean, 2 kv heads of 128: 6.2 -> 7.2) lose.
template <int D>
bool prefers_small(const Prompt<uint16_t>& a, int group) {
  if (a.requests == 0) return false;
  const int64_t groups = small_groups(a, group), mean = a.tokens / a.requests;
  constexpr int64_t kMost = 768;
  return D == 64 ? mean >= 96 && groups <= std::min(kMost, mean * 8 / 7) : mean >= 320 && groups <= std::min(kMost, mean);
}
template <int D>
void launch_kernel(const Prompt<uint16_t>& a, int group, hipStream_t stream) {
  if (prefers_small<D>(a, group)) return launch_small<uint16_t, D>(a, group, stream);
  const int64_t tiles = (a.tokens * group + kTileRows - 1) / kTileRows + a.requests;
  prompt_kernel<uint16_t, D><<<dim3((unsigned)(tiles * a.kv_heads)), kThreads, 0, stream>>>(a, group);
}

template <typename T>
hipError_t launch(const Prompt<T>& a, int head_dim, hipStream_t stream) {
  const int group = a.q_heads / a.kv_heads;
  if (head_dim == 64) launch_kernel<64>(a, group, stream);
  else launch_kernel<128>(a, group, stream);
  return hipGetLastError();
}

}  // namespace
}  // namespace attention

hipError_t launch_attention_prompt(const Prompt<uint16_t>& a, int head_dim, hipStream_t stream) { return attention::launch(a, head_dim, stream); }
hipError_t launch_attention_prompt(const Prompt<float>& a, int head_dim, hipStream_t stream) { return attention::launch(a, head_dim, stream); }

}  // namespace ssq
