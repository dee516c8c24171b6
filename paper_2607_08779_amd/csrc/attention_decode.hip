// Attention of a few new tokens of each request over the paged cache, with a prefix that all
// requests share (see include/ssq_attention.h).
//
// The cache's bytes are the floor: keys are loaded once for each tile of rows, the prefix for 128
// rows of all requests (32 in binary32), a request's own keys for 32 rows of it.  Two kinds of
// workgroups share one launch, and a second launch joins what they found, where there is more than
// one part:
//
// * wide: 128 query rows (all requests' new tokens and the group's heads) against a stretch
//   of the shared prefix, 64 keys at a time through two stages of LDS that the four
//   wavefronts share.
// * narrow: up to 32 query rows (one request's; or all requests', against the prefix, where they
//   are no more than 32 in all, and in binary32) against a stretch of keys that the four
//   wavefronts take 32 at a time, each through LDS of its own and without barriers: the next
//   keys are loaded as soon as the scores of these are formed, the next values after the
//   product.  In bf16 rows beside the used ones cost nothing that is scarce; in binary32, whose
//   products run at a sixteenth of the rate, they do (one user's 16383 tokens 37 us, 26 of bytes).
//
// Bound by memory where the keys are the requests' own: one user's 16383 tokens (8 heads of 128)
// take 18 us, of which 9.7 are the walk over the keys at 6.9 TB/s, the rest the start, the end and
// the launch that joins.  64 users behind a shared prefix of 8192 tokens, 1 to 1024 of their own,
// take 42 us where the cache lies partly in the Infinity Cache and 49 where it does not (175 MB,
// 3.6 TB/s): workgroups of 2 to 20 us of work on 512 places end unevenly.
//
// Parts leave O unnormalised in binary32 with its reference and sum, and are joined as
//   out = sum_s 2^(m_s - M) O_s / sum_s 2^(m_s - M) l_s,   M = max_s m_s.
#include <algorithm>
#include <type_traits>

#include "attention_tiles.h"

namespace ssq {
namespace attention {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves, kWideRows = 32 * kWaves, kWideKeys = 64, kNarrowRows = 32;
constexpr int kNarrowKeys = 32 * kWaves;              // keys that a narrow workgroup takes at a time
constexpr int kMaxParts = 64;
constexpr int64_t kWaveJoinRows = 1536;               // rows of out from which a wavefront joins a row

enum Share : int { kShareNone = 0, kShareWide, kShareNarrow };

struct Plan {
  int group;             // query heads of a key/value head
  int rows;              // requests * fresh * group: rows of a key/value head
  int share;             // how the prefix is taken
  int prefix_tiles, prefix_parts;
  int own_tiles, own_parts;
  int64_t line_rows;     // requests * fresh * q_heads: rows of out
  int parts() const { return own_parts + (share != kShareNone ? prefix_parts : 0); }
  int64_t prefix_groups() const { return share != kShareNone ? (int64_t)prefix_tiles * prefix_parts : 0; }
};

struct Parts {           // of every row: [part][row] and [part][row][D]
  float2* ml;            // null: one part, straight to out
  float* o;
};

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Parts of the prefix, for `tiles` workgroups a part: the quickest by a fit of its time (us).  A
// tile of 64 keys takes a workgroup 1.1 where it has a CU to itself and 1.57 where it shares one, of
// 512 places in all; a workgroup's start and end take about 4 tiles' time; and every part of a row
// is written and read again.  So parts grow until the CUs have a workgroup each; beyond that, only
// where whole tiles fill them badly (18 x 8 tiles behind 9589 keys, 79 requests of 7 tokens: 3 parts
// 115 us, 2 parts 147, 4 parts 138; 2 x 8 tiles behind 8192 keys: 16 parts 41.8 us, 24 parts 46.3).
// The fit is that of bf16 and tiles of 128 rows.  Binary32 takes the same number of parts, in tiles of 32
// rows, one workgroup a CU in heads of 128, without a fit of its own (16 users behind 4096 tokens 42 us).
int choose_prefix_parts(int64_t tiles, int64_t prefix, int64_t line_rows) {
  const int64_t most = std::min<int64_t>(kMaxParts / 2, ceil_div(prefix, 256));
  int best = 1;
  double best_us = 0.0;
  for (int n = 1; n <= most; ++n) {
    const int64_t groups = tiles * n;
    const double tile_us = groups <= 256 ? 1.1 : 1.57 * (double)ceil_div(groups, 512);
    const double us = tile_us * (double)(ceil_div(ceil_div(prefix, n), kWideKeys) + 4) + 0.25e-3 * (double)(n * line_rows);
    if (n == 1 || us < best_us) best = n, best_us = us;
  }
  return best;
}

Plan make_plan(int64_t requests, int fresh, int q_heads, int kv_heads, int64_t max_len, int64_t prefix, bool split, bool wide) {
  Plan p = {};
  p.group = q_heads / kv_heads;
  p.rows = (int)(requests * fresh * p.group);
  p.line_rows = requests * fresh * q_heads;
  p.own_tiles = (int)ceil_div((int64_t)fresh * p.group, kNarrowRows);
  p.own_parts = 1;
  p.share = kShareNone;
  if (!split) return p;
  constexpr int64_t kGroups = 512;       // two workgroups for each of 256 CUs
  prefix = std::min(prefix, max_len);
  if (requests > 1 && prefix > 0) {
    p.share = p.rows > kNarrowRows && wide ? kShareWide : kShareNarrow;
    p.prefix_tiles = (int)ceil_div(p.rows, p.share == kShareWide ? kWideRows : kNarrowRows);
    p.prefix_parts = choose_prefix_parts(ceil_div(p.rows, kWideRows) * kv_heads, prefix, p.line_rows);
  } else {
    prefix = 0;
  }
  // Fewest keys of a part of a request's own, of which a workgroup takes 128 in about a us.  Beside a
  // prefix 768: its parts take that long, and are joined in any case (30 requests of up to 300 keys
  // behind 300: 14.0 us a step, 16.7 with parts of 256).  Else one part up to 384 keys, whose join
  // would take longer (300 keys: 8.0 us, 9.4 in two parts); then 128 where the parts have a CU
  // each (900 keys: 8.4, 9.4 with 256), and 256 where they do not (4 requests of 2048: 12.7, 13.8
  // with 128).
  const int64_t behind = max_len - prefix, groups = requests * kv_heads * p.own_tiles;
  const int64_t fewest = p.share != kShareNone ? 768 : behind <= 384 ? 384 : groups * ceil_div(behind, kNarrowKeys) <= 256 ? kNarrowKeys : 256;
  p.own_parts = (int)std::clamp(ceil_div(kGroups, groups), (int64_t)1,
                                std::min<int64_t>(kMaxParts / 2, std::max<int64_t>(1, ceil_div(behind, fewest))));
  // nothing is shared or split where a launch could not hold it: own_tiles alone fit one (checked before)
  if ((p.prefix_groups() + requests * p.own_tiles * p.own_parts) * kv_heads >= kMaxGroups || p.line_rows >= kThreads / 64 * kMaxGroups)
    return make_plan(requests, fresh, q_heads, kv_heads, max_len, 0, false, false);
  return p;
}

// Rows of this wavefront: lane's column, where it goes and the last key it sees.
struct Row {
  bool present;
  int64_t line;          // row of q and out
  int column;            // head
  int last;
};

// The pages of one table row, and the descriptors of 16 keys in them.
// The entry is read through the constant address space: a scalar load, which does not wait
// behind the loads of keys and values in flight as a vector load's result would.
struct Pages {
  const int32_t* row;
  template <typename T>
  __device__ __forceinline__ bool find(const Cache<T>& c, int j, int64_t* page) const {
    typedef const __attribute__((address_space(4))) int32_t* uniform_ptr;
    *page = ((uniform_ptr)row)[j >> c.page_shift];
    return (uint64_t)*page < (uint64_t)c.pages;
  }
};

template <typename T, int D>
__device__ __forceinline__ int64_t group_offset(const Decode<T>& a, int head, int64_t page, int j) {
  return (((page * a.kv_heads + head) << a.cache.page_shift) + (j & ((1 << a.cache.page_shift) - 1))) * D;
}

template <typename T>
__device__ __forceinline__ int request_len(const Decode<T>& a, int request) {
  const int64_t room = min(a.max_len, a.table_stride << a.cache.page_shift);
  return (int)min((int64_t)max(a.lens[request], 0), room);
}

// The request that takes place `i` where those of each 64 stand longest first, so that what starts
// last is short.
template <typename T>
__device__ __forceinline__ int longest_first(const Decode<T>& a, int i) {
  const int lane = threadIdx.x & 63, base = i & ~63, r = base + lane;
  const bool there = r < a.requests;
  const uint32_t key = (there ? (uint32_t)(min(max(a.lens[there ? r : base], 0), (1 << 25) - 1) + 1) << 6 : 0u) | (uint32_t)(63 - lane);
  int before = 0;
#pragma unroll 16
  for (int j = 0; j < 64; ++j) before += (uint32_t)__builtin_amdgcn_readlane((int)key, j) > key ? 1 : 0;
  return base + __builtin_ctzll(__builtin_amdgcn_ballot_w64(before == (i & 63)));
}

// Four consecutive outputs of a row, of one part or of all.
template <typename T, int D>
__device__ __forceinline__ void put(const Decode<T>& a, const Plan& p, const Parts& parts, int part, const Row& row,
                                    int at, f32x4 o, float m, float l) {
  if (parts.ml == nullptr) {
    const float by = inverse_of(l);
    T* to = a.out.p + row.line * a.out.stride + row.column * D + at;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<u32x2*>(to) = u32x2{pack_bf16x2(o[0] * by, o[1] * by), pack_bf16x2(o[2] * by, o[3] * by)};
    else *reinterpret_cast<f32x4*>(to) = f32x4{o[0] * by, o[1] * by, o[2] * by, o[3] * by};
  } else {
    const int64_t r = part * p.line_rows + row.line * a.q_heads + row.column;
    *reinterpret_cast<f32x4*>(parts.o + r * D + at) = o;
    if (at == 0) parts.ml[r] = float2{m, l};
  }
}

template <typename T, int D>
__device__ void wide(const Decode<T>& a, const Plan& p, const Parts& parts, int head, int tile, int part, uint8_t* lds, int* spoiled) {
  using S = Shape<T, D>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int prefix = (int)min(a.prefix, min(a.max_len, a.table_stride << a.cache.page_shift));
  const int per = ((prefix + p.prefix_parts - 1) / p.prefix_parts + kWideKeys - 1) / kWideKeys * kWideKeys;
  const int begin = min(part * per, prefix), end = min(begin + per, prefix);
  const int index = tile * kWideRows + 32 * wave + (lane & 31);
  Row row;
  row.present = index < p.rows;
  const int line = index / p.group, request = line / a.fresh;
  row.line = line;
  row.column = head * p.group + index - line * p.group;
  row.last = row.present ? min(request_len(a, request) - a.fresh + (line - request * a.fresh), prefix - 1) : -1;
  const int wave_first = wave_min(row.present ? row.last : 0x7fffffff), wave_last = -wave_min(-row.last);

  Rows32<T, D> r;
  r.load_query(a.q.p + row.line * a.q.stride + row.column * D, row.present, lane);
  const Loader<T, D> load(lane, S::kRow);
  const float scale = a.scale * kLog2e;
  const Pages pages = {a.table};
  auto walk = [&](auto careful) {
    uint32_t absent = 0, next_absent = 0;                 // groups of 16 keys of this tile and the next whose page is
    int64_t at = 0;                                       // this wavefront's group of the next tile
    uint32_t bytes = 0;
    walk_shared<decltype(careful)::value>(
        r, lds, (end - begin + kWideKeys - 1) / kWideKeys, wave_last < begin ? 0 : (min(wave_last, end - 1) - begin) / kWideKeys + 1, scale, lane,
        [&](int t) {
          const int j = begin + kWideKeys * t, first = j + 16 * wave;
          absent = next_absent;
          next_absent = 0;
          bytes = 0;
          int64_t page;
          if (first < end && pages.find(a.cache, first, &page)) {
            at = group_offset<T, D>(a, head, page, first);
            bytes = (uint32_t)(min(end - first, 16) * S::kRow);
          }
#pragma unroll
          for (int g = 0; g < 4; ++g)
            if (j + 16 * g < end && !pages.find(a.cache, j + 16 * g, &page)) next_absent |= 1u << g;
        },
        [&](uint8_t* to) { load.keys(describe(a.cache.k + at, bytes), to + wave * S::kGroup); },
        [&](uint8_t* to) { load.values(describe(a.cache.v + at, bytes), to + wave * S::kGroup); },
        [&](int t) { return begin + kWideKeys * (t + 1) - 1 > min(wave_first, end - 1) || absent != 0; },
        [&](int t, f32x16 (&s)[2]) { return Rows32<T, D>::template mask<2>(s, 0, min(row.last, end - 1) - begin - kWideKeys * t, absent, lane); },
        [&](int t) { return min(row.last, end - 1) - begin - kWideKeys * t; });
  };
  if (threadIdx.x == 0) *spoiled = 0;
  walk(std::false_type{});
  __syncthreads();
  if (row.present && r.spoiled()) *spoiled = 1;
  __syncthreads();
  if (*spoiled != 0) walk(std::true_type{});
  const float l = sum_across(r.l);
  if (!row.present) return;
#pragma unroll
  for (int t = 0; t < S::kOut; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i)
      put<T, D>(a, p, parts, part, row, 32 * t + 8 * i + 4 * (lane / 32), f32x4{r.o[t][4 * i], r.o[t][4 * i + 1], r.o[t][4 * i + 2], r.o[t][4 * i + 3]}, r.m, l);
}

// Keys [begin, end) of a table row.
struct Range {
  const int32_t* row;
  int begin, end;
};

// Rows from `index0` on of `request` (of all requests if it is negative) against two ranges.
template <typename T, int D>
__device__ void narrow(const Decode<T>& a, const Plan& p, const Parts& parts, int head, int request, int index0,
                       const Range (&range)[2], int part, uint8_t* lds, float2* ml) {
  using S = Shape<T, D>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = request < 0 ? p.rows : a.fresh * p.group;
  auto find_row = [&](int n) {
    Row row;
    const int index = index0 + n, token = index / p.group;
    row.present = index < rows;
    const int of = request < 0 ? token / a.fresh : request;
    row.line = request < 0 ? token : (int64_t)request * a.fresh + token;
    row.column = head * p.group + index - token * p.group;
    row.last = row.present ? request_len(a, of) - a.fresh + (int)(row.line - (int64_t)of * a.fresh) : -1;
    return row;
  };
  const Row row = find_row(lane & 31);
  const int wave_first = wave_min(row.present ? row.last : 0x7fffffff);

  Rows32<T, D> r;
  r.load_query(a.q.p + row.line * a.q.stride + row.column * D, row.present, lane);
  const Loader<T, D> load(lane, S::kRow);
  const float scale = a.scale * kLog2e;
  auto walk = [&](auto careful) {
    r.start(lane);
#pragma unroll 1
    for (int s = 0; s < 2; ++s) {
      const int lo = s == 0 ? range[0].begin : range[1].begin, hi = s == 0 ? range[0].end : range[1].end;
      const Pages of = {s == 0 ? range[0].row : range[1].row};
      walk_private<decltype(careful)::value>(r, lds, load, load, wave, kWaves, lo, hi, wave_first, row.last, scale, lane, [&](int first) {
        Group<T> g = {a.cache.k, a.cache.v, 0u, 0u, false};
        const int count = min(hi - first, 16);
        if (count > 0) {
          int64_t page;
          g.absent = !of.find(a.cache, first, &page);
          if (!g.absent) {
            const int64_t at = group_offset<T, D>(a, head, page, first);
            g.k += at;
            g.v += at;
            g.k_bytes = g.v_bytes = (uint32_t)(count * S::kRow);
          }
        }
        return g;
      });
    }
  };
  walk(std::false_type{});
  if (__builtin_amdgcn_ballot_w64(row.present && r.spoiled()) != 0) walk(std::true_type{});
  join_waves<kWaves>(r, lds, ml, min(rows - index0, kNarrowRows), wave, lane,
                     [&](int of, int at, f32x4 o, float m, float l) { put<T, D>(a, p, parts, part, find_row(of), at, o, m, l); });
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 ? 2 : 1) void decode_kernel(const Decode<T> a, const Plan p, const Parts parts, int prefix_groups, bool sorted) {
  constexpr int kTile = 64 * Shape<T, D>::kRow;
  __shared__ __align__(1024) uint8_t lds[4 * kTile];
  __shared__ float2 ml[kWaves * 32];
  __shared__ int spoiled;
  const int prefix = (int)min(a.prefix, min(a.max_len, a.table_stride << a.cache.page_shift));
  // The heads in turn; of the rest, work on the prefix (arithmetic, and long) before the requests' own
  // keys (memory): workgroups go to the XCDs, their shader engines and CUs in turn, so that each CU
  // gets some of both.  With the two kinds taken in turn some shader engines got long ones only, and
  // held up all that came after (79 requests of 7 tokens
  // behind 9589 keys: 227 us against 147).
  const int head = (int)blockIdx.x % a.kv_heads, turn = (int)blockIdx.x / a.kv_heads;
  const bool on_prefix = turn < prefix_groups;
  const int i0 = on_prefix ? turn : turn - prefix_groups;
  // what lies in the prefix comes from the first request's pages, shared or not
  Range range[2] = {{a.table, 0, 0}, {a.table, 0, 0}};
  int request = -1, index0 = 0, part;
  if (on_prefix) {
    const int tile = i0 % p.prefix_tiles;
    part = i0 / p.prefix_tiles;
    if constexpr (sizeof(T) == 2) {
      if (p.share == kShareWide) return wide<T, D>(a, p, parts, head, tile, part, lds, &spoiled);
    }
    index0 = tile * kNarrowRows;
    const int per = ((prefix + p.prefix_parts - 1) / p.prefix_parts + kNarrowKeys - 1) / kNarrowKeys * kNarrowKeys;
    range[0].begin = min(part * per, prefix);
    range[0].end = min(range[0].begin + per, prefix);
  } else {
    int i = i0;
    part = i % p.own_parts;
    i /= p.own_parts;
    index0 = i % p.own_tiles * kNarrowRows;
    request = i / p.own_tiles;
    if (sorted) request = longest_first(a, request);
    const int len = request_len(a, request), from = min(p.share != kShareNone ? prefix : 0, len);
    const int per = ((len - from + p.own_parts - 1) / p.own_parts + kNarrowKeys - 1) / kNarrowKeys * kNarrowKeys;
    const int lo = min(from + part * per, len), hi = min(lo + per, len);
    range[0].begin = lo;
    range[0].end = min(hi, prefix);
    range[1] = {a.table + request * a.table_stride, max(lo, prefix), hi};
    if (p.share != kShareNone) part += p.prefix_parts;
  }
  narrow<T, D>(a, p, parts, head, request, index0, range, part, lds, ml);
}

// One row of out from its parts, by R lanes, a wavefront or a workgroup of them: D / 4 lanes hold the
// row, and the groups of so many lanes take the parts in turn, so that their loads are under way
// together.
template <typename T, int D, int R>
__global__ __launch_bounds__(kThreads) void join_kernel(const Decode<T> a, int64_t line_rows, int count, const Parts parts) {
  constexpr int kLanes = D / 4, kGroups = R / kLanes;
  const int lane = threadIdx.x & 63, at = (int)threadIdx.x % kLanes, group = (int)threadIdx.x % R / kLanes;
  const int64_t row = blockIdx.x * (int64_t)(kThreads / R) + threadIdx.x / R;
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
  put<T, D>(a, Plan{}, Parts{nullptr, nullptr}, 0, to, 4 * at, sum, 0.0f, l);
}

size_t part_bytes(const Plan& p, int head_dim) {
  return p.parts() > 1 ? (size_t)p.parts() * (size_t)p.line_rows * (8 + 4 * (size_t)head_dim) : 0;
}

template <typename T, int D>
hipError_t launch(const Decode<T>& a, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  Plan p = make_plan(a.requests, a.fresh, a.q_heads, a.kv_heads, a.max_len, a.prefix, true, sizeof(T) == 2);
  size_t need = part_bytes(p, D);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) {
    p = make_plan(a.requests, a.fresh, a.q_heads, a.kv_heads, a.max_len, a.prefix, false, false);
    need = 0;
  }
  Parts parts = {nullptr, nullptr};
  if (need > 0) {
    parts.o = static_cast<float*>(workspace);
    parts.ml = reinterpret_cast<float2*>(parts.o + (size_t)p.parts() * p.line_rows * D);
  }
  const int64_t prefix_groups = p.prefix_groups(), own_groups = a.requests * p.own_tiles * p.own_parts;
  // Longest requests first where workgroups outnumber their places, two on each of 256 CUs, and the
  // longest walk 512 keys or more: 64 users of 1 to 1024 tokens behind 8192 (8 key/value heads)
  // 54.2 -> 49.4 us, 32 of up to 2048 behind 4096 (64 heads) 45.8 -> 41.0.  Shorter walks do not gain
  // what finding the order takes: 128 requests of up to 100 tokens 14.5 -> 17.3, behind 4096 32.0 -> 34.4.
  const int64_t behind = a.max_len - std::min(a.max_len, p.share != kShareNone ? a.prefix : 0);
  const bool sorted = a.requests > 1 && (prefix_groups + own_groups) * a.kv_heads > 512 && behind / p.own_parts >= 512;
  decode_kernel<T, D><<<dim3((unsigned)((prefix_groups + own_groups) * a.kv_heads)), kThreads, 0, stream>>>(a, p, parts, (int)prefix_groups, sorted);
  if (need > 0) {
    // A wavefront a row where the rows fill the chip (2560 rows of 7 parts: a step of 20.3 us against
    // 21.2 with a workgroup a row), a workgroup a row where they do not (32 rows of 32 parts: 18.9
    // against 21.9; equal at about 1000 rows).
    constexpr int kPerGroup = kThreads / 64;
    if (p.line_rows >= kWaveJoinRows) join_kernel<T, D, 64><<<dim3((unsigned)((p.line_rows + kPerGroup - 1) / kPerGroup)), kThreads, 0, stream>>>(a, p.line_rows, p.parts(), parts);
    else join_kernel<T, D, kThreads><<<dim3((unsigned)p.line_rows), kThreads, 0, stream>>>(a, p.line_rows, p.parts(), parts);
  }
  return hipGetLastError();
}

}  // namespace
}  // namespace attention

size_t attention_decode_workspace_bytes(int64_t requests, int fresh, int q_heads, int kv_heads, int head_dim,
                                        int64_t max_len, int64_t prefix) {
  return attention::part_bytes(attention::make_plan(requests, fresh, q_heads, kv_heads, max_len, prefix, true, true), head_dim);
}

template <typename T>
static hipError_t launch_by_dim(const Decode<T>& a, int head_dim, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return head_dim == 64 ? attention::launch<T, 64>(a, workspace, workspace_bytes, stream)
                        : attention::launch<T, 128>(a, workspace, workspace_bytes, stream);
}
hipError_t launch_attention_decode(const Decode<uint16_t>& a, int head_dim, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return launch_by_dim(a, head_dim, workspace, workspace_bytes, stream);
}
hipError_t launch_attention_decode(const Decode<float>& a, int head_dim, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return launch_by_dim(a, head_dim, workspace, workspace_bytes, stream);
}

}  // namespace ssq
