// Attention of a few new tokens of each request over a paged cache held in 4 bits, with a prefix that
// all requests share (see include/ssq_cache.h; the cache's layout: kv4.h).
//
// A wavefront takes 32 keys at a time against tiles of 16 query rows, with the 16x16x32 matrix
// instruction.  Scores are formed transposed, S^T = K Q^T, so that lane 16 h + x holds query x and the
// keys 4 h ... 4 h + 3 of each 16; the weights are then the B operand of O^T += V^T P^T as they are, with
// the terms of the sum in an order of their own that the values' layout follows.  Codes go straight
// from memory into the operands, without LDS: in bf16 a code u enters as 128 + u, two per instruction
// ((w & mask) | magic), and the 136 too many are taken out again by a product with a constant: for the scores
// once per query (the accumulator's start), for the values once per 32 keys, so that no sum grows
// beyond what it stands for.  In binary32 the codes enter as they are, and queries and weights
// as three bf16 terms each, which hold all 24 bits.
//
// Scales are applied in binary32: a score is the sum of its groups' products, each times that key's
// scale; and the weights are multiplied by the value's scale, group by group, before they are rounded
// to bf16 (in bf16; off by up to 2^-9 each, as in attention_tiles.h).
//
// A row's softmax is kept as in attention_tiles.h: weights relative to a reference that moves only
// when a tile's maximum of that row exceeds it by more than kSlack, a sum of -0 for rows that saw no
// key.  Codes are finite whatever their bits, so that what is hidden can only enter through its
// scales: they are set to zero, and the scores to -inf, in tiles that hold hidden keys.
//
// Workgroups are of two kinds: on a request's own keys, up to 8, 16 or 32 rows of it; on a shared
// prefix, 32 rows of all requests.  Their four wavefronts take the keys 32 at a time, each for itself, and
// meet in LDS at the end; parts of a row are joined by a second launch (attention_join.h).  The next keys
// are loaded into the registers of these as soon as the scores are formed, the next values after
// the product, so that three or four workgroups fit a CU (48 requests of 4096 to 8191 keys, 8 key/value
// heads: 91 us with two sets of registers and two workgroups a CU, 71 so).
//
// Own keys are bound by memory: 96 requests of 8192 keys (908 MB) take 158 us, 5.75 TB/s; reading the
// same bytes in the same order, without arithmetic, takes 148.  48 requests of 4096 to 8191 keys (337 MB):
// 71 us, of which 4.8 are the joining launch and the rest ends unevenly.  One request of 16383 keys: 12.1,
// of which 3.4 are the joining launch; the walk's 9 are a launch, four loads that wait for each other and
// four tiles.  On a prefix 16 rows and 32 keys take about 170 instructions, a third of which unpack (shared
// by two tiles of rows) and half of which apply scales, beside 24 products: 64 requests of 1 to 1024 keys
// behind 8192 take 34.5 us (50 MB, 9.2 GFLOP), in which vector instructions have 45 % of the SIMDs' cycles and
// products 17 %; the rest is waiting and the uneven end.
#include "attention_join.h"
#include "kv4.h"

namespace ssq {
namespace attention {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves, kTileKeys = 32;
constexpr int kStepKeys = kTileKeys * kWaves;         // keys that a workgroup takes at a time
constexpr int kWideRows = 32;                         // rows of a workgroup where they are many (two tiles of 16)

struct Kv4Plan {
  int group;             // query heads of a key/value head
  int rows;              // requests * fresh * group: rows of a key/value head
  int own_rows;          // rows of a workgroup on a request's own keys: 8, 16 or 32
  bool share;            // whether the prefix is taken for all requests at once
  int prefix_tiles, prefix_parts;
  int own_tiles, own_parts;
  int64_t line_rows;     // requests * fresh * q_heads: rows of out
  int parts() const { return own_parts + (share ? prefix_parts : 0); }
  int64_t prefix_groups() const { return share ? (int64_t)prefix_tiles * prefix_parts : 0; }
};

constexpr int kPartCounts[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};      // that are looked at
static_assert(kPartCounts[sizeof(kPartCounts) / sizeof(int) - 1] == kMaxParts);
int64_t steps_of(int64_t keys, int parts) { return ceil_div(ceil_div(keys, parts), kStepKeys); }

// Parts of the requests' own keys where no prefix is shared, for `groups` workgroups a part: the quickest by a fit
// of its time (us).  A step of 128 keys takes a workgroup 1.1 where it has a CU to itself, two beside each other
// 1.8, three 2.35, and a CU full of them 0.8 each; parts have to be joined, by a launch of 3 and their traffic.  These
// constants were read on an earlier state of the walk, with up to 8 rows in bf16; what they choose was read again on
// this one, with the other forms (8 key/value heads, us, * the choice; the best is at most 7 % quicker):
//   1 request of 16383 keys          16, 24, 32*, 48, 64 parts 15.0, 13.5, 12.2, 13.6, 13.6
//   16 of 1024                       1, 2, 4*, 8 parts         12.0, 12.0, 11.9, 12.7
//   32 of 4096                       1, 2, 3*, 4, 8 parts      35.6, 30.6, 31.3, 31.7, 35.4
//   48 of 4096 to 8191               1, 2*, 3, 4, 6, 8 parts   78.5, 71.4, 76.9, 76.2, 76.0, 76.5
//   64 of 1024                       1*, 2, 4 parts            16.6, 20.1, 23.0
//   32 of 4096, 4 tokens (16 rows)   1, 2, 3*, 4 parts         38.2, 34.2, 36.4, 40.0
//   32 of 4096, 8 tokens (32 rows)   1*, 2, 3, 4 parts         49.7, 48.1, 54.9, 58.4
//   1 of 8704, 512 tokens            1, 2*, 4, 8 parts         138, 149, 163, 191
//   binary32: 1 of 16383             16, 32*, 64 parts         30.1, 21.2, 22.5
//   binary32: 48 of 4096 to 8191     1, 2*, 3, 4, 8 parts      257, 172, 183, 174, 182
int choose_parts(int64_t groups, int64_t keys, int64_t line_rows) {
  int best = 1;
  double best_us = 0.0;
  for (const int n : kPartCounts) {
    if (n > 1 && (n - 1) * kStepKeys >= keys) break;
    const int64_t beside = ceil_div(groups * n, 256);
    const double step_us = beside == 1 ? 1.1 : beside == 2 ? 1.8 : beside == 3 ? 2.35 : 0.8 * (double)beside;
    const double us = step_us * (double)steps_of(keys, n) + (n > 1 ? 3.0 : 0.0) + n * (0.04 + 0.6e-3 * (double)line_rows);
    if (n == 1 || us < best_us) best = n, best_us = us;
  }
  return best;
}

// The same beside a prefix, whose workgroups take 1.3 for a step of 128 keys and 32 rows, 2.3 where a CU has two of
// them, and in between where it has work on own keys too; a CU that is full does a step in 1.15, one of a
// request's own keys in 0.8.  Together: the work, or the longest workgroup.  64 requests of one key behind 8192 (256 rows, 8 key/value
// heads): 2, 3, 4 (the choice), 6, 8 parts 49.7, 37.9, 31.2, 33.9, 31.2 us; behind 16384: 4, 6, 8 (the choice), 12 parts
// 51.0, 54.5, 44.2, 49.1; of 1 to 1024 keys behind 8192, undivided: 3, 4 (the choice), 6, 8 parts 39.8, 35.0, 38.4, 40.7.  Binary32
// goes by the same: 16 requests of 4 tokens and 4 to 700 keys behind 1000 take 11.3 in 8 parts and 4 of their own (the
// choice), 12.4 in 4 and 2, 13.9 in 8 and 1, 15.2 in 2 and 1.
void choose_shared_parts(Kv4Plan& p, int64_t requests, int kv_heads, int64_t prefix, int64_t behind) {
  const int64_t wide = (int64_t)p.prefix_tiles * kv_heads, own = requests * p.own_tiles * kv_heads;
  double best_us = 0.0;
  for (const int n : kPartCounts) {
    if (n > kMaxParts / 2 || (n > 1 && (n - 1) * kStepKeys >= prefix)) break;
    for (const int m : {1, 2, 4, 8}) {
      if (m > 1 && (m - 1) * kStepKeys >= behind) break;
      const double wide_steps = (double)steps_of(prefix, n), own_steps = (double)steps_of(behind, m);
      const double wide_us = 1.15 * wide_steps * (double)(wide * n) / 256.0, own_us = 0.8 * own_steps * (double)(own * m) / 256.0;
      const double pace = wide * n > 256 ? 2.3 : 1.3 + 0.6 * std::min(1.0, own_us / wide_us), all = wide_us + own_us;
      const double longest = std::max(wide_steps * pace, own_steps * 1.5);
      const double us = std::max(all, longest) + 0.25e-3 * (double)((n + m) * p.line_rows);
      if ((n == 1 && m == 1) || us < best_us) p.prefix_parts = n, p.own_parts = m, best_us = us;
    }
  }
}

Kv4Plan make_kv4_plan(int64_t requests, int fresh, int q_heads, int kv_heads, int64_t max_len, int64_t prefix, bool split) {
  Kv4Plan p = {};
  p.group = q_heads / kv_heads;
  p.rows = (int)(requests * fresh * p.group);
  p.line_rows = requests * fresh * q_heads;
  const int64_t mine = (int64_t)fresh * p.group;
  p.own_rows = mine <= 8 ? 8 : mine <= 16 ? 16 : kWideRows;
  p.own_tiles = (int)ceil_div(mine, p.own_rows);
  p.own_parts = 1;
  if (!split) return p;
  prefix = std::min(prefix, max_len);
  if (requests > 1 && prefix > 0) {
    p.share = true;
    p.prefix_tiles = (int)ceil_div(p.rows, kWideRows);
    choose_shared_parts(p, requests, kv_heads, prefix, max_len - prefix);
  } else {
    p.own_parts = choose_parts(requests * kv_heads * p.own_tiles, max_len, p.line_rows);
  }
  // nothing is shared or split where a launch could not hold it: own_tiles alone fit one (checked before)
  if ((p.prefix_groups() + requests * p.own_tiles * p.own_parts) * kv_heads >= kMaxGroups || p.line_rows >= kJoinThreads / 64 * kMaxGroups)
    return make_kv4_plan(requests, fresh, q_heads, kv_heads, max_len, 0, false);
  return p;
}

// F = 2: two column groups share a product's 16 columns.  With up to 8 rows, column 8 cg + i of it is query i against
// half of the head's groups of 32, cg * kSets ... cg * kSets + kSets - 1, alone (its operands are zero for the others).
// So a chain of two products leaves two groups' sums in one accumulator, each lane scales its own groups only, and the
// columns are added up once they are scores; the weights are scaled likewise, and of an output tile the columns of
// its own groups count.  96 requests of 8192 keys, 4 or 5 rows: 158 us, 164 with F = 1 (four column groups for up to
// 4 rows: 158 too, and not kept).
template <int D, int F>
struct Fold {
  static constexpr int kGroups = D / 32, kSets = kGroups / F, kRows = 16 / F;
  static_assert(F == 1 || F == 2, "folded, a lane's groups share a word of scales");
};

// The scales of four keys, for the groups of a lane: binary16, where `of` finds them.
template <int D, int F>
struct Spread {
  using S = Fold<D, F>;
  u32x4 w[F == 1 ? S::kGroups / 2 : 1];          // [key][group]; folded: a word a key
  __device__ __forceinline__ float of(int key, int set) const {
    const int at = F == 1 ? key * S::kGroups + set : 2 * key + set;
    const uint32_t pair = w[at / 8][at / 2 % 4];
    return at % 2 == 0 ? f16_lo(pair) : f16_hi(pair);
  }
  // Zeros for keys without their bit in `seen`.
  __device__ __forceinline__ void keep(uint32_t seen) {
#pragma unroll
    for (int n = 0; n < (int)(sizeof(w) / sizeof(w[0])); ++n) {
      u32x4 mask;
#pragma unroll
      for (int i = 0; i < 4; ++i) mask[i] = 0u - (seen >> (F == 1 ? (8 * n + 2 * i) / S::kGroups : i) & 1u);
      w[n] &= mask;
    }
  }
};

// As they are loaded.  Folded, a lane loads the word of one key of its four, which the four lanes side by side exchange.
template <int D, int F>
struct Scales {
  uint32_t w;
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, int at, int base) {
    if constexpr (Fold<D, F>::kSets == 1) w = __builtin_amdgcn_raw_buffer_load_b16(r, at, base, 0);
    else w = __builtin_amdgcn_raw_buffer_load_b32(r, at, base, 0);
  }
  static __device__ __forceinline__ int lane_at(int h, int col) {
    return (4 * h + (col & 3)) * Kv4<D>::kScales + col / Fold<D, F>::kRows * 2 * Fold<D, F>::kSets;
  }
  template <int KEY>
  __device__ __forceinline__ uint32_t of_key() const { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, 0x55 * KEY, 0xF, 0xF, true); }
  __device__ __forceinline__ Spread<D, F> spread() const { return {{u32x4{of_key<0>(), of_key<1>(), of_key<2>(), of_key<3>()}}}; }
};
template <int D>
struct Scales<D, 1> {
  Spread<D, 1> all;
  __device__ __forceinline__ void load(__amdgpu_buffer_rsrc_t r, int at, int base) {
#pragma unroll
    for (int n = 0; n < D / 64; ++n) all.w[n] = __builtin_amdgcn_raw_buffer_load_b128(r, at + 16 * n, base, 0);
  }
  static __device__ __forceinline__ int lane_at(int h, int) { return 4 * h * Kv4<D>::kScales; }
  __device__ __forceinline__ Spread<D, 1> spread() const { return all; }
};

// What a lane loads of 16 keys and their values: the words of kv4.h, and scales.
template <int D, int F>
struct Half {
  static constexpr int kGroups = D / 32;
  typedef uint32_t Words __attribute__((ext_vector_type(kGroups)));
  Words k, v;
  Scales<D, F> k_scale, v_scale;
};

__device__ __forceinline__ void load_words(__amdgpu_buffer_rsrc_t r, int at, int base, u32x4& w) { w = __builtin_amdgcn_raw_buffer_load_b128(r, at, base, 0); }
__device__ __forceinline__ void load_words(__amdgpu_buffer_rsrc_t r, int at, int base, u32x2& w) { w = __builtin_amdgcn_raw_buffer_load_b64(r, at, base, 0); }

__device__ __forceinline__ float max_of_row(float v) {        // of the four lanes that hold a query
  const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return max_across(fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1])));
}
__device__ __forceinline__ float sum_of_row(float v) {
  const auto s = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return sum_across(__uint_as_float(s[0]) + __uint_as_float(s[1]));
}

__device__ __forceinline__ f32x4 product(const u32x4& a, const u32x4& b, const f32x4& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

constexpr uint32_t kLess136 = 0xC308C308u;            // -136 in bf16, twice

// What depends on the element type: how many bf16 terms a query or a weight has, and how codes enter.
template <typename T>
struct Terms;
template <>
struct Terms<uint16_t> {
  static constexpr int kCount = 1;
  uint32_t mask, magic;
  __device__ __forceinline__ Terms() : mask(opaque_s(0x000F000Fu)), magic(opaque_v(0x43004300u)) {}
  // Codes 4 i and 16 + 4 i bits up in w, as 128 + u.
  __device__ __forceinline__ uint32_t codes(uint32_t w, int i) const { return ((w >> (4 * i)) & mask) | magic; }
  static __device__ __forceinline__ void split(float a, float b, uint32_t (&t)[1]) { t[0] = pack_bf16x2(a, b); }
  // 8 elements of a query in the codes' order: 0, 4, 1, 5, 2, 6, 3, 7.
  static __device__ __forceinline__ void query(const uint16_t* p, u32x4 (&t)[1]) {
    const u32x4 d = *reinterpret_cast<const u32x4*>(p);
    t[0] = u32x4{__builtin_amdgcn_perm(d[2], d[0], 0x05040100u), __builtin_amdgcn_perm(d[2], d[0], 0x07060302u),
                 __builtin_amdgcn_perm(d[3], d[1], 0x05040100u), __builtin_amdgcn_perm(d[3], d[1], 0x07060302u)};
  }
};
template <>
struct Terms<float> {
  static constexpr int kCount = 3;
  __device__ __forceinline__ Terms() {}
  __device__ __forceinline__ uint32_t codes(uint32_t w, int i) const {
    return pack_bf16x2((float)((int)(w >> (4 * i) & 15u) - 8), (float)((int)(w >> (16 + 4 * i) & 15u) - 8));
  }
  // Each term is what the ones before leave, rounded to bf16: 8 bits and a sign each.
  static __device__ __forceinline__ void split(float a, float b, uint32_t (&t)[3]) {
#pragma unroll
    for (int i = 0; i < 3; ++i) {
      t[i] = pack_bf16x2(a, b);
      a -= bf16_lo(t[i]);
      b -= bf16_hi(t[i]);
    }
  }
  static __device__ __forceinline__ void query(const float* p, u32x4 (&t)[3]) {
    const f32x4 lo = *reinterpret_cast<const f32x4*>(p), hi = *reinterpret_cast<const f32x4*>(p + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t d[3];
      split(lo[i], hi[i], d);
#pragma unroll
      for (int n = 0; n < 3; ++n) t[n][i] = d[n];
    }
  }
};

// RT tiles of 16 / F query rows of a wavefront.
template <typename T, int D, int RT, int F>
struct Kv4Rows {
  using S = Fold<D, F>;
  static constexpr int kGroups = S::kGroups, kSets = S::kSets, kTerms = Terms<T>::kCount;
  static constexpr bool kOffset = kTerms == 1;         // whether codes enter with 136 too many
  Terms<T> terms;
  u32x4 q[RT][kGroups][kTerms];
  f32x4 start[RT][kSets];                // -136 times the sum of the groups' elements
  f32x4 o[RT][2 * kGroups];              // element 16 t + 4 h + i of the column's query, in tile t's register i
  float m[RT], l[RT];

  __device__ __forceinline__ void load_query(int rt, const T* row, bool present, int h, int col) {
#pragma unroll
    for (int j = 0; j < kSets; ++j) start[rt][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
#pragma unroll
      for (int n = 0; n < kTerms; ++n) q[rt][g][n] = u32x4{0u, 0u, 0u, 0u};
      if (present && col / S::kRows == g / kSets) Terms<T>::query(row + 32 * g + 8 * h, q[rt][g]);
      if constexpr (kOffset) start[rt][g % kSets] = product(u32x4{kLess136, kLess136, kLess136, kLess136}, q[rt][g][0], start[rt][g % kSets]);
    }
    m[rt] = -FLT_MAX;
    l[rt] = 0.0f;
#pragma unroll
    for (int t = 0; t < 2 * kGroups; ++t) o[rt][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  // Scores of two halves' keys.
  __device__ __forceinline__ void score(const Half<D, F> (&x)[2], f32x4 (&s)[RT][2]) const {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const Spread<D, F> by = x[u].k_scale.spread();
#pragma unroll
      for (int j = 0; j < kSets; ++j) {
        f32x4 part[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) part[rt] = start[rt][j];
#pragma unroll
        for (int g = j; g < kGroups; g += kSets) {
          const uint32_t w = x[u].k[g];
          const u32x4 key = {terms.codes(w, 0), terms.codes(w, 1), terms.codes(w, 2), terms.codes(w, 3)};
#pragma unroll
          for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int n = kTerms - 1; n >= 0; --n) part[rt] = product(key, q[rt][g][n], part[rt]);
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[rt][u][i] = __builtin_fmaf(part[rt][i], by.of(i, j), j == 0 ? 0.0f : s[rt][u][i]);
      }
      if constexpr (F > 1) {               // over the column groups; every column has the sum
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[rt][u][i] += other_half(s[rt][u][i]);
      }
    }
  }

  // The value 8 columns further, round the 16.
  static __device__ __forceinline__ float other_half(float v) {
    return __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(v), 0x128, 0xF, 0xF, true));
  }

  // The values' codes of two halves, elements 16 t ... 16 t + 15, as an A operand.
  __device__ __forceinline__ u32x4 value(const Half<D, F> (&x)[2], int t) const {
    const uint32_t w[2] = {x[0].v[t / 2], x[1].v[t / 2]};
    // tokens 0 and 2 of a lane's four, then 1 and 3
    return u32x4{terms.codes(w[0], t % 2), terms.codes(w[0], t % 2 + 2), terms.codes(w[1], t % 2), terms.codes(w[1], t % 2 + 2)};
  }

  // What scores of tile rt add: the softmax's step and the product with the values.
  __device__ __forceinline__ void add(int rt, const Half<D, F> (&x)[2], const Spread<D, F> (&by)[2], const f32x4 (&s)[2], float scale) {
    float most = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) most = fmaxf(most, s[u][i]);
    if (__builtin_amdgcn_ballot_w64(most * scale > m[rt] + kSlack) != 0) move(rt, most * scale);
    float p[2][4];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        p[u][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i], scale, -m[rt]));
        l[rt] += p[u][i];
      }
#pragma unroll
    for (int j = 0; j < kSets; ++j) {
      u32x4 w[kTerms];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t d[kTerms];
          // a fused product and sum, whose factors may be binary16 as they are
          Terms<T>::split(__builtin_fmaf(p[u][i], by[u].of(i, j), 0.0f), __builtin_fmaf(p[u][i + 2], by[u].of(i + 2, j), 0.0f), d);
#pragma unroll
          for (int n = 0; n < kTerms; ++n) w[n][2 * u + i] = d[n];
        }
#pragma unroll
      for (int g = j; g < kGroups; g += kSets) {
        const u32x4 values[2] = {value(x, 2 * g), value(x, 2 * g + 1)};
#pragma unroll
        for (int n = kTerms - 1; n >= 0; --n)
#pragma unroll
          for (int e = 0; e < 2; ++e) o[rt][2 * g + e] = product(values[e], w[n], o[rt][2 * g + e]);
        if constexpr (kOffset)
#pragma unroll
          for (int e = 0; e < 2; ++e) o[rt][2 * g + e] = product(u32x4{kLess136, kLess136, kLess136, kLess136}, w[0], o[rt][2 * g + e]);
      }
    }
  }

  // The references of rows whose maximum is more than kSlack above them, from the lanes' own maxima.
  __device__ __forceinline__ void move(int rt, float most) {
    most = max_of_row(most);
    const float to = most > m[rt] + kSlack ? most : m[rt], by = __builtin_amdgcn_exp2f(m[rt] - to);
    m[rt] = to;
    l[rt] *= by;
#pragma unroll
    for (int t = 0; t < 2 * kGroups; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) o[rt][t][i] *= by;
  }
};

// Keys [begin, end) of a table row, in tiles of 32 from the last multiple of 16 at or before `begin` on.
struct KeyRange {
  const int32_t* row;
  int begin, end;
  __device__ __forceinline__ int tiles() const { return end > begin ? (end - (begin & ~15) + kTileKeys - 1) / kTileKeys : 0; }
};

// What a workgroup's wavefronts leave in LDS, of ROWS rows.
template <int D, int ROWS>
struct Shared {
  static constexpr int kPitch = D + 4;
  float o[kWaves][ROWS][kPitch];
  float2 ml[kWaves][ROWS];
};

// Up to RT * 16 / F rows from index0 on, of `request` (of all requests if it is negative), against two ranges.
template <typename T, int D, int RT, int F>
__device__ __forceinline__ void walk_rows(const Decode<T>& a, const uint8_t* cache, const Kv4Plan& p, const Parts& parts, int head, int request,
                                          int index0, const KeyRange (&range)[2], int part, Shared<D, RT * 16 / F>& lds) {
  using S = Fold<D, F>;
  constexpr int kGroups = S::kGroups, kRows = RT * S::kRows;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane / 16, col = lane & 15;
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
  Kv4Rows<T, D, RT, F> r;
  int last[RT], first_last = 0x7fffffff;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const Row row = find_row(rt * S::kRows + col % S::kRows);
    last[rt] = row.last;
    if (row.present) first_last = min(first_last, row.last);
    r.load_query(rt, a.q.p + row.line * a.q.stride + row.column * D, row.present, h, col);
  }
  const int wave_first = wave_min(first_last);
  const float scale = a.scale * kLog2e;
  const int shift = a.cache.page_shift, in_page = (1 << shift) - 1, part_bytes = Kv4<D>::part(shift), scales = Kv4<D>::kCodes << shift;
  const int k_at = col * Kv4<D>::kCodes + h * 4 * kGroups, v_at = lane * 4 * kGroups, scale_at = Scales<D, F>::lane_at(h, col);
  const uint8_t* of_head = cache + head * (int64_t)(2 * part_bytes);
  const int64_t page_bytes = (int64_t)a.kv_heads * (2 * part_bytes);
  const int tiles0 = range[0].tiles(), tiles = tiles0 + range[1].tiles(), first0 = range[0].begin & ~15, first1 = range[1].begin & ~15;

  struct Place {                          // a tile: its first key, its range's ends, and the table's entries for its halves
    int first, begin, end;
    int32_t page[2];
  };
  auto place = [&](int t) {               // entries are looked at a tile later: nothing waits for them here
    Place at;
    const int of = min(t, tiles - 1);     // behind the last tile its entries again, and no keys
    const bool one = of >= tiles0;
    at.first = one ? first1 + kTileKeys * (of - tiles0) : first0 + kTileKeys * of;
    at.begin = one ? range[1].begin : range[0].begin;
    const int end = one ? range[1].end : range[0].end;
    at.end = t < tiles ? end : 0;
    typedef const __attribute__((address_space(4))) int32_t* uniform_ptr;
    const uniform_ptr row = (uniform_ptr)(one ? range[1].row : range[0].row);
#pragma unroll
    for (int u = 0; u < 2; ++u) at.page[u] = row[min(at.first + 16 * u, end - 1) >> shift];
    return at;
  };
  auto present = [&](const Place& at, int u) { return ((uint32_t)at.page[u] < (uint32_t)a.cache.pages) & (at.first + 16 * u < at.end); };
  struct Source {                         // where a tile's halves are loaded from: their pages' record, and the first token there
    __amdgpu_buffer_rsrc_t of[2];
    int codes[2], scales[2];
  };
  auto source = [&](const Place& at) {
    Source from;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const bool here = present(at, u);
      from.of[u] = make_rsrc(of_head + (uint32_t)(here ? at.page[u] : 0) * page_bytes, here ? 2 * part_bytes : 0);
      const int t0 = (at.first + 16 * u) & in_page;
      from.codes[u] = t0 * Kv4<D>::kCodes;
      from.scales[u] = scales + t0 * Kv4<D>::kScales;
    }
    return from;
  };
  Half<D, F> x[2];
  auto load_keys = [&](const Source& from) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      load_words(from.of[u], k_at, from.codes[u], x[u].k);
      x[u].k_scale.load(from.of[u], scale_at, from.scales[u]);
    }
  };
  auto load_value_scales = [&](const Source& from) {
#pragma unroll
    for (int u = 0; u < 2; ++u) x[u].v_scale.load(from.of[u], scale_at, part_bytes + from.scales[u]);
  };
  auto load_values = [&](const Source& from) {
#pragma unroll
    for (int u = 0; u < 2; ++u) load_words(from.of[u], v_at, part_bytes + from.codes[u], x[u].v);
    load_value_scales(from);
  };
  uint32_t saw[RT] = {};                  // whether a lane has seen a key
  bool all_saw = false;                   // a tile of which every row sees every key
  Place at = {}, then = {};
  if (wave < tiles) {
    at = place(wave);
    then = place(wave + kWaves);
    const Source from = source(at);
    load_keys(from);
    __builtin_amdgcn_sched_barrier(0);    // in the loop's order, which its waits count by
    load_values(from);
  }
#pragma unroll 1
  for (int t = wave; t < tiles; t += kWaves) {
    const Place later = place(t + 2 * kWaves);
    const Source from = source(then);
    const bool whole = ((at.first >= at.begin) & (at.first + kTileKeys - 1 <= min(wave_first, at.end - 1)) & present(at, 0) & present(at, 1)) != 0;
    all_saw |= whole;
    f32x4 s[RT][2];
    r.score(x, s);
    // the next keys take these ones' registers: all that reads them stays before the loads
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int u = 0; u < 2; ++u) asm volatile("" : "+v"(s[rt][u]));
    __builtin_amdgcn_sched_barrier(0);
    load_keys(from);
    __builtin_amdgcn_sched_barrier(0);
    uint32_t seen[RT][2] = {};            // bit i: whether a lane sees key i of its four of half u
    if (!whole) {
      asm volatile("");                   // a branch, not selects in every tile
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int j = at.first + 16 * u + 4 * h + i;
            const bool sees = present(at, u) && j >= at.begin && j <= min(last[rt], at.end - 1);
            s[rt][u][i] = sees ? s[rt][u][i] : -INFINITY;
            seen[rt][u] |= sees ? 1u << i : 0u;
          }
        saw[rt] |= seen[rt][0] | seen[rt][1];
      }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      // the scales of keys that tile rt's rows do not see are zero
      if constexpr (F == 1) {
        if (!whole) {
          if (rt > 0) load_value_scales(source(at));
#pragma unroll
          for (int u = 0; u < 2; ++u) x[u].v_scale.all.keep(seen[rt][u]);
        }
        r.add(rt, x, {x[0].v_scale.all, x[1].v_scale.all}, s[rt], scale);
      } else {
        Spread<D, F> by[2] = {x[0].v_scale.spread(), x[1].v_scale.spread()};
        if (!whole) {
#pragma unroll
          for (int u = 0; u < 2; ++u) by[u].keep(seen[rt][u]);
        }
        r.add(rt, x, by, s[rt], scale);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    load_values(from);
    at = then;
    then = later;
  }

  // The wavefronts' results, through LDS: all on the largest reference, then summed.
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int n = rt * S::kRows + col % S::kRows;
    const bool saw_one = all_saw || max_of_row((float)saw[rt]) != 0.0f;
    const float l = saw_one ? sum_of_row(r.l[rt]) : __uint_as_float(kSawNone);
    if (h == 0 && col < S::kRows) lds.ml[wave][n] = float2{r.m[rt], l};
#pragma unroll
    for (int t = 0; t < 2 * kGroups; ++t)
      if (F == 1 || col / S::kRows == t / 2 / S::kSets) *reinterpret_cast<f32x4*>(&lds.o[wave][n][16 * t + 4 * h]) = r.o[rt][t];
  }
  __syncthreads();
  constexpr int kChunks = D / 4;
#pragma unroll
  for (int c = threadIdx.x; c < kRows * kChunks; c += kThreads) {
    const int n = c / kChunks, d = 4 * (c % kChunks);
    if (index0 + n >= rows) continue;
    float m = -FLT_MAX, l = __uint_as_float(kSawNone);
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      if (__float_as_uint(lds.ml[w][n].y) != kSawNone) m = fmaxf(m, lds.ml[w][n].x);
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float2 of = lds.ml[w][n];
      if (__float_as_uint(of.y) == kSawNone) continue;
      const float by = __builtin_amdgcn_exp2f(of.x - m);
      l = __builtin_fmaf(by, of.y, l);
      const f32x4 add = *reinterpret_cast<const f32x4*>(&lds.o[w][n][d]);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = __builtin_fmaf(by, add[i], o[i]);
    }
    put<T, D>(a, p.line_rows, parts, part, find_row(n), d, o, m, l);
  }
}

// SHARE: some workgroups take the prefix for all requests.
template <typename T, int D, int RT, int F, bool SHARE>
__global__ __launch_bounds__(kThreads, SHARE || RT > 1 ? 2 : F > 1 ? 4 : 3) void decode_kv4_kernel(const Decode<T> a, const uint8_t* cache, const Kv4Plan p, const Parts parts, int prefix_groups) {
  constexpr int kOwnRows = RT * 16 / F;
  __shared__ union {
    Shared<D, kOwnRows> own;
    Shared<D, SHARE ? kWideRows : kOwnRows> wide;
  } lds;
  const int prefix = (int)min(a.prefix, min(a.max_len, a.table_stride << a.cache.page_shift));
  // the heads in turn; of the rest, work on the prefix (long) before the requests' own keys
  const int head = (int)blockIdx.x % a.kv_heads, turn = (int)blockIdx.x / a.kv_heads;
  KeyRange range[2] = {{a.table, 0, 0}, {a.table, 0, 0}};
  if constexpr (SHARE) {
    if (turn < prefix_groups) {
      const int index0 = turn % p.prefix_tiles * kWideRows, part = turn / p.prefix_tiles;
      const int per = ((prefix + p.prefix_parts - 1) / p.prefix_parts + kStepKeys - 1) / kStepKeys * kStepKeys;
      range[0].begin = min(part * per, prefix);
      range[0].end = min(range[0].begin + per, prefix);
      return walk_rows<T, D, kWideRows / 16, 1>(a, cache, p, parts, head, -1, index0, range, part, lds.wide);
    }
  }
  int i = turn - prefix_groups, part = i % p.own_parts;
  i /= p.own_parts;
  const int index0 = i % p.own_tiles * kOwnRows;
  const int request = i / p.own_tiles;
  const int len = request_len(a, request), from = min(SHARE ? prefix : 0, len), base = from & ~(kTileKeys - 1);
  const int per = ((len - base + p.own_parts - 1) / p.own_parts + kStepKeys - 1) / kStepKeys * kStepKeys;
  const int lo = max(min(base + part * per, len), from), hi = min(base + (part + 1) * per, len);
  range[0].begin = lo;
  range[0].end = min(hi, prefix);
  range[1] = {a.table + request * a.table_stride, max(lo, prefix), hi};
  if (SHARE) part += p.prefix_parts;
  walk_rows<T, D, RT, F>(a, cache, p, parts, head, request, index0, range, part, lds.own);
}

template <typename T, int D, int RT, int F>
hipError_t launch_kv4(const Decode<T>& a, const uint8_t* cache, const Kv4Plan& p, const Parts& parts, hipStream_t stream) {
  const int64_t prefix_groups = p.prefix_groups(), own_groups = a.requests * p.own_tiles * p.own_parts;
  const dim3 grid((unsigned)((prefix_groups + own_groups) * a.kv_heads));
  if (p.share) decode_kv4_kernel<T, D, RT, F, true><<<grid, kThreads, 0, stream>>>(a, cache, p, parts, (int)prefix_groups);
  else decode_kv4_kernel<T, D, RT, F, false><<<grid, kThreads, 0, stream>>>(a, cache, p, parts, 0);
  if (p.parts() > 1) launch_join<T, D>(a, p.line_rows, p.parts(), parts, stream);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_kv4_dim(const Decode<T>& a, const uint8_t* cache, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  Kv4Plan p = make_kv4_plan(a.requests, a.fresh, a.q_heads, a.kv_heads, a.max_len, a.prefix, true);
  const size_t need = parts_bytes(p.parts(), p.line_rows, D);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) p = make_kv4_plan(a.requests, a.fresh, a.q_heads, a.kv_heads, a.max_len, a.prefix, false);
  const Parts parts = p.parts() > 1 ? place_parts<D>(workspace, p.parts(), p.line_rows) : Parts{nullptr, nullptr};
  switch (p.own_rows) {
    case 8: return launch_kv4<T, D, 1, 2>(a, cache, p, parts, stream);
    case 16: return launch_kv4<T, D, 1, 1>(a, cache, p, parts, stream);
    default: return launch_kv4<T, D, 2, 1>(a, cache, p, parts, stream);
  }
}

}  // namespace
}  // namespace attention

size_t attention_decode_kv4_workspace_bytes(int64_t requests, int fresh, int q_heads, int kv_heads, int head_dim, int64_t max_len, int64_t prefix) {
  const attention::Kv4Plan p = attention::make_kv4_plan(requests, fresh, q_heads, kv_heads, max_len, prefix, true);
  return attention::parts_bytes(p.parts(), p.line_rows, head_dim);
}

template <typename T>
static hipError_t launch_kv4_by_dim(const Decode<T>& a, const uint8_t* cache, int head_dim, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return head_dim == 64 ? attention::launch_kv4_dim<T, 64>(a, cache, workspace, workspace_bytes, stream)
                        : attention::launch_kv4_dim<T, 128>(a, cache, workspace, workspace_bytes, stream);
}
hipError_t launch_attention_decode_kv4(const Decode<uint16_t>& a, const uint8_t* cache, int head_dim, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return launch_kv4_by_dim(a, cache, head_dim, workspace, workspace_bytes, stream);
}
hipError_t launch_attention_decode_kv4(const Decode<float>& a, const uint8_t* cache, int head_dim, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return launch_kv4_by_dim(a, cache, head_dim, workspace, workspace_bytes, stream);
}

}  // namespace ssq
