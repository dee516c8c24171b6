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
#include "attention_join.h"
#include "kv4.h"

namespace ssq {
namespace attention {
namespace {

constexpr int kWaves = 4, kThreads = 64 * kWaves, kRows = 16, kTileKeys = 32;
constexpr int kStepKeys = kTileKeys * kWaves;         // keys that a workgroup takes at a time

struct Kv4Plan {
  int group;             // query heads of a key/value head
  int rows;              // requests * fresh * group: rows of a key/value head
  bool share;            // whether the prefix is taken for all requests at once
  int prefix_tiles, prefix_parts;
  int own_tiles, own_parts;
  int64_t line_rows;     // requests * fresh * q_heads: rows of out
  int parts() const { return own_parts + (share ? prefix_parts : 0); }
  int64_t prefix_groups() const { return share ? (int64_t)prefix_tiles * prefix_parts : 0; }
};




Kv4Plan make_kv4_plan(int64_t requests, int fresh, int q_heads, int kv_heads, int64_t max_len, int64_t prefix, bool split) {
  Kv4Plan p = {};
  p.group = q_heads / kv_heads;
  p.rows = (int)(requests * fresh * p.group);
  p.line_rows = requests * fresh * q_heads;
  p.own_tiles = (int)ceil_div((int64_t)fresh * p.group, kRows);
  p.own_parts = 1;
  if (!split) return p;
  constexpr int64_t kGroups = 512;       // two workgroups for each of 256 CUs
  prefix = std::min(prefix, max_len);
  if (requests > 1 && prefix > 0) {
    p.share = true;
    p.prefix_tiles = (int)ceil_div(p.rows, kRows);
    p.prefix_parts = (int)std::clamp(ceil_div(kGroups, (int64_t)p.prefix_tiles * kv_heads), (int64_t)1,
                                     std::min<int64_t>(kMaxParts / 2, ceil_div(prefix, 2 * kStepKeys)));
  } else {
    prefix = 0;
  }
  const int64_t behind = max_len - prefix, groups = requests * kv_heads * p.own_tiles;
  p.own_parts = (int)std::clamp(ceil_div(kGroups, groups), (int64_t)1,
                                std::min<int64_t>(kMaxParts / 2, std::max<int64_t>(1, ceil_div(behind, 2 * kStepKeys))));
  // nothing is shared or split where a launch could not hold it: own_tiles alone fit one (checked before)
  if ((p.prefix_groups() + requests * p.own_tiles * p.own_parts) * kv_heads >= kMaxGroups || p.line_rows >= kJoinThreads / 64 * kMaxGroups)
    return make_kv4_plan(requests, fresh, q_heads, kv_heads, max_len, 0, false);
  return p;
}

// What a lane loads of 16 keys and their values: the words of kv4.h, and the scales of four keys.
template <int D>
struct Half {
  static constexpr int kGroups = D / 32;
  typedef uint32_t Words __attribute__((ext_vector_type(kGroups)));
  Words k, v;
  u32x4 k_scale[kGroups / 2], v_scale[kGroups / 2];          // [key][group] in binary16
};

__device__ __forceinline__ void load_words(__amdgpu_buffer_rsrc_t r, int at, int base, u32x4& w) { w = __builtin_amdgcn_raw_buffer_load_b128(r, at, base, 0); }
__device__ __forceinline__ void load_words(__amdgpu_buffer_rsrc_t r, int at, int base, u32x2& w) { w = __builtin_amdgcn_raw_buffer_load_b64(r, at, base, 0); }
template <int N>
__device__ __forceinline__ void load_words(__amdgpu_buffer_rsrc_t r, int at, int base, u32x4 (&w)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) load_words(r, at + 16 * i, base, w[i]);
}

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

// RT tiles of 16 query rows of a wavefront.
template <typename T, int D, int RT>
struct Kv4Rows {
  static constexpr int kGroups = D / 32, kTerms = Terms<T>::kCount;
  Terms<T> terms;
  u32x4 q[RT][kGroups][kTerms];
  f32x4 start[RT][kGroups];              // -136 times the sum of the group's elements, in bf16
  f32x4 o[RT][2 * kGroups];              // element 16 t + 4 h + i of query x, in tile t's register i
  float m[RT], l[RT];

  __device__ __forceinline__ void load_query(int rt, const T* row, bool present, int h) {
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
#pragma unroll
      for (int n = 0; n < kTerms; ++n) q[rt][g][n] = u32x4{0u, 0u, 0u, 0u};
      if (present) Terms<T>::query(row + 32 * g + 8 * h, q[rt][g]);
      start[rt][g] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
      if constexpr (kTerms == 1) start[rt][g] = product(u32x4{kLess136, kLess136, kLess136, kLess136}, q[rt][g][0], start[rt][g]);
    }
    m[rt] = -FLT_MAX;
    l[rt] = 0.0f;
#pragma unroll
    for (int t = 0; t < 2 * kGroups; ++t) o[rt][t] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }

  // Scores of two halves' keys.
  __device__ __forceinline__ void score(const Half<D> (&x)[2], f32x4 (&s)[RT][2]) const {
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        const uint32_t w = x[u].k[g];
        const u32x4 key = {terms.codes(w, 0), terms.codes(w, 1), terms.codes(w, 2), terms.codes(w, 3)};
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          f32x4 part = start[rt][g];
#pragma unroll
          for (int n = kTerms - 1; n >= 0; --n) part = product(key, q[rt][g][n], part);
#pragma unroll
          for (int i = 0; i < 4; ++i) s[rt][u][i] = __builtin_fmaf(part[i], scale_of(x[u].k_scale, i, g), g == 0 ? 0.0f : s[rt][u][i]);
        }
      }
  }

  // The values' codes of two halves, elements 16 t ... 16 t + 15, as an A operand.
  __device__ __forceinline__ u32x4 value(const Half<D> (&x)[2], int t) const {
    const uint32_t w[2] = {x[0].v[t / 2], x[1].v[t / 2]};
    // tokens 0 and 2 of a lane's four, then 1 and 3
    return u32x4{terms.codes(w[0], t % 2), terms.codes(w[0], t % 2 + 2), terms.codes(w[1], t % 2), terms.codes(w[1], t % 2 + 2)};
  }

  // What scores of tile rt add: the softmax's step and the product with the values, whose scales x holds.
  __device__ __forceinline__ void add(int rt, const Half<D> (&x)[2], const f32x4 (&s)[2], float scale) {
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
    for (int g = 0; g < kGroups; ++g) {
      u32x4 w[kTerms];
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          uint32_t d[kTerms];
          // a fused product and sum, whose factors may be binary16 as they are
          Terms<T>::split(__builtin_fmaf(p[u][i], scale_of(x[u].v_scale, i, g), 0.0f), __builtin_fmaf(p[u][i + 2], scale_of(x[u].v_scale, i + 2, g), 0.0f), d);
#pragma unroll
          for (int n = 0; n < kTerms; ++n) w[n][2 * u + i] = d[n];
        }
      const u32x4 values[2] = {value(x, 2 * g), value(x, 2 * g + 1)};
#pragma unroll
      for (int n = kTerms - 1; n >= 0; --n)
#pragma unroll
        for (int e = 0; e < 2; ++e) o[rt][2 * g + e] = product(values[e], w[n], o[rt][2 * g + e]);
      if constexpr (kTerms == 1)
#pragma unroll
        for (int e = 0; e < 2; ++e) o[rt][2 * g + e] = product(u32x4{kLess136, kLess136, kLess136, kLess136}, w[0], o[rt][2 * g + e]);
    }
  }

  static __device__ __forceinline__ float scale_of(const u32x4 (&w)[kGroups / 2], int key, int g) {
    const int at = key * kGroups + g;
    const uint32_t pair = w[at / 8][at / 2 % 4];
    return at % 2 == 0 ? f16_lo(pair) : f16_hi(pair);
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

// Up to RT tiles of rows from index0 on, of `request` (of all requests if it is negative), against two ranges.
template <typename T, int D, int RT>
__device__ __forceinline__ void walk_rows(const Decode<T>& a, const uint8_t* cache, const Kv4Plan& p, const Parts& parts, int head, int request,
                                          int index0, const KeyRange (&range)[2], int part, float* lds, float2 (*ml)[RT * kRows]) {
  constexpr int kGroups = D / 32;
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
  Kv4Rows<T, D, RT> r;
  int last[RT], first_last = 0x7fffffff;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const Row row = find_row(rt * kRows + col);
    last[rt] = row.last;
    if (row.present) first_last = min(first_last, row.last);
    r.load_query(rt, a.q.p + row.line * a.q.stride + row.column * D, row.present, h);
  }
  const int wave_first = wave_min(first_last);
  const float scale = a.scale * kLog2e;
  const int shift = a.cache.page_shift, in_page = (1 << shift) - 1, part_bytes = Kv4<D>::part(shift);
  const int k_at = col * Kv4<D>::kCodes + h * 4 * kGroups, v_at = lane * 4 * kGroups, scale_at = h * 4 * Kv4<D>::kScales;
  const int tiles0 = range[0].tiles(), tiles = tiles0 + range[1].tiles();

  struct Place {                          // a tile's halves: first key, and the pages they lie in (-1: absent)
    int first, begin, end;
    int32_t page[2];
  };
  auto place = [&](int t) {
    Place at = {0, 0, 0, {-1, -1}};
    if (t >= tiles) return at;
    const bool one = t >= tiles0;
    const KeyRange& of = one ? range[1] : range[0];
    at.begin = of.begin, at.end = of.end;
    at.first = (of.begin & ~15) + kTileKeys * (one ? t - tiles0 : t);
    typedef const __attribute__((address_space(4))) int32_t* uniform_ptr;
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int j = at.first + 16 * u;
      if (j >= at.end) continue;
      const int32_t page = ((uniform_ptr)of.row)[j >> shift];
      at.page[u] = (int64_t)page < a.cache.pages ? page : -1;
    }
    return at;
  };
  auto record = [&](const Place& at, int u) {
    const bool here = at.page[u] >= 0;
    return make_rsrc(cache + ((here ? at.page[u] : 0) * (int64_t)a.kv_heads + head) * (int64_t)(2 * part_bytes), here ? 2 * part_bytes : 0);
  };
  Half<D> x[2];
  auto load_keys = [&](const Place& at) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const __amdgpu_buffer_rsrc_t rsrc = record(at, u);
      const int t0 = (at.first + 16 * u) & in_page;
      load_words(rsrc, k_at, t0 * Kv4<D>::kCodes, x[u].k);
      load_words(rsrc, scale_at, (Kv4<D>::kCodes << shift) + t0 * Kv4<D>::kScales, x[u].k_scale);
    }
  };
  auto load_value_scales = [&](const Place& at) {
#pragma unroll
    for (int u = 0; u < 2; ++u)
      load_words(record(at, u), scale_at, part_bytes + (Kv4<D>::kCodes << shift) + ((at.first + 16 * u) & in_page) * Kv4<D>::kScales, x[u].v_scale);
  };
  auto load_values = [&](const Place& at) {
#pragma unroll
    for (int u = 0; u < 2; ++u) load_words(record(at, u), v_at, part_bytes + ((at.first + 16 * u) & in_page) * Kv4<D>::kCodes, x[u].v);
    load_value_scales(at);
  };
  uint32_t saw[RT] = {};                  // whether a lane has seen a key
  bool all_saw = false;                   // a tile of which every row sees every key
  Place at = place(wave), then = place(wave + kWaves);
  if (wave < tiles) {
    load_keys(at);
    load_values(at);
  }
#pragma unroll 1
  for (int t = wave; t < tiles; t += kWaves) {
    const Place later = place(t + 2 * kWaves);
    const bool whole = ((at.first >= at.begin) & (at.first + kTileKeys - 1 <= min(wave_first, at.end - 1)) & ((at.page[0] | at.page[1]) >= 0)) != 0;
    all_saw |= whole;
    f32x4 s[RT][2];
    r.score(x, s);
    // the next keys take these ones' registers: all that reads them stays before the loads
#pragma unroll
    for (int rt = 0; rt < RT; ++rt)
#pragma unroll
      for (int u = 0; u < 2; ++u) asm volatile("" : "+v"(s[rt][u]));
    __builtin_amdgcn_sched_barrier(0);
    load_keys(then);
    __builtin_amdgcn_sched_barrier(0);
    uint32_t seen[RT] = {};               // bit 4 u + i: whether a lane sees key i of its four of half u
    if (!whole) {
      asm volatile("");                   // a branch, not selects in every tile
#pragma unroll
      for (int rt = 0; rt < RT; ++rt)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int j = at.first + 16 * u + 4 * h + i;
            const bool sees = at.page[u] >= 0 && j >= at.begin && j <= min(last[rt], at.end - 1);
            s[rt][u][i] = sees ? s[rt][u][i] : -INFINITY;
            seen[rt] |= sees ? 1u << (4 * u + i) : 0u;
          }
    }
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      if (!whole) {                       // the scales of keys that tile rt's rows do not see
        if (rt > 0) load_value_scales(at);
        saw[rt] |= seen[rt];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int n = 0; n < kGroups / 2; ++n) {           // 8 / kGroups keys each
            u32x4 keep;
#pragma unroll
            for (int i = 0; i < 4; ++i) keep[i] = 0u - (seen[rt] >> (4 * u + (8 * n + 2 * i) / kGroups) & 1u);
            x[u].v_scale[n] &= keep;
          }
      }
      r.add(rt, x, s[rt], scale);
    }
    __builtin_amdgcn_sched_barrier(0);
    load_values(then);
    at = then;
    then = later;
  }

  // The wavefronts' results, through LDS: all on the largest reference, then summed.
  constexpr int kPitch = D + 4;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const bool saw_one = all_saw || max_of_row((float)saw[rt]) != 0.0f;
    const float l = saw_one ? sum_of_row(r.l[rt]) : __uint_as_float(kSawNone);
    if (h == 0) ml[wave][rt * kRows + col] = float2{r.m[rt], l};
#pragma unroll
    for (int t = 0; t < 2 * kGroups; ++t)
      *reinterpret_cast<f32x4*>(lds + (wave * RT * kRows + rt * kRows + col) * kPitch + 16 * t + 4 * h) = r.o[rt][t];
  }
  __syncthreads();
  constexpr int kChunks = D / 4;
#pragma unroll
  for (int c = threadIdx.x; c < RT * kRows * kChunks; c += kThreads) {
    const int n = c / kChunks, d = 4 * (c % kChunks);
    if (index0 + n >= rows) continue;
    float m = -FLT_MAX, l = __uint_as_float(kSawNone);
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      if (__float_as_uint(ml[w][n].y) != kSawNone) m = fmaxf(m, ml[w][n].x);
    f32x4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float2 of = ml[w][n];
      if (__float_as_uint(of.y) == kSawNone) continue;
      const float by = __builtin_amdgcn_exp2f(of.x - m);
      l = __builtin_fmaf(by, of.y, l);
      const f32x4 add = *reinterpret_cast<const f32x4*>(lds + (w * RT * kRows + n) * kPitch + d);
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = __builtin_fmaf(by, add[i], o[i]);
    }
    put<T, D>(a, p.line_rows, parts, part, find_row(n), d, o, m, l);
  }
}

template <typename T, int D, int RT>
__global__ __launch_bounds__(kThreads, sizeof(T) == 2 && RT == 1 ? 3 : 2) void decode_kv4_kernel(const Decode<T> a, const uint8_t* cache, const Kv4Plan p, const Parts parts, int prefix_groups, bool sorted) {
  __shared__ __align__(16) float lds[kWaves * RT * kRows * (D + 4)];
  __shared__ float2 ml[kWaves][RT * kRows];
  const int prefix = (int)min(a.prefix, min(a.max_len, a.table_stride << a.cache.page_shift));
  // the heads in turn; of the rest, work on the prefix (long) before the requests' own keys
  const int head = (int)blockIdx.x % a.kv_heads, turn = (int)blockIdx.x / a.kv_heads;
  KeyRange range[2] = {{a.table, 0, 0}, {a.table, 0, 0}};
  int request = -1, index0, part;
  if (turn < prefix_groups) {
    index0 = turn % p.prefix_tiles * (RT * kRows);
    part = turn / p.prefix_tiles;
    const int per = ((prefix + p.prefix_parts - 1) / p.prefix_parts + kStepKeys - 1) / kStepKeys * kStepKeys;
    range[0].begin = min(part * per, prefix);
    range[0].end = min(range[0].begin + per, prefix);
  } else {
    int i = turn - prefix_groups;
    part = i % p.own_parts;
    i /= p.own_parts;
    index0 = i % p.own_tiles * (RT * kRows);
    request = i / p.own_tiles;
    if (sorted) request = longest_first(a, request);
    const int len = request_len(a, request), from = min(p.share ? prefix : 0, len), base = from & ~(kTileKeys - 1);
    const int per = ((len - base + p.own_parts - 1) / p.own_parts + kStepKeys - 1) / kStepKeys * kStepKeys;
    const int lo = max(min(base + part * per, len), from), hi = min(base + (part + 1) * per, len);
    range[0].begin = lo;
    range[0].end = min(hi, prefix);
    range[1] = {a.table + request * a.table_stride, max(lo, prefix), hi};
    if (p.share) part += p.prefix_parts;
  }
  walk_rows<T, D, RT>(a, cache, p, parts, head, request, index0, range, part, lds, ml);
}

template <typename T, int D, int RT>
hipError_t launch_kv4(const Decode<T>& a, const uint8_t* cache, const Kv4Plan& p, const Parts& parts, hipStream_t stream) {
  const int64_t prefix_groups = p.prefix_groups(), own_groups = a.requests * p.own_tiles * p.own_parts;
  decode_kv4_kernel<T, D, RT><<<dim3((unsigned)((prefix_groups + own_groups) * a.kv_heads)), kThreads, 0, stream>>>(a, cache, p, parts, (int)prefix_groups, false);
  if (p.parts() > 1) launch_join<T, D>(a, p.line_rows, p.parts(), parts, stream);
  return hipGetLastError();
}

template <typename T, int D>
hipError_t launch_kv4_dim(const Decode<T>& a, const uint8_t* cache, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  Kv4Plan p = make_kv4_plan(a.requests, a.fresh, a.q_heads, a.kv_heads, a.max_len, a.prefix, true);
  const size_t need = parts_bytes(p.parts(), p.line_rows, D);
  if (need > 0 && (workspace == nullptr || workspace_bytes < need)) p = make_kv4_plan(a.requests, a.fresh, a.q_heads, a.kv_heads, a.max_len, a.prefix, false);
  const Parts parts = p.parts() > 1 ? place_parts<D>(workspace, p.parts(), p.line_rows) : Parts{nullptr, nullptr};
  return launch_kv4<T, D, 1>(a, cache, p, parts, stream);
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
