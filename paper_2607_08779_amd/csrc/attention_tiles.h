// Attention of 32 query rows against tiles of 32 keys on the matrix cores, in bf16 or binary32:
// the parts that the prompt and the decode kernels are made of.
//
// A wavefront holds 32 query rows (a row is one token's one head; the heads of a group share
// their keys, so rows of several heads and tokens go together).  Scores are formed
// transposed, S^T = K Q^T, so that a lane holds one query (column lane % 32) and half of a
// tile's keys: key 8 (i / 4) + 4 (lane / 32) + i % 4 in register i.  The softmax then runs
// inside a lane, with one exchange between lane and lane ^ 32 for the maximum of a tile, and
// its weights are already the B operand of O^T += V^T P^T, keys permuted within 16 (the
// order of a sum's terms is free): slots 0-3 of a lane are keys 4 h + (0..3), slots 4-7
// keys 8 + 4 h + (0..3).  V^T is read from row-major V in LDS by transposing reads in that order.
//
// O and the sum of the weights are relative to a running reference m (log2 units) of each row:
// weights are 2^(scale log2(e) s - m).  m only moves, and O is only rescaled, when a tile's
// maximum of that row exceeds it by more than kSlack: weights stay at or below 2^kSlack, far from any
// overflow.  In bf16 the weights are rounded to 8 significant bits for the product, because the
// matrix cores take both operands in one type; each is off by up to 2^-9 of itself, whatever m is,
// though by how much depends on m's fraction.  A second product with what the rounding leaves was
// measured and not taken: results come from 2.0e-3 to 1.65e-3 of those in 64 bits (relative norm; the
// output's own rounding is 1.63e-3), and eight ragged prompts go from 252 to 315 us, a prompt of 16384
// tokens from 1.96 to 2.68 ms, one user's 16383 cached tokens from 17.8 to 18.9 us, 64 users behind
// 8192 from 49.2 to 51.2, eight requests of 100 to 300 from 7.8 to 8.5.
//
// The sum starts at -0 and leaves it with the first tile of which the row sees a key.  So a sum of -0
// is that of a row that saw none, which gives zeros, and +0 that of one whose scores were all -inf,
// which gives NaN as their softmax does (inverse_of).
//
// Both tiles live in LDS as rows of D elements, 16-byte chunks XOR-swizzled so that the 16 lanes
// an access serves at once spread over all banks; the swizzle is applied to the global address
// of a direct-to-LDS load, whose LDS side is linear.
#pragma once

#include <float.h>

#include <type_traits>

#include "attention_internal.h"
#include "mfma_dequant.h"

namespace ssq {
namespace attention {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4* lds_s16x4;
typedef __attribute__((address_space(3))) void* lds_void;

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kSlack = 8.0f;
constexpr uint32_t kNowhere = 0x80000000u;      // past every descriptor's bytes: loads zeros

template <typename T, int D>
struct Shape {
  static constexpr int kRow = (int)sizeof(T) * D;             // bytes of a key's row
  static constexpr int kChunks = kRow / 16;                   // 16-byte chunks of it
  static constexpr int kOut = D / 32;                         // MFMA tiles of outputs along the head
  static constexpr int kGroup = 16 * kRow;                    // bytes of 16 keys, the unit of loading
  static constexpr int kLoads = kGroup / 1024;                // 1 KB loads of a wavefront for it
  static constexpr int kLoadRows = 1024 / kRow;
  static constexpr int kQuery = D / 2;                        // a lane's half of a query, in elements
};

// XOR of a row's chunk numbers in LDS: 16 rows at one chunk (keys), and 4 rows at a run of
// 64 bytes (bf16 values), then touch every bank once.
template <typename T, int D>
__device__ __forceinline__ int key_swizzle(int row) { return sizeof(T) == 2 && D == 64 ? (row >> 1) & 7 : row & 15; }
template <typename T, int D>
__device__ __forceinline__ int value_swizzle(int row) {
  return sizeof(T) == 4 ? 0 : D == 128 ? 4 * (row & 3) : 4 * ((row >> 1) & 1);
}

__device__ __forceinline__ bool is_finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }

__device__ __forceinline__ float max_across(float v) {       // of lane and lane ^ 32
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
__device__ __forceinline__ float sum_across(float v) {
  const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

constexpr uint32_t kSawNone = 0x80000000u;      // the bits of -0

// What the outputs are multiplied by for the sum l of a row's weights.
__device__ __forceinline__ float inverse_of(float l) { return __float_as_uint(l) == kSawNone ? 0.0f : 1.0f / l; }

// A reduction over the wavefront's 64 lanes in six DPP moves (shifts within rows of 16 lanes, then
// broadcasts across them), an eighth of the latency of as many exchanges through LDS; lanes that a
// move gives nothing keep their own value, twice.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_or_own(uint32_t v) { return __builtin_amdgcn_update_dpp(v, v, CTRL, ROWS, 0xF, false); }
template <typename Op>
__device__ __forceinline__ uint32_t wave_reduce(uint32_t v, Op op) {
  v = op(v, dpp_or_own<0x111, 0xF>(v));
  v = op(v, dpp_or_own<0x112, 0xF>(v));
  v = op(v, dpp_or_own<0x114, 0xF>(v));
  v = op(v, dpp_or_own<0x118, 0xF>(v));
  v = op(v, dpp_or_own<0x142, 0xA>(v));
  v = op(v, dpp_or_own<0x143, 0xC>(v));
  return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
__device__ __forceinline__ int wave_min(int v) {
  return (int)wave_reduce((uint32_t)v, [](uint32_t x, uint32_t y) { return (uint32_t)min((int)x, (int)y); });
}
__device__ __forceinline__ float wave_max(float v) {
  return __uint_as_float(wave_reduce(__float_as_uint(v), [](uint32_t x, uint32_t y) { return __float_as_uint(fmaxf(__uint_as_float(x), __uint_as_float(y))); }));
}
// Sums need zeros where a move gives nothing.
__device__ __forceinline__ float wave_sum(float v) {
  auto step = [&](auto ctrl, auto rows) {
    v += __uint_as_float(__builtin_amdgcn_update_dpp(0u, __float_as_uint(v), decltype(ctrl)::value, decltype(rows)::value, 0xF, true));
  };
  std::integral_constant<int, 0xF> all;
  step(std::integral_constant<int, 0x111>(), all);
  step(std::integral_constant<int, 0x112>(), all);
  step(std::integral_constant<int, 0x114>(), all);
  step(std::integral_constant<int, 0x118>(), all);
  step(std::integral_constant<int, 0x142>(), std::integral_constant<int, 0xA>());
  step(std::integral_constant<int, 0x143>(), std::integral_constant<int, 0xC>());
  return __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(v), 63));
}

// Every load but the last N has landed, for this wavefront: what it reads from LDS is read after.
template <int N>
__device__ __forceinline__ void landed() {
  wait_vmcnt<N>();
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}
// This wavefront's LDS reads have returned: what they read may be loaded over.
__device__ __forceinline__ void have_read() {
  __builtin_amdgcn_s_waitcnt(0xC07F);             // lgkmcnt(0)
  asm volatile("" ::: "memory");
  __builtin_amdgcn_sched_barrier(0);
}

// A raw buffer descriptor in four scalar registers.
typedef u32x4 Descriptor;
__device__ __forceinline__ Descriptor describe(const void* base, uint32_t bytes) {
  const uint64_t p = (uint64_t)base;
  return Descriptor{(uint32_t)p, (uint32_t)(p >> 32) & 0xffffu, bytes, (uint32_t)kBufferWord3};
}
// 16 bytes of each lane into LDS at `to` + 16 lane (`to` uniform), straight from memory.  Written
// out because the compiler, which does not see which of several such loads a read of LDS
// depends on, waits for all of them before reads that depend on none; here the wait is the
// caller's (landed, or wait_vmcnt and a barrier), and nothing is returned in registers.  M0 is
// nobody else's in these kernels.
__device__ __forceinline__ void load_lds(const Descriptor& d, uint8_t* to, uint32_t offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
               :
               : "s"((uint32_t)(uintptr_t)(lds_void)to), "v"(offset), "s"(d)
               : "m0");
}

// Loads of 16 keys into LDS by one wavefront: `stride` bytes between rows, row0 the first row of
// the group that is to be loaded (earlier ones become zeros, as do rows past the descriptor's
// bytes; the whole offset is the lane's, so that all of it counts in that check).
template <typename T, int D>
struct Loader {
  using S = Shape<T, D>;
  uint32_t k_off[S::kLoads], v_off[S::kLoads];
  int row;
  __device__ __forceinline__ Loader(int lane, uint32_t stride) {
    row = lane / S::kChunks;
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) {
      const int r = row + i * S::kLoadRows, c = lane % S::kChunks;
      k_off[i] = (uint32_t)r * stride + 16u * (uint32_t)(c ^ key_swizzle<T, D>(r));
      v_off[i] = (uint32_t)r * stride + 16u * (uint32_t)(c ^ value_swizzle<T, D>(r));
    }
  }
  __device__ __forceinline__ void load(const Descriptor& d, uint8_t* to, const uint32_t (&off)[S::kLoads], int row0) const {
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) load_lds(d, to + 1024 * i, row + i * S::kLoadRows < row0 ? kNowhere : off[i]);
  }
  __device__ __forceinline__ void keys(const Descriptor& d, uint8_t* to, int row0 = 0) const { load(d, to, k_off, row0); }
  __device__ __forceinline__ void values(const Descriptor& d, uint8_t* to, int row0 = 0) const { load(d, to, v_off, row0); }
};

// The products of 32 query rows with tiles of 32 keys: what depends on the element type.
template <typename T, int D>
struct Products;

template <int D>
struct Products<uint16_t, D> {
  using S = Shape<uint16_t, D>;
  static constexpr int kSteps = D / 16;
  bf16x8 q[kSteps];
  uint32_t k_at, v_at;            // of piece 0; the other pieces' addresses differ in bits that an XOR sets
  template <int KT>
  struct Weights {
    u32x4 w[2 * KT];               // B operands of 16 keys each
  };

  __device__ __forceinline__ void start(int lane) {
    const int h = lane / 32, i = lane & 15;
    k_at = (uint32_t)((lane & 31) * S::kRow + 16 * (h ^ key_swizzle<uint16_t, D>(lane & 31)));
    v_at = (uint32_t)((4 * h + i / 4) * S::kRow + 16 * ((2 * ((lane / 16) & 1) + (i & 3) / 2) ^ value_swizzle<uint16_t, D>(i / 4)) + 8 * (i & 1));
  }
  __device__ __forceinline__ void load_query(const uint16_t* row, bool present, int lane) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      u32x4 d = {0u, 0u, 0u, 0u};
      if (present) d = *reinterpret_cast<const u32x4*>(row + 16 * s + 8 * (lane / 32));
      q[s] = __builtin_bit_cast(bf16x8, d);
    }
  }
  static constexpr int kPieces = kSteps;
  typedef bf16x8 Piece;            // of 32 keys, as an A operand
  __device__ __forceinline__ Piece key(const uint8_t* keys, int k) const { return *reinterpret_cast<const bf16x8*>(keys + (k_at ^ (uint32_t)(32 * k))); }
  __device__ __forceinline__ void score(const Piece& key, int k, f32x16& s) const {
    s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key, q[k], s, 0, 0, 0);
  }
  // Weights w[2 i], w[2 i + 1] of a lane's half of tile kt, rounded to bf16.
  template <int KT>
  static __device__ __forceinline__ void set(Weights<KT>& p, int kt, int i, float a, float b) {
    p.w[2 * kt + i / 4][i % 4] = pack_bf16x2(a, b);
  }
  template <int KT>
  static __device__ __forceinline__ float add_weights(const Weights<KT>& p, int kt, int i, float sum) {
    const uint32_t pair = p.w[2 * kt + i / 4][i % 4];      // a value first: a bit cast of a vector's element casts the vector
    return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), __builtin_bit_cast(bf16x2, 0x3F803F80u), sum, false);
  }
  // V^T of 16 keys (chunk c of the tile) and 32 outputs (tile t), as an A operand.
  __device__ __forceinline__ bf16x8 value(const uint8_t* values, int c, int t) const {
    s16x4 d[2];
#pragma unroll
    for (int s = 0; s < 2; ++s)
      d[s] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4)(values + (v_at ^ (uint32_t)(64 * t)) + (16 * c + 8 * s) * S::kRow));
    const auto lo = __builtin_bit_cast(u32x2, d[0]), hi = __builtin_bit_cast(u32x2, d[1]);
    return __builtin_bit_cast(bf16x8, u32x4{lo.x, lo.y, hi.x, hi.y});
  }
  // The same with zeros for infinities and NaN.
  static __device__ __forceinline__ bf16x8 finite(bf16x8 v) {
    u32x4 d = __builtin_bit_cast(u32x4, v);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      d[i] &= ((d[i] & 0x7f80u) == 0x7f80u ? 0u : 0xffffu) | ((d[i] & 0x7f800000u) == 0x7f800000u ? 0u : 0xffff0000u);
    return __builtin_bit_cast(bf16x8, d);
  }
  template <bool FINITE, int KT>
  __device__ __forceinline__ void accumulate(const uint8_t* values, const Weights<KT>& p, f32x16 (&o)[S::kOut]) const {
#pragma unroll
    for (int c = 0; c < 2 * KT; ++c)
#pragma unroll
      for (int t = 0; t < S::kOut; ++t) {
        const bf16x8 v = value(values, c, t);
        o[t] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(FINITE ? finite(v) : v, __builtin_bit_cast(bf16x8, p.w[c]), o[t], 0, 0, 0);
      }
  }
  // One key's weight for this lane's column, and four of its values.
  template <int KT>
  static __device__ __forceinline__ float weight_of(const Weights<KT>& p, int key) {
    const int slot = (key % 16) / 8 * 4 + key % 4, word = key / 16 * 4 + slot / 2;
    uint32_t d = 0;
#pragma unroll
    for (int i = 0; i < 8 * KT; ++i) d = i == word ? p.w[i / 4][i % 4] : d;
    const auto s = __builtin_amdgcn_permlane32_swap(d, d, false, false);
    d = (key / 4) % 2 ? s[1] : s[0];
    return slot % 2 ? bf16_hi(d) : bf16_lo(d);
  }
  static __device__ __forceinline__ f32x4 values_of(const uint8_t* values, int key, int at) {
    const u32x2 d = *reinterpret_cast<const u32x2*>(values + key * S::kRow + 16 * (at / 8 ^ value_swizzle<uint16_t, D>(key)) + 2 * (at % 8));
    return f32x4{bf16_lo(d.x), bf16_hi(d.x), bf16_lo(d.y), bf16_hi(d.y)};
  }
};

// Binary32: the same tiles on v_mfma_f32_32x32x2_f32 (one key or dimension of each half a
// step).  The dimensions of a head are taken in the order in which a lane reads them, 16
// bytes at a time: step 4 u + e multiplies dimensions 8 u + e and 8 u + 4 + e.
template <int D>
struct Products<float, D> {
  using S = Shape<float, D>;
  float q[D / 2];
  uint32_t k_base, v_base;
  int k_swz;
  template <int KT>
  struct Weights {
    f32x16 w[KT];
  };

  __device__ __forceinline__ void start(int lane) {
    k_base = (uint32_t)((lane & 31) * S::kRow);
    k_swz = key_swizzle<float, D>(lane & 31) ^ (lane / 32);
    v_base = (uint32_t)(4 * (lane / 32) * S::kRow + 4 * (lane & 31));
  }
  __device__ __forceinline__ void load_query(const float* row, bool present, int lane) {
#pragma unroll
    for (int u = 0; u < D / 8; ++u) {
      f32x4 d = {0.0f, 0.0f, 0.0f, 0.0f};
      if (present) d = *reinterpret_cast<const f32x4*>(row + 8 * u + 4 * (lane / 32));
#pragma unroll
      for (int e = 0; e < 4; ++e) q[4 * u + e] = d[e];
    }
  }
  static constexpr int kPieces = D / 8;
  typedef f32x4 Piece;
  __device__ __forceinline__ Piece key(const uint8_t* keys, int u) const { return *reinterpret_cast<const f32x4*>(keys + k_base + 16 * ((2 * u) ^ k_swz)); }
  __device__ __forceinline__ void score(const Piece& key, int u, f32x16& s) const {
#pragma unroll
    for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(key[e], q[4 * u + e], s, 0, 0, 0);
  }
  template <int KT>
  static __device__ __forceinline__ void set(Weights<KT>& p, int kt, int i, float a, float b) {
    p.w[kt][2 * i] = a;
    p.w[kt][2 * i + 1] = b;
  }
  template <int KT>
  static __device__ __forceinline__ float add_weights(const Weights<KT>& p, int kt, int i, float sum) {
    return sum + (p.w[kt][2 * i] + p.w[kt][2 * i + 1]);
  }
  template <bool FINITE, int KT>
  __device__ __forceinline__ void accumulate(const uint8_t* values, const Weights<KT>& p, f32x16 (&o)[S::kOut]) const {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int t = 0; t < S::kOut; ++t) {
          const float v = *reinterpret_cast<const float*>(values + v_base + (32 * kt + 8 * (i / 4) + i % 4) * S::kRow + 128 * t);
          o[t] = __builtin_amdgcn_mfma_f32_32x32x2f32(FINITE && !is_finite(v) ? 0.0f : v, p.w[kt][i], o[t], 0, 0, 0);
        }
  }
  template <int KT>
  static __device__ __forceinline__ float weight_of(const Weights<KT>& p, int key) {
    const int reg = key / 32 * 16 + (key % 32) / 8 * 4 + key % 4;
    float w = 0.0f;
#pragma unroll
    for (int i = 0; i < 16 * KT; ++i) w = i == reg ? p.w[i / 16][i % 16] : w;
    const auto s = __builtin_amdgcn_permlane32_swap(__float_as_uint(w), __float_as_uint(w), false, false);
    return __uint_as_float((key / 4) % 2 ? s[1] : s[0]);
  }
  static __device__ __forceinline__ f32x4 values_of(const uint8_t* values, int key, int at) {
    return *reinterpret_cast<const f32x4*>(values + key * S::kRow + 4 * at);
  }
};

// 32 query rows of a wavefront and what they have gathered so far.
template <typename T, int D>
struct Rows32 {
  using S = Shape<T, D>;
  using P = Products<T, D>;
  P x;
  f32x16 o[S::kOut];
  float m, l;                     // reference (log2 units) and this lane's share of the sum

  // `row` points at the query of this lane's column; absent ones are zeros.
  __device__ __forceinline__ void load_query(const T* row, bool present, int lane) { x.load_query(row, present, lane); }
  __device__ __forceinline__ void start(int lane) {
    x.start(lane);
#pragma unroll
    for (int t = 0; t < S::kOut; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[t][i] = 0.0f;
    m = -FLT_MAX;
    l = __uint_as_float(kSawNone);
  }

  // S^T of 32 KT keys: the tiles in turn, each piece of the keys read four products ahead.
  template <int KT>
  __device__ __forceinline__ void scores(const uint8_t* keys, f32x16 (&s)[KT]) const {
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) s[kt][i] = 0.0f;
#pragma unroll
    for (int k = 0; k < P::kPieces; ++k)
#pragma unroll
      for (int kt = 0; kt < KT; ++kt) x.score(x.key(keys + 32 * kt * S::kRow, k), k, s[kt]);
    if constexpr (sizeof(T) == 2) {
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
      for (int i = 0; i < P::kPieces * KT - 4; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, 4, 0);
    }
  }

  // Scores of keys outside [first, last], counted from the tile's first key, and of absent
  // groups of 16 (bits of `absent`) become those of keys that are not seen; true if one is.
  template <int KT>
  static __device__ __forceinline__ bool mask(f32x16 (&s)[KT], int first, int last, uint32_t absent, int lane) {
    const int h4 = 4 * (lane / 32);
    bool seen = false;
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int key = 32 * kt + 8 * (i / 4) + i % 4 + h4;
        const bool hidden = (key < first) | (key > last) | ((absent >> (2 * kt + i / 8) & 1u) != 0);
        s[kt][i] = hidden ? -__builtin_inff() : s[kt][i];
        seen |= !hidden;
      }
    return seen;
  }

  // Moves a row's reference where a score of its own exceeds it by more than kSlack, and no other
  // row's: weights are rounded relative to it, so what shares the tile would show in the result.
  // A NaN score leaves it as it is and spoils its row by its weight.
  template <int KT>
  __device__ __forceinline__ void raise(const f32x16 (&s)[KT], float scale) {
    float top = s[0][0];
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = __builtin_elementwise_maximum(top, s[kt][i]);
    top = max_across(top) * scale;
    if (__builtin_expect(__builtin_amdgcn_ballot_w64(top > m + kSlack) != 0, 0)) {
      const float to = top > m + kSlack ? top : m, by = __builtin_amdgcn_exp2f(m - to);
      m = to;
      l *= by;
#pragma unroll
      for (int t = 0; t < S::kOut; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] *= by;
    }
  }

  // Weights of 32 KT keys from their scores, and the running sum; `seen`: the row sees one of them.
  // The sum is that of the weights as the product takes them, so that their rounding is one of weights
  // that still add up to one (in bf16: a row of one or a few keys comes out as exact as its values are).
  template <int KT>
  __device__ __forceinline__ void weights(const f32x16 (&s)[KT], float scale, bool seen, typename P::template Weights<KT>& p) {
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int kt = 0; kt < KT; ++kt)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float a = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][2 * i], scale, -m));
        const float b = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kt][2 * i + 1], scale, -m));
        P::set(p, kt, i, a, b);
        sum[i % 2] = P::add_weights(p, kt, i, sum[i % 2]);
      }
    l = seen ? l + (sum[0] + sum[1]) : l;
  }

  // What values that are infinite or NaN add, key by key and only to the rows that see the key: a
  // weight of zero times such a value of a hidden key is NaN, and the matrix cores add the product
  // to every row of a tile.  The finite ones stay with the matrix cores, so that a row's bits are
  // the same whatever is hidden from it.
  template <int KT>
  __device__ __forceinline__ void accumulate_others(const uint8_t* values, const typename P::template Weights<KT>& p, int last, int lane) {
#pragma unroll 1
    for (int key = 0; key < 32 * KT; ++key) {
      const float w = P::weight_of(p, key);
#pragma unroll
      for (int t = 0; t < S::kOut; ++t)
#pragma unroll
        for (int a = 0; a < 4; ++a) {
          const f32x4 v = P::values_of(values, key, 32 * t + 8 * a + 4 * (lane / 32));
#pragma unroll
          for (int e = 0; e < 4; ++e) o[t][4 * a + e] = key <= last && !is_finite(v[e]) ? __builtin_fmaf(w, v[e], o[t][4 * a + e]) : o[t][4 * a + e];
        }
    }
  }

  template <bool CAREFUL, int KT>
  __device__ __forceinline__ void add(const uint8_t* values, const typename P::template Weights<KT>& p, bool edge, int last, int lane) {
    if constexpr (CAREFUL) {
      if (edge) {
        x.template accumulate<true, KT>(values, p, o);
        return accumulate_others<KT>(values, p, last, lane);
      }
    }
    x.template accumulate<false, KT>(values, p, o);
  }

  // Whether an output of this lane's row is not finite.
  __device__ __forceinline__ bool spoiled() const {
    float z = 0.0f;
#pragma unroll
    for (int t = 0; t < S::kOut; ++t)
#pragma unroll
      for (int i = 0; i < 16; ++i) z = __builtin_fmaf(o[t][i], 0.0f, z);
    return !(z == 0.0f);
  }

  // Outputs times `by` to the row at `out`, in bf16: lane and lane ^ 32 exchange halves so that each
  // stores 16 bytes.
  __device__ __forceinline__ void store(uint16_t* out, bool present, float by, int lane) const {
#pragma unroll
    for (int t = 0; t < S::kOut; ++t)
#pragma unroll
      for (int a = 0; a < 4; a += 2) {
        const auto x = __builtin_amdgcn_permlane32_swap(pack_bf16x2(o[t][4 * a] * by, o[t][4 * a + 1] * by),
                                                        pack_bf16x2(o[t][4 * a + 4] * by, o[t][4 * a + 5] * by), false, false);
        const auto y = __builtin_amdgcn_permlane32_swap(pack_bf16x2(o[t][4 * a + 2] * by, o[t][4 * a + 3] * by),
                                                        pack_bf16x2(o[t][4 * a + 6] * by, o[t][4 * a + 7] * by), false, false);
        if (present) *reinterpret_cast<u32x4*>(out + 32 * t + 8 * a + 8 * (lane / 32)) = u32x4{x[0], y[0], x[1], y[1]};
      }
  }
};

// Four wavefronts of 32 rows each against the same keys, which come 64 at a time through two
// stages of LDS, the next 64 on their way while these are used.  `ahead(t)` looks up what the
// loads of tile t need, before the wait for those of tile t - 1, `keys(buffer)` and
// `values(buffer)` load this wavefront's quarter of the next 64, in order; `tiles` are walked by
// all, the first `mine` of them matter to this wavefront's rows; `edge(t)` says whether some row
// does not see all keys of tile t, `hide(t, s)` then masks its scores and says whether the lane's
// row sees one, and `last(t)` is the last key of tile t that it sees.
template <bool CAREFUL, typename T, int D, typename Ahead, typename Keys, typename Values, typename Edge, typename Hide, typename Last>
__device__ __forceinline__ void walk_shared(Rows32<T, D>& r, uint8_t* lds, int tiles, int mine, float scale, int lane, Ahead ahead,
                                            Keys keys, Values values, Edge edge, Hide hide, Last last) {
  using S = Shape<T, D>;
  constexpr int kTile = 64 * S::kRow;
  r.start(lane);
  auto turn = [&](int t, uint8_t* next) {              // tile t is there, t + 1 on its way
    ahead(t + 1);
    wait_vmcnt<0>();
    lds_barrier();
    if (t + 1 < tiles) {
      keys(next);
      values(next + kTile);
    }
  };
  auto step = [&](int t, uint8_t* now, uint8_t* next) {
    turn(t, next);
    f32x16 s[2];
    r.scores(now, s);
    const bool hidden = edge(t);
    bool seen = true;
    if (__builtin_expect(hidden, 0)) seen = hide(t, s);
    r.template raise<2>(s, scale);
    typename Products<T, D>::template Weights<2> p;
    r.template weights<2>(s, scale, seen, p);
    r.template add<CAREFUL, 2>(now + kTile, p, CAREFUL && hidden, CAREFUL ? last(t) : 0, lane);
  };
  uint8_t *const a = lds, *const b = lds + 2 * kTile;
  if (tiles > 0) {
    ahead(0);
    keys(a);
    values(a + kTile);
  }
  for (int t = 0; t < mine; t += 2) {
    step(t, a, b);
    if (t + 1 < mine) step(t + 1, b, a);
  }
  for (int t = mine; t < tiles; ++t) turn(t, t & 1 ? a : b);       // the others' tiles
}

// Keys and values of up to 16 keys: where they begin and how many bytes are there.
template <typename T>
struct Group {
  const T* k;
  const T* v;
  uint32_t k_bytes, v_bytes;
  bool absent;
};

// The same 32 rows in each of `waves` wavefronts, which take keys [lo, hi) 32 at a time in turn,
// each through its own LDS (64 rows at lds + wave * 64 rows) and without barriers: the next keys are
// loaded as soon as the scores of these are formed, the next values after the product.
// `find(first)` is the group of 16 keys that begins at `first`, a multiple of 16; every row sees
// the keys up to `all`, the lane's row those up to `last`.
template <bool CAREFUL, typename T, int D, typename Find>
__device__ __forceinline__ void walk_private(Rows32<T, D>& r, uint8_t* lds, const Loader<T, D>& load_k, const Loader<T, D>& load_v, int wave,
                                             int waves, int lo, int hi, int all, int last, float scale, int lane, Find find) {
  using S = Shape<T, D>;
  if (lo >= hi) return;
  uint8_t *const k = lds + wave * 4 * S::kGroup, *const v = k + 2 * S::kGroup;
  int j = (lo & ~15) + 32 * wave;
  Group<T> now[2] = {find(j), find(j + 16)};
#pragma unroll
  for (int g = 0; g < 2; ++g) load_k.keys(describe(now[g].k, now[g].k_bytes), k + g * S::kGroup, lo - (j + 16 * g));
#pragma unroll
  for (int g = 0; g < 2; ++g) load_v.values(describe(now[g].v, now[g].v_bytes), v + g * S::kGroup, lo - (j + 16 * g));
  for (; j < hi; j += 32 * waves) {
    const int next_j = j + 32 * waves;
    const Group<T> next[2] = {find(next_j), find(next_j + 16)};
    const uint32_t absent = (now[0].absent ? 1u : 0u) | (now[1].absent ? 2u : 0u);
    const bool edge = j + 31 > min(all, hi - 1) || j < lo || absent != 0;
    landed<2 * S::kLoads>();
    f32x16 s[1];
    r.scores(k, s);
    have_read();
#pragma unroll
    for (int g = 0; g < 2; ++g) load_k.keys(describe(next[g].k, next[g].k_bytes), k + g * S::kGroup);
    bool seen = true;
    if (edge) seen = Rows32<T, D>::template mask<1>(s, lo - j, min(last, hi - 1) - j, absent, lane);
    r.template raise<1>(s, scale);
    typename Products<T, D>::template Weights<1> p;
    r.template weights<1>(s, scale, seen, p);
    landed<2 * S::kLoads>();
    r.template add<CAREFUL, 1>(v, p, edge, min(last, hi - 1) - j, lane);
    have_read();
#pragma unroll
    for (int g = 0; g < 2; ++g) load_v.values(describe(next[g].v, next[g].v_bytes), v + g * S::kGroup);
    now[0] = next[0];
    now[1] = next[1];
  }
  landed<0>();
}

// What the wavefronts of a workgroup gathered for the same `count` rows, joined through LDS (16-byte
// pieces swizzled by row) and handed on four outputs at a time: put(row, at, o, m, l).
template <int WAVES, typename T, int D, typename Put>
__device__ __forceinline__ void join_waves(const Rows32<T, D>& r, uint8_t* lds, float2* ml, int count, int wave, int lane, Put put) {
  constexpr int kPieces = D / 4;
  const float l = sum_across(r.l);
  __syncthreads();
  f32x4* const o = reinterpret_cast<f32x4*>(lds);
  const int n = lane & 31;
  if (n < count) {
#pragma unroll
    for (int t = 0; t < D / 32; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        o[(wave * 32 + n) * kPieces + ((8 * t + 2 * i + lane / 32) ^ (n % kPieces))] = f32x4{r.o[t][4 * i], r.o[t][4 * i + 1], r.o[t][4 * i + 2], r.o[t][4 * i + 3]};
    if (lane < 32) ml[wave * 32 + n] = float2{r.m, l};
  }
  __syncthreads();
  for (int i = threadIdx.x; i < count * kPieces; i += 64 * WAVES) {
    const int at = i % kPieces, of = i / kPieces;
    float m = ml[of].x, sum = __uint_as_float(kSawNone);
#pragma unroll
    for (int w = 1; w < WAVES; ++w) m = fmaxf(m, ml[w * 32 + of].x);
    f32x4 all = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const float2 x = ml[w * 32 + of];
      if (x.y == 0.0f) {
        sum += x.y;                       // for its sign
        continue;
      }
      const float by = __builtin_amdgcn_exp2f(x.x - m);
      const f32x4 y = o[(w * 32 + of) * kPieces + (at ^ (of % kPieces))];
      sum = __builtin_fmaf(by, x.y, sum);
#pragma unroll
      for (int e = 0; e < 4; ++e) all[e] = __builtin_fmaf(by, y[e], all[e]);
    }
    put(of, 4 * at, all, m, sum);
  }
}

}  // namespace attention
}  // namespace ssq
