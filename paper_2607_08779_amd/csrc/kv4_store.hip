// Keys and values of new tokens into a paged cache in 4 bits (see include/ssq_cache.h, kv4.h).
//
// The grid is that of ssq_quantize: s = gamma M / 8 in binary32, codes clip(rne(fl32(w / s)), -8, 7) against
// that s, the stored scale s in binary16.  A thread takes 8 elements of a head's key and of its value,
// four threads a group, whose maxima they exchange in DPP moves.
//
// Long runs are bound by the rows' bytes: 4099 tokens of 8 heads of 128 with the rows as held (38 MB)
// 10.2 us, of which a copy of as many bytes takes 7.4 and the launch 2; all loads, then all stores are under way
// together.  With a division for each element and tokens of a head spread over workgroups it was 12.7.
// In binary32, which divides for each element, they take 18.5 (72 MB: a copy 13.8).  One token takes 2.8, the launch.
#include "kv4.h"
#include "mfma_dequant.h"

namespace ssq {
namespace {

constexpr int kThreads = 256;

template <int CTRL>
__device__ __forceinline__ uint32_t of_quad(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true); }

constexpr float kRound = 8388616.0f;         // 2^23 + 8: t + kRound is rne(t) + 8 in its lowest bits

// Eight elements of a row as they are loaded.
template <typename T>
struct Eight;
template <>
struct Eight<uint16_t> {
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  typedef int16_t i16x2 __attribute__((ext_vector_type(2)));
  static constexpr uint32_t kSign = 0x8000u, kInfinity = 0x7F80u;
  u32x4 d;
  __device__ __forceinline__ void load(const uint16_t* p) { d = load_stream16(p); }
  __device__ __forceinline__ float of(int i) const { return i % 2 == 0 ? bf16_lo(d[i / 2]) : bf16_hi(d[i / 2]); }
  // The largest of their bits, unsigned and signed, two elements at a time.
  __device__ __forceinline__ void largest(uint32_t* any, int* positive) const {
    u16x2 u = __builtin_bit_cast(u16x2, (uint32_t)d[0]);
    i16x2 s = __builtin_bit_cast(i16x2, (uint32_t)d[0]);
#pragma unroll
    for (int i = 1; i < 4; ++i) {
      u = __builtin_elementwise_max(u, __builtin_bit_cast(u16x2, (uint32_t)d[i]));
      s = __builtin_elementwise_max(s, __builtin_bit_cast(i16x2, (uint32_t)d[i]));
    }
    *any = max((uint32_t)u[0], (uint32_t)u[1]);
    *positive = max((int)s[0], (int)s[1]);
  }
  static __device__ __forceinline__ float value(uint32_t bits) { return __uint_as_float(bits << 16); }
  // c = rne(fl32(w / s)) + 8 in a float's lowest bits.  With M and w of 8 significant bits w / s = 8 w / M is a half-integer, or at least 2^-11 from every one; w times the
  // reciprocal of s is within 2^-18 of it.  Rounded to a multiple of 2^-13 (the spacing about 1.5 * 2^10) it is the
  // half-integer again in the first case and on the same side in the second, so that rounding it to even gives
  // rne(fl32(w / s)).  Outside the range of s where the reciprocal is that close, divide.
  __device__ __forceinline__ void over(float s, float most, float (&c)[8]) const {
    if (most >= 0x1p-100f && most <= 0x1p100f) {
      const float by = __builtin_amdgcn_rcpf(s);
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] = __builtin_fmaf(of(i), by, 0x1.8p10f) + (kRound - 0x1.8p10f);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] = of(i) / s + kRound;
    }
  }
  static __device__ __forceinline__ void store(uint16_t* p, const float (&w)[8]) {
    *reinterpret_cast<u32x4*>(p) = u32x4{pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3]), pack_bf16x2(w[4], w[5]), pack_bf16x2(w[6], w[7])};
  }
};
template <>
struct Eight<float> {
  static constexpr uint32_t kSign = 0x80000000u, kInfinity = 0x7F800000u;
  u32x4 d[2];
  __device__ __forceinline__ void load(const float* p) {
    d[0] = load_stream16(p);
    d[1] = load_stream16(p + 4);
  }
  __device__ __forceinline__ float of(int i) const { return __uint_as_float(d[i / 4][i % 4]); }
  __device__ __forceinline__ void largest(uint32_t* any, int* positive) const {
    *any = d[0][0];
    *positive = (int)d[0][0];
#pragma unroll
    for (int i = 1; i < 8; ++i) {
      *any = max(*any, (uint32_t)d[i / 4][i % 4]);
      *positive = max(*positive, (int)d[i / 4][i % 4]);
    }
  }
  static __device__ __forceinline__ float value(uint32_t bits) { return __uint_as_float(bits); }
  // Where s is below the normal numbers, rounded or zero, quotients go below -8 too; 0 / 0 counts as -8, as in
  // ssq_quantize_f32.  (In bf16 M / 8 is exact, and no quotient is below -8.)
  __device__ __forceinline__ void over(float s, float, float (&c)[8]) const {
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = fmaxf(of(i) / s + kRound, kRound - 8.0f);
  }
  static __device__ __forceinline__ void store(float* p, const float (&w)[8]) {
    *reinterpret_cast<f32x4*>(p) = f32x4{w[0], w[1], w[2], w[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{w[4], w[5], w[6], w[7]};
  }
};

// The codes of 8 elements (+ 8, lowest first) and their group's scale in binary16; `held`, where wanted: what they stand for.  A
// group that holds an infinity or a NaN, or whose scale binary16 does not reach, has codes 8 and the scale NaN, so
// that all of it reads as NaN.
template <typename T>
__device__ __forceinline__ uint32_t on_grid(const Eight<T>& x, uint32_t* scale, bool want, float (&held)[8]) {
  using E = Eight<T>;
  // As whole numbers, the bits of positive elements are in their order, and those of negative ones in that of their
  // sizes: the signed maximum is the largest positive element, if there is one, the unsigned one the largest
  // negative, if there is one; NaN are larger than all.
  uint32_t any;
  int positive;
  x.largest(&any, &positive);
  any = max(any, of_quad<0xB1>(any));
  positive = max(positive, (int)of_quad<0xB1>((uint32_t)positive));
  any = max(any, of_quad<0x4E>(any));
  positive = max(positive, (int)of_quad<0x4E>((uint32_t)positive));
  const uint32_t up = (uint32_t)max(positive, 0), down = any >= E::kSign ? any - E::kSign : 0u, size = max(up, down);
  const float most = E::value(size), s = up > down ? -0.125f * most : 0.125f * most;
  uint32_t bits = f32_to_f16_bits(s);
  if (size >= E::kInfinity || (bits & 0x7C00u) == 0x7C00u) bits = 0x7E00u;
  const float by = f16_bits_to_f32(bits);
  float c[8];
  if (size == 0 || bits == 0x7E00u) {
#pragma unroll
    for (int i = 0; i < 8; ++i) c[i] = kRound;
  } else {
    x.over(s, most, c);
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) c[i] = fminf(c[i], kRound + 7.0f);
  // The bits of 2^23 above each code: 0x4B000000 once, and 16 times it; higher ones fall out.
  uint32_t codes = __float_as_uint(c[7]);
#pragma unroll
  for (int i = 6; i >= 0; --i) codes = (codes << 4) + __float_as_uint(c[i]);
  codes -= 0xFB000000u;
  if (want) {
#pragma unroll
    for (int i = 0; i < 8; ++i) held[i] = (c[i] - kRound) * by;
  }
  *scale = bits;
  return codes;
}

// A workgroup takes consecutive tokens of one head, whose places in a page lie side by side: what they write fills
// whole cache lines.
template <typename T, int D>
__global__ __launch_bounds__(kThreads) void kv4_store_kernel(const Kv4Store<T> a) {
  using L = Kv4<D>;
  constexpr int kPieces = D / 8, kTokens = kThreads / kPieces;                 // threads of a token; tokens of a workgroup
  const uint32_t head = blockIdx.x % (uint32_t)a.kv_heads, piece = threadIdx.x % kPieces;
  const int64_t token = (int64_t)(blockIdx.x / (uint32_t)a.kv_heads) * kTokens + threadIdx.x / kPieces;
  if (token >= a.tokens) return;                                // whole groups of threads
  const int64_t at = (int64_t)head * D + 8 * piece;
  Eight<T> k, v;
  k.load(a.k.p + token * a.k.stride + at);
  v.load(a.v.p + token * a.v.stride + at);
  const int64_t slot = a.slots[token];
  uint32_t k_scale, v_scale;
  float held[8];
  const uint32_t kc = on_grid(k, &k_scale, a.k_held.p != nullptr, held);
  if (a.k_held.p != nullptr) Eight<T>::store(a.k_held.p + token * a.k_held.stride + at, held);
  const uint32_t vc = on_grid(v, &v_scale, a.v_held.p != nullptr, held);
  if (a.v_held.p != nullptr) Eight<T>::store(a.v_held.p + token * a.v_held.stride + at, held);
  const int64_t page = slot >> a.page_shift;
  const uint32_t g = piece / 4, h = piece % 4;
  const uint32_t other = of_quad<0x4E>(vc);                     // of lane ^ 2: the group's other half
  if (slot < 0 || page >= a.pages) return;
  const int in_page = (int)slot & ((1 << a.page_shift) - 1), part = L::part(a.page_shift);
  uint8_t* to = a.cache + (page * a.kv_heads + head) * (int64_t)(2 * part);
  *reinterpret_cast<uint32_t*>(to + in_page * L::kCodes + 4 * (h * L::kGroups + g)) = kc;
  // four of the group's 16 bytes, each an element of its first half and one of its second
  uint8_t* to_v = to + part;
  const uint32_t shift = h < 2 ? 0 : 16, low = (h < 2 ? vc : other) >> shift, high = (h < 2 ? other : vc) >> shift;
  const uint32_t x0 = 8 * (h % 2) + (h < 2 ? 0 : 4);
  uint8_t* quad = to_v + (in_page / 4) * (4 * L::kCodes) + 4 * g + in_page % 4;
#pragma unroll
  for (uint32_t j = 0; j < 4; ++j)
    quad[(x0 + j) * 4 * L::kGroups] = (uint8_t)(((low >> (4 * j)) & 15u) | ((high >> (4 * j)) & 15u) << 4);
  if (h < 2) {
    const int scales = (L::kCodes << a.page_shift) + in_page * L::kScales + 2 * (int)g;
    *reinterpret_cast<uint16_t*>((h == 0 ? to : to_v) + scales) = (uint16_t)(h == 0 ? k_scale : v_scale);
  }
}

template <typename T>
hipError_t launch(const Kv4Store<T>& a, int head_dim, hipStream_t stream) {
  const int64_t tokens = kThreads / (head_dim / 8);             // of a workgroup
  const dim3 grid((unsigned)((a.tokens + tokens - 1) / tokens * a.kv_heads));
  if (head_dim == 64) kv4_store_kernel<T, 64><<<grid, kThreads, 0, stream>>>(a);
  else kv4_store_kernel<T, 128><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_store(const Kv4Store<uint16_t>& a, int head_dim, hipStream_t stream) { return launch(a, head_dim, stream); }
hipError_t launch_kv4_store(const Kv4Store<float>& a, int head_dim, hipStream_t stream) { return launch(a, head_dim, stream); }

}  // namespace ssq
