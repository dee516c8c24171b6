// Norms of queries and keys for each head, the position rotation and the store into the
// paged cache, in one pass (see include/ssq_attention.h).
//
//   n = x / sqrt(mean(x^2) + eps) * gain;   out = (n1 cos - n2 sin, n2 cos + n1 sin)
//
// with n1, n2 the halves of a head.  Bound by memory: every head is read once and written
// once (keys twice where a cache is given, values once), the arithmetic is a few
// instructions per element.  A lane holds 16 bytes of each half, so that the rotation needs
// no exchange between lanes and every access is 16 bytes wide; 4 to 16 neighbouring lanes
// hold a head and add their squares with DPP moves.  4099 tokens of 40/8 heads of 128 into a cache:
// 27 us, 4.7 TB/s, 91 % of a large copy's rate; one token of 32/8 heads: 2.8 us, a launch.  Heads of all tokens form one list that
// the grid covers: the rotation row is read again for every head of a token, from L1.
#include "attention_internal.h"

namespace ssq {
namespace {

constexpr int kThreads = 256;

template <typename T>
struct Piece;                                 // 16 bytes of a head in binary32
template <>
struct Piece<uint16_t> {
  static constexpr int kCount = 8;
  static __device__ __forceinline__ void load(const uint16_t* p, float (&v)[8]) {
    const u32x4 d = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[2 * i] = bf16_lo(d[i]), v[2 * i + 1] = bf16_hi(d[i]);
  }
  static __device__ __forceinline__ u32x4 packed(const float (&v)[8]) {
    u32x4 d;
#pragma unroll
    for (int i = 0; i < 4; ++i) d[i] = (uint32_t)f32_to_bf16_bits(v[2 * i]) | (uint32_t)f32_to_bf16_bits(v[2 * i + 1]) << 16;
    return d;
  }
};
template <>
struct Piece<float> {
  static constexpr int kCount = 4;
  static __device__ __forceinline__ void load(const float* p, float (&v)[4]) {
    const float4 d = *reinterpret_cast<const float4*>(p);
    v[0] = d.x, v[1] = d.y, v[2] = d.z, v[3] = d.w;
  }
  static __device__ __forceinline__ u32x4 packed(const float (&v)[4]) {
    return u32x4{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
  }
};

// Sum over aligned groups of 4, 8 or 16 lanes, in every lane of the group.
template <int WIDTH>
__device__ __forceinline__ float lanes_sum(float v) {
  v = dpp_add<0xB1, 0xF>(v);                              // quad_perm [1,0,3,2]
  v = dpp_add<0x4E, 0xF>(v);                              // quad_perm [2,3,0,1]
  if constexpr (WIDTH >= 8) v = dpp_add<0x141, 0xF>(v);   // row_half_mirror
  if constexpr (WIDTH >= 16) v = dpp_add<0x140, 0xF>(v);  // row_mirror
  return v;
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void qk_norm_rope_kernel(const NormRope<T> a, int per_token, int total) {
  using P = Piece<T>;
  constexpr int E = P::kCount, L = D / 2 / E, kHeads = kThreads / L;
  const int unit = (int)blockIdx.x * kHeads + (int)threadIdx.x / L, at = (int)threadIdx.x % L * E;
  if (unit >= total) return;                  // whole groups of L lanes leave together
  const int t = unit / per_token, u = unit - t * per_token;
  const bool is_q = u < a.q_heads, is_v = u >= a.q_heads + a.kv_heads;
  const int h = is_q ? u : is_v ? u - a.q_heads - a.kv_heads : u - a.q_heads;

  int64_t place = -1;                         // element offset of the head in the cache
  if (!is_q && a.slots != nullptr) {
    const int slot = a.slots[t];
    const int64_t page = slot >> a.cache.page_shift;
    if (slot >= 0 && page < a.cache.pages)
      place = ((((page * a.kv_heads + h) << a.cache.page_shift) + (slot & ((1 << a.cache.page_shift) - 1))) * D) + at;
  }
  if (is_v) {
    if (place < 0) return;
    const T* x = a.v.p + t * a.v.stride + h * D + at;
    const u32x4 lo = *reinterpret_cast<const u32x4*>(x), hi = *reinterpret_cast<const u32x4*>(x + D / 2);
    *reinterpret_cast<u32x4*>(a.cache.v + place) = lo;
    *reinterpret_cast<u32x4*>(a.cache.v + place + D / 2) = hi;
    return;
  }

  const Rows<const T> in = is_q ? a.q : a.k;
  const T* x = in.p + t * in.stride + h * D + at;
  float lo[E], hi[E], c[E], s[E];
  P::load(x, lo);
  P::load(x + D / 2, hi);
  const int position = a.positions[t];
  if (position >= 0 && position < a.rope_rows) {
    const float* row = a.rope + (int64_t)position * D + at;
#pragma unroll
    for (int i = 0; i < E; i += 4) {
      const float4 x4 = *reinterpret_cast<const float4*>(row + i), y4 = *reinterpret_cast<const float4*>(row + D / 2 + i);
      c[i] = x4.x, c[i + 1] = x4.y, c[i + 2] = x4.z, c[i + 3] = x4.w;
      s[i] = y4.x, s[i + 1] = y4.y, s[i + 2] = y4.z, s[i + 3] = y4.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < E; ++i) c[i] = s[i] = __uint_as_float(0x7fc00000u);
  }
  const T* gain = is_q ? a.q_gain : a.k_gain;
  if (gain != nullptr) {
    float sum = 0.0f, g[E];
#pragma unroll
    for (int i = 0; i < E; ++i) sum = __builtin_fmaf(lo[i], lo[i], __builtin_fmaf(hi[i], hi[i], sum));
    const float r = rsqrtf(lanes_sum<L>(sum) * (1.0f / (float)D) + a.eps);
    P::load(gain + at, g);
#pragma unroll
    for (int i = 0; i < E; ++i) lo[i] = lo[i] * r * g[i];
    P::load(gain + at + D / 2, g);
#pragma unroll
    for (int i = 0; i < E; ++i) hi[i] = hi[i] * r * g[i];
  }
  float out[E], out2[E];
#pragma unroll
  for (int i = 0; i < E; ++i) {
    out[i] = __builtin_fmaf(lo[i], c[i], -(hi[i] * s[i]));
    out2[i] = __builtin_fmaf(hi[i], c[i], lo[i] * s[i]);
  }
  const u32x4 p = P::packed(out), p2 = P::packed(out2);
  const Rows<T> to = is_q ? a.q_out : a.k_out;
  if (to.p != nullptr) {
    T* y = to.p + t * to.stride + h * D + at;
    *reinterpret_cast<u32x4*>(y) = p;
    *reinterpret_cast<u32x4*>(y + D / 2) = p2;
  }
  if (place >= 0) {
    *reinterpret_cast<u32x4*>(a.cache.k + place) = p;
    *reinterpret_cast<u32x4*>(a.cache.k + place + D / 2) = p2;
  }
}

template <typename T>
hipError_t launch(const NormRope<T>& a, int head_dim, hipStream_t stream) {
  const int per_token = a.q_heads + (a.slots != nullptr ? 2 : 1) * a.kv_heads;
  const int total = (int)(a.tokens * per_token);
  const int heads = kThreads / (head_dim / 2 / Piece<T>::kCount);
  const dim3 grid((unsigned)((total + (int64_t)heads - 1) / heads));
  if (head_dim == 64) qk_norm_rope_kernel<T, 64><<<grid, kThreads, 0, stream>>>(a, per_token, total);
  else qk_norm_rope_kernel<T, 128><<<grid, kThreads, 0, stream>>>(a, per_token, total);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_qk_norm_rope(const NormRope<uint16_t>& a, int head_dim, hipStream_t stream) { return launch(a, head_dim, stream); }
hipError_t launch_qk_norm_rope(const NormRope<float>& a, int head_dim, hipStream_t stream) { return launch(a, head_dim, stream); }

}  // namespace ssq
