// Keys and values of new tokens into a paged cache in 4 bits (see include/ssq_cache.h, kv4.h).
//
// The grid is that of ssq_quantize: s = gamma M / 8 in binary32, codes clip(rne(fl32(w / s)), -8, 7) against
// that s, the stored scale s in binary16.  A thread takes 8 elements of a head's key and of its value,
// four threads a group, whose maxima they exchange in DPP moves.  Bound by the rows' bytes in long
// runs, by the launch where tokens are few.
#include "kv4.h"
#include "mfma_dequant.h"

namespace ssq {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ void load8(const uint16_t* p, float (&w)[8]) {
  const u32x4 d = load_stream16(p);
#pragma unroll
  for (int i = 0; i < 4; ++i) w[2 * i] = bf16_lo(d[i]), w[2 * i + 1] = bf16_hi(d[i]);
}
__device__ __forceinline__ void load8(const float* p, float (&w)[8]) {
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const u32x4 d = load_stream16(p + 4 * j);
#pragma unroll
    for (int i = 0; i < 4; ++i) w[4 * j + i] = __uint_as_float(d[i]);
  }
}
__device__ __forceinline__ void store8(uint16_t* p, const float (&w)[8]) {
  *reinterpret_cast<u32x4*>(p) = u32x4{pack_bf16x2(w[0], w[1]), pack_bf16x2(w[2], w[3]), pack_bf16x2(w[4], w[5]), pack_bf16x2(w[6], w[7])};
}
__device__ __forceinline__ void store8(float* p, const float (&w)[8]) {
  *reinterpret_cast<f32x4*>(p) = f32x4{w[0], w[1], w[2], w[3]};
  *reinterpret_cast<f32x4*>(p + 4) = f32x4{w[4], w[5], w[6], w[7]};
}

// The codes of 8 elements (+ 8, lowest first) and their group's scale in binary16; `w` becomes what they
// stand for.  A group that holds an infinity or a NaN, or whose scale binary16 does not reach, has the
// scale NaN, so that all of it reads as NaN.
__device__ __forceinline__ uint32_t on_grid(float (&w)[8], uint16_t* scale) {
  float hi = w[0], lo = w[0], not_finite = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    hi = fmaxf(hi, w[i]);
    lo = fminf(lo, w[i]);
    not_finite = __builtin_fmaf(w[i], 0.0f, not_finite);       // NaN from the first such element on
  }
  hi = group_max<4>(hi);
  const float down = group_max<4>(-lo);
  const float bad = group_max<4>(not_finite == 0.0f ? 0.0f : 1.0f);
  const float most = fmaxf(hi, down);
  const float s = most > 0.0f ? (hi > down ? -most : most) * 0.125f : 0.0f;       // of zeros alone +0, whatever their signs
  uint32_t bits = f32_to_f16_bits(s);
  if (bad != 0.0f || (bits & 0x7C00u) == 0x7C00u) bits = 0x7E00u;
  const float held = f16_bits_to_f32(bits);
  uint32_t codes = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float c = most > 0.0f ? fminf(fmaxf(rintf(w[i] / s), -8.0f), 7.0f) : 0.0f;
    codes |= (uint32_t)((int)c + 8) << (4 * i);
    w[i] = c * held;
  }
  *scale = (uint16_t)bits;
  return codes;
}

template <typename T, int D>
__global__ __launch_bounds__(kThreads) void kv4_store_kernel(const Kv4Store<T> a) {
  using L = Kv4<D>;
  constexpr int kPieces = D / 8;                                // threads of a head
  const uint32_t i = blockIdx.x * (uint32_t)kThreads + threadIdx.x, piece = i % kPieces, row = i / kPieces;
  const uint32_t token = row / (uint32_t)a.kv_heads, head = row - token * (uint32_t)a.kv_heads;
  if (token >= a.tokens) return;                                // whole groups of threads
  const int64_t at = (int64_t)head * D + 8 * piece;
  float k[8], v[8];
  load8(a.k.p + token * a.k.stride + at, k);
  load8(a.v.p + token * a.v.stride + at, v);
  const int64_t slot = a.slots[token];
  uint16_t k_scale, v_scale;
  const uint32_t kc = on_grid(k, &k_scale), vc = on_grid(v, &v_scale);
  if (a.k_held.p != nullptr) store8(a.k_held.p + token * a.k_held.stride + at, k);
  if (a.v_held.p != nullptr) store8(a.v_held.p + token * a.v_held.stride + at, v);
  const int64_t page = slot >> a.page_shift;
  const uint32_t g = piece / 4, h = piece % 4;
  const uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)vc, 0x4E, 0xF, 0xF, false);     // of lane ^ 2: the group's other half
  if (slot < 0 || page >= a.pages) return;
  const int in_page = (int)slot & ((1 << a.page_shift) - 1), part = L::part(a.page_shift);
  uint8_t* to = a.cache + (page * a.kv_heads + head) * (int64_t)(2 * part);
  *reinterpret_cast<uint32_t*>(to + in_page * L::kCodes + 4 * (h * L::kGroups + g)) = kc;
  uint8_t* to_v = to + part;
  const uint32_t shift = h < 2 ? 0 : 16, low = (h < 2 ? vc : other) >> shift, high = (h < 2 ? other : vc) >> shift;
  const uint32_t x0 = 8 * (h % 2) + (h < 2 ? 0 : 4);            // four of the group's 16 bytes
  uint8_t* quad = to_v + (in_page / 4) * (4 * L::kCodes) + 4 * g + in_page % 4;
#pragma unroll
  for (uint32_t j = 0; j < 4; ++j)
    quad[(x0 + j) * 4 * L::kGroups] = (uint8_t)(((low >> (4 * j)) & 15u) | ((high >> (4 * j)) & 15u) << 4);
  if (h < 2) {
    const int scales = (L::kCodes << a.page_shift) + in_page * L::kScales + 2 * (int)g;
    *reinterpret_cast<uint16_t*>((h == 0 ? to : to_v) + scales) = h == 0 ? k_scale : v_scale;
  }
}

template <typename T>
hipError_t launch(const Kv4Store<T>& a, int head_dim, hipStream_t stream) {
  const int64_t threads = a.tokens * a.kv_heads * (head_dim / 8);
  const dim3 grid((unsigned)((threads + kThreads - 1) / kThreads));
  if (head_dim == 64) kv4_store_kernel<T, 64><<<grid, kThreads, 0, stream>>>(a);
  else kv4_store_kernel<T, 128><<<grid, kThreads, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_kv4_store(const Kv4Store<uint16_t>& a, int head_dim, hipStream_t stream) { return launch(a, head_dim, stream); }
hipError_t launch_kv4_store(const Kv4Store<float>& a, int head_dim, hipStream_t stream) { return launch(a, head_dim, stream); }

}  // namespace ssq
