// The paged cache in 4 bits (see include/ssq_cache.h): for each page and key/value head the keys' part,
// then the values', each the codes of the page's tokens and behind them their scales.
//
// Both layouts are those in which a wavefront takes 16 tokens as operands of the 16x16x32 matrix
// instruction without moving a bit between lanes.  There lane 16 h + x holds row x and the terms
// 8 h ... 8 h + 7 of the 32 that are summed:
//
// * keys (row: token, terms: a group's 32 elements): the lane needs the words of elements
//   8 h ... 8 h + 7 of every group of its token, which stand side by side: word h * groups + g of a
//   token holds elements 32 g + 8 h + (0..7), lowest in the lowest bits.
// * values (row: element, terms: tokens): four tokens interleave, so that a word holds two elements of
//   each: byte i of word x * groups + g of a quad holds elements 32 g + x (low half) and
//   32 g + 16 + x (high half) of its token i.  A token's codes are whole bytes: tokens of a quad
//   are stored by whoever has them, with byte stores.
//
// Either way a lane's words of 16 tokens are D / 8 consecutive bytes.
#pragma once

#include "attention_internal.h"

namespace ssq {

template <int D>
struct Kv4 {
  static constexpr int kGroups = D / 32;                       // groups of 32 elements, one scale each
  static constexpr int kCodes = D / 2, kScales = D / 16;       // bytes of a token
  static __host__ __device__ __forceinline__ int part(int page_shift) { return (kCodes + kScales) << page_shift; }
};

template <typename T>
struct Kv4Store {
  Rows<const T> k, v;
  Rows<T> k_held, v_held;        // p null: not wanted
  const int32_t* slots;
  uint8_t* cache;
  int64_t tokens, pages;
  int kv_heads, page_shift;
};
hipError_t launch_kv4_store(const Kv4Store<uint16_t>& a, int head_dim, hipStream_t stream);
hipError_t launch_kv4_store(const Kv4Store<float>& a, int head_dim, hipStream_t stream);

// Decode's arguments, whose cache pointers are null, and the cache in their place.
hipError_t launch_attention_decode_kv4(const Decode<uint16_t>& a, const uint8_t* cache, int head_dim, void* workspace,
                                       size_t workspace_bytes, hipStream_t stream);
hipError_t launch_attention_decode_kv4(const Decode<float>& a, const uint8_t* cache, int head_dim, void* workspace,
                                       size_t workspace_bytes, hipStream_t stream);
size_t attention_decode_kv4_workspace_bytes(int64_t requests, int fresh, int q_heads, int kv_heads, int head_dim,
                                            int64_t max_len, int64_t prefix);

}  // namespace ssq
