// Internal declarations of the attention operators (see include/ssq_attention.h).
#pragma once

#include "ssq_internal.h"

namespace ssq {

constexpr int64_t kMaxGroups = int64_t(1) << 24;     // workgroups of 256 threads: a grid holds fewer than 2^32 threads

// Packed rows of heads: row t starts `stride` elements after row t - 1.
template <typename T>
struct Rows {
  T* p;
  int64_t stride;
};

// The paged cache: [pages, kv_heads, 1 << page_shift, head_dim].
template <typename T>
struct Cache {
  T* k;
  T* v;
  int64_t pages;
  int page_shift;
};

hipError_t launch_page_tables(const int32_t* held, const int32_t* added, int64_t requests, const int32_t* free_pages,
                              int64_t free_count, const int32_t* taken, int page_shift, int32_t* table,
                              int64_t table_stride, int64_t tokens, int32_t* starts, int32_t* lens, int32_t* positions,
                              int32_t* slots, int32_t* taken_after, hipStream_t stream);

template <typename T>
struct NormRope {
  Rows<const T> q, k, v;
  Rows<T> q_out, k_out;          // k_out.p may be null
  const T* q_gain;
  const T* k_gain;
  const int32_t* positions;
  const float* rope;
  const int32_t* slots;          // null: no cache
  Cache<T> cache;
  int64_t tokens, rope_rows;
  int q_heads, kv_heads;
  float eps;
};
hipError_t launch_qk_norm_rope(const NormRope<uint16_t>& a, int head_dim, hipStream_t stream);
hipError_t launch_qk_norm_rope(const NormRope<float>& a, int head_dim, hipStream_t stream);

template <typename T>
struct Prompt {
  Rows<const T> q, k, v;
  Rows<T> out;
  const int32_t* starts;
  int64_t requests, tokens;
  int q_heads, kv_heads;
  float scale;
};
hipError_t launch_attention_prompt(const Prompt<uint16_t>& a, int head_dim, hipStream_t stream);
hipError_t launch_attention_prompt(const Prompt<float>& a, int head_dim, hipStream_t stream);

template <typename T>
struct Decode {
  Rows<const T> q;
  Rows<T> out;
  Cache<const T> cache;
  const int32_t* table;
  int64_t table_stride;
  const int32_t* lens;
  int64_t requests, max_len, prefix;
  int fresh, q_heads, kv_heads;
  float scale;
};
hipError_t launch_attention_decode(const Decode<uint16_t>& a, int head_dim, void* workspace, size_t workspace_bytes,
                                   hipStream_t stream);
hipError_t launch_attention_decode(const Decode<float>& a, int head_dim, void* workspace, size_t workspace_bytes,
                                   hipStream_t stream);
size_t attention_decode_workspace_bytes(int64_t requests, int fresh, int q_heads, int kv_heads, int head_dim,
                                        int64_t max_len, int64_t prefix);

}  // namespace ssq
