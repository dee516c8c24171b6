// C ABI of the attention operators: argument validation and dispatch (see
// include/ssq_attention.h).  Every check runs on the host before any HIP call.
#include "ssq_attention.h"

#include "attention_checks.h"

namespace {

constexpr int64_t kMaxRopeBytes = int64_t(127) << 30; // of all heads: 32 bytes a thread, of which a grid holds fewer than 2^32

int check_page_tables(const int32_t* held, const int32_t* added, int64_t requests, const int32_t* free_pages,
                      int64_t free_count, const int32_t* taken, int page_size, const int32_t* table, int64_t table_stride,
                      int64_t tokens, const int32_t* starts, const int32_t* lens, const int32_t* positions,
                      const int32_t* slots, const int32_t* taken_after) {
  if (requests < 0 || requests > kMaxRequests || free_count < 0 || free_count > INT32_MAX || !valid_page(page_size) ||
      table_stride < 0 || table_stride > INT32_MAX || tokens < 0 || tokens > kMaxLen)
    return SSQ_EINVAL;
  if (starts == nullptr || taken_after == nullptr || taken_after == taken || (free_count > 0 && free_pages == nullptr) ||
      (tokens > 0 && (positions == nullptr || slots == nullptr)) ||
      (requests > 0 && (held == nullptr || added == nullptr || lens == nullptr || (table_stride > 0 && table == nullptr))))
    return SSQ_EINVAL;
  for (const void* p : {held, added, free_pages, taken, table, starts, lens, positions, slots, taken_after})
    if (!aligned(p, 4)) return SSQ_EALIGN;
  // Every workgroup reads the lengths, the free list and the rows while others write: an output over
  // any of them, or over another output, is a race.
  const Span arrays[] = {{table, requests * table_stride}, {starts, requests + 1}, {lens, requests}, {positions, tokens}, {slots, tokens},
                         {taken_after, 1}, {held, requests}, {added, requests}, {free_pages, free_count}, {taken, taken != nullptr}};
  constexpr int kWritten = 6, kArrays = sizeof(arrays) / sizeof(arrays[0]);
  for (int i = 0; i < kWritten; ++i)
    for (int j = i + 1; j < kArrays; ++j)
      if (overlap(arrays[i], arrays[j])) return SSQ_EINVAL;
  return SSQ_OK;
}

template <typename T>
int norm_rope(const T* q, int64_t q_stride, const T* k, int64_t k_stride, const T* v, int64_t v_stride, int64_t tokens,
              int q_heads, int kv_heads, int head_dim, const T* q_gain, const T* k_gain, float eps, const int32_t* positions,
              const float* rope, int64_t rope_rows, T* q_out, int64_t q_out_stride, T* k_out, int64_t k_out_stride,
              const int32_t* slots, T* k_pages, T* v_pages, int64_t pages, int page_size, hipStream_t stream) {
  if (tokens < 0 || !valid_heads(q_heads, kv_heads) || !valid_dim(head_dim) || !(eps >= 0.0f) || !std::isfinite(eps) ||
      rope_rows < 0 || rope_rows > INT32_MAX)
    return SSQ_EINVAL;
  if (tokens > kMaxLen || tokens * ((int64_t)q_heads + 2 * kv_heads) > kMaxRopeBytes / (head_dim * (int64_t)sizeof(T))) return SSQ_EINVAL;
  const bool cache = slots != nullptr;
  if (cache != (k_pages != nullptr) || cache != (v_pages != nullptr)) return SSQ_EINVAL;
  if (cache && (!valid_page(page_size) || pages < 0 || pages > INT32_MAX / page_size)) return SSQ_EINVAL;
  if (!valid_stride<T>(q_stride, q_heads, head_dim) || !valid_stride<T>(k_stride, kv_heads, head_dim) ||
      !valid_stride<T>(q_out_stride, q_heads, head_dim) || (k_out != nullptr && !valid_stride<T>(k_out_stride, kv_heads, head_dim)) ||
      (cache && !valid_stride<T>(v_stride, kv_heads, head_dim)))
    return SSQ_EINVAL;
  if (tokens == 0) return SSQ_OK;
  if (q == nullptr || k == nullptr || positions == nullptr || rope == nullptr || q_out == nullptr ||
      (k_out == nullptr && !cache) || (cache && v == nullptr))
    return SSQ_EINVAL;
  if ((q_out == q && q_out_stride != q_stride) || (k_out == k && k_out_stride != k_stride)) return SSQ_EINVAL;
  for (const void* p : {(const void*)q, (const void*)k, (const void*)v, (const void*)q_gain, (const void*)k_gain,
                        (const void*)rope, (const void*)q_out, (const void*)k_out, (const void*)k_pages, (const void*)v_pages})
    if (!aligned(p, 16)) return SSQ_EALIGN;
  if (!aligned(positions, 4) || !aligned(slots, 4)) return SSQ_EALIGN;
  const ssq::NormRope<T> a = {{q, q_stride}, {k, k_stride}, {v, v_stride}, {q_out, q_out_stride}, {k_out, k_out_stride},
                              q_gain, k_gain, positions, rope, slots, {k_pages, v_pages, pages, cache ? shift_of(page_size) : 0},
                              tokens, rope_rows, q_heads, kv_heads, eps};
  return status_of(ssq::launch_qk_norm_rope(a, head_dim, stream));
}

template <typename T>
int prompt(const T* q, int64_t q_stride, const T* k, int64_t k_stride, const T* v, int64_t v_stride, const int32_t* starts,
           int64_t requests, int64_t tokens, int q_heads, int kv_heads, int head_dim, float scale, T* out, int64_t out_stride,
           hipStream_t stream) {
  if (tokens < 0 || requests < 0 || requests > kMaxRequests || !valid_heads(q_heads, kv_heads) || !valid_dim(head_dim) ||
      !(scale > 0.0f) || !std::isfinite(scale))
    return SSQ_EINVAL;
  constexpr int64_t kRows = sizeof(T) == 2 ? 128 : 32;      // of a workgroup; where bf16 takes 32, it launches few
  if (tokens > kMaxLen || tokens * q_heads + kRows * (requests + 1) * kv_heads >= kRows * ssq::kMaxGroups) return SSQ_EINVAL;
  if (!valid_stride<T>(q_stride, q_heads, head_dim) || !valid_stride<T>(out_stride, q_heads, head_dim) ||
      !valid_stride<T>(k_stride, kv_heads, head_dim) || !valid_stride<T>(v_stride, kv_heads, head_dim))
    return SSQ_EINVAL;
  if (tokens == 0) return SSQ_OK;
  if (q == nullptr || k == nullptr || v == nullptr || out == nullptr || starts == nullptr) return SSQ_EINVAL;
  for (const void* p : {(const void*)q, (const void*)k, (const void*)v, (const void*)out})
    if (!aligned(p, 16)) return SSQ_EALIGN;
  if (!aligned(starts, 4)) return SSQ_EALIGN;
  const ssq::Prompt<T> a = {{q, q_stride}, {k, k_stride}, {v, v_stride}, {out, out_stride}, starts, requests, tokens, q_heads, kv_heads, scale};
  return status_of(ssq::launch_attention_prompt(a, head_dim, stream));
}

template <typename T>
int decode(const T* q, int64_t q_stride, int64_t requests, int fresh, int q_heads, int kv_heads, int head_dim, float scale,
           const T* k_pages, const T* v_pages, int64_t pages, int page_size, const int32_t* table, int64_t table_stride,
           const int32_t* lens, int64_t max_len, int64_t prefix, T* out, int64_t out_stride, void* workspace,
           size_t workspace_bytes, hipStream_t stream) {
  if (!valid_decode_sizes(requests, fresh, q_heads, kv_heads, head_dim, max_len, prefix) || !(scale > 0.0f) || !std::isfinite(scale) ||
      !valid_page(page_size) || pages < 0 || pages > INT32_MAX / page_size || table_stride < 0 || table_stride > INT32_MAX)
    return SSQ_EINVAL;
  if (!valid_stride<T>(q_stride, q_heads, head_dim) || !valid_stride<T>(out_stride, q_heads, head_dim)) return SSQ_EINVAL;
  if (requests == 0) return SSQ_OK;
  if (q == nullptr || out == nullptr || lens == nullptr || (table_stride > 0 && max_len > 0 && table == nullptr) ||
      (pages > 0 && max_len > 0 && (k_pages == nullptr || v_pages == nullptr)))
    return SSQ_EINVAL;
  for (const void* p : {(const void*)q, (const void*)k_pages, (const void*)v_pages, (const void*)out})
    if (!aligned(p, 16)) return SSQ_EALIGN;
  if (!aligned(table, 4) || !aligned(lens, 4) || !aligned(workspace, 256)) return SSQ_EALIGN;
  const ssq::Decode<T> a = {{q, q_stride}, {out, out_stride}, {k_pages, v_pages, pages, shift_of(page_size)}, table, table_stride, lens,
                            requests, max_len, prefix, fresh, q_heads, kv_heads, scale};
  return status_of(ssq::launch_attention_decode(a, head_dim, workspace, workspace_bytes, stream));
}

}  // namespace

extern "C" {

int ssq_page_tables(const int32_t* held, const int32_t* added, int64_t requests, const int32_t* free_pages,
                    int64_t free_count, const int32_t* taken, int page_size, int32_t* table, int64_t table_stride,
                    int64_t tokens, int32_t* starts, int32_t* lens, int32_t* positions, int32_t* slots,
                    int32_t* taken_after, hipStream_t stream) {
  const int st = check_page_tables(held, added, requests, free_pages, free_count, taken, page_size, table, table_stride, tokens,
                                   starts, lens, positions, slots, taken_after);
  if (st != SSQ_OK) return st;
  return status_of(ssq::launch_page_tables(held, added, requests, free_pages, free_count, taken, shift_of(page_size), table,
                                           table_stride, tokens, starts, lens, positions, slots, taken_after, stream));
}

int ssq_qk_norm_rope(const uint16_t* q, int64_t q_stride, const uint16_t* k, int64_t k_stride, const uint16_t* v,
                     int64_t v_stride, int64_t tokens, int q_heads, int kv_heads, int head_dim, const uint16_t* q_gain,
                     const uint16_t* k_gain, float eps, const int32_t* positions, const float* rope, int64_t rope_rows,
                     uint16_t* q_out, int64_t q_out_stride, uint16_t* k_out, int64_t k_out_stride, const int32_t* slots,
                     uint16_t* k_pages, uint16_t* v_pages, int64_t pages, int page_size, hipStream_t stream) {
  return norm_rope(q, q_stride, k, k_stride, v, v_stride, tokens, q_heads, kv_heads, head_dim, q_gain, k_gain, eps, positions, rope,
                   rope_rows, q_out, q_out_stride, k_out, k_out_stride, slots, k_pages, v_pages, pages, page_size, stream);
}

int ssq_qk_norm_rope_f32(const float* q, int64_t q_stride, const float* k, int64_t k_stride, const float* v, int64_t v_stride,
                         int64_t tokens, int q_heads, int kv_heads, int head_dim, const float* q_gain, const float* k_gain,
                         float eps, const int32_t* positions, const float* rope, int64_t rope_rows, float* q_out,
                         int64_t q_out_stride, float* k_out, int64_t k_out_stride, const int32_t* slots, float* k_pages,
                         float* v_pages, int64_t pages, int page_size, hipStream_t stream) {
  return norm_rope(q, q_stride, k, k_stride, v, v_stride, tokens, q_heads, kv_heads, head_dim, q_gain, k_gain, eps, positions, rope,
                   rope_rows, q_out, q_out_stride, k_out, k_out_stride, slots, k_pages, v_pages, pages, page_size, stream);
}

int ssq_attention_prompt(const uint16_t* q, int64_t q_stride, const uint16_t* k, int64_t k_stride, const uint16_t* v,
                         int64_t v_stride, const int32_t* starts, int64_t requests, int64_t tokens, int q_heads, int kv_heads,
                         int head_dim, float scale, uint16_t* out, int64_t out_stride, hipStream_t stream) {
  return prompt(q, q_stride, k, k_stride, v, v_stride, starts, requests, tokens, q_heads, kv_heads, head_dim, scale, out, out_stride, stream);
}

int ssq_attention_prompt_f32(const float* q, int64_t q_stride, const float* k, int64_t k_stride, const float* v, int64_t v_stride,
                             const int32_t* starts, int64_t requests, int64_t tokens, int q_heads, int kv_heads, int head_dim,
                             float scale, float* out, int64_t out_stride, hipStream_t stream) {
  return prompt(q, q_stride, k, k_stride, v, v_stride, starts, requests, tokens, q_heads, kv_heads, head_dim, scale, out, out_stride, stream);
}

int ssq_attention_decode(const uint16_t* q, int64_t q_stride, int64_t requests, int fresh, int q_heads, int kv_heads, int head_dim,
                         float scale, const uint16_t* k_pages, const uint16_t* v_pages, int64_t pages, int page_size,
                         const int32_t* table, int64_t table_stride, const int32_t* lens, int64_t max_len, int64_t prefix,
                         uint16_t* out, int64_t out_stride, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return decode(q, q_stride, requests, fresh, q_heads, kv_heads, head_dim, scale, k_pages, v_pages, pages, page_size, table,
                table_stride, lens, max_len, prefix, out, out_stride, workspace, workspace_bytes, stream);
}

int ssq_attention_decode_f32(const float* q, int64_t q_stride, int64_t requests, int fresh, int q_heads, int kv_heads, int head_dim,
                             float scale, const float* k_pages, const float* v_pages, int64_t pages, int page_size,
                             const int32_t* table, int64_t table_stride, const int32_t* lens, int64_t max_len, int64_t prefix,
                             float* out, int64_t out_stride, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return decode(q, q_stride, requests, fresh, q_heads, kv_heads, head_dim, scale, k_pages, v_pages, pages, page_size, table,
                table_stride, lens, max_len, prefix, out, out_stride, workspace, workspace_bytes, stream);
}

size_t ssq_attention_decode_workspace_size(int64_t requests, int fresh, int q_heads, int kv_heads, int head_dim, int64_t max_len,
                                           int64_t prefix) {
  if (!valid_decode_sizes(requests, fresh, q_heads, kv_heads, head_dim, max_len, prefix) || requests == 0) return 0;
  return ssq::attention_decode_workspace_bytes(requests, fresh, q_heads, kv_heads, head_dim, max_len, prefix);
}

}  // extern "C"
