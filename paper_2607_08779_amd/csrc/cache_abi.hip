// C ABI of the 4-bit cache and of the operators on pages: argument validation and dispatch (see
// include/ssq_cache.h).  Every check runs on the host before any HIP call.
#include "ssq_cache.h"

#include <algorithm>

#include "attention_checks.h"
#include "kv4.h"
#include "page_lists.h"

namespace {

constexpr int kDecodeTile = 16;          // rows of a workgroup of the 4-bit decode kernel

// No array that is written (the first `written`) over another.
template <int N>
bool separate(const Span (&arrays)[N], int written) {
  for (int i = 0; i < written; ++i)
    for (int j = i + 1; j < N; ++j)
      if (overlap(arrays[i], arrays[j])) return false;
  return true;
}

// `count` rows of `bytes` bytes, `stride` bytes apart; no rows: an array that is not given.
struct RowSpan {
  const void* p;
  int64_t count, bytes, stride;
};
bool same(const RowSpan& a, const RowSpan& b) { return a.p == b.p && a.stride == b.stride; }
// Whether a byte is in a row of both.  Not by their ends alone: k and v lie between each other in the rows of a fused
// projection, as may the rows that are written.
bool overlap(const RowSpan& a, const RowSpan& b) {
  if (a.count == 0 || b.count == 0) return false;
  const int64_t d = (int64_t)(reinterpret_cast<uintptr_t>(b.p) - reinterpret_cast<uintptr_t>(a.p));
  if (d >= (a.count - 1) * a.stride + a.bytes || -d >= (b.count - 1) * b.stride + b.bytes) return false;
  if (a.count > b.count) return overlap(b, a);
  // whether a row of a that begins `at` bytes behind b's first one meets the first of b's rows, from `from` on, that ends behind `at`
  auto meets = [&](int64_t at, int64_t from) {
    const int64_t x = at - b.bytes, floor = x / b.stride - (x % b.stride < 0), j = std::max(floor + 1, from);
    return j < b.count && j * b.stride < at + a.bytes;
  };
  if (a.stride == b.stride) return meets(-d, 1 - a.count);        // the difference of two rows' numbers is what counts
  for (int64_t i = 0; i < a.count; ++i)
    if (meets(i * a.stride - d, 0)) return true;
  return false;
}

template <typename T>
int kv4_store(const T* k, int64_t k_stride, const T* v, int64_t v_stride, int64_t tokens, int kv_heads, int head_dim, const int32_t* slots,
              uint8_t* cache, int64_t pages, int page_size, T* k_held, int64_t k_held_stride, T* v_held, int64_t v_held_stride,
              hipStream_t stream) {
  if (tokens < 0 || tokens > kMaxLen || !valid_heads(kv_heads, kv_heads) || !valid_dim(head_dim) || !valid_page(page_size) || pages < 0 ||
      pages > INT32_MAX / page_size)
    return SSQ_EINVAL;
  const int64_t together = 256 / (head_dim / 8);            // tokens of a head that a workgroup takes
  if ((tokens + together - 1) / together * kv_heads >= ssq::kMaxGroups) return SSQ_EINVAL;
  if (!valid_stride<T>(k_stride, kv_heads, head_dim) || !valid_stride<T>(v_stride, kv_heads, head_dim) ||
      (k_held != nullptr && !valid_stride<T>(k_held_stride, kv_heads, head_dim)) || (v_held != nullptr && !valid_stride<T>(v_held_stride, kv_heads, head_dim)))
    return SSQ_EINVAL;
  if (tokens == 0) return SSQ_OK;
  if (k == nullptr || v == nullptr || slots == nullptr || (pages > 0 && cache == nullptr)) return SSQ_EINVAL;
  if ((k_held == k && k_held_stride != k_stride) || (v_held == v && v_held_stride != v_stride)) return SSQ_EINVAL;
  for (const void* p : {(const void*)k, (const void*)v, (const void*)cache, (const void*)k_held, (const void*)v_held})
    if (!aligned(p, 16)) return SSQ_EALIGN;
  if (!aligned(slots, 4)) return SSQ_EALIGN;
  // Of rows that are written, a thread reads and writes the same elements of k, v and both outputs; so k_held may be k, and where
  // k and v are the same rows all four may be.
  auto rows = [&](const T* p, int64_t stride) { return RowSpan{p, p != nullptr ? tokens : 0, (int64_t)sizeof(T) * kv_heads * head_dim, (int64_t)sizeof(T) * stride}; };
  const RowSpan kr = rows(k, k_stride), vr = rows(v, v_stride), kh = rows(k_held, k_held_stride), vh = rows(v_held, v_held_stride);
  const int64_t cache_bytes = pages * kv_heads * page_size * (head_dim + head_dim / 8);
  const RowSpan cached = {cache, cache_bytes > 0, cache_bytes, cache_bytes}, places = {slots, 1, 4 * tokens, 4 * tokens};
  const bool one = same(kr, vr);
  if ((overlap(kh, kr) && !same(kh, kr)) || (overlap(kh, vr) && !(one && same(kh, vr))) || (overlap(vh, vr) && !same(vh, vr)) ||
      (overlap(vh, kr) && !(one && same(vh, kr))) || (overlap(kh, vh) && !(one && same(kh, vh))))
    return SSQ_EINVAL;
  for (const RowSpan& x : {kr, vr, kh, vh, places})
    if (overlap(cached, x)) return SSQ_EINVAL;
  if (overlap(kh, places) || overlap(vh, places)) return SSQ_EINVAL;
  const ssq::Kv4Store<T> a = {{k, k_stride}, {v, v_stride}, {k_held, k_held_stride}, {v_held, v_held_stride}, slots, cache, tokens, pages, kv_heads, shift_of(page_size)};
  return status_of(ssq::launch_kv4_store(a, head_dim, stream));
}

template <typename T>
int decode_kv4(const T* q, int64_t q_stride, int64_t requests, int fresh, int q_heads, int kv_heads, int head_dim, float scale, const uint8_t* cache,
               int64_t pages, int page_size, const int32_t* table, int64_t table_stride, const int32_t* lens, int64_t max_len, int64_t prefix, T* out,
               int64_t out_stride, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  if (!valid_decode_sizes(requests, fresh, q_heads, kv_heads, head_dim, max_len, prefix, kDecodeTile) || !(scale > 0.0f) || !std::isfinite(scale) ||
      !valid_page(page_size) || pages < 0 || pages > INT32_MAX / page_size || table_stride < 0 || table_stride > INT32_MAX)
    return SSQ_EINVAL;
  if (!valid_stride<T>(q_stride, q_heads, head_dim) || !valid_stride<T>(out_stride, q_heads, head_dim)) return SSQ_EINVAL;
  if (requests == 0) return SSQ_OK;
  if (q == nullptr || out == nullptr || lens == nullptr || (table_stride > 0 && max_len > 0 && table == nullptr) || (pages > 0 && max_len > 0 && cache == nullptr))
    return SSQ_EINVAL;
  for (const void* p : {(const void*)q, (const void*)cache, (const void*)out})
    if (!aligned(p, 16)) return SSQ_EALIGN;
  if (!aligned(table, 4) || !aligned(lens, 4) || !aligned(workspace, 256)) return SSQ_EALIGN;
  const ssq::Decode<T> a = {{q, q_stride}, {out, out_stride}, {nullptr, nullptr, pages, shift_of(page_size)}, table, table_stride, lens,
                            requests, max_len, prefix, fresh, q_heads, kv_heads, scale};
  return status_of(ssq::launch_attention_decode_kv4(a, cache, head_dim, workspace, workspace_bytes, stream));
}

int collect(const int32_t* lens, int64_t requests, const int32_t* table, int64_t table_stride, int page_size, int64_t pages, const uint8_t* pinned,
            bool compact, int32_t* table_out, int32_t* free_pages, int32_t* count, int32_t* src, int32_t* dst, int32_t* moved, void* workspace,
            size_t workspace_bytes, hipStream_t stream) {
  if (requests < 0 || requests > kMaxRequests || table_stride < 0 || table_stride > INT32_MAX || !valid_page(page_size) || pages < 0 ||
      pages > INT32_MAX / page_size || requests * ((table_stride + 1023) / 1024) >= ssq::kMaxGroups)
    return SSQ_EINVAL;
  const bool rows = requests > 0 && table_stride > 0;
  if (!rows) requests = 0;                 // of rows without entries not even the lengths are read: lens may be null
  if (count == nullptr || (pages > 0 && free_pages == nullptr) || (rows && (lens == nullptr || table == nullptr)) || workspace == nullptr ||
      workspace_bytes < ssq::page_collect_workspace_bytes(pages, compact))
    return SSQ_EINVAL;
  if (compact && (moved == nullptr || (rows && table_out == nullptr) || (pages > 1 && (src == nullptr || dst == nullptr)))) return SSQ_EINVAL;
  for (const void* p : {lens, table, (const int32_t*)table_out, (const int32_t*)free_pages, (const int32_t*)count, (const int32_t*)src, (const int32_t*)dst, (const int32_t*)moved})
    if (!aligned(p, 4)) return SSQ_EALIGN;
  if (!aligned(workspace, 256)) return SSQ_EALIGN;
  const int64_t entries = requests * table_stride, half = compact ? pages / 2 : 0;
  const bool in_place = compact && table_out == table;      // one array, which is written
  const Span arrays[] = {{free_pages, pages}, {count, 1}, {src, half}, {dst, half}, {moved, compact}, {workspace, (int64_t)workspace_bytes, 1},
                         {table_out, compact ? entries : 0}, {lens, requests}, {table, in_place ? 0 : entries}, {pinned, pinned != nullptr ? pages : 0, 1}};
  if (!separate(arrays, 7)) return SSQ_EINVAL;
  const ssq::PageCollect a = {lens, table, pinned, table_out, free_pages, count, src, dst, moved, requests, table_stride, pages, shift_of(page_size)};
  return status_of(ssq::launch_page_collect(a, compact, workspace, stream));
}

}  // namespace

extern "C" {

int ssq_kv4_store(const uint16_t* k, int64_t k_stride, const uint16_t* v, int64_t v_stride, int64_t tokens, int kv_heads, int head_dim,
                  const int32_t* slots, uint8_t* cache, int64_t pages, int page_size, uint16_t* k_held, int64_t k_held_stride, uint16_t* v_held,
                  int64_t v_held_stride, hipStream_t stream) {
  return kv4_store(k, k_stride, v, v_stride, tokens, kv_heads, head_dim, slots, cache, pages, page_size, k_held, k_held_stride, v_held, v_held_stride, stream);
}

int ssq_kv4_store_f32(const float* k, int64_t k_stride, const float* v, int64_t v_stride, int64_t tokens, int kv_heads, int head_dim,
                      const int32_t* slots, uint8_t* cache, int64_t pages, int page_size, float* k_held, int64_t k_held_stride, float* v_held,
                      int64_t v_held_stride, hipStream_t stream) {
  return kv4_store(k, k_stride, v, v_stride, tokens, kv_heads, head_dim, slots, cache, pages, page_size, k_held, k_held_stride, v_held, v_held_stride, stream);
}

int ssq_attention_decode_kv4(const uint16_t* q, int64_t q_stride, int64_t requests, int fresh, int q_heads, int kv_heads, int head_dim, float scale,
                             const uint8_t* cache, int64_t pages, int page_size, const int32_t* table, int64_t table_stride, const int32_t* lens,
                             int64_t max_len, int64_t prefix, uint16_t* out, int64_t out_stride, void* workspace, size_t workspace_bytes,
                             hipStream_t stream) {
  return decode_kv4(q, q_stride, requests, fresh, q_heads, kv_heads, head_dim, scale, cache, pages, page_size, table, table_stride, lens, max_len, prefix,
                    out, out_stride, workspace, workspace_bytes, stream);
}

int ssq_attention_decode_kv4_f32(const float* q, int64_t q_stride, int64_t requests, int fresh, int q_heads, int kv_heads, int head_dim, float scale,
                                 const uint8_t* cache, int64_t pages, int page_size, const int32_t* table, int64_t table_stride, const int32_t* lens,
                                 int64_t max_len, int64_t prefix, float* out, int64_t out_stride, void* workspace, size_t workspace_bytes,
                                 hipStream_t stream) {
  return decode_kv4(q, q_stride, requests, fresh, q_heads, kv_heads, head_dim, scale, cache, pages, page_size, table, table_stride, lens, max_len, prefix,
                    out, out_stride, workspace, workspace_bytes, stream);
}

size_t ssq_attention_decode_kv4_workspace_size(int64_t requests, int fresh, int q_heads, int kv_heads, int head_dim, int64_t max_len, int64_t prefix) {
  if (!valid_decode_sizes(requests, fresh, q_heads, kv_heads, head_dim, max_len, prefix, kDecodeTile) || requests == 0) return 0;
  return ssq::attention_decode_kv4_workspace_bytes(requests, fresh, q_heads, kv_heads, head_dim, max_len, prefix);
}

int ssq_page_fork(const int32_t* parents, int64_t requests, const int32_t* lens, const int32_t* table, int64_t rows, int64_t table_stride,
                  const int32_t* free_pages, int64_t free_count, const int32_t* taken, int page_size, int32_t* table_out, int64_t table_out_stride,
                  int32_t* lens_out, int32_t* src, int32_t* dst, int32_t* taken_after, hipStream_t stream) {
  if (requests < 0 || requests > ssq::kMaxForkRows || rows < 0 || rows > ssq::kMaxForkRows || table_stride < 0 || table_stride > INT32_MAX ||
      table_out_stride < 0 || table_out_stride > INT32_MAX || free_count < 0 || free_count > INT32_MAX || !valid_page(page_size))
    return SSQ_EINVAL;
  if (taken_after == nullptr || (free_count > 0 && free_pages == nullptr) || (rows > 0 && (lens == nullptr || (table_stride > 0 && table == nullptr))) ||
      (requests > 0 && (parents == nullptr || lens_out == nullptr || src == nullptr || dst == nullptr || (table_out_stride > 0 && table_out == nullptr))))
    return SSQ_EINVAL;
  for (const int32_t* p : {parents, lens, table, free_pages, taken, (const int32_t*)table_out, (const int32_t*)lens_out, (const int32_t*)src, (const int32_t*)dst,
                           (const int32_t*)taken_after})
    if (!aligned(p, 4)) return SSQ_EALIGN;
  const Span arrays[] = {{table_out, requests * table_out_stride}, {lens_out, requests}, {src, requests}, {dst, requests}, {taken_after, 1}, {parents, requests},
                         {lens, rows}, {table, rows * table_stride}, {free_pages, free_count}, {taken, taken != nullptr}};
  if (!separate(arrays, 5)) return SSQ_EINVAL;
  const ssq::PageFork a = {parents, lens, table, free_pages, taken, table_out, lens_out, src, dst, taken_after, requests, rows, table_stride, table_out_stride,
                           free_count, shift_of(page_size)};
  return status_of(ssq::launch_page_fork(a, stream));
}

int ssq_page_collect(const int32_t* lens, int64_t requests, const int32_t* table, int64_t table_stride, int page_size, int64_t pages, const uint8_t* pinned,
                     int32_t* free_pages, int32_t* count, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  return collect(lens, requests, table, table_stride, page_size, pages, pinned, false, nullptr, free_pages, count, nullptr, nullptr, nullptr, workspace,
                 workspace_bytes, stream);
}

int ssq_page_compact(const int32_t* lens, int64_t requests, const int32_t* table, int64_t table_stride, int page_size, int64_t pages, const uint8_t* pinned,
                     int32_t* table_out, int32_t* free_pages, int32_t* count, int32_t* src, int32_t* dst, int32_t* moved, void* workspace,
                     size_t workspace_bytes, hipStream_t stream) {
  return collect(lens, requests, table, table_stride, page_size, pages, pinned, true, table_out, free_pages, count, src, dst, moved, workspace, workspace_bytes,
                 stream);
}

size_t ssq_page_collect_workspace_size(int64_t pages, int compact) {
  return pages < 0 || pages > INT32_MAX / 16 ? 0 : ssq::page_collect_workspace_bytes(pages, compact != 0);
}

int ssq_page_copy(void* const* caches, int count, int64_t page_bytes, int64_t pages, const int32_t* src, const int32_t* dst, int64_t entries,
                  hipStream_t stream) {
  if (count < 0 || count > (1 << 16) || page_bytes <= 0 || page_bytes > kMaxLen || page_bytes % 16 != 0 || pages < 0 || pages > INT32_MAX || entries < 0 ||
      entries > kMaxLen)
    return SSQ_EINVAL;
  if (count == 0 || entries == 0 || pages == 0) return SSQ_OK;
  if (caches == nullptr || src == nullptr || dst == nullptr) return SSQ_EINVAL;
  for (int i = 0; i < count; ++i) {
    if (caches[i] == nullptr) return SSQ_EINVAL;
    if (!aligned(caches[i], 16)) return SSQ_EALIGN;
  }
  if (!aligned(src, 4) || !aligned(dst, 4)) return SSQ_EALIGN;
  for (int i = 0; i < count; ++i) {         // other workgroups still read the lists
    const Span cache = {caches[i], pages, page_bytes};
    if (overlap(cache, {src, entries}) || overlap(cache, {dst, entries})) return SSQ_EINVAL;
  }
  return status_of(ssq::launch_page_copy(reinterpret_cast<uint8_t* const*>(caches), count, src, dst, entries, pages, page_bytes, stream));
}

}  // extern "C"
