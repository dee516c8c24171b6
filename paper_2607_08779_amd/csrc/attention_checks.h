// Checks of arguments that the entry points of include/ssq_attention.h share.
#pragma once

#include <cmath>

#include "attention_internal.h"
#include "ssq.h"

namespace {

constexpr int64_t kMaxRequests = int64_t(1) << 20;
constexpr int64_t kMaxRows = int64_t(1) << 31;       // kernels index rows in int
constexpr int64_t kMaxStride = int64_t(1) << 24;     // elements between rows (32-bit tile offsets)
constexpr int64_t kMaxLen = int64_t(1) << 30;
constexpr int kMaxHeadCount = 1 << 16;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
int status_of(hipError_t e) { return e == hipSuccess ? SSQ_OK : SSQ_EHIP; }
bool valid_dim(int d) { return d == 64 || d == 128; }
bool valid_page(int p) { return p >= 16 && p <= 1024 && (p & (p - 1)) == 0; }
bool valid_heads(int q_heads, int kv_heads) {
  return q_heads > 0 && kv_heads > 0 && q_heads <= kMaxHeadCount && q_heads % kv_heads == 0;
}
int shift_of(int page_size) { return __builtin_ctz((unsigned)page_size); }

// An array of 4-byte elements (of `size` bytes), which may be empty.
struct Span {
  const void* p;
  int64_t count;
  int64_t size = 4;
};
bool overlap(const Span& a, const Span& b) {
  const auto x = reinterpret_cast<uintptr_t>(a.p), y = reinterpret_cast<uintptr_t>(b.p);
  return a.count > 0 && b.count > 0 && x < y + (uintptr_t)(b.size * b.count) && y < x + (uintptr_t)(a.size * a.count);
}

// Rows of `heads` heads: a stride that holds them, in whole 16-byte pieces.
template <typename T>
bool valid_stride(int64_t stride, int heads, int head_dim) {
  return stride >= (int64_t)heads * head_dim && stride <= kMaxStride && stride % (int64_t)(16 / sizeof(T)) == 0;
}

bool valid_decode_sizes(int64_t requests, int fresh, int q_heads, int kv_heads, int head_dim, int64_t max_len, int64_t prefix,
                        int tile = 32) {
  if (requests < 0 || requests > kMaxRequests || fresh < 1 || !valid_heads(q_heads, kv_heads) || !valid_dim(head_dim) ||
      max_len < 0 || max_len > kMaxLen || prefix < 0)
    return false;
  return fresh <= kMaxLen && requests * fresh < kMaxRows &&
         requests * fresh * q_heads + tile * requests * kv_heads < tile * ssq::kMaxGroups;      // own rows, `tile` a workgroup
}

}  // namespace
