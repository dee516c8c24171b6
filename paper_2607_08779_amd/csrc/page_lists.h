// Internal declarations of the operators on tables and pools of pages (see include/ssq_cache.h).
#pragma once

#include "attention_internal.h"

namespace ssq {

constexpr int kMaxForkRows = 1 << 14;        // rows of a table that is forked: 4 bytes of LDS each
constexpr int kCopyArrays = 64;              // caches of one launch

struct PageFork {
  const int32_t* parents;
  const int32_t* lens;
  const int32_t* table;
  const int32_t* free_pages;
  const int32_t* taken;          // null: 0
  int32_t* table_out;
  int32_t* lens_out;
  int32_t* src;
  int32_t* dst;
  int32_t* taken_after;
  int64_t requests, rows, stride, stride_out, free_count;
  int shift;
};
hipError_t launch_page_fork(const PageFork& a, hipStream_t stream);

struct PageCollect {
  const int32_t* lens;
  const int32_t* table;
  const uint8_t* pinned;         // null: none
  int32_t* table_out;            // compact only, as are src, dst and moved
  int32_t* free_pages;
  int32_t* count;
  int32_t* src;
  int32_t* dst;
  int32_t* moved;
  int64_t requests, stride, pages;
  int shift;
};
hipError_t launch_page_collect(const PageCollect& a, bool compact, void* workspace, hipStream_t stream);
size_t page_collect_workspace_bytes(int64_t pages, bool compact);

hipError_t launch_page_copy(uint8_t* const* arrays, int count, const int32_t* src, const int32_t* dst, int64_t entries, int64_t pages,
                            int64_t page_bytes, hipStream_t stream);

}  // namespace ssq
