// The paged cache's shape, as its kernels and the rotation that writes into it take it.
#pragma once

#include <cstdint>

#include "rgd.h"

namespace rgd {

constexpr int kPageSize = 16;
constexpr int kPlanThreads = 1024;
// Rows (or pairs, or tokens) at most: the numbers that a last block gives to those past the end are still an int.
constexpr int32_t kMaxRows = 0x7fffffff - kPlanThreads;

struct CacheView {
  int32_t layers, pages, heads, dim;
  int64_t layer_stride;  // elements between a layer's pool and the next
};

// Checks a caller's shape under the name `fn`.
int check_cache_shape(const char* fn, const rgd_cache_shape* s, CacheView& c);

}  // namespace rgd
