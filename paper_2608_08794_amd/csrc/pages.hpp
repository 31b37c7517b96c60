// What the calls over strided tensors and paged caches share: extents and
// overlap of strided planes on the host, division by a page's rows, and a
// pool's addressing on the device.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>
#include <initializer_list>
#include <utility>

#include "common.hpp"

namespace apack {

constexpr int kMaxLayers = 64;
constexpr int64_t kMaxThreads = int64_t(1) << 32;   // threads of a launch's first dimension, exclusive

// n / d for 0 <= n < 2^31 and 1 <= d < 2^31 as (n * m) >> (31 + s) with
// s = ceil(log2 d) and m = ceil(2^(31+s) / d) < 2^32: m*d exceeds 2^(31+s) by
// less than d <= 2^s, so the quotient is exact while n < 2^31.
struct FastDiv {
  uint32_t d = 1, m = 0x80000000u, s = 0;
  FastDiv() = default;
  explicit FastDiv(uint32_t div) : d(div) {
    while ((uint64_t(1) << s) < div) ++s;
    m = (uint32_t)(((uint64_t(1) << (31 + s)) + div - 1) / div);
  }
  __host__ __device__ __forceinline__ uint32_t div(uint32_t n) const {
    return (uint32_t)(((uint64_t)n * m) >> (31 + s));
  }
};

// The elements of a tensor of up to three strided dimensions over contiguous
// runs: `ok` when all of them are distinct, `extent` elements from the first
// to the last, and the outermost dimension's stride and what lies within one
// step of it.
struct Strided {
  const void* data = nullptr;
  size_t es = 2;
  bool ok = true;
  int64_t extent = 0, outer_stride = 0, inner = 0;
  int n = 0;                 // dimensions of more than one step
};

// run: contiguous elements; (stride, count) pairs in any order.
inline Strided strided(const void* data, size_t es, int64_t run,
                       std::initializer_list<std::pair<int64_t, int64_t>> dims) {
  Strided t;
  t.data = data;
  t.es = es;
  t.inner = run;
  std::pair<int64_t, int64_t> by[3];
  for (auto& dim : dims)
    if (dim.second > 1) by[t.n++] = dim;
  std::sort(by, by + t.n);
  __int128 at = run;
  for (int i = 0; i < t.n; ++i) {
    t.ok &= by[i].first >= at;
    t.inner = (int64_t)at;
    t.outer_stride = by[i].first;
    at += (__int128)by[i].first * (by[i].second - 1);
    t.ok &= at >= 0 && at <= (__int128(1) << 46);
    if (!t.ok) return t;
  }
  t.extent = (int64_t)at;
  return t;
}

// Whether no element of a is one of b: their byte ranges are apart, or they
// interleave (equal strides, as slices of one tensor, each within its part of
// the outermost step).
inline bool apart(const Strided& a, const Strided& b) {
  if (!overlaps(a.data, (size_t)a.extent * a.es, b.data, (size_t)b.extent * b.es)) return true;
  if (a.es != b.es || !a.n || !b.n || a.outer_stride != b.outer_stride) return false;
  const int64_t bytes = (int64_t)((uintptr_t)b.data - (uintptr_t)a.data);
  if (bytes % (int64_t)a.es) return false;
  int64_t at = bytes / (int64_t)a.es % a.outer_stride;
  if (at < 0) at += a.outer_stride;
  return at >= a.inner && a.outer_stride - at >= b.inner;
}

// A contiguous range as a Strided.
inline Strided range(const void* data, size_t bytes) { return strided(data, 1, (int64_t)bytes, {}); }

// `rows` rows of `width` elements at a stride (host checks of tables, masks, position ids).
inline Strided rows_of_stride(const void* data, size_t es, int64_t rows, int64_t stride, int64_t width) {
  return data && rows ? strided(data, es, width, {{stride, rows}}) : range(data, 0);
}

// Addressing of a pool (one page that holds the packed rows without a table).
struct PoolDev {
  const int32_t* table;
  int64_t table_stride, page_stride, head_stride, row_stride;
  int32_t table_width, n_pages;
  FastDiv rows;   // rows of a page
};

// Checks a pool and fills `dev` and the extent of one layer's K (or V).
apack_status check_pages(const apack_pages* p, const char* what, PoolDev* dev, Strided* plane);

// Checks a [heads][rows][d] tensor and fills its extent.
apack_status check_heads(const apack_heads* t, const char* what, int64_t rows, int32_t d, size_t es, Strided* s);

}  // namespace apack
