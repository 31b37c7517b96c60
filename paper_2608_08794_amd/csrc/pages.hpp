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
// to the last, and the dimensions of more than one step as (stride, steps), the
// innermost first: a stride is no shorter than what lies within it.
struct Strided {
  const void* data = nullptr;
  size_t es = 2;
  bool ok = true;
  int64_t extent = 0, run = 0;
  std::pair<int64_t, int64_t> dim[3];
  int n = 0;
};

// run: contiguous elements; (stride, count) pairs in any order.
inline Strided strided(const void* data, size_t es, int64_t run,
                       std::initializer_list<std::pair<int64_t, int64_t>> dims) {
  Strided t;
  t.data = data;
  t.es = es;
  t.run = run;
  for (auto& dim : dims)
    if (dim.second > 1) t.dim[t.n++] = dim;
  std::sort(t.dim, t.dim + t.n);
  __int128 at = run;
  for (int i = 0; i < t.n; ++i) {
    t.ok &= t.dim[i].first >= at;
    at += (__int128)t.dim[i].first * (t.dim[i].second - 1);
    t.ok &= at >= 0 && at <= (__int128(1) << 46);
    if (!t.ok) return t;
  }
  t.extent = (int64_t)at;
  return t;
}

// Whether the elements of a's la inner dimensions are none of those of b's lb inner
// ones, ea and eb elements long, with b's first `at` elements after a's: their ranges
// are apart, or they interleave at equal strides S.  Two elements of steps i and j of
// S then meet only where i S + x = at + j S + y; x and y lie in [0, S), so with
// at = q S + m, 0 <= m < S, either i - j = q and x = y + m, or i - j = q + 1 and
// x = y + m - S.
inline bool apart_at(const Strided& a, int la, int64_t ea, const Strided& b, int lb, int64_t eb, int64_t at) {
  if (at >= ea || at + eb <= 0) return true;
  if (!la || !lb || a.dim[la - 1].first != b.dim[lb - 1].first) return false;
  const int64_t stride = a.dim[la - 1].first, i = a.dim[la - 1].second - 1, j = b.dim[lb - 1].second - 1;
  const int64_t q = at / stride - (at % stride < 0), m = at - q * stride;
  ea -= stride * i;
  eb -= stride * j;
  return (q < -j || q > i || apart_at(a, la - 1, ea, b, lb - 1, eb, m)) &&
         (q + 1 < -j || q + 1 > i || apart_at(a, la - 1, ea, b, lb - 1, eb, m - stride));
}

// Whether no element of a is one of b: their byte ranges are apart, or they interleave
// at equal strides (slices of one tensor, of any of its dimensions).
inline bool apart(const Strided& a, const Strided& b) {
  if (!overlaps(a.data, (size_t)a.extent * a.es, b.data, (size_t)b.extent * b.es)) return true;
  const int64_t bytes = (int64_t)((uintptr_t)b.data - (uintptr_t)a.data);
  if (a.es != b.es || bytes % (int64_t)a.es) return false;
  return apart_at(a, a.n, a.extent, b, b.n, b.extent, bytes / (int64_t)a.es);
}

// A contiguous range as a Strided.
inline Strided range(const void* data, size_t bytes) { return strided(data, 1, (int64_t)bytes, {}); }

// `rows` rows of `width` elements at a stride, one row at a stride of 0 (host checks of
// tables, masks, position ids).
inline Strided rows_of_stride(const void* data, size_t es, int64_t rows, int64_t stride, int64_t width) {
  return data && rows ? strided(data, es, width, {{stride, stride ? rows : 1}}) : range(data, 0);
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
