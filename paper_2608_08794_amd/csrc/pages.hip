// A cache of pages: bookkeeping of a pool on the host, copies of pages, and the
// gather of kept rows (Section 3.2, last sentence; Algorithm 1, "slice their
// KV-cache entries") into, out of and between pages.
//
// Both kernels move bytes and are bound by HBM, in units of 16 bytes (smaller ones
// for rows whose size or address is no multiple of them).  One unit a thread keeps
// enough of them in flight: four cost the copy 11% (591 pages of 28 layers 180 us,
// 6.0 TB/s, against 200), by more bytes in flight than the L2 holds.
#include <cstring>
#include <new>
#include <vector>

#include "pages.hpp"

namespace apack {

apack_status check_pages(const apack_pages* p, const char* what, PoolDev* dev, Strided* plane) {
  APACK_CHECK(p, APACK_E_ARG, "%s is NULL", what);
  APACK_CHECK(dtype_ok(p->dtype), APACK_E_DTYPE, "%s: unknown dtype %d", what, (int)p->dtype);
  APACK_CHECK(p->reserved == 0, APACK_E_ARG, "%s: reserved must be 0", what);
  APACK_CHECK(p->n_layers >= 1 && p->n_layers <= kMaxLayers, APACK_E_ARG, "%s: n_layers must lie in [1, %d]", what,
              kMaxLayers);
  APACK_CHECK(p->n_pages >= 1 && p->page_rows >= 1 && p->hkv >= 1 && p->d >= 1, APACK_E_SHAPE,
              "%s: n_pages, page_rows, hkv and d must be positive", what);
  APACK_CHECK(p->k, APACK_E_ARG, "%s: the K pointer table is NULL", what);
  for (int l = 0; l < p->n_layers; ++l)
    APACK_CHECK(p->k[l] && (!p->v || p->v[l]), APACK_E_ARG, "%s: layer %d: NULL K/V pointer", what, l);
  if (p->table)
    APACK_CHECK(p->table_width >= 0 && (p->table_stride >= p->table_width || p->table_stride == 0), APACK_E_SHAPE,
                "%s: table_stride must be >= table_width >= 0, or 0", what);
  const int64_t ps = p->n_pages > 1 ? p->page_stride : 0;
  const int64_t hs = p->hkv > 1 ? p->head_stride : 0;
  const int64_t rs = p->page_rows > 1 ? p->row_stride : 0;
  *plane = strided(p->k[0], dtype_size(p->dtype), p->d, {{ps, p->n_pages}, {hs, p->hkv}, {rs, p->page_rows}});
  APACK_CHECK(plane->ok, APACK_E_SHAPE, "%s: strides must keep every row apart (and a plane below 2^46 elements)", what);
  dev->table = p->table;
  dev->table_stride = p->table_stride;
  dev->table_width = p->table ? p->table_width : 0;
  dev->n_pages = p->n_pages;
  dev->page_stride = ps;
  dev->head_stride = hs;
  dev->row_stride = rs;
  dev->rows = FastDiv((uint32_t)p->page_rows);
  return APACK_OK;
}

apack_status check_heads(const apack_heads* t, const char* what, int64_t rows, int32_t d, size_t es, Strided* s) {
  APACK_CHECK(t, APACK_E_ARG, "%s is NULL", what);
  APACK_CHECK(t->reserved == 0, APACK_E_ARG, "%s: reserved must be 0", what);
  APACK_CHECK(t->heads >= 1, APACK_E_SHAPE, "%s: heads must be positive", what);
  APACK_CHECK(t->heads < 65536, APACK_E_UNSUPPORTED, "%s: 65536 heads or more", what);
  *s = range(t->data, 0);
  if (rows == 0) return APACK_OK;
  APACK_CHECK(t->data, APACK_E_ARG, "%s: data is NULL", what);
  *s = strided(t->data, es, d, {{t->head_stride, t->heads}, {t->row_stride, rows}});
  APACK_CHECK(s->ok, APACK_E_SHAPE, "%s: strides must keep every row apart (and the tensor below 2^46 elements)", what);
  return APACK_OK;
}

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;

// The widest unit of 16, 4 or 2 bytes that divides every byte count given.
inline int64_t unit_bytes(std::initializer_list<int64_t> counts, uintptr_t addresses) {
  uint64_t all = addresses;
  for (int64_t c : counts) all |= (uint64_t)c;
  return all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : 2;
}

// ---------------------------------------------------------------------------
// Page copies
// ---------------------------------------------------------------------------

// A page of a plane is runs[1] x runs[0] runs of `run` units (contiguous parts
// of a page are one run).
struct CopyArgs {
  const int32_t* pairs;
  int32_t n_pages;
  int32_t slabs;                // workgroups of one page
  int64_t page_units;           // units of one page
  int64_t page_stride;          // in units
  int64_t run, stride0, stride1;
  FastDiv by_run, by_count0;
  void* plane[2 * kMaxLayers];
};

template <class U>
__global__ __launch_bounds__(kThreads) void k_copy_pages(const CopyArgs a) {
  const uint32_t pair = blockIdx.x / (unsigned)a.slabs;
  const uint32_t u = (blockIdx.x - pair * a.slabs) * kThreads + threadIdx.x;
  const int32_t src = a.pairs[2 * (int64_t)pair], dst = a.pairs[2 * (int64_t)pair + 1];
  if (u >= a.page_units || src < 0 || src >= a.n_pages || dst < 0 || dst >= a.n_pages) return;
  const uint32_t r = a.by_run.div(u), r1 = a.by_count0.div(r);
  const int64_t at = (u - (int64_t)r * a.run) + (int64_t)(r - r1 * a.by_count0.d) * a.stride0 + r1 * a.stride1;
  U* plane = static_cast<U*>(a.plane[blockIdx.y]);
  __builtin_nontemporal_store(__builtin_nontemporal_load(plane + src * a.page_stride + at), plane + dst * a.page_stride + at);
}

template <class U>
void launch_copy(const CopyArgs& a, dim3 grid, hipStream_t s) {
  hipLaunchKernelGGL(k_copy_pages<U>, grid, dim3(kThreads), 0, s, a);
}

// ---------------------------------------------------------------------------
// Gather between pages and planes
// ---------------------------------------------------------------------------

constexpr int kMaxMoves = 48;   // sequences per launch (they travel as an argument)
constexpr int kPlanes = 4;      // planes of a thread

struct MoveArgs {
  const int32_t* kept;
  PoolDev in, out;              // strides in units
  int32_t n_seq, seq0;          // sequences of this launch, the first one's number
  int32_t heads, planes;
  int32_t row_units;            // units of a row
  FastDiv by_units;
  int32_t end[kMaxMoves + 1];   // first out row of each sequence, from kept[kept0]
  int32_t src_off[kMaxMoves], n_in[kMaxMoves], dst_off[kMaxMoves];
  const void* src[2 * kMaxLayers];
  void* dst[2 * kMaxLayers];
};

// Offset of a row in a plane, in units; -1 when it is in no page.
__device__ __forceinline__ int64_t row_offset(const PoolDev& p, int seq, int64_t row) {
  const uint32_t page_rows = p.rows.d;
  if (!p.table) return row < page_rows ? row * p.row_stride : -1;
  const uint32_t at = p.rows.div((uint32_t)row);
  if (at >= (uint32_t)p.table_width) return -1;
  const int32_t page = p.table[seq * p.table_stride + at];
  if (page < 0 || page >= p.n_pages) return -1;
  return page * p.page_stride + (row - (int64_t)at * page_rows) * p.row_stride;
}

// Each thread finds where its unit comes from and goes to (the lanes of a row
// read the same words: no LDS, no barrier) and copies it in kPlanes planes (layer
// x {K, V} x head), whose rows lie alike.  All loads come before the stores: they
// complete in order, so a load after a store would wait for it.  47014 of 94028 rows
// of 28 layers, 5.4 GB: 961 us between pages in random order, 893 in ascending order
// (6.0 TB/s); with one plane a thread 1576 (the look-ups' chain), with eight loaded
// ahead of stores 1003.
template <class U>
__global__ __launch_bounds__(kThreads) void k_move_rows(const MoveArgs a) {
  const uint32_t u = blockIdx.x * (uint32_t)kThreads + threadIdx.x;   // < 2^31
  const int row = (int)a.by_units.div(u);
  if (row >= a.end[a.n_seq]) return;
  const int64_t kept = a.kept ? a.kept[row] : 0;
  int s = 0, hi = a.n_seq;            // the last sequence whose first out row is <= row
  while (hi - s > 1) {
    const int mid = (s + hi) >> 1;
    if (a.end[mid] <= row) s = mid;
    else hi = mid;
  }
  const int at = row - a.end[s];
  const int64_t local = a.kept ? kept - a.src_off[s] : at;
  if (local < 0 || local >= a.n_in[s]) return;
  const int64_t to_row = row_offset(a.out, a.seq0 + s, (int64_t)a.dst_off[s] + at);
  const int64_t from_row = row_offset(a.in, a.seq0 + s, a.in.table ? local : local + a.src_off[s]);
  if (from_row < 0 || to_row < 0) return;
  const int64_t c = u - (uint32_t)row * (uint32_t)a.row_units, from = from_row + c, to = to_row + c;

  const int p0 = blockIdx.y * kPlanes;
  auto load = [&](int i) {
    const int p = min(p0 + i, a.planes - 1), tensor = p / a.heads;
    return __builtin_nontemporal_load(static_cast<const U*>(a.src[tensor]) + (p - tensor * a.heads) * a.in.head_stride + from);
  };
  U x[kPlanes];
#pragma unroll
  for (int i = 0; i < kPlanes; ++i) x[i] = load(i);
#pragma unroll
  for (int i = 0; i < kPlanes; ++i) {
    const int p = p0 + i, tensor = p / a.heads;
    if (p >= a.planes) break;
    __builtin_nontemporal_store(x[i], static_cast<U*>(a.dst[tensor]) + (p - tensor * a.heads) * a.out.head_stride + to);
  }
}

template <class U>
void launch_move(const MoveArgs& a, unsigned blocks, hipStream_t s) {
  const dim3 grid(blocks, (unsigned)((a.planes + kPlanes - 1) / kPlanes));
  hipLaunchKernelGGL(k_move_rows<U>, grid, dim3(kThreads), 0, s, a);
}

inline void to_units(PoolDev& p, int64_t es, int64_t ub) {
  p.page_stride = p.page_stride * es / ub;
  p.head_stride = p.head_stride * es / ub;
  p.row_stride = p.row_stride * es / ub;
}

// Addresses and strides of a pool, or'ed for the choice of the unit.
inline uintptr_t bits_of(const apack_pages* p, const PoolDev& dev, int64_t es) {
  uintptr_t all = (uintptr_t)(dev.page_stride * es) | (uintptr_t)(dev.head_stride * es) |
                  (uintptr_t)(dev.row_stride * es);
  for (int l = 0; l < p->n_layers; ++l) all |= (uintptr_t)p->k[l] | (p->v ? (uintptr_t)p->v[l] : 0);
  return all;
}

inline bool same_pool(const apack_pages* a, const apack_pages* b, const PoolDev& x, const PoolDev& y) {
  if (!a->table || !b->table || a->n_pages != b->n_pages || a->page_rows != b->page_rows ||
      x.page_stride != y.page_stride || x.head_stride != y.head_stride || x.row_stride != y.row_stride)
    return false;
  for (int l = 0; l < a->n_layers; ++l)
    if (a->k[l] != b->k[l] || (a->v && a->v[l] != b->v[l])) return false;
  return true;
}

inline Strided at(Strided t, const void* p) {
  t.data = p;
  return t;
}

}  // namespace
}  // namespace apack

using namespace apack;

extern "C" {

apack_status apack_pages_alloc(int32_t n_pages, int32_t* refs, int64_t n, int32_t* pages) {
  clear_error();
  APACK_CHECK(n_pages >= 0 && n >= 0, APACK_E_ARG, "negative n_pages or n");
  APACK_CHECK((n_pages == 0 || refs) && (n == 0 || pages), APACK_E_ARG, "refs or pages is NULL");
  int64_t got = 0;
  for (int32_t p = 0; p < n_pages && got < n; ++p)
    if (refs[p] == 0) ++got;
  APACK_CHECK(got == n, APACK_E_SHAPE, "%lld pages asked for, %lld free", (long long)n, (long long)got);
  got = 0;
  for (int32_t p = 0; got < n; ++p)
    if (refs[p] == 0) {
      refs[p] = 1;
      pages[got++] = p;
    }
  return APACK_OK;
}

apack_status apack_pages_free(int32_t n_pages, int32_t* refs, int64_t n, const int32_t* pages) {
  clear_error();
  APACK_CHECK(n_pages >= 0 && n >= 0, APACK_E_ARG, "negative n_pages or n");
  APACK_CHECK((n_pages == 0 || refs) && (n == 0 || pages), APACK_E_ARG, "refs or pages is NULL");
  for (int64_t i = 0; i < n; ++i) {
    const int32_t p = pages[i];
    if (p >= 0 && p < n_pages && refs[p] > 0) {
      --refs[p];
      continue;
    }
    for (int64_t j = 0; j < i; ++j) ++refs[pages[j]];   // as it was
    return p < 0 || p >= n_pages ? fail(APACK_E_SHAPE, "page %d is outside [0, %d)", p, n_pages)
                                 : fail(APACK_E_SHAPE, "page %d is freed more often than it is held", p);
  }
  return APACK_OK;
}

apack_status apack_pages_fork(int32_t n_pages, int32_t* refs, int32_t page_rows, int64_t n_rows, const int32_t* parent,
                              int32_t n_children, int32_t* children, int32_t* copies, int64_t* n_copies) {
  clear_error();
  APACK_CHECK(n_pages >= 0 && page_rows >= 1 && n_rows >= 0 && n_children >= 0, APACK_E_ARG,
              "n_pages, n_rows and n_children must be >= 0, page_rows >= 1");
  APACK_CHECK(n_copies, APACK_E_ARG, "n_copies is NULL");
  const int64_t full = n_rows / page_rows;
  const bool part = n_rows % page_rows != 0;
  const int64_t n = full + part;
  if (n_children > 0 && n > 0)
    APACK_CHECK(refs && parent && children && (!part || copies), APACK_E_ARG,
                "refs, parent, children or copies is NULL");
  for (int64_t i = 0; i < n; ++i) {
    const int32_t p = n_children > 0 ? parent[i] : 0;
    if (n_children == 0) break;
    APACK_CHECK(p >= 0 && p < n_pages && refs[p] > 0, APACK_E_SHAPE, "parent page %d is not a held page of the pool", p);
    APACK_CHECK(refs[p] <= INT32_MAX - n_children, APACK_E_UNSUPPORTED, "page %d: too many references", p);
  }
  if (part) {
    int64_t free_pages = 0;
    for (int32_t p = 0; p < n_pages && free_pages < n_children; ++p) free_pages += refs[p] == 0;
    APACK_CHECK(free_pages >= n_children, APACK_E_SHAPE, "%d pages needed, %lld free", n_children, (long long)free_pages);
  }
  int32_t next = 0;
  for (int32_t c = 0; c < n_children; ++c) {
    int32_t* mine = children + (int64_t)c * n;
    for (int64_t i = 0; i < full; ++i) {
      mine[i] = parent[i];
      ++refs[parent[i]];
    }
    if (part) {
      while (refs[next] != 0) ++next;
      refs[next] = 1;
      mine[full] = next;
      copies[2 * (int64_t)c] = parent[full];
      copies[2 * (int64_t)c + 1] = next;
    }
  }
  *n_copies = part ? n_children : 0;
  return APACK_OK;
}

apack_status apack_pages_copy(const apack_pages* pages, int64_t n_pairs, const int32_t* pairs, void* stream) {
  clear_error();
  PoolDev dev;
  Strided plane;
  apack_status st = check_pages(pages, "pages", &dev, &plane);
  if (st != APACK_OK) return st;
  APACK_CHECK(n_pairs >= 0, APACK_E_ARG, "n_pairs must be >= 0");
  APACK_CHECK(n_pairs < (int64_t(1) << 31), APACK_E_UNSUPPORTED, "n_pairs must be < 2^31");
  APACK_CHECK(n_pairs == 0 || pairs, APACK_E_ARG, "pairs is NULL");
  const int64_t es = (int64_t)dtype_size(pages->dtype);
  for (int l = 0; l < pages->n_layers; ++l)
    for (int kv = 0; kv < (pages->v ? 2 : 1); ++kv)
      APACK_CHECK(apart(range(pairs, (size_t)n_pairs * 8), at(plane, kv ? pages->v[l] : pages->k[l])), APACK_E_ALIAS,
                  "pairs overlaps the pool");
  if (n_pairs == 0) return APACK_OK;

  // Heads and rows of a page in the order of their strides, contiguous ones as one run.
  int64_t run = pages->d;
  int64_t dim[2][2] = {{0, 1}, {0, 1}};
  int n = 0;
  const std::pair<int64_t, int64_t> hr[2] = {{dev.head_stride, pages->hkv}, {dev.row_stride, pages->page_rows}};
  const int first = pages->hkv > 1 && pages->page_rows > 1 && hr[0].first < hr[1].first ? 0 : 1;
  for (int i = 0; i < 2; ++i) {
    const auto& [stride, count] = hr[i == 0 ? first : 1 - first];
    if (count == 1) continue;
    if (n == 0 && stride == run) {
      run *= count;
    } else {
      dim[n][0] = stride;
      dim[n++][1] = count;
    }
  }
  const int64_t ub = unit_bytes({run * es, dim[0][0] * es, dim[1][0] * es}, bits_of(pages, dev, es));
  CopyArgs a;
  std::memset(&a, 0, sizeof a);
  a.pairs = pairs;
  a.n_pages = pages->n_pages;
  a.run = run * es / ub;
  a.page_units = a.run * dim[0][1] * dim[1][1];
  a.page_stride = dev.page_stride * es / ub;
  a.stride0 = dim[0][0] * es / ub;
  a.stride1 = dim[1][0] * es / ub;
  const int64_t slabs = (a.page_units + kThreads - 1) / kThreads;
  APACK_CHECK(a.page_units + kThreads < (int64_t(1) << 31) && n_pairs < kMaxThreads / kThreads / slabs,
              APACK_E_UNSUPPORTED, "2^31 units of %d bytes in a page, or 2^32 in one layer's pages copied", (int)ub);
  a.slabs = (int32_t)slabs;
  a.by_run = FastDiv((uint32_t)a.run);
  a.by_count0 = FastDiv((uint32_t)dim[0][1]);
  int planes = 0;
  for (int l = 0; l < pages->n_layers; ++l) {
    a.plane[planes++] = pages->k[l];
    if (pages->v) a.plane[planes++] = pages->v[l];
  }
  const dim3 grid((unsigned)(slabs * n_pairs), (unsigned)planes);
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (ub == 16) launch_copy<u32x4>(a, grid, hs);
  else if (ub == 4) launch_copy<uint32_t>(a, grid, hs);
  else launch_copy<uint16_t>(a, grid, hs);
  return launch_status("k_copy_pages");
}

apack_status apack_compact_kv_pages(int32_t n_seq, const apack_move* seqs, const int32_t* src_rows,
                                    const apack_pages* in, const apack_pages* out, void* stream) {
  clear_error();
  PoolDev pin, pout;
  Strided tin, tout;
  apack_status st = check_pages(in, "in", &pin, &tin);
  if (st == APACK_OK) st = check_pages(out, "out", &pout, &tout);
  if (st != APACK_OK) return st;
  APACK_CHECK(in->n_layers == out->n_layers && in->hkv == out->hkv && in->d == out->d && !in->v == !out->v,
              APACK_E_SHAPE, "in and out differ in layers, heads, d, or in whether there is a v");
  APACK_CHECK(in->dtype == out->dtype, APACK_E_DTYPE, "in and out differ in dtype");
  APACK_CHECK(n_seq >= 0, APACK_E_ARG, "n_seq must be >= 0");
  if (n_seq == 0) return APACK_OK;
  APACK_CHECK(seqs, APACK_E_ARG, "seqs is NULL");
  APACK_CHECK((in->table || in->n_pages == 1) && (out->table || out->n_pages == 1), APACK_E_SHAPE,
              "planes (no table) are one page");
  constexpr int64_t kLim = int64_t(1) << 31;
  int64_t total = 0;
  for (int32_t s = 0; s < n_seq; ++s) {
    const apack_move& m = seqs[s];
    APACK_CHECK(m.src_off >= 0 && m.n_in >= 0 && m.dst_off >= 0 && m.n_out >= 0, APACK_E_SHAPE,
                "sequence %d: negative offset or row count", s);
    APACK_CHECK(m.src_off < kLim && m.n_in < kLim && m.dst_off < kLim && m.n_out < kLim &&
                    m.src_off + m.n_in < kLim && m.dst_off + m.n_out < kLim,
                APACK_E_UNSUPPORTED, "sequence %d: rows must be < 2^31", s);
    APACK_CHECK(src_rows || m.n_out <= m.n_in, APACK_E_SHAPE, "sequence %d: n_out > n_in without src_rows", s);
    if (!in->table)
      APACK_CHECK(m.src_off + m.n_in <= in->page_rows, APACK_E_SHAPE, "sequence %d: rows past the input planes", s);
    if (!out->table)
      APACK_CHECK(m.dst_off + m.n_out <= out->page_rows, APACK_E_SHAPE, "sequence %d: rows past the output planes", s);
    else
      APACK_CHECK((m.dst_off + m.n_out + out->page_rows - 1) / out->page_rows <= out->table_width, APACK_E_SHAPE,
                  "sequence %d: rows past the output table", s);
    total += m.n_out;
    APACK_CHECK(total < kLim, APACK_E_UNSUPPORTED, "2^31 kept rows or more");
  }
  const bool one = same_pool(in, out, pin, pout);
  std::vector<const void*> ins, outs;
  try {
    for (int l = 0; l < in->n_layers; ++l) {
      ins.push_back(in->k[l]);
      outs.push_back(out->k[l]);
      if (in->v) {
        ins.push_back(in->v[l]);
        outs.push_back(out->v[l]);
      }
    }
  } catch (const std::bad_alloc&) {
    return fail(APACK_E_HIP, "out of host memory");
  }
  const Strided kept = range(src_rows, (size_t)(src_rows ? total : 0) * 4);
  const Strided t_in = rows_of_stride(in->table, 4, n_seq, in->table_stride, in->table_width);
  const Strided t_out = rows_of_stride(out->table, 4, n_seq, out->table_stride, out->table_width);
  APACK_CHECK(t_in.ok && t_out.ok, APACK_E_SHAPE, "a table of 2^46 entries or more");
  Strided o = tout, other_in = tin, other_out = tout;
  for (size_t i = 0; i < outs.size(); ++i) {
    o.data = outs[i];
    APACK_CHECK(apart(o, kept) && apart(o, t_in) && apart(o, t_out), APACK_E_ALIAS,
                "an output overlaps src_rows or a table");
    for (size_t j = 0; j < ins.size(); ++j) {
      other_in.data = ins[j];
      other_out.data = outs[j];
      APACK_CHECK((one && i == j) || apart(o, other_in), APACK_E_ALIAS, "an output overlaps an input");
      APACK_CHECK(j <= i || apart(o, other_out), APACK_E_ALIAS, "two outputs overlap");
    }
  }
  if (total == 0) return APACK_OK;

  const int64_t es = (int64_t)dtype_size(in->dtype);
  const int64_t ub = unit_bytes({in->d * es}, bits_of(in, pin, es) | bits_of(out, pout, es));
  MoveArgs a;
  std::memset(static_cast<void*>(&a), 0, sizeof a);
  a.in = pin;
  a.out = pout;
  to_units(a.in, es, ub);
  to_units(a.out, es, ub);
  a.row_units = (int32_t)(in->d * es / ub);
  a.by_units = FastDiv((uint32_t)a.row_units);
  APACK_CHECK(in->d * es / ub < kLim && total * a.row_units + kThreads < kLim, APACK_E_UNSUPPORTED,
              "2^31 units of %d bytes or more in a plane", (int)ub);
  a.heads = in->hkv;
  const int64_t planes = (int64_t)in->hkv * (int64_t)ins.size();
  APACK_CHECK(planes < 65536, APACK_E_UNSUPPORTED, "65536 planes or more");
  a.planes = (int32_t)planes;
  for (size_t i = 0; i < ins.size(); ++i) {
    a.src[i] = ins[i];
    a.dst[i] = const_cast<void*>(outs[i]);
  }
  hipStream_t hs = static_cast<hipStream_t>(stream);
  int64_t done = 0;
  for (int64_t s0 = 0; s0 < n_seq; s0 += kMaxMoves) {
    a.n_seq = (int32_t)std::min<int64_t>(kMaxMoves, n_seq - s0);
    a.seq0 = (int32_t)s0;
    a.kept = src_rows ? src_rows + done : nullptr;
    int64_t rows = 0;
    for (int32_t s = 0; s < a.n_seq; ++s) {
      const apack_move& m = seqs[s0 + s];
      a.end[s] = (int32_t)rows;
      a.src_off[s] = (int32_t)m.src_off;
      a.n_in[s] = (int32_t)m.n_in;
      a.dst_off[s] = (int32_t)m.dst_off;
      rows += m.n_out;
    }
    a.end[a.n_seq] = (int32_t)rows;
    done += rows;
    if (rows == 0) continue;
    const int64_t blocks = (rows * a.row_units + kThreads - 1) / kThreads;
    if (ub == 16) launch_move<u32x4>(a, (unsigned)blocks, hs);
    else if (ub == 4) launch_move<uint32_t>(a, (unsigned)blocks, hs);
    else launch_move<uint16_t>(a, (unsigned)blocks, hs);
    st = launch_status("k_move_rows");
    if (st != APACK_OK) return st;
  }
  return APACK_OK;
}

}  // extern "C"
