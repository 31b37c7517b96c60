// Attention of one query row per sequence over its rows of a paged cache:
//   o = sum_j p_j v_j,  p = softmax_j(scale q.k_j).
//
// Every row's K and V is read once: 4 D bytes (bf16) for 4 D flops per query
// head of its group, so the call is bound by HBM, or by latency where the cache
// is small.  The query heads that share a key head (up to 16 at a time) are the
// columns of one MFMA, and one pass over the rows keeps a running maximum and
// sum.  Both operands that come from the cache go from global memory into
// registers as their rows lie, with no LDS:
//   logits  C[key][head] = K Q^T: lane l holds head l % 16 and, of each 16 keys,
//           keys 4 (l/16) .. + 3;
//   output  C[d][head] = V^T P^T.  The contraction's order over keys is free, so
//           lane l contracts exactly the keys whose logits it holds, and its V
//           operand is D/16 consecutive elements of those keys' rows: loads of
//           whole rows, then a transpose of 16-bit values between registers.
// Probabilities, maxima, sums and rescaling of a head all sit in its lane.
//
// The rows of all sequences and key heads, in tiles of 32, are dealt to the
// workgroups in equal shares (those of a few sequences key head by key head), whatever
// the lengths on the device are.  Where a share's border falls inside a sequence's
// key head, each side leaves its maximum, sum and unnormalised output, and a second
// kernel joins them.
//
// Measured (bf16, 28 heads over 4 of 128, pages of 16 rows), of 6.8 to 7.1 TB/s at
// which nontemporal loads read this much alone: 64 sequences of 700 to 9454 rows
// (0.68 GB) 108 + 5 us, 6.2 TB/s in the first kernel; one of 94028 rows (0.19 GB)
// 34 + 4 us, 5.6 TB/s.  What is left is the launches, the first loads' chain (length,
// page id, row) and the join.
#include <cmath>
#include <cstring>

#include "pages.hpp"

namespace apack {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kHeads = 16;        // query heads of a workgroup: an MFMA's columns
constexpr int kTile = 32;         // rows of a tile
constexpr int kWaves = 4;         // of a workgroup
// Eight waves a compute unit are what the registers let run at once (the steps
// loaded ahead take 128 of them); a share is a tile at least: with four, one a wave,
// four fp32 sequences of up to 1312 rows take 11.6 us, not 8.6.
constexpr int kShares = 2048 / kWaves;
template <int D> constexpr int kPart = D + 4;   // floats of a head's part: output, maximum, sum, 16-byte aligned
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

struct AttnArgs {
  const void* q;
  void* out;
  float* lse;
  const void* k;
  const void* v;
  const int32_t* lens;
  const uint8_t* mask;
  int32_t* split;                 // [seq][item]: parts, first part's slot, first share
  float* part;                    // [slot][head][kPart<D>]
  int64_t q_head, q_row, out_head, out_row, mask_stride;   // elements
  int64_t max_len, window;
  int64_t n_seq;
  int32_t hkv, group;             // key heads; query heads of each
  int32_t tiles;                  // ceil(group / kHeads)
  int32_t shares;
  float scale;
  PoolDev pages;
};

// Rows [base + skip, base + n) are those that a sequence attends to, base a
// multiple of 16; n rows lie in so many tiles (one, of no rows, when there are
// none, so that the output is written).
struct Rows {
  int64_t base;
  int skip, n, tiles;
};
__device__ __forceinline__ Rows rows_of(const AttnArgs& a, int64_t seq) {
  const int64_t have = a.lens[seq];
  const int64_t len = max((int64_t)0, min(have, min(a.max_len, (int64_t)a.pages.table_width * a.pages.rows.d)));
  const int64_t lo = a.window > 0 ? max((int64_t)0, have - a.window) : 0;
  const int64_t base = lo & ~(int64_t)15;
  const int n = len > lo ? (int)(len - base) : 0;
  return {base, (int)(lo - base), n, max(1, (n + kTile - 1) / kTile)};
}

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// A value that all lanes hold, as the scalar that the compiler cannot see it is.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Over the four lanes that hold a head.
__device__ __forceinline__ float max_of_head(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum_of_head(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// K and V pass once: nontemporal loads, 6.8 TB/s where plain ones read 192 MB at 5.9.
template <class V>
__device__ __forceinline__ V stream(const V* p) {
  return __builtin_nontemporal_load(p);
}

template <class T> struct Elem;

template <> struct Elem<uint16_t> {   // bf16 bits
  static constexpr int kRow16 = 2;    // 16-row logit tiles per step
  static __device__ __forceinline__ void put(float x, uint16_t* y) {
    const __bf16 b = (__bf16)x;
    *y = __builtin_bit_cast(uint16_t, b);
  }
};
template <> struct Elem<float> {
  static constexpr int kRow16 = 1;
  static __device__ __forceinline__ void put(float x, float* y) { *y = x; }
};

// A lane's part of one step: K rows l % 16 (+ 16) and V rows of its own keys.
template <class T, int D> struct Step;

template <int D> struct Step<uint16_t, D> {
  static constexpr int kQ = D / 32;           // 16-byte fragments of a query or key row
  static constexpr int kV = D / 16;           // elements of a V row per lane
  using VRow = std::conditional_t<D == 128, u32x4, u32x2>;
  u32x4 k[2][kQ];
  VRow v[8];
  uint32_t seen[2];     // mask bytes of the lane's keys

  static __device__ __forceinline__ int k_off(int g, int j) { return j * 32 + g * 8; }

  __device__ __forceinline__ void logits(const u32x4 (&q)[kQ], f32x4 (&x)[2]) const {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      x[t] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < kQ; ++j)
        x[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[t][j]),
                                                       __builtin_bit_cast(bf16x8, q[j]), x[t], 0, 0, 0);
    }
  }

  __device__ __forceinline__ void add(const float (&p)[8], f32x4 (&acc)[kV]) const {
    // Two bf16 parts hold 16 bits of each probability: their rounding stays below
    // that of the result, and the second product costs nothing beside the loads.
    bf16x8 hi, lo;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      hi[i] = (__bf16)p[i];
      lo[i] = (__bf16)(p[i] - (float)hi[i]);
    }
#pragma unroll
    for (int s = 0; s < kV; ++s) {
      u32x4 a;
#pragma unroll
      for (int j = 0; j < 4; ++j)   // element s of keys 2j and 2j + 1
        a[j] = __builtin_amdgcn_perm(v[2 * j + 1][s / 2], v[2 * j][s / 2], s % 2 ? 0x07060302u : 0x05040100u);
      acc[s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), hi, acc[s], 0, 0, 0);
      acc[s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), lo, acc[s], 0, 0, 0);
    }
  }
};

template <int D> struct Step<float, D> {
  static constexpr int kQ = D / 16;
  static constexpr int kV = D / 16;
  typedef unsigned int VRow __attribute__((ext_vector_type(kV)));
  u32x4 k[1][kQ];
  VRow v[4];
  uint32_t seen[1];

  static __device__ __forceinline__ int k_off(int g, int j) { return j * 16 + g * 4; }

  __device__ __forceinline__ void logits(const u32x4 (&q)[kQ], f32x4 (&x)[1]) const {
    x[0] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < kQ; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        x[0] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[0][j][e]), __uint_as_float(q[j][e]), x[0], 0, 0, 0);
  }

  __device__ __forceinline__ void add(const float (&p)[4], f32x4 (&acc)[kV]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int s = 0; s < kV; ++s)
        acc[s] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[i][s]), p[i], acc[s], 0, 0, 0);
  }
};

// A wave's state over one item (key head and up to 16 of its query heads) of a
// sequence: per lane, for its head l % 16, the running maximum, its keys' part of
// the sum, and acc[s][i], element (4 (l/16) + i) kV + s of the output.
//
// kAligned: pages hold a multiple of 16 rows, so the 16 rows of a logit tile lie
// in one page.  A tile's address is then the wave's (scalar) plus an offset that a
// lane keeps, and page ids sit in one register, lane by lane.  Otherwise every lane
// looks its rows' pages up.  kMask: there is a mask.
template <class T, int D, bool kAligned, bool kMask>
struct Wave {
  using S = Step<T, D>;
  static constexpr int kR = Elem<T>::kRow16, kKeys = 4 * kR, kStep = 16 * kR;
  static constexpr int kIdSteps = 64 / kR;         // steps whose page ids a wave holds

  const AttnArgs& a;
  const int64_t seq;
  const Rows of;
  const int kh, h0, heads;                         // key head; first query head of its group, and how many
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const float c = a.scale * kLog2e;
  u32x4 q[S::kQ];
  float m = -INFINITY, l = 0;
  f32x4 acc[S::kV] = {};
  const T *kb, *vb;

  __device__ __forceinline__ Wave(const AttnArgs& args, int64_t s, const Rows& rows, int item)
      : a(args), seq(s), of(rows), kh(item / args.tiles), h0((item % args.tiles) * kHeads),
        heads(min(kHeads, args.group - h0)) {
    // The query rows; heads past the group read its last one and are never stored.
    const int h = kh * a.group + h0 + min(n, heads - 1);
    const T* src = static_cast<const T*>(a.q) + h * a.q_head + seq * a.q_row;
#pragma unroll
    for (int j = 0; j < S::kQ; ++j) q[j] = *reinterpret_cast<const u32x4*>(src + S::k_off(g, j));
    kb = static_cast<const T*>(a.k) + kh * a.pages.head_stride;
    vb = static_cast<const T*>(a.v) + kh * a.pages.head_stride;
  }

  // The mask from the sequence's first row on, and whether a step from r0 on lies inside it: its
  // bytes are then loaded with the step's rows, four at a time.
  __device__ __forceinline__ const uint8_t* mask_row() const { return a.mask + seq * a.mask_stride + of.base; }
  __device__ __forceinline__ bool mask_whole(int r0) const { return of.base + r0 + kStep <= a.max_len; }
  __device__ __forceinline__ void load_mask(S& st, int r0) const {
    if (!kMask || !mask_whole(r0)) return;
#pragma unroll
    for (int t = 0; t < kR; ++t) __builtin_memcpy(&st.seen[t], mask_row() + r0 + 16 * t + 4 * g, 4);
  }

  // Takes a loaded step of rows from r0 on; page_in(i): whether key i lies in a page.  `holes`: some may not.
  template <class F>
  __device__ __forceinline__ void take(S& st, int r0, bool holes, F page_in) {
    f32x4 xt[kR];
    st.logits(q, xt);
    float x[kKeys];
#pragma unroll
    for (int i = 0; i < kKeys; ++i) x[i] = xt[i / 4][i % 4];
    if (kMask || holes || r0 < of.skip || r0 + kStep > of.n) {
      // Rows left out: their logit is -inf whatever they hold, their V is 0.
      bool in[kKeys];
#pragma unroll
      for (int i = 0; i < kKeys; ++i) {
        const int r = r0 + 16 * (i / 4) + 4 * g + i % 4;
        in[i] = (r >= of.skip) & (r < of.n) & (!holes || page_in(i));
      }
      if constexpr (kMask) {
        uint8_t seen[kKeys];
        if (mask_whole(r0)) {
#pragma unroll
          for (int i = 0; i < kKeys; ++i) seen[i] = (uint8_t)(st.seen[i / 4] >> 8 * (i % 4));
        } else {
#pragma unroll
          for (int i = 0; i < kKeys; ++i) seen[i] = mask_row()[min(r0 + 16 * (i / 4) + 4 * g + i % 4, of.n - 1)];
        }
#pragma unroll
        for (int i = 0; i < kKeys; ++i) in[i] &= seen[i] != 0;
      }
#pragma unroll
      for (int i = 0; i < kKeys; ++i) {
        x[i] = in[i] ? x[i] : -INFINITY;
        const uint32_t keep = in[i] ? ~0u : 0u;
#pragma unroll
        for (int e = 0; e < (int)(sizeof(typename S::VRow) / 4); ++e) st.v[i][e] &= keep;
      }
    }
    float top = x[0];
#pragma unroll
    for (int i = 1; i < kKeys; ++i) top = fmaxf(top, x[i]);
    top = fmaxf(m, max_of_head(top));
    const float at = top == -INFINITY ? 0.0f : top;   // no row yet: every exponent below is -inf
    const float alpha = exp2_((m - at) * c);
    m = top;
    float sum = 0, p[kKeys];
#pragma unroll
    for (int i = 0; i < kKeys; ++i) {
      p[i] = exp2_((x[i] - at) * c);
      sum += p[i];
    }
    l = l * alpha + sum;
#pragma unroll
    for (int s = 0; s < S::kV; ++s) acc[s] *= alpha;
    st.add(p, acc);
  }

  // Steps of rows first, first + stride, ... before `end`.  Each is loaded while the
  // one before it is taken; a load past the last step reads one place of the pool.
  __device__ __forceinline__ void rows_aligned(int first, int end, int stride) {
    if (first >= end) return;
    const int steps = (end - first + stride - 1) / stride;
    const int last = (of.n - 1) & ~15;              // first row of the last 16 that hold one
    const uint32_t page_rows = a.pages.rows.d;
    // Byte offsets of a lane's K row and first V row within 16 rows, and of a row.
    const uint32_t row = (uint32_t)a.pages.row_stride * sizeof(T);
    const uint32_t k_lane = n * row + S::k_off(g, 0) * sizeof(T);
    const uint32_t v_lane = 4 * g * row + n * S::kV * sizeof(T);
    auto row_of = [&](int s, int t) { return min(first + s * stride + 16 * t, last); };
    int32_t ids;
    auto fetch_ids = [&](int s) {
      if (s >= steps) return;
      const uint32_t p = a.pages.rows.div((uint32_t)(of.base + row_of(s + lane / kR, lane % kR)));
      ids = a.pages.table[seq * a.pages.table_stride + p];
      asm volatile("" : "+v"(ids));                 // arrives here, not where it is read
    };
    auto load = [&](S& st, bool (&bad)[kR], int s) {
      const bool live = s < steps;
      const uint32_t ko = live ? k_lane : 0, vo = live ? v_lane : 0, step = live ? row : 0;
#pragma unroll
      for (int t = 0; t < kR; ++t) {
        const int32_t id = __builtin_amdgcn_readlane(ids, s % kIdSteps * kR + t);
        bad[t] = (uint32_t)id >= (uint32_t)a.pages.n_pages;
        const uint32_t r = (uint32_t)of.base + row_of(s, t);
        const int64_t at = (bad[t] || !live ? 0 : id) * a.pages.page_stride * (int64_t)sizeof(T) +
                           (int64_t)(r - a.pages.rows.div(r) * page_rows) * row;
        const char *k = reinterpret_cast<const char*>(kb) + at, *v = reinterpret_cast<const char*>(vb) + at;
#pragma unroll
        for (int j = 0; j < S::kQ; ++j)
          st.k[t][j] = stream(reinterpret_cast<const u32x4*>(k + ko + (S::k_off(0, j) - S::k_off(0, 0)) * sizeof(T)));
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t off = vo + i * step;
          st.v[4 * t + i] = stream(reinterpret_cast<const typename S::VRow*>(v + off));
        }
      }
      if (live) load_mask(st, first + s * stride);
    };
    auto step = [&](S& st, const bool (&bad)[kR], int s) {
      bool holes = false;
#pragma unroll
      for (int t = 0; t < kR; ++t) holes |= bad[t];
      take(st, first + s * stride, holes, [&](int i) { return !bad[i / 4]; });
    };
    S x, y;
    bool bx[kR], by[kR];
    // Loads are issued before the step that they overlap is begun.
    fetch_ids(0);
    load(x, bx, 0);
    int s = 0;
    for (; s + 1 < steps; s += 2) {
      load(y, by, s + 1);
      __builtin_amdgcn_sched_barrier(0);
      step(x, bx, s);
      if ((s + 2) % kIdSteps == 0) fetch_ids(s + 2);
      load(x, bx, s + 2);
      __builtin_amdgcn_sched_barrier(0);
      step(y, by, s + 1);
    }
    if (s < steps) step(x, bx, s);
  }

  // The same for pages of any size; the next step's page ids are looked up while one is loaded.
  __device__ __forceinline__ void rows_general(int first, int end, int stride) {
    const uint32_t page_rows = a.pages.rows.d;
    const int32_t* table = a.pages.table + seq * a.pages.table_stride;
    // Row of the sequence that lane holds as K row t and as key i.
    auto k_row = [&](int r0, int t) { return (uint32_t)(of.base + min(r0 + 16 * t + n, of.n - 1)); };
    auto v_row = [&](int r0, int i) { return (uint32_t)(of.base + min(r0 + 16 * (i / 4) + 4 * g + i % 4, of.n - 1)); };
    int32_t k_id[kR], v_id[kKeys];
    auto fetch_ids = [&](int r0) {
#pragma unroll
      for (int t = 0; t < kR; ++t) k_id[t] = table[a.pages.rows.div(k_row(r0, t))];
#pragma unroll
      for (int i = 0; i < kKeys; ++i) v_id[i] = table[a.pages.rows.div(v_row(r0, i))];
    };
    // Offset of row r in a plane, of a page that may be none (page 0 stands in).
    auto at = [&](uint32_t r, int32_t id) {
      return ((uint32_t)id < (uint32_t)a.pages.n_pages ? id : 0) * a.pages.page_stride +
             (int64_t)(r - a.pages.rows.div(r) * page_rows) * a.pages.row_stride;
    };
    if (first < end) fetch_ids(first);
    for (int r0 = first; r0 < end; r0 += stride) {
      S st;
      bool bad[kKeys], any = false;
#pragma unroll
      for (int t = 0; t < kR; ++t) {
        const T* src = kb + at(k_row(r0, t), k_id[t]);
#pragma unroll
        for (int j = 0; j < S::kQ; ++j) st.k[t][j] = stream(reinterpret_cast<const u32x4*>(src + S::k_off(g, j)));
      }
#pragma unroll
      for (int i = 0; i < kKeys; ++i) {
        bad[i] = (uint32_t)v_id[i] >= (uint32_t)a.pages.n_pages;
        any |= bad[i];
        st.v[i] = stream(reinterpret_cast<const typename S::VRow*>(vb + at(v_row(r0, i), v_id[i]) + n * S::kV));
      }
      load_mask(st, r0);
      if (r0 + stride < end) fetch_ids(r0 + stride);
      take(st, r0, __any(any), [&](int i) { return !bad[i]; });
    }
  }

  __device__ __forceinline__ void rows(int first, int end, int stride) {
    if constexpr (kAligned) rows_aligned(first, end, stride);
    else rows_general(first, end, stride);
    l = sum_of_head(l);
  }

  __device__ __forceinline__ int64_t head(int h) const { return (int64_t)kh * a.group + h0 + h; }
  __device__ __forceinline__ void put_lse(int h, float top, float sum) const {
    if (a.lse) a.lse[head(h) * a.n_seq + seq] = sum != 0 ? top * a.scale + __log2f(sum) * kLn2 : -INFINITY;
  }
};

// What the waves of a workgroup leave in LDS.
template <int D>
struct Joint {
  float part[kWaves][kHeads][D + 4];
  float stat[kWaves][kHeads][2];

  // Joins the waves' states and writes the output (a sum of 0: no row; NaN stays NaN), or its part.  Every thread
  // calls it.
  template <class W, class T>
  __device__ __forceinline__ void join(const W& w, T* out, float* to_part) {
    const int wave = threadIdx.x >> 6;
    if (w.g == 0) {
      stat[wave][w.n][0] = w.m;
      stat[wave][w.n][1] = w.l;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int s = 0; s < W::S::kV; s += 4)
        *reinterpret_cast<f32x4*>(&part[wave][w.n][(4 * w.g + i) * W::S::kV + s]) =
            f32x4{w.acc[s][i], w.acc[s + 1][i], w.acc[s + 2][i], w.acc[s + 3][i]};
    __syncthreads();
    for (int i = threadIdx.x; i < w.heads * D; i += 64 * kWaves) {
      const int h = i / D, e = i % D;
      float top = -INFINITY;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) top = fmaxf(top, stat[v][h][0]);
      const float at = top == -INFINITY ? 0.0f : top;
      float sum = 0, o = 0;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) {
        const float f = exp2_((stat[v][h][0] - at) * w.c);
        sum += stat[v][h][1] * f;
        o += part[v][h][e] * f;
      }
      if (to_part) {
        float* to = to_part + h * kPart<D>;
        to[e] = o;
        if (e == 0) {
          to[D] = top;
          to[D + 1] = sum;
        }
      } else {
        Elem<T>::put(sum != 0 ? o / sum : 0.0f, out + w.head(h) * w.a.out_head + w.seq * w.a.out_row + e);
        if (e == 0) w.put_lse(h, top, sum);
      }
    }
  }
};

// One workgroup for each sequence and item: its waves take the steps in turn.
template <class T, int D, bool kAligned, bool kMask>
__global__ __launch_bounds__(64 * kWaves, 2) void k_attend_whole(const AttnArgs a) {
  using W = Wave<T, D, kAligned, kMask>;
  __shared__ Joint<D> sh;
  const Rows of = rows_of(a, blockIdx.y);
  W w(a, blockIdx.y, of, blockIdx.x);
  w.rows(uniform((int)threadIdx.x >> 6) * W::kStep, of.n, kWaves * W::kStep);
  sh.join(w, static_cast<T*>(a.out), nullptr);
}

// a / b for 0 <= a < 2^50 and b > 0: the fp64 quotient is off by less than one.
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  int64_t q = (int64_t)((double)a * (1.0 / (double)b));
  const int64_t r = a - q * b;
  return r < 0 ? q - 1 : r >= b ? q + 1 : q;
}

// Sum of x over the lanes up to and with this one.
__device__ __forceinline__ uint32_t sum_upto(uint32_t x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr:1, 2, 4, 8: within 16 lanes
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast:15 into rows 1 and 3
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // row_bcast:31 into rows 2 and 3
  return x;
}

// Share w of `all` tiles: those from w all / shares on, rounded down.
__device__ __forceinline__ int64_t share_start(int64_t w, int64_t all, int64_t shares) {
  return quotient(w * all, shares);
}

__device__ __forceinline__ uint32_t of_lane(uint32_t x, int lane) { return (uint32_t)__builtin_amdgcn_readlane(x, lane); }

template <class T, int D, bool kAligned, bool kMask>
__global__ __launch_bounds__(64 * kWaves, 2) void k_attend_shares(const AttnArgs a) {
  const int items = a.hkv * a.tiles;
  const int share = blockIdx.x;
  __shared__ Joint<D> sh;

  // Tiles of all sequences: each lane adds up a run of them.
  const int lane = threadIdx.x & 63;
  const int64_t per = (a.n_seq + 63) / 64;
  uint32_t mine = 0;
  for (int64_t i = 0; i < per; ++i)
    if (lane * per + i < a.n_seq) mine += rows_of(a, lane * per + i).tiles;
  const uint32_t upto = sum_upto(mine);
  const int64_t all = (int64_t)of_lane(upto, 63) * items;
  const int64_t shares = min((int64_t)a.shares, all);   // no share is smaller than a tile

  // A border inside a share costs it the chain of first loads once more.  With few
  // sequences it is spared: each item is dealt in parts of its own, of up to `most`
  // tiles, as long as that makes a share at most two tiles longer than an equal one
  // (three sequences of 1000 to 4000 rows 14.1 us, 17.2 in equal shares; ten of 136 to
  // 1090 13.1, 16.0; sixteen of 1024, whose borders happen to be the shares', lose: 16.3,
  // 14.5).  One sequence's borders are too few to count (94028 rows 40.9 us, 38.7 in equal
  // shares), and a tile each leaves none inside.
  const int64_t pieces = a.n_seq * items;
  const bool own = a.n_seq > 1 && all > shares && pieces < shares && all * pieces <= 2 * shares * (shares - pieces);

  int64_t seq, base = 0, x0 = 0, x1;
  int item = 0, t0 = 0, t1 = 0, parts = 0;
  Rows of;
  if (own) {
    const int most = (int)quotient(all - 1, shares - pieces) + 1;   // so that all / most + pieces <= shares
    auto parts_of = [&](const Rows& r) { return (int)quotient(r.tiles - 1, most) + 1; };
    uint32_t my_parts = 0;
    for (int64_t i = 0; i < per; ++i)
      if (lane * per + i < a.n_seq) my_parts += parts_of(rows_of(a, lane * per + i));
    const uint32_t parts_upto = sum_upto(my_parts);
    if (share >= (int64_t)of_lane(parts_upto, 63) * items) return;
    const int owner = __popcll(__ballot((int64_t)parts_upto * items <= share));   // the lane whose run holds the share
    int left = share - (int)(of_lane(parts_upto, owner) - of_lane(my_parts, owner)) * items;
    seq = owner * per;
    of = rows_of(a, seq);
    parts = parts_of(of);
    while (left >= parts * items) {
      left -= parts * items;
      of = rows_of(a, ++seq);
      parts = parts_of(of);
    }
    item = (int)quotient(left, parts);
    const int64_t part = left - item * parts;
    t0 = (int)quotient(part * of.tiles, parts);
    t1 = (int)quotient((part + 1) * of.tiles, parts);
    x1 = t1 - t0;
  } else {
    if (share >= shares) return;
    x0 = share_start(share, all, shares);
    x1 = share_start(share + 1, all, shares);
    const int owner = __popcll(__ballot((int64_t)upto * items <= x0));   // the lane whose run holds tile x0
    base = (int64_t)(of_lane(upto, owner) - of_lane(mine, owner)) * items;
    seq = owner * per;
    of = rows_of(a, seq);
    while (x0 >= base + (int64_t)of.tiles * items) {
      base += (int64_t)of.tiles * items;
      of = rows_of(a, ++seq);
    }
  }
  for (int64_t x = x0; x < x1;) {
    int64_t first = 0;             // the item's first tile
    if (!own) {
      item = (int)quotient(x - base, of.tiles);
      first = base + (int64_t)item * of.tiles;
      t0 = (int)(x - first);
      t1 = (int)min((int64_t)of.tiles, t0 + (x1 - x));
    }
    const bool whole = t0 == 0 && t1 == of.tiles;
    const int slot = 2 * share + (x == x0 ? 0 : 1);
    Wave<T, D, kAligned, kMask> w(a, seq, of, item);
    w.rows(t0 * kTile + uniform((int)threadIdx.x >> 6) * w.kStep, min(of.n, t1 * kTile), kWaves * w.kStep);
    if (x > x0) __syncthreads();   // the item before has been read from LDS
    sh.join(w, static_cast<T*>(a.out), whole ? nullptr : a.part + (int64_t)slot * min(kHeads, a.group) * kPart<D>);
    if (threadIdx.x == 0 && t0 == 0) {
      // An item's last equal share is the last one that starts before its end.
      if (!own) parts = whole ? 1 : (int)(quotient((first + of.tiles) * shares - 1, all) - share) + 1;
      int32_t* to = a.split + 3 * (seq * items + item);
      to[0] = whole ? 0 : parts;
      to[1] = slot;
      to[2] = share;
    }
    x += t1 - t0;
    if (x < x1 && x == base + (int64_t)items * of.tiles) {
      base = x;
      of = rows_of(a, ++seq);
    }
  }
}

// Joins the parts of one head of one sequence: groups of D/4 lanes each run over
// every kGroups-th part, in order, and the groups are joined in order.
template <class T, int D, int kThreads>
__global__ __launch_bounds__(kThreads) void k_join_parts(const AttnArgs a) {
  constexpr int kGroups = kThreads / (D / 4);
  __shared__ f32x4 out[kGroups][D / 4];
  __shared__ float stat[kGroups][2];
  const int head = blockIdx.x;
  const int64_t seq = blockIdx.y;
  const int kh = head / a.group, h = head % a.group;
  const int32_t* sp = a.split + 3 * (seq * a.hkv * a.tiles + (int64_t)kh * a.tiles + h / kHeads);
  const int n = sp[0], slot0 = sp[1], w0 = sp[2];
  if (n == 0) return;   // its output is written
  const int64_t step = (int64_t)min(kHeads, a.group) * kPart<D>;
  const float* base = a.part + (h % kHeads) * kPart<D>;
  const float c = a.scale * kLog2e;
  const int e4 = threadIdx.x % (D / 4), group = threadIdx.x / (D / 4);
  float m = -INFINITY, sum = 0;
  f32x4 o = {0, 0, 0, 0};
#pragma unroll 4
  for (int i = group; i < n; i += kGroups) {
    const float* p = base + (i == 0 ? slot0 : 2 * (w0 + i)) * step;
    const f32x4 x = *reinterpret_cast<const f32x4*>(p + 4 * e4);
    const float mi = p[D], si = p[D + 1];
    const float top = fmaxf(m, mi), at = top == -INFINITY ? 0.0f : top;
    const float f = exp2_((m - at) * c), fi = exp2_((mi - at) * c);
    o = o * f + x * fi;
    sum = sum * f + si * fi;
    m = top;
  }
  out[group][e4] = o;
  if (e4 == 0) {
    stat[group][0] = m;
    stat[group][1] = sum;
  }
  __syncthreads();
  for (int e = threadIdx.x; e < D; e += kThreads) {
    float top = -INFINITY, r = 0, s = 0;
#pragma unroll
    for (int i = 0; i < kGroups; ++i) top = fmaxf(top, stat[i][0]);
    const float at = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int i = 0; i < kGroups; ++i) {
      const float f = exp2_((stat[i][0] - at) * c);
      r += out[i][e / 4][e % 4] * f;
      s += stat[i][1] * f;
    }
    Elem<T>::put(s != 0 ? r / s : 0.0f, static_cast<T*>(a.out) + head * a.out_head + seq * a.out_row + e);
    if (e == 0 && a.lse) a.lse[head * a.n_seq + seq] = s != 0 ? top * a.scale + __log2f(s) * kLn2 : -INFINITY;
  }
}

// Spans that one workgroup takes whole: at most kWholeSpan rows (one sequence of 512
// rows of 28 heads over 4: 8.4 us, 9.5 in shares and a join), and more where items are
// many, kRowsPerItem for each of them (32 sequences, 128 items: of 500 to 1024 rows
// 18.8 us, 21.4 in shares; to 1400 rows 24.2 either way; to 2048 rows 33.5, 28.8), up to
// kWholeSpanMany (64 sequences of 1000 to 2048 rows: 39 us, 42 in shares).  Longer ones
// of few items would leave most of the chip idle: one sequence of 1024 rows takes 13 us
// whole, 9 in shares.
constexpr int64_t kWholeSpan = 512, kWholeSpanMany = 2048, kRowsPerItem = 11;

// Shares of k_attend_shares, 0 for one workgroup per sequence and item.
int64_t plan(int64_t n_seq, int64_t items, int64_t span) {
  const int64_t tiles = std::max<int64_t>(1, (span + kTile - 1) / kTile);
  if (span <= std::max(kWholeSpan, std::min(kWholeSpanMany, kRowsPerItem * n_seq * items))) return 0;
  return std::min<int64_t>(kShares, n_seq * items * tiles);
}

// Row numbers, up to a few thousand past max_len where steps are looked ahead, are 32-bit; tiles of all sequences
// are counted in 32 bits, and times key heads and shares stay below 2^50.
bool sizes_ok(int64_t n_seq, int32_t hq, int32_t hkv, int32_t d, int64_t max_len) {
  return n_seq >= 0 && n_seq < 65536 && hkv >= 1 && hkv < 256 && hq >= hkv && hq % hkv == 0 && hq < 4096 &&
         (d == 64 || d == 128) && max_len >= 0 && max_len <= (int64_t(1) << 31) - (1 << 16) &&
         n_seq * (max_len / kTile + 1) < (int64_t(1) << 31);
}

struct Layout {
  int32_t* split;
  float* part;
  size_t bytes;
};

// `shares` workgroups' parts, and which items are split.
Layout layout(void* ws, int64_t shares, int64_t n_seq, int64_t items, int32_t group, int32_t d) {
  Carver c(ws);
  Layout l{nullptr, nullptr, 0};
  if (shares) {
    l.split = c.take<int32_t>(3 * (size_t)(n_seq * items));
    l.part = c.take<float>((size_t)2 * shares * std::min(kHeads, group) * (d + 4));
  }
  l.bytes = c.used;
  return l;
}

template <class T, int D, bool kAligned, bool kMask>
apack_status launch(const AttnArgs& a, int32_t hq, hipStream_t s) {
  const unsigned items = (unsigned)(a.hkv * a.tiles);
  if (a.shares == 0) {
    hipLaunchKernelGGL((k_attend_whole<T, D, kAligned, kMask>), dim3(items, (unsigned)a.n_seq), dim3(64 * kWaves), 0, s, a);
    return launch_status("k_attend_whole");
  }
  hipLaunchKernelGGL((k_attend_shares<T, D, kAligned, kMask>), dim3((unsigned)a.shares), dim3(64 * kWaves), 0, s, a);
  apack_status st = launch_status("k_attend_shares");
  if (st != APACK_OK) return st;
  // Few parts each: one wave a head; many: eight.
  if (a.shares <= 8 * items * a.n_seq)
    hipLaunchKernelGGL((k_join_parts<T, D, 64>), dim3((unsigned)hq, (unsigned)a.n_seq), dim3(64), 0, s, a);
  else
    hipLaunchKernelGGL((k_join_parts<T, D, 512>), dim3((unsigned)hq, (unsigned)a.n_seq), dim3(512), 0, s, a);
  return launch_status("k_join_parts");
}

template <class T, int D>
apack_status run(const AttnArgs& a, int32_t hq, hipStream_t s) {
  // 16 rows in one page, and offsets within them that 32 bits hold.
  const bool aligned = a.pages.rows.d % 16 == 0 && a.pages.row_stride < (int64_t(1) << 26);
  if (a.mask) return aligned ? launch<T, D, true, true>(a, hq, s) : launch<T, D, false, true>(a, hq, s);
  return aligned ? launch<T, D, true, false>(a, hq, s) : launch<T, D, false, false>(a, hq, s);
}

}  // namespace
}  // namespace apack

using namespace apack;

extern "C" {

size_t apack_paged_attention_workspace(int64_t n_seq, int32_t hq, int32_t hkv, int32_t d, int64_t max_len) {
  if (!sizes_ok(n_seq, hq, hkv, d, max_len)) return 0;
  const int group = hq / hkv;
  const int64_t items = (int64_t)hkv * ((group + kHeads - 1) / kHeads);
  // The largest need up to these sizes: where so many sequences are taken whole, the most
  // that are dealt in shares.
  int64_t n = n_seq;
  if (plan(n, items, max_len) == 0) n = max_len > kWholeSpan ? std::min(n, (max_len - 1) / (kRowsPerItem * items)) : 0;
  return std::max<size_t>(kAlign, layout(nullptr, plan(n, items, max_len), n, items, group, d).bytes);
}

apack_status apack_paged_attention(int64_t n_seq, int32_t hq, const apack_heads* q, const apack_heads* out, float* lse,
                                   const apack_pages* pages, const int32_t* lens, int64_t max_len, const uint8_t* mask,
                                   int64_t mask_stride, int64_t window, double scale, void* ws, size_t ws_bytes,
                                   void* stream) {
  clear_error();
  AttnArgs a;
  std::memset(static_cast<void*>(&a), 0, sizeof a);
  Strided plane;
  apack_status st = check_pages(pages, "pages", &a.pages, &plane);
  if (st != APACK_OK) return st;
  APACK_CHECK(pages->n_layers == 1 && pages->v && (pages->table || n_seq == 0), APACK_E_ARG,
              "pages must be one layer with v and a table");
  APACK_CHECK(pages->d == 64 || pages->d == 128, APACK_E_UNSUPPORTED, "d must be 64 or 128");
  APACK_CHECK(hq >= 1 && hq % pages->hkv == 0, APACK_E_SHAPE, "hq must be a positive multiple of hkv");
  APACK_CHECK(n_seq >= 0 && max_len >= 0, APACK_E_SHAPE, "n_seq and max_len must be >= 0");
  APACK_CHECK(sizes_ok(n_seq, hq, pages->hkv, pages->d, max_len), APACK_E_UNSUPPORTED,
              "n_seq, heads or max_len too large");
  APACK_CHECK(window >= 0, APACK_E_ARG, "window must be >= 0");
  APACK_CHECK(scale == 0 || (scale >= 1e-30 && scale <= 1e30), APACK_E_ARG,
              "scale must lie in [1e-30, 1e30], or be 0 for 1/sqrt(d)");
  APACK_CHECK(n_seq == 0 || lens, APACK_E_ARG, "lens is NULL");
  APACK_CHECK(!mask || mask_stride >= max_len || mask_stride == 0, APACK_E_SHAPE, "mask_stride must be >= max_len, or 0");
  const size_t es = dtype_size(pages->dtype);
  Strided tq, to;
  st = check_heads(q, "q", n_seq, pages->d, es, &tq);
  if (st == APACK_OK) st = check_heads(out, "out", n_seq, pages->d, es, &to);
  if (st != APACK_OK) return st;
  APACK_CHECK(q->heads == hq && out->heads == hq, APACK_E_SHAPE, "q and out must have hq heads");
  if (n_seq == 0) return APACK_OK;

  a.q_head = hq > 1 ? q->head_stride : 0;
  a.q_row = n_seq > 1 ? q->row_stride : 0;
  a.out_head = hq > 1 ? out->head_stride : 0;
  a.out_row = n_seq > 1 ? out->row_stride : 0;
  const uintptr_t bits = (uintptr_t)q->data | (uintptr_t)pages->k[0] | (uintptr_t)pages->v[0] |
                         (uintptr_t)((a.q_head | a.q_row | a.pages.page_stride | a.pages.head_stride |
                                      a.pages.row_stride) * (int64_t)es);
  APACK_CHECK(bits % 16 == 0, APACK_E_UNSUPPORTED, "rows of q and of the pages must start 16-byte aligned");
  const int64_t span = window > 0 ? std::min(window, max_len) : max_len;
  a.hkv = pages->hkv;
  a.group = hq / pages->hkv;
  a.tiles = (a.group + kHeads - 1) / kHeads;
  const int64_t items = (int64_t)a.hkv * a.tiles;
  a.shares = (int32_t)plan(n_seq, items, span);
  const Layout lay = layout(ws, a.shares, n_seq, items, a.group, pages->d);
  const size_t need = lay.bytes;
  if (need) {
    APACK_CHECK(ws && (uintptr_t)ws % kAlign == 0, APACK_E_WORKSPACE, "workspace must be non-NULL and 256-byte aligned");
    APACK_CHECK(ws_bytes >= need, APACK_E_WORKSPACE, "workspace %zu < %zu needed", ws_bytes, need);
  }
  Strided pk = plane, pv = plane;
  pk.data = pages->k[0];
  pv.data = pages->v[0];
  const Strided reads[] = {tq, pk, pv, range(lens, (size_t)n_seq * 4),
                           rows_of_stride(pages->table, 4, n_seq, pages->table_stride, pages->table_width),
                           rows_of_stride(mask, 1, n_seq, mask_stride, max_len)};
  for (const Strided& r : reads) APACK_CHECK(r.ok, APACK_E_SHAPE, "a table or mask of 2^46 elements or more");
  const Strided writes[] = {to, range(lse, lse ? (size_t)hq * n_seq * 4 : 0), range(ws, need)};
  for (int i = 0; i < 3; ++i) {
    for (const Strided& r : reads) APACK_CHECK(apart(writes[i], r), APACK_E_ALIAS, "an output or the workspace overlaps an input");
    for (int j = i + 1; j < 3; ++j) APACK_CHECK(apart(writes[i], writes[j]), APACK_E_ALIAS, "outputs or the workspace overlap");
  }
  a.q = q->data;
  a.out = out->data;
  a.lse = lse;
  a.k = pages->k[0];
  a.v = pages->v[0];
  a.lens = lens;
  a.mask = mask;
  a.split = lay.split;
  a.part = lay.part;
  a.mask_stride = mask_stride;
  a.max_len = max_len;
  a.window = window;
  a.n_seq = n_seq;
  a.scale = scale > 0 ? (float)scale : (float)(1.0 / std::sqrt((double)pages->d));
  hipStream_t hs = static_cast<hipStream_t>(stream);
  if (pages->dtype == APACK_BF16) return pages->d == 128 ? run<uint16_t, 128>(a, hq, hs) : run<uint16_t, 64>(a, hq, hs);
  return pages->d == 128 ? run<float, 128>(a, hq, hs) : run<float, 64>(a, hq, hs);
}

}  // extern "C"
