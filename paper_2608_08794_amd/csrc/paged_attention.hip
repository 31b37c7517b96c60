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
// workgroups in equal shares, whatever the lengths on the device are.  Where a
// share's border falls inside a sequence's key head, each side leaves its
// maximum, sum and unnormalised output, and a second kernel joins them.
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
constexpr int kChunk = 2048;      // rows whose page ids lie in LDS at a time
constexpr int kShareWaves = 4;    // waves of a workgroup that takes a share
constexpr int kWholeWaves = 8;    // ... that takes a sequence's key head whole
constexpr int kShares = 512;      // two workgroups a compute unit: what the registers let run at once
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
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)((uint64_t)(uint32_t)uniform((int)x) | (uint64_t)(uint32_t)uniform((int)(x >> 32)) << 32);
}

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
  static __device__ __forceinline__ float get(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
  static __device__ __forceinline__ void put(float x, uint16_t* y) {
    const __bf16 b = (__bf16)x;
    *y = __builtin_bit_cast(uint16_t, b);
  }
};
template <> struct Elem<float> {
  static constexpr int kRow16 = 1;
  static __device__ __forceinline__ float get(float x) { return x; }
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
    bf16x8 pb;
#pragma unroll
    for (int i = 0; i < 8; ++i) pb[i] = (__bf16)p[i];
#pragma unroll
    for (int s = 0; s < kV; ++s) {
      u32x4 a;
#pragma unroll
      for (int j = 0; j < 4; ++j)   // element s of keys 2j and 2j + 1
        a[j] = __builtin_amdgcn_perm(v[2 * j + 1][s / 2], v[2 * j][s / 2], s % 2 ? 0x07060302u : 0x05040100u);
      acc[s] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), pb, acc[s], 0, 0, 0);
    }
  }
};

template <int D> struct Step<float, D> {
  static constexpr int kQ = D / 16;
  static constexpr int kV = D / 16;
  typedef unsigned int VRow __attribute__((ext_vector_type(kV)));
  u32x4 k[1][kQ];
  VRow v[4];

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

// A workgroup's state: per lane, for its head l % 16, the running maximum, its
// keys' part of the sum, and acc[s][i], element (4 (l/16) + i) kV + s of the output.
//
// kAligned: pages hold a multiple of 16 rows, so the 16 rows of a logit tile lie
// in one page.  A tile's address is then the wave's (scalar) plus an offset that a
// lane keeps, and page ids sit in one register, lane by lane.  Otherwise every lane
// looks its rows up in a list of page ids in LDS.
template <class T, int D, int kWaves, bool kAligned>
struct Worker {
  using S = Step<T, D>;
  static constexpr int kR = Elem<T>::kRow16, kKeys = 4 * kR, kStep = 16 * kR, kThreads = 64 * kWaves;
  static constexpr int kIdSteps = 64 / kR;         // steps whose page ids a wave holds
  struct Shared {
    int32_t page[kAligned ? 1 : kChunk + 1];       // ids of the pages of a chunk's rows, -1 where there is none
    float part[kWaves][kHeads][D + 4];
    float stat[kWaves][kHeads][2];
  };

  const AttnArgs& a;
  Shared& sh;
  const int64_t seq;
  const Rows of;
  const int kh, h0;                                // key head; first query head of its group
  const int lane = threadIdx.x & 63, wave = uniform((int)threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
  const float c = a.scale * kLog2e;
  u32x4 q[S::kQ];
  float m = -INFINITY, l = 0;
  f32x4 acc[S::kV] = {};
  const T *kb, *vb;

  __device__ __forceinline__ Worker(const AttnArgs& args, Shared& shared, int64_t s, const Rows& rows, int item)
      : a(args), sh(shared), seq(s), of(rows), kh(item / args.tiles), h0((item % args.tiles) * kHeads) {
    // The query rows; heads past the group read its last one and are never stored.
    const int h = kh * a.group + min(h0 + n, a.group - 1);
    const T* src = static_cast<const T*>(a.q) + h * a.q_head + seq * a.q_row;
#pragma unroll
    for (int j = 0; j < S::kQ; ++j) q[j] = *reinterpret_cast<const u32x4*>(src + S::k_off(g, j));
    kb = static_cast<const T*>(a.k) + kh * a.pages.head_stride;
    vb = static_cast<const T*>(a.v) + kh * a.pages.head_stride;
  }

  // Takes a loaded step of rows from r0 on; page_in(i): whether key i lies in a page.  `holes`: some may not.
  template <class F>
  __device__ __forceinline__ void take(S& st, int r0, bool holes, F page_in) {
    f32x4 xt[kR];
    st.logits(q, xt);
    float x[kKeys];
#pragma unroll
    for (int i = 0; i < kKeys; ++i) x[i] = xt[i / 4][i % 4];
    if (holes || a.mask || r0 < of.skip || r0 + kStep > of.n) {
      // Rows left out: their logit is -inf whatever they hold, their V is 0.
      bool in[kKeys];
#pragma unroll
      for (int i = 0; i < kKeys; ++i) {
        const int r = r0 + 16 * (i / 4) + 4 * g + i % 4;
        in[i] = (r >= of.skip) & (r < of.n) & (!holes || page_in(i));
      }
      if (a.mask) {
        const uint8_t* row = a.mask + seq * a.mask_stride + of.base;
        uint8_t seen[kKeys];
#pragma unroll
        for (int i = 0; i < kKeys; ++i) seen[i] = row[min(r0 + 16 * (i / 4) + 4 * g + i % 4, of.n - 1)];
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

  // Rows [first, end), the waves' steps in turn.  Each step is loaded while the
  // one before it is taken; a load past the last step reads one place of the pool.
  __device__ __forceinline__ void rows_aligned(int first, int end) {
    const int steps = max(0, (end - first - wave * kStep + kWaves * kStep - 1) / (kWaves * kStep));
    if (steps == 0) return;
    const int last = (of.n - 1) & ~15;              // first row of the last 16 that hold one
    const uint32_t page_rows = a.pages.rows.d;
    // Byte offsets of a lane's K row and first V row within 16 rows, and of a row.
    const uint32_t row = (uint32_t)a.pages.row_stride * sizeof(T);
    const uint32_t k_lane = n * row + S::k_off(g, 0) * sizeof(T);
    const uint32_t v_lane = 4 * g * row + n * S::kV * sizeof(T);
    auto row_of = [&](int s, int t) { return min(first + (wave + kWaves * s) * kStep + 16 * t, last); };
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
    };
    auto step = [&](S& st, const bool (&bad)[kR], int s) {
      bool holes = false;
#pragma unroll
      for (int t = 0; t < kR; ++t) holes |= bad[t];
      take(st, first + (wave + kWaves * s) * kStep, holes, [&](int i) { return !bad[i / 4]; });
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

  __device__ __forceinline__ void rows_general(int first, int end) {
    const uint32_t page_rows = a.pages.rows.d;
    for (; first < end; first += kChunk) {
      const int rows = min(kChunk, end - first);
      const int64_t r0 = of.base + first;
      const uint32_t p0 = a.pages.rows.div((uint32_t)r0);
      const int pages = (int)(a.pages.rows.div((uint32_t)(r0 + rows - 1)) - p0) + 1;
      __syncthreads();   // the last chunk's ids have been read
      for (int i = threadIdx.x; i < pages; i += kThreads) {
        const int32_t p = a.pages.table[seq * a.pages.table_stride + p0 + i];
        sh.page[i] = p >= 0 && p < a.pages.n_pages ? p : -1;
      }
      __syncthreads();
      // Offset of row i of the chunk in a plane (page 0 stands in where there is no page), and its page.
      auto row_at = [&](int i, int32_t* page) {
        const uint32_t r = (uint32_t)(r0 + min(i, rows - 1)), p = a.pages.rows.div(r);
        *page = sh.page[p - p0];
        return max(*page, 0) * a.pages.page_stride + (int64_t)(r - p * page_rows) * a.pages.row_stride;
      };
      for (int i0 = wave * kStep; i0 < rows; i0 += kWaves * kStep) {
        S st;
        int32_t page, least = 0, in[kKeys];
#pragma unroll
        for (int t = 0; t < kR; ++t) {
          const T* src = kb + row_at(i0 + 16 * t + n, &page);
#pragma unroll
          for (int j = 0; j < S::kQ; ++j) st.k[t][j] = stream(reinterpret_cast<const u32x4*>(src + S::k_off(g, j)));
        }
#pragma unroll
        for (int i = 0; i < kKeys; ++i) {
          const T* src = vb + row_at(i0 + 16 * (i / 4) + 4 * g + i % 4, &in[i]) + n * S::kV;
          st.v[i] = stream(reinterpret_cast<const typename S::VRow*>(src));
          least = min(least, in[i]);
        }
        take(st, first + i0, __any(least < 0), [&](int i) { return in[i] >= 0; });
      }
    }
  }

  // Joins the waves and writes the output, or with part != nullptr its parts.
  __device__ __forceinline__ void finish(float* part) {
    const int heads = min(kHeads, a.group - h0);
    l = sum_of_head(l);
    if (g == 0) {
      sh.stat[wave][n][0] = m;
      sh.stat[wave][n][1] = l;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int s = 0; s < S::kV; s += 4)
        *reinterpret_cast<f32x4*>(&sh.part[wave][n][(4 * g + i) * S::kV + s]) =
            f32x4{acc[s][i], acc[s + 1][i], acc[s + 2][i], acc[s + 3][i]};
    __syncthreads();
    for (int i = threadIdx.x; i < heads * D; i += kThreads) {
      const int h = i / D, e = i % D;
      float top = -INFINITY;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) top = fmaxf(top, sh.stat[w][h][0]);
      const float at = top == -INFINITY ? 0.0f : top;
      float sum = 0, o = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        const float f = exp2_((sh.stat[w][h][0] - at) * c);
        sum += sh.stat[w][h][1] * f;
        o += sh.part[w][h][e] * f;
      }
      if (part) {
        float* to = part + h * kPart<D>;
        to[e] = o;
        if (e == 0) {
          to[D] = top;
          to[D + 1] = sum;
        }
      } else {
        const int64_t head = (int64_t)kh * a.group + h0 + h;
        Elem<T>::put(sum > 0 ? o / sum : 0.0f, static_cast<T*>(a.out) + head * a.out_head + seq * a.out_row + e);
        if (e == 0 && a.lse) a.lse[head * a.n_seq + seq] = sum > 0 ? top * a.scale + __log2f(sum) * kLn2 : -INFINITY;
      }
    }
    __syncthreads();   // before the next item's parts
  }

  // Tiles [t0, t1) of item `item` (key head and 16 query heads) of a sequence.
  static __device__ __forceinline__ void run(const AttnArgs& a, Shared& sh, int64_t seq, const Rows& of, int item, int t0,
                                             int t1, float* part) {
    Worker w(a, sh, seq, of, item);
    const int end = min(of.n, t1 * kTile);
    if constexpr (kAligned) w.rows_aligned(t0 * kTile, end);
    else w.rows_general(t0 * kTile, end);
    w.finish(part);
  }
};

// One workgroup for each sequence and item.
template <class T, int D, bool kAligned>
__global__ __launch_bounds__(64 * kWholeWaves) void k_attend_whole(const AttnArgs a) {
  using W = Worker<T, D, kWholeWaves, kAligned>;
  __shared__ typename W::Shared sh;
  const Rows of = rows_of(a, blockIdx.y);
  W::run(a, sh, blockIdx.y, of, blockIdx.x, 0, of.tiles, nullptr);
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

template <class T, int D, bool kAligned>
__global__ __launch_bounds__(64 * kShareWaves, 2) void k_attend_shares(const AttnArgs a) {
  using W = Worker<T, D, kShareWaves, kAligned>;
  __shared__ typename W::Shared sh;
  const int items = a.hkv * a.tiles;

  // Tiles of all sequences, and the sequence of this share's first one: each
  // lane adds up a run of sequences, every wave for itself (no barrier).
  const int lane = threadIdx.x & 63;
  const int64_t per = (a.n_seq + 63) / 64;
  uint32_t mine = 0;
  for (int64_t i = 0; i < per; ++i)
    if (lane * per + i < a.n_seq) mine += rows_of(a, lane * per + i).tiles;
  const uint32_t upto = sum_upto(mine);
  const int64_t all = (int64_t)(uint32_t)__builtin_amdgcn_readlane(upto, 63) * items;
  // No more shares than give each wave a tile; none is empty.
  const int64_t shares = max((int64_t)1, min((int64_t)a.shares, all / kShareWaves));
  if (blockIdx.x >= shares) return;
  const int64_t x0 = share_start(blockIdx.x, all, shares), x1 = share_start(blockIdx.x + 1, all, shares);
  const int owner = __popcll(__ballot((int64_t)upto * items <= x0));   // the lane whose run holds tile x0
  int64_t seq = owner * per;
  int64_t base = (int64_t)(uint32_t)(__builtin_amdgcn_readlane(upto, owner) - __builtin_amdgcn_readlane(mine, owner)) * items;
  Rows of = rows_of(a, seq);
  while (x0 >= base + (int64_t)of.tiles * items) {
    base += (int64_t)of.tiles * items;
    of = rows_of(a, ++seq);
  }
  for (int64_t x = x0; x < x1;) {
    const int item = (int)quotient(x - base, of.tiles);
    const int64_t first = base + (int64_t)item * of.tiles;   // the item's first tile
    const int t0 = (int)(x - first), t1 = (int)min((int64_t)of.tiles, t0 + (x1 - x));
    const bool whole = t0 == 0 && t1 == of.tiles;
    const int slot = 2 * (int)blockIdx.x + (x == x0 ? 0 : 1);
    if (threadIdx.x == 0 && t0 == 0) {
      // The item's last share is the last w with w all < (its last tile + 1) shares.
      const int64_t last = whole ? 0 : quotient((first + of.tiles) * shares - 1, all);
      int32_t* to = a.split + 3 * (seq * items + item);
      to[0] = whole ? 0 : (int32_t)(last - blockIdx.x) + 1;
      to[1] = slot;
      to[2] = blockIdx.x;
    }
    float* part = whole ? nullptr : a.part + (int64_t)slot * min(kHeads, a.group) * kPart<D>;
    W::run(a, sh, seq, of, item, t0, t1, part);
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
    Elem<T>::put(s > 0 ? r / s : 0.0f, static_cast<T*>(a.out) + head * a.out_head + seq * a.out_row + e);
    if (e == 0 && a.lse) a.lse[head * a.n_seq + seq] = s > 0 ? top * a.scale + __log2f(s) * kLn2 : -INFINITY;
  }
}

constexpr int64_t kWholeSpan = 512;

// Workgroups of k_attend_shares, 0 for one workgroup per sequence and item.
int64_t plan(int64_t n_seq, int64_t items, int64_t span) {
  const int64_t tiles = std::max<int64_t>(1, (span + kTile - 1) / kTile);
  if (span <= kWholeSpan) return 0;
  return std::min<int64_t>(kShares, (n_seq * items * tiles + kShareWaves - 1) / kShareWaves);
}

// Tiles of all sequences are counted in 32 bits, and times key heads and shares stay below 2^50.
bool sizes_ok(int64_t n_seq, int32_t hq, int32_t hkv, int32_t d, int64_t max_len) {
  return n_seq >= 0 && n_seq < 65536 && hkv >= 1 && hkv < 256 && hq >= hkv && hq % hkv == 0 && hq < 4096 &&
         (d == 64 || d == 128) && max_len >= 0 && max_len < (int64_t(1) << 31) - kChunk &&
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

template <class T, int D, bool kAligned>
apack_status launch(const AttnArgs& a, int32_t hq, hipStream_t s) {
  const unsigned items = (unsigned)(a.hkv * a.tiles);
  if (a.shares == 0) {
    hipLaunchKernelGGL((k_attend_whole<T, D, kAligned>), dim3(items, (unsigned)a.n_seq), dim3(64 * kWholeWaves), 0, s, a);
    return launch_status("k_attend_whole");
  }
  hipLaunchKernelGGL((k_attend_shares<T, D, kAligned>), dim3((unsigned)a.shares), dim3(64 * kShareWaves), 0, s, a);
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
  return aligned ? launch<T, D, true>(a, hq, s) : launch<T, D, false>(a, hq, s);
}

}  // namespace
}  // namespace apack

using namespace apack;

extern "C" {

size_t apack_paged_attention_workspace(int64_t n_seq, int32_t hq, int32_t hkv, int32_t d, int64_t max_len) {
  if (!sizes_ok(n_seq, hq, hkv, d, max_len)) return 0;
  const int group = hq / hkv;
  const int64_t items = (int64_t)hkv * ((group + kHeads - 1) / kHeads);
  return std::max<size_t>(kAlign, layout(nullptr, plan(n_seq, items, max_len), n_seq, items, group, d).bytes);
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
  APACK_CHECK(scale >= 0 && std::isfinite((float)scale), APACK_E_ARG, "scale must be finite, and > 0 or 0 for 1/sqrt(d)");
  APACK_CHECK(n_seq == 0 || lens, APACK_E_ARG, "lens is NULL");
  APACK_CHECK(!mask || mask_stride >= max_len, APACK_E_SHAPE, "mask_stride must be >= max_len");
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
                           range(pages->table, (size_t)((n_seq - 1) * pages->table_stride + pages->table_width) * 4),
                           range(mask, mask ? (size_t)((n_seq - 1) * mask_stride + max_len) : 0)};
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
