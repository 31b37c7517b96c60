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
// The rows of a sequence are split over workgroups (chunks of a size that fills
// the chip); each leaves its maximum, sum and unnormalised output, and a second
// kernel joins them.
#include <cmath>
#include <cstring>

#include "pages.hpp"

namespace apack {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kWaves = 4;
constexpr int kThreads = 64 * kWaves;
constexpr int kHeads = 16;        // query heads of a workgroup: an MFMA's columns
constexpr int kTile = 32;         // rows of a wave's step
constexpr int kMinChunk = kWaves * kTile;
constexpr int kMaxChunk = 2048;   // rows of a workgroup; its page ids lie in LDS
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
  float* part;                    // [seq][head][chunk][D + 2]: output, maximum, sum
  int64_t q_head, q_row, out_head, out_row, mask_stride;   // elements
  int64_t max_len, window;
  int64_t n_seq;
  int32_t hkv, group;             // key heads; query heads of each
  int32_t tiles;                  // ceil(group / kHeads)
  int32_t chunk, chunks;          // rows of a workgroup; workgroups of a sequence's key head
  float scale;
  PoolDev pages;
};

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }

// Over the four lanes that hold a head.
__device__ __forceinline__ float max_of_head(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum_of_head(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
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
  struct VRow {
    u32x4 w[kV / 4];
  };
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
        acc[s] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(v[i].w[s / 4][s % 4]), p[i], acc[s], 0, 0, 0);
  }
};

template <class T, int D>
__global__ __launch_bounds__(kThreads) void k_paged_attention(const AttnArgs a) {
  using S = Step<T, D>;
  constexpr int kR = Elem<T>::kRow16, kKeys = 4 * kR, kStep = 16 * kR;
  constexpr int kPad = D + 4;
  __shared__ int32_t page_of[kMaxChunk + 1];
  __shared__ float part[kWaves][kHeads][kPad];
  __shared__ float stat[kWaves][kHeads][2];
  __shared__ int any_bad;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int n = lane & 15, g = lane >> 4;
  const int chunk = blockIdx.x;
  const int kh = blockIdx.y / a.tiles, h0 = (blockIdx.y % a.tiles) * kHeads;   // key head; first head of its group
  const int64_t seq = blockIdx.z;
  const int heads = min(kHeads, a.group - h0);

  // Rows [r0, r1) of this workgroup.
  const uint32_t page_rows = a.pages.rows.d;
  int64_t len = min((int64_t)a.lens[seq], min(a.max_len, (int64_t)a.pages.table_width * page_rows));
  len = max(len, (int64_t)0);
  const int64_t lo = a.window > 0 ? max((int64_t)0, (int64_t)a.lens[seq] - a.window) : 0;
  const int64_t r0 = lo + (int64_t)chunk * a.chunk;
  const int rows = (int)max((int64_t)0, min((int64_t)a.chunk, len - r0));
  if (rows == 0 && a.chunks > 1) return;   // the join counts chunks itself

  const uint32_t p0 = a.pages.rows.div((uint32_t)r0);
  if (threadIdx.x == 0) any_bad = 0;
  __syncthreads();
  if (rows > 0) {
    const int pages = (int)(a.pages.rows.div((uint32_t)(r0 + rows - 1)) - p0) + 1;
    for (int i = threadIdx.x; i < pages; i += kThreads) {
      int32_t p = a.pages.table[seq * a.pages.table_stride + p0 + i];
      if (p < 0 || p >= a.pages.n_pages) {
        p = -1;
        any_bad = 1;
      }
      page_of[i] = p;
    }
  }
  __syncthreads();
  const bool holes = any_bad || a.mask;

  // The query rows; heads past the group read its last one and are never stored.
  u32x4 q[S::kQ];
  {
    const int h = kh * a.group + h0 + min(n, heads - 1);
    const T* src = static_cast<const T*>(a.q) + h * a.q_head + seq * a.q_row;
#pragma unroll
    for (int j = 0; j < S::kQ; ++j) q[j] = *reinterpret_cast<const u32x4*>(src + S::k_off(g, j));
  }
  const T* kb = static_cast<const T*>(a.k) + kh * a.pages.head_stride;
  const T* vb = static_cast<const T*>(a.v) + kh * a.pages.head_stride;
  // Row i of the chunk, in a page (page 0 stands in where there is none).
  auto row_at = [&](const T* base, int i) {
    const uint32_t r = (uint32_t)(r0 + i), p = a.pages.rows.div(r);
    return base + max(page_of[p - p0], 0) * a.pages.page_stride + (int64_t)(r - p * page_rows) * a.pages.row_stride;
  };

  const float c = a.scale * kLog2e;
  float m = -INFINITY, l = 0;
  f32x4 acc[S::kV] = {};
  for (int i0 = wave * kStep; i0 < rows; i0 += kWaves * kStep) {
    S st;
#pragma unroll
    for (int t = 0; t < kR; ++t) {
      const T* src = row_at(kb, min(i0 + 16 * t + n, rows - 1));
#pragma unroll
      for (int j = 0; j < S::kQ; ++j) st.k[t][j] = *reinterpret_cast<const u32x4*>(src + S::k_off(g, j));
    }
#pragma unroll
    for (int i = 0; i < kKeys; ++i)
      st.v[i] = *reinterpret_cast<const typename S::VRow*>(
          row_at(vb, min(i0 + 16 * (i / 4) + 4 * g + i % 4, rows - 1)) + n * S::kV);
    f32x4 xt[kR];
    st.logits(q, xt);
    float x[kKeys];
#pragma unroll
    for (int i = 0; i < kKeys; ++i) x[i] = xt[i / 4][i % 4];
    if (holes || i0 + kStep > rows) {
      // Rows left out: their logit is -inf whatever they hold, their V is 0.
#pragma unroll
      for (int i = 0; i < kKeys; ++i) {
        const int r = i0 + 16 * (i / 4) + 4 * g + i % 4;
        bool in = r < rows;
        if (in && holes) {
          in = page_of[a.pages.rows.div((uint32_t)(r0 + r)) - p0] >= 0;
          if (in && a.mask) in = a.mask[seq * a.mask_stride + r0 + r] != 0;
        }
        if (!in) {
          x[i] = -INFINITY;
          st.v[i] = typename S::VRow{};
        }
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
  l = sum_of_head(l);

  // Join the waves.  acc[s][i] is element (4 g + i) kV + s of head n.
  if (g == 0) {
    stat[wave][n][0] = m;
    stat[wave][n][1] = l;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int s = 0; s < S::kV; ++s) part[wave][n][(4 * g + i) * S::kV + s] = acc[s][i];
  __syncthreads();
  for (int i = threadIdx.x; i < heads * D; i += kThreads) {
    const int h = i / D, e = i % D;
    float top = -INFINITY;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, stat[w][h][0]);
    const float at = top == -INFINITY ? 0.0f : top;
    float sum = 0, o = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f = exp2_((stat[w][h][0] - at) * c);
      sum += stat[w][h][1] * f;
      o += part[w][h][e] * f;
    }
    const int64_t head = (int64_t)kh * a.group + h0 + h;
    if (a.chunks > 1) {
      float* to = a.part + ((seq * a.hkv * a.group + head) * a.chunks + chunk) * (D + 2);
      to[e] = o;
      if (e == 0) {
        to[D] = top;
        to[D + 1] = sum;
      }
    } else {
      Elem<T>::put(sum > 0 ? o / sum : 0.0f, static_cast<T*>(a.out) + head * a.out_head + seq * a.out_row + e);
      if (e == 0 && a.lse) a.lse[head * a.n_seq + seq] = sum > 0 ? top * a.scale + __log2f(sum) * kLn2 : -INFINITY;
    }
  }
}

// Joins the chunks of one head of one sequence.
template <class T, int D>
__global__ __launch_bounds__(kThreads) void k_join_chunks(const AttnArgs a) {
  constexpr int kLanes = kThreads / D;
  __shared__ float red[kThreads];
  __shared__ float sums[kThreads];
  const int64_t head = blockIdx.x, seq = blockIdx.y;
  const int64_t width = (int64_t)a.pages.table_width * a.pages.rows.d;
  const int64_t len = max((int64_t)0, min((int64_t)a.lens[seq], min(a.max_len, width)));
  const int64_t lo = a.window > 0 ? max((int64_t)0, (int64_t)a.lens[seq] - a.window) : 0;
  const int n = (int)((max((int64_t)0, len - lo) + a.chunk - 1) / a.chunk);
  const float* part = a.part + (seq * a.hkv * a.group + head) * a.chunks * (D + 2);
  const float c = a.scale * kLog2e;
  float top = -INFINITY;
  for (int i = threadIdx.x; i < n; i += kThreads) top = fmaxf(top, part[(int64_t)i * (D + 2) + D]);
  red[threadIdx.x] = top;
  __syncthreads();
  for (int s = kThreads / 2; s > 0; s >>= 1) {
    if (threadIdx.x < s) red[threadIdx.x] = fmaxf(red[threadIdx.x], red[threadIdx.x + s]);
    __syncthreads();
  }
  top = red[0];
  __syncthreads();
  const float at = top == -INFINITY ? 0.0f : top;
  const int e = threadIdx.x % D;
  float o = 0, sum = 0;
  for (int i = threadIdx.x / D; i < n; i += kLanes) {
    const float* p = part + (int64_t)i * (D + 2);
    const float f = exp2_((p[D] - at) * c);
    o += p[e] * f;
    sum += p[D + 1] * f;
  }
  red[threadIdx.x] = o;
  sums[threadIdx.x] = sum;
  __syncthreads();
  if (threadIdx.x < D) {
    o = sum = 0;
#pragma unroll
    for (int i = 0; i < kLanes; ++i) {
      o += red[i * D + e];
      sum += sums[i * D + e];
    }
    Elem<T>::put(sum > 0 ? o / sum : 0.0f, static_cast<T*>(a.out) + head * a.out_head + seq * a.out_row + e);
    if (e == 0 && a.lse) a.lse[head * a.n_seq + seq] = sum > 0 ? top * a.scale + __log2f(sum) * kLn2 : -INFINITY;
  }
}

// Rows of a chunk: whole steps of a workgroup, as many as leave 1024 workgroups.
void plan(int64_t n_seq, int64_t items, int64_t span, int32_t* chunk, int32_t* chunks) {
  const int64_t want = std::max<int64_t>(1, 1024 / std::max<int64_t>(1, n_seq * items));
  int64_t c = (span + want - 1) / want;
  c = (c + kMinChunk - 1) / kMinChunk * kMinChunk;
  c = std::min<int64_t>(std::max<int64_t>(c, kMinChunk), kMaxChunk);
  *chunk = (int32_t)c;
  *chunks = (int32_t)std::max<int64_t>(1, (span + c - 1) / c);
}

bool sizes_ok(int64_t n_seq, int32_t hq, int32_t hkv, int32_t d, int64_t max_len) {
  return n_seq >= 0 && n_seq < 65536 && hkv >= 1 && hkv < 65536 && hq >= hkv && hq % hkv == 0 && hq < 65536 &&
         (d == 64 || d == 128) && max_len >= 0 && max_len < (int64_t(1) << 31) - kMaxChunk;
}

// Bytes for the chunks of any span up to max_len.
size_t workspace(int64_t n_seq, int32_t hq, int32_t hkv, int32_t d, int64_t max_len) {
  const int64_t items = n_seq * hkv * ((hq / hkv + kHeads - 1) / kHeads);
  const int64_t want = std::max<int64_t>(1, 1024 / std::max<int64_t>(1, items));
  const int64_t chunks = std::max(std::min(want, (max_len + kMinChunk - 1) / kMinChunk), (max_len + kMaxChunk - 1) / kMaxChunk);
  return chunks > 1 ? align_up((size_t)n_seq * hq * chunks * (d + 2) * sizeof(float)) : 0;
}

template <class T, int D>
apack_status run(const AttnArgs& a, int32_t hq, hipStream_t s) {
  hipLaunchKernelGGL((k_paged_attention<T, D>), dim3((unsigned)a.chunks, (unsigned)(a.hkv * a.tiles), (unsigned)a.n_seq),
                     dim3(kThreads), 0, s, a);
  apack_status st = launch_status("k_paged_attention");
  if (st != APACK_OK || a.chunks == 1) return st;
  hipLaunchKernelGGL((k_join_chunks<T, D>), dim3((unsigned)hq, (unsigned)a.n_seq), dim3(kThreads), 0, s, a);
  return launch_status("k_join_chunks");
}

}  // namespace
}  // namespace apack

using namespace apack;

extern "C" {

size_t apack_paged_attention_workspace(int64_t n_seq, int32_t hq, int32_t hkv, int32_t d, int64_t max_len) {
  if (!sizes_ok(n_seq, hq, hkv, d, max_len)) return 0;
  return std::max<size_t>(kAlign, workspace(n_seq, hq, hkv, d, max_len));
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
  APACK_CHECK((int64_t)a.hkv * a.tiles < 65536, APACK_E_UNSUPPORTED, "too many heads");
  plan(n_seq, (int64_t)a.hkv * a.tiles, span, &a.chunk, &a.chunks);
  const size_t need = a.chunks > 1 ? workspace(n_seq, hq, pages->hkv, pages->d, max_len) : 0;
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
  a.part = static_cast<float*>(ws);
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
