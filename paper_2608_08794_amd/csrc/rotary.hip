// Rotary positions: pair i of a head's first rot_dim elements turns by
// theta = pos * f_i,
//   a' = factor (a cos - b sin),  b' = factor (a sin + b cos),
// alone (apack_rotary) or together with a decode step's append of K and V to a
// paged cache (apack_rotary_append).
//
// One read and one write of every element: bound by HBM, by launch latency for
// the few rows of a decode step.  The angle depends on the row and the pair but
// not on the head, so a thread owns one row and 2 * VEC elements (VEC pairs),
// forms their sines and cosines once and applies them to a run of heads.
#include <cmath>
#include <cstring>

#include "pages.hpp"

namespace apack {
namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kMaxDim = 512;
constexpr int kUnroll = 2;      // heads in flight per thread
constexpr double kTwoPi = 6.283185307179586476925286766559;

struct HeadsDev {
  const void* in;
  void* out;
  int64_t in_head, in_row, out_head, out_row;   // strides, elements
  int32_t heads;
};

struct RotaryArgs {
  const int32_t* pos;
  int64_t pos_stride, rows;
  int32_t d, rot, pos_rows;
  int32_t chunks, rows_per_wg;   // threads of a row; rows of a workgroup
  int32_t chunk_magic;           // ceil(2^16 / chunks)
  int32_t heads_per_wg;          // heads of a workgroup, of all tensors
  int32_t bound[3];              // first pair of sections 1, 2 and 3
  float factor, sign;
  HeadsDev t[3];                 // q, k, v (v is copied)
  const int32_t* lens;           // append: rows of pool `pages` take k and v
  PoolDev pages;
  double turns[APACK_ROPE_MAX_PAIRS];   // freq / 2 pi
};

template <class T, int VEC>
struct alignas(sizeof(T) * VEC) Vec {
  T v[VEC];
};

// kStream: nontemporal, for tensors that pass once (16-byte vectors only).
template <bool kStream, class T, int VEC>
__device__ __forceinline__ void get(const T* p, Vec<T, VEC>* v) {
  if constexpr (kStream && VEC > 1) {
    const u32x4 x = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    __builtin_memcpy(v, &x, 16);
  } else {
    *v = *reinterpret_cast<const Vec<T, VEC>*>(p);
  }
}
template <bool kStream, class T, int VEC>
__device__ __forceinline__ void put(const Vec<T, VEC>& v, T* p) {
  if constexpr (kStream && VEC > 1) {
    u32x4 x;
    __builtin_memcpy(&x, &v, 16);
    __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(p));
  } else {
    *reinterpret_cast<Vec<T, VEC>*>(p) = v;
  }
}

__device__ __forceinline__ float to_f(float x) { return x; }
__device__ __forceinline__ float to_f(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ void from_f(float x, float* y) { *y = x; }
__device__ __forceinline__ void from_f(float x, uint16_t* y) {   // to nearest, ties to even; NaN stays NaN
  const __bf16 b = (__bf16)x;
  *y = __builtin_bit_cast(uint16_t, b);
}

// The products and sums are written out, so that every variant rounds alike.
template <class T>
__device__ __forceinline__ void turn_pair(float a, float b, float c, float s, T* x, T* y) {
  from_f(__builtin_fmaf(a, c, -(b * s)), x);
  from_f(__builtin_fmaf(a, s, b * c), y);
}

// Sine and cosine of x turns, |x| <= 1/2: an eighth of a turn or less from a whole
// quarter, where the Taylor series to the 9th and 10th power are off by less than 2^-28.
// Half as long as the library's, which takes any angle: 12998 rows of 18 heads of 64
// take 16.0 us, 17.2 with it, one row's append 3.9, 4.2.
__device__ __forceinline__ void sincos_turns(float x, float* s, float* c) {
  const float q = __builtin_rintf(4.0f * x), r = __builtin_fmaf(q, -0.25f, x), t = r * r;
  float a = __builtin_fmaf(t, 4.205869394e+01f, -7.670585975e+01f);
  a = __builtin_fmaf(t, a, 8.160524928e+01f);
  a = __builtin_fmaf(t, a, -4.134170224e+01f);
  a = r * __builtin_fmaf(t, a, 6.283185307e+00f);
  float b = __builtin_fmaf(t, -2.642625678e+01f, 6.024464137e+01f);
  b = __builtin_fmaf(t, b, -8.545681721e+01f);
  b = __builtin_fmaf(t, b, 6.493939402e+01f);
  b = __builtin_fmaf(t, b, -1.973920880e+01f);
  b = __builtin_fmaf(t, b, 1.0f);
  const int n = (int)q;                     // quarters: -2 to 2
  const uint32_t sn = __float_as_uint(n & 1 ? b : a), cn = __float_as_uint(n & 1 ? a : b);
  *s = __uint_as_float(sn ^ ((uint32_t)n & 2) << 30);
  *c = __uint_as_float(cn ^ ((uint32_t)(n + 1) & 2) << 30);
}

// T: uint16_t (bf16 bits) or float.  A thread has VEC elements from e0 and VEC from
// e1 on, half of what turns (or of what does not) apart, so that the lanes of either
// load lie side by side.  The VEC pairs are (e0 + j, e1 + j) (kHalf), or two by two
// within each; single elements (VEC 1) are neighbours then.
template <class T, int VEC, bool kHalf, bool kAppend>
__global__ __launch_bounds__(kThreads) void k_rotary(const RotaryArgs a) {
  using V = Vec<T, VEC>;
  const int rl = (threadIdx.x * a.chunk_magic) >> 16, c = threadIdx.x - rl * a.chunks;
  const int64_t row = (int64_t)blockIdx.x * a.rows_per_wg + rl;
  if (rl >= a.rows_per_wg || row >= a.rows) return;
  const int half = a.rot >> 1;
  const bool turned = c * VEC < half;
  int e0, e1, pair0, pair1;      // the first pair of either half of the pairs
  if (turned) {
    const bool apart = kHalf || VEC > 1;
    e0 = apart ? c * VEC : 2 * c;
    e1 = apart ? e0 + half : e0 + 1;
    pair0 = kHalf || VEC == 1 ? c * VEC : e0 / 2;
    pair1 = kHalf || VEC == 1 ? pair0 + VEC / 2 : e1 / 2;
  } else {                       // elements that do not turn
    e0 = a.rot + (c * VEC - half);
    e1 = e0 + (a.d - a.rot + 1) / 2;
    pair0 = pair1 = 0;
  }
  const bool second = e1 < a.d;  // an odd d ends in a single element

  // Vectors: the positions are asked for first, the rows' elements next, and the
  // angles come while those are on their way (which takes 0.9 us off 256 sequences'
  // append).  Single elements, many heads a thread, have them before.
  int32_t p[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) p[j] = turned && j < a.pos_rows ? a.pos[j * a.pos_stride + row] : 0;
  float cs[VEC], sn[VEC];
  bool angles = false;
  auto form_angles = [&]() {
    angles = true;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
      const int i = VEC > 1 && j >= VEC / 2 ? pair1 + j - VEC / 2 : pair0 + j;
      const int32_t at = i < a.bound[0] ? p[0] : i < a.bound[1] ? p[1] : i < a.bound[2] ? p[2] : p[3];
      // fp64 up to the fraction of a turn: a position of 2^31 is still off by
      // less than 2^-24 turns, where an fp32 angle would be off by whole turns.
      const double x = __builtin_rint((double)at * a.turns[i]);
      float s, k;
      sincos_turns((float)__builtin_fma((double)at, a.turns[i], -x), &s, &k);
      cs[j] = k * a.factor;
      sn[j] = s * a.factor * a.sign;
    }
  };

  if (VEC == 1 && turned) form_angles();

  int64_t page_off = -1;         // append: the new row's place in the pool
  if constexpr (kAppend) {
    const int64_t at = (int64_t)a.lens[row] - 1;
    if (at >= 0) {
      const uint32_t n = a.pages.rows.div((uint32_t)at);
      if (n < (uint32_t)a.pages.table_width) {
        const int32_t page = a.pages.table[row * a.pages.table_stride + n];
        if (page >= 0 && page < a.pages.n_pages)
          page_off = page * a.pages.page_stride + (at - (int64_t)n * a.pages.rows.d) * a.pages.row_stride;
      }
    }
  }

  int h0 = blockIdx.y * a.heads_per_wg, left = a.heads_per_wg;
#pragma unroll
  for (int ti = 0; ti < (kAppend ? 3 : 2); ++ti) {
    const HeadsDev& t = a.t[ti];
    if (h0 >= t.heads) {
      h0 -= t.heads;
      continue;
    }
    const int n = min(left, t.heads - h0);
    const T* in = static_cast<const T*>(t.in) + row * t.in_row + h0 * t.in_head;
    T* out = static_cast<T*>(t.out) + h0 * t.out_head;
    bool write = true;
    if (kAppend && ti > 0) {
      write = page_off >= 0;
      out += page_off;
    } else {
      out += row * t.out_row;
    }
    const bool turn = turned && ti < 2;
    if (write)
      for (int h = 0; h < n; h += kUnroll) {
        V x[kUnroll], y[kUnroll];
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
          if (h + u < n) {
            get<!kAppend>(in + (h + u) * t.in_head + e0, &x[u]);
            if (second) get<!kAppend>(in + (h + u) * t.in_head + e1, &y[u]);
          }
        if (VEC > 1 && turn && !angles) form_angles();
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
          if (h + u < n) {
            if (turn) {
              if constexpr (kHalf || VEC == 1) {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                  const float p = to_f(x[u].v[j]), q = to_f(y[u].v[j]);
                  turn_pair(p, q, cs[j], sn[j], &x[u].v[j], &y[u].v[j]);
                }
              } else {
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                  V& w = j < VEC / 2 ? x[u] : y[u];
                  const int i = 2 * j % VEC;
                  const float p = to_f(w.v[i]), q = to_f(w.v[i + 1]);
                  turn_pair(p, q, cs[j], sn[j], &w.v[i], &w.v[i + 1]);
                }
              }
            }
            put<!kAppend>(x[u], out + (h + u) * t.out_head + e0);
            if (second) put<!kAppend>(y[u], out + (h + u) * t.out_head + e1);
          }
      }
    left -= n;
    h0 = 0;
    if (left <= 0) return;
  }
}

template <class T, int VEC>
void launch(const RotaryArgs& a, bool half, bool append, dim3 grid, hipStream_t s) {
  if (append) {
    if (half) hipLaunchKernelGGL((k_rotary<T, VEC, true, true>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((k_rotary<T, VEC, false, true>), grid, dim3(kThreads), 0, s, a);
  } else {
    if (half) hipLaunchKernelGGL((k_rotary<T, VEC, true, false>), grid, dim3(kThreads), 0, s, a);
    else hipLaunchKernelGGL((k_rotary<T, VEC, false, false>), grid, dim3(kThreads), 0, s, a);
  }
}

apack_status check_rope(const apack_rope* r, int32_t d, RotaryArgs* a) {
  APACK_CHECK(r, APACK_E_ARG, "rope is NULL");
  APACK_CHECK(r->rot_dim >= 2 && r->rot_dim <= 2 * APACK_ROPE_MAX_PAIRS && r->rot_dim % 2 == 0, APACK_E_SHAPE,
              "rot_dim must be even and lie in [2, %d]", 2 * APACK_ROPE_MAX_PAIRS);
  APACK_CHECK(r->layout == APACK_ROPE_HALF || r->layout == APACK_ROPE_INTERLEAVED, APACK_E_ARG, "unknown layout %d",
              r->layout);
  APACK_CHECK(r->transpose == 0 || r->transpose == 1, APACK_E_ARG, "transpose must be 0 or 1");
  APACK_CHECK(r->pos_rows >= 1 && r->pos_rows <= 4, APACK_E_ARG, "pos_rows must lie in [1, 4]");
  APACK_CHECK(d >= 1 && d <= kMaxDim, APACK_E_UNSUPPORTED, "d must lie in [1, %d]", kMaxDim);
  APACK_CHECK(r->rot_dim <= d, APACK_E_SHAPE, "rot_dim %d > d %d", r->rot_dim, d);
  const int half = r->rot_dim / 2;
  int64_t sum = 0;
  for (int j = 0; j < r->pos_rows; ++j) {
    APACK_CHECK(r->sections[j] >= 0, APACK_E_SHAPE, "negative section");
    sum += r->sections[j];
    if (j < 3) a->bound[j] = (int32_t)std::min<int64_t>(sum, half);
  }
  APACK_CHECK(sum == half, APACK_E_SHAPE, "the sections turn %lld pairs of %d", (long long)sum, half);
  for (int j = r->pos_rows; j < 3; ++j) a->bound[j] = half;
  APACK_CHECK(std::isfinite((float)r->factor), APACK_E_ARG, "factor is not finite in fp32");
  for (int i = 0; i < half; ++i) {
    APACK_CHECK(std::isfinite(r->freq[i]), APACK_E_ARG, "freq[%d] is not finite", i);
    a->turns[i] = r->freq[i] / kTwoPi;
  }
  a->d = d;
  a->rot = r->rot_dim;
  a->pos_rows = r->pos_rows;
  a->factor = (float)r->factor;
  a->sign = r->transpose ? -1.0f : 1.0f;
  return APACK_OK;
}

bool same_heads(const apack_heads* a, const apack_heads* b, int64_t rows) {
  return a->data == b->data && (a->heads == 1 || a->head_stride == b->head_stride) &&
         (rows <= 1 || a->row_stride == b->row_stride);
}

HeadsDev dev_heads(const apack_heads* in, const apack_heads* out) {
  return HeadsDev{in->data, out ? out->data : nullptr, in->head_stride, in->row_stride,
                  out ? out->head_stride : 0, out ? out->row_stride : 0, in->heads};
}

// Vectors of 16 bytes when the pairs, every stride and every address allow it,
// else single elements; then one workgroup per rows_per_wg rows and heads_per_wg
// heads.
apack_status run(RotaryArgs& a, const apack_rope* rope, apack_dtype dtype, bool append, hipStream_t stream) {
  const int64_t es = (int64_t)dtype_size(dtype);
  const int vec = (int)(16 / es);
  uintptr_t all = 0;
  int heads = 0;
  for (int i = 0; i < 3; ++i) {
    const HeadsDev& t = a.t[i];
    if (!t.heads) continue;
    heads += t.heads;
    all |= (uintptr_t)t.in | (uintptr_t)t.out | (uintptr_t)(t.in_head * es) | (uintptr_t)(t.in_row * es) |
           (uintptr_t)(t.out_head * es) | (uintptr_t)(t.out_row * es);
  }
  if (append) all |= (uintptr_t)(a.pages.page_stride * es) | (uintptr_t)(a.pages.row_stride * es);
  const bool wide = all % 16 == 0 && (a.rot / 2) % vec == 0 && a.d % (2 * vec) == 0;
  const int v = wide ? vec : 1;
  a.chunks = (a.d + 2 * v - 1) / (2 * v);
  a.chunk_magic = (65536 + a.chunks - 1) / a.chunks;
  a.rows_per_wg = kThreads / a.chunks;
  const int64_t blocks = (a.rows + a.rows_per_wg - 1) / a.rows_per_wg;
  APACK_CHECK(blocks < kMaxThreads / kThreads, APACK_E_UNSUPPORTED, "too many rows of %d elements for one call", a.d);
  // Heads are split over workgroups until there are 1024 of them, and to two a
  // thread where vectors of it are in flight: 94028 rows of 32 heads of 128 take 261 us
  // so, 275 with eight heads a thread; single elements take 84 us for 20000 rows with
  // all heads, 116 with two.
  const int64_t split = std::max<int64_t>(1, std::min<int64_t>(heads, 1024 / blocks));
  a.heads_per_wg = (int32_t)((heads + split - 1) / split);
  if (wide) a.heads_per_wg = std::min(a.heads_per_wg, kUnroll);
  const int gy = (heads + a.heads_per_wg - 1) / a.heads_per_wg;
  APACK_CHECK(gy < 65536, APACK_E_UNSUPPORTED, "65536 heads or more in all");
  const dim3 grid((unsigned)blocks, (unsigned)gy);
  const bool half = rope->layout == APACK_ROPE_HALF;
  if (dtype == APACK_BF16) {
    if (wide) launch<uint16_t, 8>(a, half, append, grid, stream);
    else launch<uint16_t, 1>(a, half, append, grid, stream);
  } else {
    if (wide) launch<float, 4>(a, half, append, grid, stream);
    else launch<float, 1>(a, half, append, grid, stream);
  }
  return launch_status("k_rotary");
}

}  // namespace
}  // namespace apack

using namespace apack;

extern "C" {

apack_status apack_rope_init(apack_rope* r, int32_t rot_dim, int32_t layout, double base, int32_t scaling, double s,
                             int64_t trained_len) {
  clear_error();
  APACK_CHECK(r, APACK_E_ARG, "rope is NULL");
  APACK_CHECK(rot_dim >= 2 && rot_dim <= 2 * APACK_ROPE_MAX_PAIRS && rot_dim % 2 == 0, APACK_E_SHAPE,
              "rot_dim must be even and lie in [2, %d]", 2 * APACK_ROPE_MAX_PAIRS);
  APACK_CHECK(layout == APACK_ROPE_HALF || layout == APACK_ROPE_INTERLEAVED, APACK_E_ARG, "unknown layout %d", layout);
  APACK_CHECK(scaling >= APACK_ROPE_SCALE_NONE && scaling <= APACK_ROPE_SCALE_BY_PARTS, APACK_E_ARG,
              "unknown scaling %d", scaling);
  APACK_CHECK(std::isfinite(base) && base > 1, APACK_E_ARG, "base must be finite and > 1");
  if (scaling != APACK_ROPE_SCALE_NONE)
    APACK_CHECK(std::isfinite(s) && s >= 1, APACK_E_ARG, "the scaling factor must be finite and >= 1");
  if (scaling == APACK_ROPE_SCALE_BY_PARTS)
    APACK_CHECK(trained_len >= 1, APACK_E_ARG, "trained_len must be >= 1");
  if (scaling == APACK_ROPE_SCALE_NTK) {
    APACK_CHECK(rot_dim > 2, APACK_E_SHAPE, "NTK scaling needs rot_dim > 2");
    base *= std::pow(s, (double)rot_dim / (rot_dim - 2));
    APACK_CHECK(std::isfinite(base), APACK_E_ARG, "the scaled base overflows");
  }
  std::memset(r, 0, sizeof *r);
  r->rot_dim = rot_dim;
  r->layout = layout;
  r->pos_rows = 1;
  r->sections[0] = rot_dim / 2;
  r->factor = scaling == APACK_ROPE_SCALE_BY_PARTS ? 0.1 * std::log(s) + 1 : 1.0;
  const double step = -2.0 * std::log(base) / rot_dim;
  for (int i = 0; i < rot_dim / 2; ++i) {
    double f = std::exp(i * step);
    if (scaling == APACK_ROPE_SCALE_LINEAR) f /= s;
    if (scaling == APACK_ROPE_SCALE_BY_PARTS) {
      const double turns = (double)trained_len * f / kTwoPi;
      const double g = std::min(1.0, std::max(0.0, (turns - 1) / (32 - 1)));
      f = (1 - g) * f / s + g * f;
    }
    r->freq[i] = f;
  }
  return APACK_OK;
}

apack_status apack_rotary(const apack_rope* rope, int64_t rows, const int32_t* pos, int64_t pos_stride,
                          apack_dtype dtype, int32_t d, const apack_heads* q_in, const apack_heads* q_out,
                          const apack_heads* k_in, const apack_heads* k_out, void* stream) {
  clear_error();
  APACK_CHECK(dtype_ok(dtype), APACK_E_DTYPE, "unknown dtype %d", (int)dtype);
  RotaryArgs a;
  std::memset(static_cast<void*>(&a), 0, sizeof a);
  apack_status st = check_rope(rope, d, &a);
  if (st != APACK_OK) return st;
  APACK_CHECK(rows >= 0, APACK_E_SHAPE, "rows must be >= 0");
  APACK_CHECK(rows < (int64_t(1) << 31), APACK_E_UNSUPPORTED, "rows must be < 2^31");
  APACK_CHECK(rows == 0 || pos, APACK_E_ARG, "pos is NULL");
  APACK_CHECK(rope->pos_rows == 1 || pos_stride >= rows || pos_stride == 0, APACK_E_SHAPE,
              "pos_stride must be >= rows, or 0");
  APACK_CHECK(!q_in == !q_out && !k_in == !k_out, APACK_E_ARG, "an input without its output, or the reverse");
  const size_t es = dtype_size(dtype);
  Strided ins[2], outs[2];
  const apack_heads* const in[2] = {q_in, k_in};
  const apack_heads* const out[2] = {q_out, k_out};
  static const char* const names[2][2] = {{"q_in", "q_out"}, {"k_in", "k_out"}};
  for (int i = 0; i < 2; ++i) {
    if (!in[i]) continue;
    st = check_heads(in[i], names[i][0], rows, d, es, &ins[i]);
    if (st == APACK_OK) st = check_heads(out[i], names[i][1], rows, d, es, &outs[i]);
    if (st != APACK_OK) return st;
    APACK_CHECK(in[i]->heads == out[i]->heads, APACK_E_SHAPE, "%s and %s differ in heads", names[i][0], names[i][1]);
    a.t[i] = dev_heads(in[i], out[i]);
  }
  const Strided p = rows_of_stride(rows ? pos : nullptr, 4, rope->pos_rows, pos_stride, rows);
  APACK_CHECK(p.ok, APACK_E_SHAPE, "pos of 2^46 elements or more");
  for (int i = 0; i < 2; ++i) {
    if (!out[i]) continue;
    APACK_CHECK(apart(outs[i], p), APACK_E_ALIAS, "%s overlaps pos", names[i][1]);
    for (int j = 0; j < 2; ++j) {
      if (!in[j]) continue;
      const bool own = i == j && same_heads(in[i], out[i], rows);
      APACK_CHECK(own || apart(outs[i], ins[j]), APACK_E_ALIAS, "%s overlaps %s", names[i][1], names[j][0]);
      APACK_CHECK(j <= i || apart(outs[i], outs[j]), APACK_E_ALIAS, "q_out overlaps k_out");
    }
  }
  if (rows == 0 || (!q_in && !k_in)) return APACK_OK;
  a.pos = pos;
  a.pos_stride = pos_stride;
  a.rows = rows;
  return run(a, rope, dtype, false, static_cast<hipStream_t>(stream));
}

apack_status apack_rotary_append(const apack_rope* rope, int64_t n_seq, const int32_t* pos, int64_t pos_stride,
                                 const int32_t* lens, const apack_heads* q_in, const apack_heads* q_out,
                                 const apack_heads* k, const apack_heads* v, const apack_pages* pages, void* stream) {
  clear_error();
  RotaryArgs a;
  std::memset(static_cast<void*>(&a), 0, sizeof a);
  Strided plane;
  apack_status st = check_pages(pages, "pages", &a.pages, &plane);
  if (st == APACK_OK) st = check_rope(rope, pages->d, &a);
  if (st != APACK_OK) return st;
  APACK_CHECK(pages->n_layers == 1 && pages->v && (pages->table || n_seq == 0), APACK_E_ARG,
              "pages must be one layer with v and a table");
  APACK_CHECK(n_seq >= 0, APACK_E_SHAPE, "n_seq must be >= 0");
  APACK_CHECK(n_seq < (int64_t(1) << 31), APACK_E_UNSUPPORTED, "n_seq must be < 2^31");
  APACK_CHECK(n_seq == 0 || (pos && lens), APACK_E_ARG, "pos or lens is NULL");
  APACK_CHECK(rope->pos_rows == 1 || pos_stride >= n_seq || pos_stride == 0, APACK_E_SHAPE,
              "pos_stride must be >= n_seq, or 0");
  const size_t es = dtype_size(pages->dtype);
  Strided ins[3], qo;
  const apack_heads* const in[3] = {q_in, k, v};
  static const char* const names[3] = {"q_in", "k", "v"};
  for (int i = 0; i < 3; ++i) {
    st = check_heads(in[i], names[i], n_seq, pages->d, es, &ins[i]);
    if (st != APACK_OK) return st;
  }
  st = check_heads(q_out, "q_out", n_seq, pages->d, es, &qo);
  if (st != APACK_OK) return st;
  APACK_CHECK(q_in->heads == q_out->heads && k->heads == pages->hkv && v->heads == pages->hkv, APACK_E_SHAPE,
              "heads of q_in and q_out, or of k, v and the pages, differ");
  Strided pk = plane, pv = plane;
  pk.data = pages->k[0];
  pv.data = pages->v[0];
  const Strided reads[3] = {rows_of_stride(n_seq ? pos : nullptr, 4, rope->pos_rows, pos_stride, n_seq),
                            range(lens, (size_t)n_seq * 4),
                            rows_of_stride(pages->table, 4, n_seq, pages->table_stride, pages->table_width)};
  APACK_CHECK(reads[0].ok && reads[2].ok, APACK_E_SHAPE, "pos or a table of 2^46 elements or more");
  for (const Strided& o : {qo, pk, pv}) {
    for (const Strided& r : reads) APACK_CHECK(apart(o, r), APACK_E_ALIAS, "an output overlaps pos, lens or the table");
    for (int i = 0; i < 3; ++i) {
      const bool own = i == 0 && o.data == qo.data && same_heads(q_in, q_out, n_seq);
      APACK_CHECK(own || apart(o, ins[i]), APACK_E_ALIAS, "an output overlaps %s", names[i]);
    }
  }
  APACK_CHECK(apart(pk, pv) && apart(qo, pk) && apart(qo, pv), APACK_E_ALIAS, "two outputs overlap");
  if (n_seq == 0) return APACK_OK;
  a.pos = pos;
  a.pos_stride = pos_stride;
  a.rows = n_seq;
  a.lens = lens;
  a.t[0] = dev_heads(q_in, q_out);
  for (int i = 1; i < 3; ++i) {
    a.t[i] = dev_heads(in[i], nullptr);
    a.t[i].out = i == 1 ? pages->k[0] : pages->v[0];
    a.t[i].out_head = a.pages.head_stride;
  }
  return run(a, rope, pages->dtype, true, static_cast<hipStream_t>(stream));
}

}  // extern "C"
