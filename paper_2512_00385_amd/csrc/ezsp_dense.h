// ezsp_dense.h -- what the dense operators of a point-embedding network
// (layer norm, product with epilogue, gated feed-forward) share: element
// types, vector accesses at any alignment, activations and their derivatives.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include "../../include/ezsp.h"
#include "ezsp_internal.h"

namespace ezsp {

typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x16_t __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// The same vectors at the alignment of their elements: gfx950 takes 16-byte
// global accesses at any address, so a row of odd length costs no scalar
// loads (only its last, incomplete vector does).
typedef bf16x8_t bf16x8_u __attribute__((aligned(2)));
typedef f32x8_t f32x8_u __attribute__((aligned(4)));
typedef u32x4_t u32x4_u2 __attribute__((aligned(2)));
typedef u32x4_t u32x4_u4 __attribute__((aligned(4)));

constexpr int kVec = 8;  // elements a lane takes at once

// cnt elements (at most kVec) from p on as fp32, the rest 0
__device__ __forceinline__ f32x8_t load8(const __bf16 *p, int cnt) {
  f32x8_t r = {0, 0, 0, 0, 0, 0, 0, 0};
  if (cnt >= kVec) {
    r = __builtin_convertvector(*reinterpret_cast<const bf16x8_u *>(p),
                                f32x8_t);
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (i < cnt) r[i] = (float)p[i];
  }
  return r;
}
__device__ __forceinline__ f32x8_t load8(const float *p, int cnt) {
  f32x8_t r = {0, 0, 0, 0, 0, 0, 0, 0};
  if (cnt >= kVec) {
    r = *reinterpret_cast<const f32x8_u *>(p);
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (i < cnt) r[i] = p[i];
  }
  return r;
}

// the first cnt of v to p, rounded to nearest even for bfloat16 (the one
// rounding of a result that was held in fp32 until here)
__device__ __forceinline__ void store8(__bf16 *p, f32x8_t v, int cnt) {
  const bf16x8_t b = __builtin_convertvector(v, bf16x8_t);
  if (cnt >= kVec) {
    *reinterpret_cast<bf16x8_u *>(p) = b;
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (i < cnt) p[i] = b[i];
  }
}
__device__ __forceinline__ void store8(float *p, f32x8_t v, int cnt) {
  if (cnt >= kVec) {
    *reinterpret_cast<f32x8_u *>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < kVec; ++i)
      if (i < cnt) p[i] = v[i];
  }
}

// A lane's kVec columns from col on, of rows of d values.  They are loaded
// without a branch, as they lie in memory: columns of an incomplete last
// vector by way of the vector that ends with the row, rows past the end as
// the last one.  settle() then shifts them into place and zeroes what does
// not exist.  Rows shorter than a vector are loaded together with what
// follows them, the table's last ones with what precedes them.
template <int V>
struct SpanOf {
  int32_t at;   // column that the load starts at
  int32_t cnt;  // columns that exist
  int32_t off;  // first of them in the load
  bool thin;    // d < V
};
typedef SpanOf<kVec> Span;
template <int V = kVec>
__device__ __forceinline__ SpanOf<V> span_of(int32_t col, int32_t d) {
  SpanOf<V> s;
  s.cnt = min(max(d - col, 0), V);
  s.at = min(col, max(d - V, 0));
  s.off = col - s.at;
  s.thin = d < V;
  return s;
}
// rows [n] of the table and their distance; n * d >= V
template <int V>
__device__ __forceinline__ int64_t span_at(int64_t row, int64_t ld, int32_t n,
                                           int32_t d, SpanOf<V> s, int32_t &back) {
  const int64_t at = min(row, (int64_t)n - 1) * ld + s.at;
  back = 0;
  if (s.thin) {
    const int64_t last = (int64_t)(n - 1) * ld + d - V;
    if (at > last) back = (int32_t)(at - last);
  }
  return at - back;
}
template <class T>
struct Vec8;  // kVec values in registers
template <>
struct Vec8<__bf16> {
  u32x4_t v;
};
template <>
struct Vec8<float> {
  f32x8_t v;
};
__device__ __forceinline__ Vec8<__bf16> raw8(const __bf16 *p) {
  return {*reinterpret_cast<const u32x4_u2 *>(p)};
}
__device__ __forceinline__ Vec8<float> raw8(const float *p) {
  return {*reinterpret_cast<const f32x8_u *>(p)};
}
// The same from load8, for tables of less than a vector.
__device__ __forceinline__ Vec8<__bf16> raw_of(f32x8_t v, const __bf16 *) {
  return {__builtin_bit_cast(u32x4_t, __builtin_convertvector(v, bf16x8_t))};
}
__device__ __forceinline__ Vec8<float> raw_of(f32x8_t v, const float *) {
  return {v};
}
__device__ __forceinline__ bf16x8_t settle(Vec8<__bf16> r, int32_t off,
                                           int32_t cnt) {
  if (off) {
    uint64_t lo = ((uint64_t)r.v[1] << 32) | r.v[0];
    uint64_t hi = ((uint64_t)r.v[3] << 32) | r.v[2];
    const int bits = 16 * off;  // those of 8 and more are zeroed below
    lo = bits >= 64 ? hi >> (bits & 63)
                    : (lo >> bits) | (hi << ((64 - bits) & 63));
    hi = bits >= 64 ? 0 : hi >> bits;
    r.v = u32x4_t{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi,
                  (uint32_t)(hi >> 32)};
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    r.v[i] = cnt > 2 * i + 1 ? r.v[i] : cnt > 2 * i ? r.v[i] & 0xffffu : 0u;
  return __builtin_bit_cast(bf16x8_t, r.v);
}
__device__ __forceinline__ f32x8_t settle(Vec8<float> r, int32_t off,
                                          int32_t cnt) {
  if (off) {
#pragma unroll
    for (int step = 4; step > 0; step >>= 1)
      if (off & step) {
#pragma unroll
        for (int i = 0; i < kVec; ++i)
          r.v[i] = i + step < kVec ? r.v[i + step] : 0.0f;
      }
  }
#pragma unroll
  for (int i = 0; i < kVec; ++i) r.v[i] = i < cnt ? r.v[i] : 0.0f;
  return r.v;
}

// Accesses whose element type is known at run time only (uniform branches).
__device__ __forceinline__ f32x8_t load8_t(const void *p, int64_t at, int type,
                                           int cnt) {
  return type == EZSP_TYPE_BF16
             ? load8(static_cast<const __bf16 *>(p) + at, cnt)
             : load8(static_cast<const float *>(p) + at, cnt);
}
__device__ __forceinline__ void store8_t(void *p, int64_t at, int type,
                                         f32x8_t v, int cnt) {
  if (type == EZSP_TYPE_BF16)
    store8(static_cast<__bf16 *>(p) + at, v, cnt);
  else
    store8(static_cast<float *>(p) + at, v, cnt);
}

// --- activations ------------------------------------------------------------
// In fp32, from the hardware's 2^x and reciprocal (one ulp each): errors of a
// few 2^-24 (1 + |z|), where the library's expf and erfcf take five times the
// instructions, 34 us of a 256 x 256 tile's epilogue.  A NaN stays a NaN;
// silu(-inf) and gelu(-inf) are NaN as their formulas give.
__device__ __forceinline__ float exp_f(float x) {
  return __builtin_amdgcn_exp2f(1.44269504f * x);
}
__device__ __forceinline__ float sigmoid_f(float z) {
  return __builtin_amdgcn_rcpf(1.0f + exp_f(-z));
}
// The normal distribution function, in two forms; gauss gets exp(-z^2 / 2).
// For bfloat16 results, Hastings' rational approximation of erfc (Abramowitz
// and Stegun 7.1.26):
//   erfc(x) = (a1 t + ... + a5 t^5) exp(-x^2), t = 1 / (1 + p x), x >= 0,
// with x = |z| / sqrt(2).  gelu is within 1.7 2^-24 (1 + |z|), its derivative
// within 4.8; relative to itself gelu is off by 5e-4 at -4 and by 4e-3, half
// an ulp of bfloat16, at -6, where it is 6e-9.
__device__ __forceinline__ float normal_cdf_f(float z, float &gauss) {
  const float x = 0.70710678f * fabsf(z);
  const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f, x, 1.0f));
  gauss = exp_f(-0.5f * z * z);
  float q = __builtin_fmaf(1.061405429f, t, -1.453152027f);
  q = __builtin_fmaf(q, t, 1.421413741f);
  q = __builtin_fmaf(q, t, -0.284496736f);
  q = __builtin_fmaf(q, t, 0.254829592f);
  const float tail = 0.5f * q * t * gauss;  // of the side away from 0
  return z < 0.0f ? tail : 1.0f - tail;
}
// For fp32 results,
//   Phi(-|z|) = exp(-z^2 / 2) t Q(1 - t),  t = 1 / (1 + 0.3 |z| / sqrt(2)),
// Q of degree 8 with Q(0) = 1/2, fitted here to the least largest relative
// error (2.3e-8 up to |z| = 17, where Phi underflows).  1 - t is formed as
// 0.3 |z| / sqrt(2) t, which is as accurate at 0 as z, so that Phi(0) loses
// nothing to it.  gelu is within 1.2 2^-24 (1 + |z|), its derivative within
// 3, the negative tail within 5 2^-24 (1 + z^2) of itself.  (With it for
// bfloat16 too: 16,384 x 4096 -> 4096 553 us for 527, the narrow gated
// backward of 1,265,474 rows 317 for 293.)
__device__ __forceinline__ float normal_cdf_fine_f(float z, float &gauss) {
  // (from 4 on, |z| = 18.9, gauss is 0; an infinite z gives no 0 inf)
  const float x = fminf(0.21213203f * fabsf(z), 4.0f);
  const float t = __builtin_amdgcn_rcpf(1.0f + x);
  const float m = x * t;
  gauss = exp_f(-0.5f * z * z);
  float q = __builtin_fmaf(-0.064491205f, m, 0.2744203f);
  q = __builtin_fmaf(q, m, -0.36878094f);
  q = __builtin_fmaf(q, m, -0.20966952f);
  q = __builtin_fmaf(q, m, 1.4443028f);
  q = __builtin_fmaf(q, m, -2.4047801f);
  q = __builtin_fmaf(q, m, 2.2942245f);
  q = __builtin_fmaf(q, m, -1.3806305f);
  q = __builtin_fmaf(q, m, 0.5f);
  const float tail = q * t * gauss;
  return z < 0.0f ? tail : 1.0f - tail;
}
// GELU's code in the kernels, by the type of what it is rounded to.
constexpr int32_t kGeluFine = EZSP_ACT_SILU + 1;
inline int32_t act_for(int32_t act, int32_t type) {
  return act == EZSP_ACT_GELU && type == EZSP_TYPE_F32 ? kGeluFine : act;
}
// value and derivative; ReLU's derivative at 0 is 0
__device__ __forceinline__ void relu_f(float z, float &v, float &dv) {
  v = z < 0.0f ? 0.0f : z;
  dv = z > 0.0f ? 1.0f : 0.0f;
}
__device__ __forceinline__ void gelu_f(float z, float &v, float &dv) {
  float gauss;
  const float cdf = normal_cdf_f(z, gauss);
  v = z * cdf;
  dv = __builtin_fmaf(0.39894228f * z, gauss, cdf);
}
__device__ __forceinline__ void gelu_fine_f(float z, float &v, float &dv) {
  float gauss;
  const float cdf = normal_cdf_fine_f(z, gauss);
  v = z * cdf;
  dv = __builtin_fmaf(0.39894228f * z, gauss, cdf);
}
__device__ __forceinline__ void silu_f(float z, float &v, float &dv) {
  const float s = sigmoid_f(z);
  v = z * s;
  dv = s * __builtin_fmaf(z, 1.0f - s, 1.0f);
}
// of eight elements, the branch on the activation taken once
__device__ __forceinline__ void act_both8(f32x8_t z, int act, f32x8_t &v,
                                          f32x8_t &dv) {
#define EZSP_EACH(F)                                  \
  do {                                                \
    _Pragma("unroll") for (int i = 0; i < kVec; ++i) { \
      float a, b;                                     \
      F(z[i], a, b);                                  \
      v[i] = a;                                       \
      dv[i] = b;                                      \
    }                                                 \
  } while (0)
  if (act == EZSP_ACT_SILU)
    EZSP_EACH(silu_f);
  else if (act == EZSP_ACT_GELU)
    EZSP_EACH(gelu_f);
  else if (act == kGeluFine)
    EZSP_EACH(gelu_fine_f);
  else if (act == EZSP_ACT_RELU)
    EZSP_EACH(relu_f);
  else {
    v = z;
    dv = f32x8_t(1.0f);
  }
#undef EZSP_EACH
}
__device__ __forceinline__ f32x8_t act8(f32x8_t z, int act) {
  f32x8_t v, dv;
  act_both8(z, act, v, dv);
  return v;
}
__device__ __forceinline__ f32x8_t act_grad8(f32x8_t z, int act) {
  f32x8_t v, dv;
  act_both8(z, act, v, dv);
  return dv;
}

inline size_t type_bytes(int type) { return type == EZSP_TYPE_BF16 ? 2 : 4; }

// Sums partial rows: out[j] = sum over p of part[p * len + j] for j < len,
// in the order of p.  The finish of every reduction over rows that blocks
// share (gradients of weights and biases): no atomics, so results do not
// depend on the order in which blocks run.
void join_rows(const float *part, int32_t n_part, int32_t len, float *out0,
               float *out1, int32_t split, hipStream_t st);

}  // namespace ezsp
