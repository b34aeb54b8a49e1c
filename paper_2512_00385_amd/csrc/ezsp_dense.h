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

__device__ __forceinline__ float bf16_to_f32(__bf16 v) { return (float)v; }

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
// In fp32.  A NaN stays a NaN in each; silu(-inf) is NaN as its formula gives.
__device__ __forceinline__ float sigmoid_f(float z) {
  return __builtin_amdgcn_rcpf(1.0f + expf(-z));
}
__device__ __forceinline__ float normal_cdf_f(float z) {
  // 0.5 erfc keeps the relative precision of the lower tail
  return 0.5f * erfcf(-0.70710678f * z);
}
__device__ __forceinline__ float act_f(float z, int act) {
  switch (act) {
    case EZSP_ACT_RELU: return z < 0.0f ? 0.0f : z;
    case EZSP_ACT_GELU: return z * normal_cdf_f(z);
    case EZSP_ACT_SILU: return z * sigmoid_f(z);
    default: return z;
  }
}
// act'(z); ReLU's derivative at 0 is 0
__device__ __forceinline__ float act_grad_f(float z, int act) {
  switch (act) {
    case EZSP_ACT_RELU: return z > 0.0f ? 1.0f : 0.0f;
    case EZSP_ACT_GELU:
      return normal_cdf_f(z) + z * 0.39894228f * expf(-0.5f * z * z);
    case EZSP_ACT_SILU: {
      const float s = sigmoid_f(z);
      return s * (1.0f + z * (1.0f - s));
    }
    default: return 1.0f;
  }
}
__device__ __forceinline__ f32x8_t act8(f32x8_t z, int act) {
  if (act != EZSP_ACT_NONE) {
#pragma unroll
    for (int i = 0; i < kVec; ++i) z[i] = act_f(z[i], act);
  }
  return z;
}
__device__ __forceinline__ f32x8_t act_grad8(f32x8_t z, int act) {
#pragma unroll
  for (int i = 0; i < kVec; ++i) z[i] = act_grad_f(z[i], act);
  return z;
}

inline size_t type_bytes(int type) { return type == EZSP_TYPE_BF16 ? 2 : 4; }

// Sums partial rows: out[j] = sum over p of part[p * len + j] for j < len,
// in the order of p.  The finish of every reduction over rows that blocks
// share (gradients of weights and biases): no atomics, so results do not
// depend on the order in which blocks run.
void join_rows(const float *part, int32_t n_part, int32_t len, float *out0,
               float *out1, int32_t split, hipStream_t st);

}  // namespace ezsp
