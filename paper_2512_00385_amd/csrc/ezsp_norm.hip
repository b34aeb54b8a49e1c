// ezsp_norm.hip -- layer norm over the rows of a matrix, forward and
// backward.
//
//   forward   mean = sum(x) / d, var = sum((x - mean)^2) / d,
//             y = (x - mean) / sqrt(var + eps) * w + b
//   backward  xh = (x - mean) rstd, g = dy w,
//             dx = (g - sum(g)/d - xh sum(g xh)/d) rstd (+ dres),
//             dw = sum over rows of dy xh, db = sum over rows of dy
//
// Both are bound by memory: every element is read once and written once, and
// a row stays in registers between its statistics and its result, so the
// variance is the centred one at no second read.  A row is held by a group of
// G lanes, kVec elements a lane and step, so that short rows share a wave and
// long ones take a block.
#include <algorithm>

#include "ezsp_dense.h"

namespace ezsp {

namespace {

constexpr int kNormNT = 256;
constexpr int64_t kNormGrid = (int64_t)1 << 22;  // blocks of a launch

// Sum over the G lanes of a group, in each of them (G = kNormNT: a block;
// red is LDS of 2 * kNormNT / kWave floats, used in turn).
template <int G>
__device__ __forceinline__ float group_sum(float v, float *red) {
#pragma unroll
  for (int off = (G < kWave ? G : kWave) / 2; off > 0; off >>= 1)
    v += __shfl_xor(v, off, kWave);
  if constexpr (G > kWave) {
    constexpr int kW = G / kWave;
    __syncthreads();  // the sum before this one has been read
    if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = v;
    __syncthreads();
    v = 0.0f;
#pragma unroll
    for (int w = 0; w < kW; ++w) v += red[w];
  }
  return v;
}

template <class TX, class TY, int G, int NV>
__global__ __launch_bounds__(kNormNT) void k_norm_fwd(
    const TX *x, int64_t ldx, int64_t n, int32_t d,
    const float *__restrict__ w, const float *__restrict__ b, float eps,
    TY *y, int64_t ldy, float *__restrict__ mean_out,
    float *__restrict__ rstd_out) {
  __shared__ float red[kNormNT / kWave];
  const int gl = threadIdx.x % G;
  for (int64_t r0 = (int64_t)blockIdx.x * (kNormNT / G); r0 < n;
       r0 += (int64_t)gridDim.x * (kNormNT / G)) {
    const int64_t row = r0 + threadIdx.x / G;
    const bool live = row < n;
    const TX *xr = x + (live ? row : 0) * ldx;
    f32x8_t v[NV];
    float s = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (gl + G * j) * kVec;
      v[j] = load8(xr + c, live ? d - c : 0);
#pragma unroll
      for (int i = 0; i < kVec; ++i) s += v[j][i];
    }
    const float inv_d = 1.0f / (float)d;
    const float mean = group_sum<G>(s, red) * inv_d;
    float q = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (gl + G * j) * kVec;
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float t = v[j][i] - mean;
        q += c + i < d ? t * t : 0.0f;
      }
    }
    const float rstd = 1.0f / sqrtf(group_sum<G>(q, red) * inv_d + eps);
    if (!live) continue;
    TY *yr = y + row * ldy;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (gl + G * j) * kVec;
      if (c >= d) break;
      f32x8_t o;
      const f32x8_t wv = w ? load8(w + c, d - c) : f32x8_t(1.0f);
      const f32x8_t bv = b ? load8(b + c, d - c) : f32x8_t(0.0f);
#pragma unroll
      for (int i = 0; i < kVec; ++i)
        o[i] = (v[j][i] - mean) * rstd * wv[i] + bv[i];
      store8(yr + c, o, d - c);
    }
    if (gl == 0) {
      if (mean_out) mean_out[row] = mean;
      if (rstd_out) rstd_out[row] = rstd;
    }
  }
}

// Rows gridDim.x * (kNormNT / G) apart; the column sums of a lane's rows stay
// in its registers and are joined over the block's groups at the end:
// part[block][0 .. d) for dw, [d .. 2d) for db.
template <class TX, class TY, int G, int NV>
__global__ __launch_bounds__(kNormNT) void k_norm_bwd(
    const TY *__restrict__ dy, int64_t lddy, const TX *__restrict__ x,
    int64_t ldx, int64_t n, int32_t d, const float *__restrict__ w,
    const float *__restrict__ mean_in, const float *__restrict__ rstd_in,
    const TX *dres, int64_t lddres, TX *dx, int64_t lddx,
    float *__restrict__ part) {
  constexpr int kRows = kNormNT / G;
  constexpr int kSpan = G * NV * kVec;  // columns of a group
  __shared__ float red[kNormNT / kWave];
  __shared__ float sums[G > kWave ? 1 : 2 * kSpan];
  const int gl = threadIdx.x % G;
  const float inv_d = 1.0f / (float)d;
  f32x8_t aw[NV], ab[NV], wv[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (gl + G * j) * kVec;
    aw[j] = ab[j] = f32x8_t(0.0f);
    wv[j] = w ? load8(w + c, d - c) : f32x8_t(1.0f);
  }
  // every lane of a block takes the same number of steps (the group sums of
  // a block-wide group hold barriers); rows past the end count as 0
  for (int64_t r0 = (int64_t)blockIdx.x * kRows; r0 < n;
       r0 += (int64_t)gridDim.x * kRows) {
    const int64_t row = r0 + threadIdx.x / G;
    const bool live = row < n;
    const int64_t at = live ? row : 0;
    const float mean = live ? mean_in[at] : 0.0f;
    const float rstd = live ? rstd_in[at] : 0.0f;
    f32x8_t xh[NV], gv[NV];
    float s1 = 0.0f, s2 = 0.0f;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (gl + G * j) * kVec;
      const int cnt = live ? d - c : 0;
      xh[j] = load8(x + at * ldx + c, cnt);
      gv[j] = load8(dy + at * lddy + c, cnt);
    }
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (gl + G * j) * kVec;
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float h = live && c + i < d ? (xh[j][i] - mean) * rstd : 0.0f;
        xh[j][i] = h;
        aw[j][i] += gv[j][i] * h;
        ab[j][i] += gv[j][i];
        const float g = gv[j][i] * wv[j][i];
        gv[j][i] = g;
        s1 += g;
        s2 += g * h;
      }
    }
    if (dx) {
      const float m1 = group_sum<G>(s1, red) * inv_d;
      const float m2 = group_sum<G>(s2, red) * inv_d;
      if (live) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          const int c = (gl + G * j) * kVec;
          if (c >= d) break;
          f32x8_t o = dres ? load8(dres + at * lddres + c, d - c)
                           : f32x8_t(0.0f);
#pragma unroll
          for (int i = 0; i < kVec; ++i)
            o[i] += (gv[j][i] - m1 - xh[j][i] * m2) * rstd;
          store8(dx + at * lddx + c, o, d - c);
        }
      }
    }
  }
  if (!part) return;
  float *pw = part + (int64_t)blockIdx.x * 2 * d;
  if constexpr (G > kWave) {  // one group: its lanes hold the block's sums
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (gl + G * j) * kVec;
      store8(pw + c, aw[j], d - c);
      store8(pw + d + c, ab[j], d - c);
    }
  } else {
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < kVec; ++i)
#pragma unroll
        for (int off = G; off < kWave; off <<= 1) {
          aw[j][i] += __shfl_xor(aw[j][i], off, kWave);
          ab[j][i] += __shfl_xor(ab[j][i], off, kWave);
        }
    // the waves add to the block's sums in turn
    const int wave = threadIdx.x / kWave;
    for (int t = 0; t < kNormNT / kWave; ++t) {
      if (wave == t && threadIdx.x % kWave < G) {
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int i = 0; i < kVec; ++i) {
            const int c = (gl + G * j) * kVec + i;
            sums[c] = (t ? sums[c] : 0.0f) + aw[j][i];
            sums[kSpan + c] = (t ? sums[kSpan + c] : 0.0f) + ab[j][i];
          }
      }
      __syncthreads();
    }
    for (int c = threadIdx.x; c < d; c += kNormNT) {
      pw[c] = sums[c];
      pw[d + c] = sums[kSpan + c];
    }
  }
}

constexpr int kJoinCols = 64;
constexpr int kJoinNT = 1024;

__global__ __launch_bounds__(kJoinNT) void k_join_rows(
    const float *__restrict__ part, int32_t n_part, int32_t len,
    float *__restrict__ out0, float *__restrict__ out1, int32_t split) {
  constexpr int kSlices = kJoinNT / kJoinCols;
  __shared__ float sl[kSlices][kJoinCols];
  const int c = threadIdx.x % kJoinCols, s = threadIdx.x / kJoinCols;
  const int32_t col = (int32_t)blockIdx.x * kJoinCols + c;
  float v = 0.0f;
  if (col < len) {
#pragma unroll 8
    for (int32_t p = s; p < n_part; p += kSlices)
      v += part[(int64_t)p * len + col];
  }
  sl[s][c] = v;
  __syncthreads();
  if (s == 0 && col < len) {
    v = 0.0f;
#pragma unroll
    for (int t = 0; t < kSlices; ++t) v += sl[t][c];
    if (col < split) {
      if (out0) out0[col] = v;
    } else {
      if (out1) out1[col - split] = v;
    }
  }
}

// Blocks of the backward pass: enough to fill the chip, few enough that the
// partial sums (8 d bytes a block) stay small next to the rows.
int32_t bwd_blocks(int64_t n, int rows_per_block) {
  return (int32_t)std::min<int64_t>((n + rows_per_block - 1) / rows_per_block,
                                    kNormParts);
}

template <class TX, class TY, int G, int NV>
void fwd(const NormArgs &a, hipStream_t st) {
  const int64_t rows = kNormNT / G;
  hipLaunchKernelGGL((k_norm_fwd<TX, TY, G, NV>),
                     dim3((unsigned)std::min<int64_t>(
                         (a.n + rows - 1) / rows, kNormGrid)),
                     dim3(kNormNT), 0, st, static_cast<const TX *>(a.x), a.ldx, a.n, a.d, a.w,
                     a.b, (float)a.eps, static_cast<TY *>(a.y), a.ldy, a.mean,
                     a.rstd);
}

template <class TX, class TY, int G, int NV>
void bwd(const NormArgs &a, hipStream_t st) {
  const int32_t blocks = bwd_blocks(a.n, kNormNT / G);
  const bool sums = a.dw || a.db;
  hipLaunchKernelGGL((k_norm_bwd<TX, TY, G, NV>), dim3((unsigned)blocks),
                     dim3(kNormNT), 0, st, static_cast<const TY *>(a.dy),
                     a.lddy, static_cast<const TX *>(a.x), a.ldx, a.n, a.d,
                     a.w, a.mean, a.rstd, static_cast<const TX *>(a.dres),
                     a.lddres, static_cast<TX *>(a.dx), a.lddx,
                     sums ? a.part : nullptr);
  if (sums)
    join_rows(a.part, blocks, 2 * a.d, a.dw, a.db, a.d, st);
}

// The group of a row: the smallest that holds it at one vector a lane, up to
// a wave of four vectors a lane, then a block.
template <class TX, class TY, bool BWD>
void dispatch(const NormArgs &a, hipStream_t st) {
  const int32_t chunks = (a.d + kVec - 1) / kVec;
#define EZSP_NORM(G, NV)            \
  do {                              \
    if constexpr (BWD)              \
      bwd<TX, TY, G, NV>(a, st);    \
    else                            \
      fwd<TX, TY, G, NV>(a, st);    \
    return;                         \
  } while (0)
  if (chunks <= 1) EZSP_NORM(1, 1);
  if (chunks <= 2) EZSP_NORM(2, 1);
  if (chunks <= 4) EZSP_NORM(4, 1);
  if (chunks <= 8) EZSP_NORM(8, 1);
  if (chunks <= 16) EZSP_NORM(16, 1);
  if (chunks <= 32) EZSP_NORM(32, 1);
  if (chunks <= 64) EZSP_NORM(64, 1);
  if (chunks <= 128) EZSP_NORM(64, 2);
  if (chunks <= 256) EZSP_NORM(64, 4);
  if (chunks <= 512) EZSP_NORM(256, 2);
  if (chunks <= 1024) EZSP_NORM(256, 4);
  EZSP_NORM(256, 8);
#undef EZSP_NORM
}

template <bool BWD>
int run(const NormArgs &a, hipStream_t st) {
  const bool xb = a.type_x == EZSP_TYPE_BF16, yb = a.type_y == EZSP_TYPE_BF16;
  prof_begin("layer_norm", st);
  if (xb && yb)
    dispatch<__bf16, __bf16, BWD>(a, st);
  else if (xb)
    dispatch<__bf16, float, BWD>(a, st);
  else if (yb)
    dispatch<float, __bf16, BWD>(a, st);
  else
    dispatch<float, float, BWD>(a, st);
  prof_end(st);
  const int rc = check_hip(hipGetLastError(), "layer norm launch");
  const double ex = (double)type_bytes(a.type_x),
               ey = (double)type_bytes(a.type_y);
  prof_bytes("layer_norm",
             (double)a.n * a.d *
                 (BWD ? ey + ex + (a.dx ? ex : 0.0) + (a.dres ? ex : 0.0)
                      : ex + ey));
  return rc;
}

}  // namespace

void join_rows(const float *part, int32_t n_part, int32_t len, float *out0,
               float *out1, int32_t split, hipStream_t st) {
  hipLaunchKernelGGL(k_join_rows,
                     dim3((unsigned)((len + kJoinCols - 1) / kJoinCols)),
                     dim3(kJoinNT), 0, st, part, n_part, len, out0, out1,
                     split);
}

int norm_fwd_run(const NormArgs &a, hipStream_t st) {
  return run<false>(a, st);
}

int norm_bwd_run(const NormArgs &a, hipStream_t st) {
  return run<true>(a, st);
}

}  // namespace ezsp
