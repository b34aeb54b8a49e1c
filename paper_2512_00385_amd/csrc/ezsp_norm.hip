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

// Threads of a block whose groups have G lanes.
constexpr int norm_nt(int G) { return G > kNormNT ? G : kNormNT; }

// Sums of N values over the G lanes of a group, in each of them.  A group
// wider than a wave is the block; red is LDS of N * G / kWave floats then.
template <int G, int N>
__device__ __forceinline__ void group_sum(float (&v)[N], float *red) {
#pragma unroll
  for (int off = (G < kWave ? G : kWave) / 2; off > 0; off >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += __shfl_xor(v[i], off, kWave);
  if constexpr (G > kWave) {
    constexpr int kW = G / kWave;
    __syncthreads();  // the sums before these have been read
    if (threadIdx.x % kWave == 0)
#pragma unroll
      for (int i = 0; i < N; ++i) red[i * kW + threadIdx.x / kWave] = v[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
      v[i] = 0.0f;
#pragma unroll
      for (int w = 0; w < kW; ++w) v[i] += red[i * kW + w];
    }
  }
}

template <class TX, class TY, int G, int NV>
__global__ __launch_bounds__(norm_nt(G)) void k_norm_fwd(
    const TX *x, int64_t ldx, int64_t n, int32_t d,
    const float *__restrict__ w, const float *__restrict__ b, float eps,
    TY *y, int64_t ldy, float *__restrict__ mean_out,
    float *__restrict__ rstd_out) {
  constexpr int kRows = norm_nt(G) / G;
  __shared__ float red[norm_nt(G) / kWave];
  const int gl = threadIdx.x % G;
  for (int64_t r0 = (int64_t)blockIdx.x * kRows; r0 < n;
       r0 += (int64_t)gridDim.x * kRows) {
    const int64_t row = r0 + threadIdx.x / G;
    const bool live = row < n;
    const TX *xr = x + (live ? row : 0) * ldx;
    f32x8_t v[NV];
    float s[1] = {0.0f}, q[1] = {0.0f};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (gl + G * j) * kVec;
      v[j] = load8(xr + c, live ? d - c : 0);
#pragma unroll
      for (int i = 0; i < kVec; ++i) s[0] += v[j][i];
    }
    const float inv_d = 1.0f / (float)d;
    group_sum<G>(s, red);
    const float mean = s[0] * inv_d;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (gl + G * j) * kVec;
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float t = v[j][i] - mean;
        q[0] += c + i < d ? t * t : 0.0f;
      }
    }
    group_sum<G>(q, red);
    const float rstd = 1.0f / sqrtf(q[0] * inv_d + eps);
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
// part_w and part_b are 2 d from block to block, or the results themselves
// where one block takes all rows.  A row's x and dy are
// replaced by the next row's as soon as they have been read, its dres at its
// end, so that a row's loads have a row's time to arrive (16,384 rows of 2048
// bfloat16 values with dres: 85 us without, 60 with).
template <class TX, class TY, int G, int NV>
__global__ __launch_bounds__(norm_nt(G)) void k_norm_bwd(
    const TY *__restrict__ dy, int64_t lddy, const TX *__restrict__ x,
    int64_t ldx, int32_t n, int32_t d, const float *__restrict__ w,
    const float *__restrict__ mean_in, const float *__restrict__ rstd_in,
    const TX *dres, int64_t lddres, TX *dx, int64_t lddx,
    float *__restrict__ part_w, float *__restrict__ part_b) {
  constexpr int kRows = norm_nt(G) / G;
  constexpr int kSpan = G * NV * kVec;  // columns of a group
  __shared__ float red[2 * norm_nt(G) / kWave];
  __shared__ float sums[G > kWave ? 1 : 2 * kSpan];
  const int gl = threadIdx.x % G;
  const float inv_d = 1.0f / (float)d;
  Span sp[NV];
  f32x8_t aw[NV], ab[NV], wv[NV];
#pragma unroll
  for (int j = 0; j < NV; ++j) {
    const int c = (gl + G * j) * kVec;
    sp[j] = span_of(c, d);
    if (n < kVec) sp[j].thin = false;
    aw[j] = ab[j] = f32x8_t(0.0f);
    wv[j] = w ? load8(w + c, d - c) : f32x8_t(1.0f);
  }
  Vec8<TX> rx[NV], rr[NV];
  Vec8<TY> ry[NV];
  float mean, rstd;
  // (a table of less than a vector has no place for raw8)
  const bool tiny = d < kVec && n < kVec;
  auto load = [&](int64_t row) {
    int32_t back;
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      if (tiny) {
        const int64_t at = min(row, (int64_t)n - 1);
        rx[j] = raw_of(load8(x + at * ldx, gl ? 0 : d), x);
        ry[j] = raw_of(load8(dy + at * lddy, gl ? 0 : d), dy);
        continue;
      }
      rx[j] = raw8(x + span_at(row, ldx, n, d, sp[j], back));
      ry[j] = raw8(dy + span_at(row, lddy, n, d, sp[j], back));
    }
    const int64_t at = min(row, (int64_t)n - 1);
    mean = mean_in[at];
    rstd = rstd_in[at];
  };
  auto load_res = [&](int64_t row) {
    int32_t back;
#pragma unroll
    for (int j = 0; j < NV; ++j)
      rr[j] = tiny ? raw_of(load8(dres + min(row, (int64_t)n - 1) * lddres,
                                  gl ? 0 : d),
                            dres)
                   : raw8(dres + span_at(row, lddres, n, d, sp[j], back));
  };
  // every lane of a block takes the same number of steps (the group sums of
  // a block-wide group hold barriers); rows past the end count as 0
  const int64_t stride = (int64_t)gridDim.x * kRows;
  const int64_t first = (int64_t)blockIdx.x * kRows + threadIdx.x / G;
  load(first);
  if (dres) load_res(first);
  for (int64_t r0 = (int64_t)blockIdx.x * kRows; r0 < n; r0 += stride) {
    const int64_t row = r0 + threadIdx.x / G;
    const bool live = row < n;
    const float rs = rstd;
    f32x8_t xh[NV], gv[NV];
    float s[2] = {0.0f, 0.0f};  // of g and of g xh
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int32_t cnt = live ? sp[j].cnt : 0;
      int32_t back;
      span_at(row, ldx, n, d, sp[j], back);
      xh[j] = __builtin_convertvector(settle(rx[j], sp[j].off + back, cnt),
                                      f32x8_t);
      span_at(row, lddy, n, d, sp[j], back);
      gv[j] = __builtin_convertvector(settle(ry[j], sp[j].off + back, cnt),
                                      f32x8_t);
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float h = i < cnt ? (xh[j][i] - mean) * rs : 0.0f;
        xh[j][i] = h;
        aw[j][i] = __builtin_fmaf(gv[j][i], h, aw[j][i]);
        ab[j][i] += gv[j][i];
        const float g = gv[j][i] * wv[j][i];
        gv[j][i] = g;
        s[0] += g;
        s[1] = __builtin_fmaf(g, h, s[1]);
      }
    }
    if (r0 + stride < n) load(row + stride);
    if (dx) {
      group_sum<G>(s, red);
      const float m1 = s[0] * inv_d, m2 = s[1] * inv_d;
      if (live) {
#pragma unroll
        for (int j = 0; j < NV; ++j) {
          if (sp[j].cnt <= 0) break;
          f32x8_t o = f32x8_t(0.0f);
          if (dres) {
            int32_t back;
            span_at(row, lddres, n, d, sp[j], back);
            o = __builtin_convertvector(
                settle(rr[j], sp[j].off + back, sp[j].cnt), f32x8_t);
          }
#pragma unroll
          for (int i = 0; i < kVec; ++i)
            o[i] = __builtin_fmaf(
                gv[j][i] - __builtin_fmaf(xh[j][i], m2, m1), rs, o[i]);
          store8(dx + row * lddx + (gl + G * j) * kVec, o, sp[j].cnt);
        }
      }
      if (dres && r0 + stride < n) load_res(row + stride);
    }
  }
  if (!part_w && !part_b) return;
  float *pw = part_w ? part_w + (int64_t)blockIdx.x * 2 * d : nullptr;
  float *pb = part_b ? part_b + (int64_t)blockIdx.x * 2 * d : nullptr;
  if constexpr (G > kWave) {  // one group: its lanes hold the block's sums
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (gl + G * j) * kVec;
      if (pw) store8(pw + c, aw[j], d - c);
      if (pb) store8(pb + c, ab[j], d - c);
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
    for (int t = 0; t < norm_nt(G) / kWave; ++t) {
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
    for (int c = threadIdx.x; c < d; c += norm_nt(G)) {
      if (pw) pw[c] = sums[c];
      if (pb) pb[c] = sums[kSpan + c];
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
int32_t bwd_blocks(int64_t n, int rows_per_block, int32_t parts) {
  return (int32_t)std::min<int64_t>((n + rows_per_block - 1) / rows_per_block,
                                    parts);
}

template <class TX, class TY, int G, int NV>
void fwd(const NormArgs &a, hipStream_t st) {
  const int64_t rows = norm_nt(G) / G;
  hipLaunchKernelGGL((k_norm_fwd<TX, TY, G, NV>),
                     dim3((unsigned)std::min<int64_t>(
                         (a.n + rows - 1) / rows, kNormGrid)),
                     dim3(norm_nt(G)), 0, st, static_cast<const TX *>(a.x), a.ldx, a.n, a.d, a.w,
                     a.b, (float)a.eps, static_cast<TY *>(a.y), a.ldy, a.mean,
                     a.rstd);
}

template <class TX, class TY, int G, int NV>
void bwd(const NormArgs &a, hipStream_t st) {
  // a few steps of one block cost less than a second launch
  const int32_t blocks =
      a.n <= 4 * (norm_nt(G) / G)
          ? 1
          : bwd_blocks(a.n, norm_nt(G) / G,
                       G > kWave ? kNormParts * 256 / norm_nt(G)
                                 : kNormParts);
  const bool join = blocks > 1 && (a.dw || a.db);
  hipLaunchKernelGGL((k_norm_bwd<TX, TY, G, NV>), dim3((unsigned)blocks),
                     dim3(norm_nt(G)), 0, st, static_cast<const TY *>(a.dy),
                     a.lddy, static_cast<const TX *>(a.x), a.ldx, (int32_t)a.n,
                     a.d, a.w, a.mean, a.rstd, static_cast<const TX *>(a.dres),
                     a.lddres, static_cast<TX *>(a.dx), a.lddx,
                     join ? a.part : a.dw, join ? a.part + a.d : a.db);
  if (join) join_rows(a.part, blocks, 2 * a.d, a.dw, a.db, a.d, st);
}

// The group of a row: the smallest that holds it at one vector a lane, or two
// from a wave on, beyond a wave a block.  (Four vectors a lane leave the
// backward pass one wave a SIMD.)
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
  if (chunks <= 256) EZSP_NORM(256, 1);
  if (chunks <= 512) EZSP_NORM(256, 2);
  if (chunks <= 1024) EZSP_NORM(512, 2);
  EZSP_NORM(512, 4);
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
