// ezsp_narrow_f32.h -- the one-pass backward of ezsp_narrow.h for fp32.
//
// The fp32 matrix instruction (16 x 16 x 4) takes one value a lane, k in any
// order that both operands share, which lets every wave work alone on 16 rows
// of its own, without a barrier:
//   a lane loads 4 neighbouring columns 4 (l / 16) of row l % 16, of x and of
//   what dz is made from.  dz's values are then already the operand of
//   dx += dz W^T (k = 4 (l / 16) + i in the i-th instruction), W's operand
//   lies in LDS in lane order;
//   for dW += x^T dz, where k runs over the rows, both are turned over in a
//   strip of LDS of the wave's own: four words written, one vector read.
// The sums stay in registers over all of a wave's rows and meet at the end.
#pragma once

#include "ezsp_narrow.h"

namespace ezsp {
namespace {

constexpr int kN32Vec = 4;
constexpr int kN32Ld = 20;                   // words from column to column
constexpr int kN32Strip = 16 * kN32Ld;       // of a strip: every bank once
constexpr int kN32Rows = 16;                 // of a wave's step

typedef f32x4_t f32x4_u __attribute__((aligned(4)));

__device__ __forceinline__ f32x4_t raw4(const float *p) {
  return *reinterpret_cast<const f32x4_u *>(p);
}
__device__ __forceinline__ f32x4_t settle4(f32x4_t v, int32_t off,
                                           int32_t cnt) {
  if (off) {
#pragma unroll
    for (int step = 2; step > 0; step >>= 1)
      if (off & step) {
#pragma unroll
        for (int i = 0; i < kN32Vec; ++i)
          v[i] = i + step < kN32Vec ? v[i + step] : 0.0f;
      }
  }
#pragma unroll
  for (int i = 0; i < kN32Vec; ++i) v[i] = i < cnt ? v[i] : 0.0f;
  return v;
}
__device__ __forceinline__ f32x8_t widen4(f32x4_t v) {
  return __builtin_shufflevector(v, v, 0, 1, 2, 3, 0, 1, 2, 3);
}
__device__ __forceinline__ f32x4_t low4(f32x8_t v) {
  return __builtin_shufflevector(v, v, 0, 1, 2, 3);
}

// DT: 16-column tiles of x, CT of dz, NB products.
// Waves a SIMD is to hold, by what a lane holds: sums, the next step's
// inputs, operands, offsets.
constexpr int narrow_waves_f32(int nb, int dt, int ct) {
  const int regs = 4 * (dt * nb * ct + nb * ct + (nb + 1) * ct) + 6 * ct +
                   16 * dt + 50;
  return regs <= 155 ? 3 : regs <= 250 ? 2 : 1;
}

template <class Op, int NB, int DT, int CT>
__global__ __launch_bounds__(kNarrowNT, narrow_waves_f32(NB, DT, CT))
void k_narrow_bwd_f32(NarrowArgs<float> g, Op op) {
  constexpr int kTiles = NB * CT;
  constexpr int kWaves = kNarrowNT / kWave;
  constexpr int kStrips = DT + NB;
  __shared__ __attribute__((aligned(16))) float wt[DT * kTiles * kWave * 4];
  __shared__ __attribute__((aligned(16)))
      float strips[kWaves][kStrips * kN32Strip];
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int lr = lane & 15, lg = lane >> 4;
  // W in the order that the lanes take it, zero past its ends
  for (int i = tid; i < DT * kTiles * kWave; i += kNarrowNT) {
    const int t = i / kWave, l = i % kWave;
    const int32_t d = t / kTiles * 16 + (l & 15);
    const int32_t c = t % kTiles % CT * 16 + 4 * (l >> 4);
    const float *w = g.w[t % kTiles / CT] + (int64_t)d * g.d_out + c;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      wt[4 * i + e] = d < g.d_in && c + e < g.d_out ? w[e] : 0.0f;
  }
  __syncthreads();

  f32x4_t sum[NB][CT], dw[DT][NB][CT];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      sum[b][c] = f32x4_t(0.0f);
#pragma unroll
      for (int i = 0; i < DT; ++i) dw[i][b][c] = f32x4_t(0.0f);
    }
  typename Op::Raw raw[CT];
  f32x4_t xraw[DT];
  auto x_at = [&](int64_t row, int i, int32_t &off, int32_t &cnt) {
    const SpanOf<4> sp = span_of<4>(16 * i + 4 * lg, g.d_in);
    int32_t back;
    const int64_t at = span_at(row, g.ldx, g.n, g.d_in, sp, back);
    off = sp.off + back;
    cnt = row < g.n ? sp.cnt : 0;
    return at;
  };

  const int64_t stride = (int64_t)gridDim.x * kWaves * kN32Rows;
  int64_t row = ((int64_t)blockIdx.x * kWaves + wave) * kN32Rows + lr;
  int32_t off, cnt;
#pragma unroll
  for (int i = 0; i < DT; ++i) xraw[i] = raw4(g.x + x_at(row, i, off, cnt));
#pragma unroll
  for (int c = 0; c < CT; ++c)
    raw[c] = op.raw(row, g.n, g.d_out, span_of<4>(16 * c + 4 * lg, g.d_out));
  float *strip = strips[wave];
  // column 4 lg + e of row lr, then rows 4 lg + 0 .. 3 of column lr
  const int put = 4 * lg * kN32Ld + lr, get = lr * kN32Ld + 4 * lg;
  auto turn = [&](float *s, f32x4_t v) {
#pragma unroll
    for (int e = 0; e < 4; ++e) s[put + e * kN32Ld] = v[e];
    __builtin_amdgcn_wave_barrier();
    const f32x4_t t = *reinterpret_cast<const f32x4_t *>(s + get);
    __builtin_amdgcn_wave_barrier();
    return t;
  };
  for (; row - lr < g.n; row += stride) {
    f32x4_t x[DT], dx[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) {
      dx[i] = f32x4_t(0.0f);
      x_at(row, i, off, cnt);
      x[i] = turn(strip + i * kN32Strip, settle4(xraw[i], off, cnt));
      // (rows past the end: the last one again)
      xraw[i] = raw4(g.x + x_at(row + stride, i, off, cnt));
    }
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      const SpanOf<4> sp = span_of<4>(16 * c + 4 * lg, g.d_out);
      f32x4_t v[NB], z[NB];
      op.value(raw[c], row, g.n, g.d_out, sp, v);
      raw[c] = op.raw(row + stride, g.n, g.d_out, sp);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        sum[b][c] += v[b];
        z[b] = turn(strip + (DT + b) * kN32Strip, v[b]);
      }
      if (g.dx) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < DT; ++i) {
            const f32x4_t w = *reinterpret_cast<const f32x4_t *>(
                wt + 4 * ((i * kTiles + b * CT + c) * kWave + lane));
#pragma unroll
            for (int e = 0; e < 4; ++e)
              dx[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[e], v[b][e],
                                                           dx[i], 0, 0, 0);
          }
      }
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            dw[i][b][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                x[i][e], z[b][e], dw[i][b][c], 0, 0, 0);
    }
    if (g.dx && row < g.n) {
      float *o = g.dx + row * g.lddx;
#pragma unroll
      for (int i = 0; i < DT; ++i) {
        const int col = 16 * i + 4 * lg;
        if (col + 4 <= g.d_in) {
          *reinterpret_cast<f32x4_u *>(o + col) = dx[i];
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (col + e < g.d_in) o[col + e] = dx[i][e];
        }
      }
    }
  }

  // the waves' sums in order: the block's parts, or the results where it is
  // alone
  const int64_t mat = (int64_t)g.d_in * g.d_out, plane = mat + g.d_out;
  const bool alone = gridDim.x == 1;
  float *part = g.part + (int64_t)blockIdx.x * NB * plane;
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          strip[i * kN32Strip + (4 * lg + e) * kN32Ld + lr] = dw[i][b][c][e];
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int m = 1; m < 16; m <<= 1)
          sum[b][c][e] += __shfl_xor(sum[b][c][e], m, kWave);
      if (lr == 0)
        *reinterpret_cast<f32x4_t *>(strip + DT * kN32Strip + 4 * lg) =
            sum[b][c];
      __syncthreads();
      const int32_t col = 16 * c + (tid & 15);
      if (col < g.d_out) {
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          const int32_t d = 16 * i + (tid >> 4);
          float t = 0.0f;
#pragma unroll
          for (int w = 0; w < kWaves; ++w)
            t += strips[w][i * kN32Strip + (tid >> 4) * kN32Ld + (tid & 15)];
          const int64_t at = (int64_t)d * g.d_out + col;
          if (d < g.d_in) {
            if (!alone)
              part[b * plane + at] = t;
            else if (g.dw[b])
              g.dw[b][at] = t;
          }
        }
        if (tid < 16) {
          float t = 0.0f;
#pragma unroll
          for (int w = 0; w < kWaves; ++w)
            t += strips[w][DT * kN32Strip + tid];
          if (!alone)
            part[b * plane + mat + col] = t;
          else if (g.db[b])
            g.db[b][col] = t;
        }
      }
    }
}

// Whether a wave's registers hold the sums, in tiles of 16 x 16.  For 200,000
// rows against dz and two products (floors at 4.9 TB/s and 150 TFLOP/s):
//                   one product          gated
//     6 ->  4     17 us for  90 (3)     19 for 145 (4)
//    32 -> 32     31 for  81 (21)       38 for 112 (26)
//    64 -> 64     62 for 105 (42)      109 for 172 (52)
//   128 -> 64    123 for 141 (63)      (too many sums)
// Up to 32 columns a step's loads and LDS bound it, from 64 on the matrix
// instructions of one wave a SIMD.
inline bool narrow_fits_f32(int64_t n, int64_t d_in, int64_t d_out,
                            int products) {
  const int64_t dt = d_in <= 16 ? 1 : d_in <= 32 ? 2 : d_in <= 64 ? 4 : 8;
  const int64_t ct = d_out <= 16 ? 1 : d_out <= 32 ? 2 : d_out <= 64 ? 4 : 8;
  return n >= kVec && d_in <= 128 && d_out <= 128 && dt * ct * products <= 32;
}

inline bool narrow_serves(int type, int64_t n, int64_t d_in, int64_t d_out,
                          int products) {
  return type == EZSP_TYPE_BF16 ? narrow_fits(n, d_in, d_out, products)
                                : narrow_fits_f32(n, d_in, d_out, products);
}

template <class Op, int NB, int DT, int CT>
void narrow_launch_f32(const NarrowArgs<float> &g, const Op &op,
                       hipStream_t st) {
  static const int64_t slots = [] {
    int per_cu = 0;
    if (hipOccupancyMaxActiveBlocksPerMultiprocessor(
            &per_cu, (const void *)k_narrow_bwd_f32<Op, NB, DT, CT>, kNarrowNT,
            0) != hipSuccess ||
        per_cu < 1)
      per_cu = 1;
    return std::min<int64_t>((int64_t)per_cu * kCus, kNarrowParts);
  }();
  const int32_t blocks = (int32_t)std::min<int64_t>(
      ((int64_t)g.n + kNarrowRows - 1) / kNarrowRows, slots);
  hipLaunchKernelGGL((k_narrow_bwd_f32<Op, NB, DT, CT>),
                     dim3((unsigned)blocks), dim3(kNarrowNT), 0, st, g, op);
  narrow_join<float, NB>(g, blocks, st);
}

template <class Op, int NB>
void narrow_f32(const NarrowArgs<float> &g, const Op &op, hipStream_t st) {
#define EZSP_NARROW(DT, CT)                          \
  do {                                               \
    if constexpr (DT * CT * NB <= 32)                \
      narrow_launch_f32<Op, NB, DT, CT>(g, op, st);  \
    return;                                          \
  } while (0)
#define EZSP_NARROW_D(DT)                    \
  do {                                       \
    if (g.d_out <= 16) EZSP_NARROW(DT, 1);   \
    if (g.d_out <= 32) EZSP_NARROW(DT, 2);   \
    if (g.d_out <= 64) EZSP_NARROW(DT, 4);   \
    EZSP_NARROW(DT, 8);                      \
  } while (0)
  if (g.d_in <= 16) EZSP_NARROW_D(1);
  if (g.d_in <= 32) EZSP_NARROW_D(2);
  if (g.d_in <= 64) EZSP_NARROW_D(4);
  EZSP_NARROW_D(8);
#undef EZSP_NARROW_D
#undef EZSP_NARROW
}

}  // namespace
}  // namespace ezsp
