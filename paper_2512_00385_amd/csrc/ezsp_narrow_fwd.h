// ezsp_narrow_fwd.h -- the forward product of many rows with few columns.
//
// What a row costs is reading it and writing its results, so nothing else may
// take long: W lies in LDS, whole, in the order that the lanes take it, and
// every wave works alone on 32 rows at a time.  A lane loads 16 bytes of
// neighbouring k of row l % 16, which is the operand of the matrix
// instruction (16 x 16 x 32, fp32: four of 16 x 16 x 4) as it lies; W's
// columns are dealt to the instructions so that a lane ends with 8
// neighbouring columns of one row, and the epilogue runs on them from the
// registers.  No barrier after W is there, no exchange through LDS.
#pragma once

#include "ezsp_narrow_f32.h"

namespace ezsp {
namespace {

constexpr int kNFwdNT = 256;
constexpr int kNFwdRows = 32;                  // of a wave's step
constexpr int kNFwdR = kNFwdRows / 16;
constexpr int kNFwdPerCu = 8;                  // blocks

__device__ __forceinline__ bf16x8_t shift_in(bf16x8_t v, int32_t off,
                                             int32_t cnt) {
  return settle(Vec8<__bf16>{__builtin_bit_cast(u32x4_t, v)}, off, cnt);
}
__device__ __forceinline__ f32x4_t shift_in(f32x4_t v, int32_t off,
                                            int32_t cnt) {
  return settle4(v, off, cnt);
}
__device__ __forceinline__ f32x4_t narrow_mfma(bf16x8_t w, bf16x8_t x,
                                               f32x4_t acc) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, x, acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4_t narrow_mfma(f32x4_t w, f32x4_t x,
                                               f32x4_t acc) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    acc = __builtin_amdgcn_mfma_f32_16x16x4f32(w[e], x[e], acc, 0, 0, 0);
  return acc;
}

// k of at most 64 bytes of a row, NB products.
template <class T, class Epi, int NB>
__global__ __launch_bounds__(kNFwdNT, 2) void k_narrow_fwd(GemmArgs<T> g,
                                                           Epi epi) {
  constexpr int V = 16 / (int)sizeof(T);  // values of a lane
  constexpr int kStep = 4 * V;            // k of a step
  typedef T vec __attribute__((ext_vector_type(V)));
  typedef vec vec_u __attribute__((aligned(sizeof(T))));
  extern __shared__ __attribute__((aligned(16))) char lds[];
  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int lr = lane & 15, lg = lane >> 4;
  const int32_t groups = (g.n + 31) / 32;
  // the 1024 bytes of columns 32 c + 8 q + 4 half + r (lane 4 q + r) begin at
  // (product * groups + c) * 2 + half
  const int32_t eights = groups * 4;
  for (int32_t i = tid; i < NB * kStep * eights; i += kNFwdNT) {
    const int32_t c8 = i % eights, k = i / eights % kStep;
    const int b = i / eights / kStep;
    const f32x8_t v = load8(g.b[b] + (int64_t)k * g.ldb + 8 * c8,
                            k < g.k ? g.n - 8 * c8 : 0);
    const int32_t c = c8 / 4, q = c8 % 4;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int32_t tile = (b * groups + c) * 2 + (e >> 2);
      const int l = 4 * q + (e & 3) + 16 * (k / V);
      reinterpret_cast<T *>(lds)[(tile * kWave + l) * V + k % V] = (T)v[e];
    }
  }
  __syncthreads();

  const int64_t stride = (int64_t)gridDim.x * (kNFwdNT / kWave) * kNFwdRows;
  int64_t row = ((int64_t)blockIdx.x * (kNFwdNT / kWave) + wave) * kNFwdRows +
                lr;
  const SpanOf<V> sp = span_of<V>(V * lg, g.k);
  int32_t back;
  vec_u raw[kNFwdR];
  auto load = [&](int64_t r) {
    return *reinterpret_cast<const vec_u *>(
        g.a[0] + span_at(r, g.lda, g.m, g.k, sp, back));
  };
#pragma unroll
  for (int i = 0; i < kNFwdR; ++i) raw[i] = load(row + 16 * i);
  for (; row - lr < g.m; row += stride) {
    vec x[kNFwdR];
#pragma unroll
    for (int i = 0; i < kNFwdR; ++i) {
      const int64_t r = row + 16 * i;
      span_at(r, g.lda, g.m, g.k, sp, back);
      x[i] = shift_in(raw[i], sp.off + back, r < g.m ? sp.cnt : 0);
      raw[i] = load(r + stride);  // (past the end: the last row again)
    }
    for (int32_t c = 0; c < groups; ++c) {
      const int32_t col = 32 * c + 8 * lg;
      const typename Epi::Lane at = epi.open(row, min(col, g.n - 1), g.n);
      f32x4_t acc[kNFwdR][NB][2];
#pragma unroll
      for (int i = 0; i < kNFwdR; ++i)
#pragma unroll
        for (int b = 0; b < NB; ++b)
          acc[i][b][0] = acc[i][b][1] = f32x4_t(0.0f);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const vec w = reinterpret_cast<const vec *>(
              lds)[((b * groups + c) * 2 + h) * kWave + lane];
#pragma unroll
          for (int i = 0; i < kNFwdR; ++i)
            acc[i][b][h] = narrow_mfma(w, x[i], acc[i][b][h]);
        }
#pragma unroll
      for (int i = 0; i < kNFwdR; ++i)
        if (row + 16 * i < g.m && col < g.n) {
          f32x8_t v[NB];
#pragma unroll
          for (int b = 0; b < NB; ++b)
            v[b] = __builtin_shufflevector(acc[i][b][0], acc[i][b][1], 0, 1, 2,
                                           3, 4, 5, 6, 7);
          epi.at(at, 16 * i, v);
        }
    }
  }
}

// Rows of up to 64 bytes, to results of up to 128.  800,000 rows, silu, for
// the tiles of ezsp_gemm.h, us (floor at 4.9 TB/s); s: with residual or
// pre-activations saved
//                    linear          linear, s        gated       gated, s
//   bf16   6 ->   6  22 for 42 ( 4)  36 for 53 ( 8)  26 for 73   31 for 82
//          6 ->  32  21 for 39 (12)  29 for 44 (33)  23 for 58   28 for 60
//         32 ->  32  22 for 27 (21)  33 for 34 (42)  24 for 40   33 for 43
//         32 ->  64  32 for 46 (31) 114 for 112 (73) 37 for 60  104 for 95
//   fp32   6 ->   6  27 for 49 ( 8)  40 for 58 (16)  38 for 85   47 for 93
//          6 ->  32  28 for 48 (25)  83 for 80 (67)  35 for 79  106 for 126
// The tiles store whole lines where a lane's rows here are half of one apart,
// which costs once the results leave the caches: with 256 bytes the saved
// forms lose more (bf16 32 -> 128, gated: 211 for 135) than the others gain
// (62 for 99).  (Which kernel serves may not depend on what is saved: h is
// the same, bit for bit, in both.)  Rows of more than 64 bytes gain from
// loads of whole lines too (200,000 rows, bf16 128 -> 32: 20 for 15), and up
// to 20,000 rows the two are alike.
template <class T>
bool narrow_fwd_serves(const GemmArgs<T> &g) {
  constexpr int64_t e = (int64_t)sizeof(T);
  return g.m >= 1024 && g.k * e <= 64 && g.n * e <= 128;
}

template <class T, int NB, class Epi>
void narrow_fwd(const GemmArgs<T> &g, const Epi &epi, hipStream_t st) {
  const int32_t bytes = NB * ((g.n + 31) / 32) * 2 * 1024;  // at most 8 KiB
  const int64_t rows = kNFwdRows * (kNFwdNT / kWave);
  const int32_t blocks = (int32_t)std::min<int64_t>(
      ((int64_t)g.m + rows - 1) / rows, (int64_t)kNFwdPerCu * kCus);
  hipLaunchKernelGGL((k_narrow_fwd<T, Epi, NB>), dim3((unsigned)blocks),
                     dim3(kNFwdNT), (unsigned)bytes, st, g, epi);
}

}  // namespace
}  // namespace ezsp
