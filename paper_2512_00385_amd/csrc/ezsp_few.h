// ezsp_few.h -- the forward product of a few rows (a token, a small batch):
// the weights are the work, and each is read once.
//
// A block takes 16 V columns and all of k, its waves taking steps of k in
// turn.  Lanes load V neighbouring weights of 8 consecutive k (bfloat16; 4 for
// fp32) straight into registers, 16 lanes to a row of W.  For the matrix
// instruction (16 x 16 x 32, fp32: four of 16 x 16 x 4) a lane has to bring
// consecutive k of one column: which column is free as long as the result is
// stored there, so lane l's c-th instruction takes column V (l % 16) + c, and
// the k pairs of a column are put together by one byte permute each.  x comes
// from the caches.  The waves' sums meet in LDS, where the epilogue is
// applied: one launch, no parts in memory.
#pragma once

#include "ezsp_gemm.h"

namespace ezsp {
namespace {

constexpr int kFewNT = 512;
constexpr int kFewWaves = kFewNT / kWave;
constexpr int kFewRows = 64;  // rows at most

// V values of T at the alignment of one.
template <class T, int V>
struct FewVec {
  uint32_t d[V * (int)sizeof(T) / 4];
};
template <int W>
__device__ __forceinline__ void few_load(const void *p, uint32_t *d) {
  typedef uint32_t vec __attribute__((ext_vector_type(W)));
  typedef vec vec_u __attribute__((aligned(2)));
  const vec v = *reinterpret_cast<const vec_u *>(p);
#pragma unroll
  for (int i = 0; i < W; ++i) d[i] = v[i];
}
template <>
__device__ __forceinline__ void few_load<1>(const void *p, uint32_t *d) {
  typedef uint32_t u32_u __attribute__((aligned(2)));
  d[0] = *reinterpret_cast<const u32_u *>(p);
}

template <class T, int V, int MT, int NB, class Epi>
__global__ __launch_bounds__(kFewNT) void k_few(GemmArgs<T> g, Epi epi) {
  constexpr int kStepK = sizeof(T) == 2 ? 32 : 16;  // k of a step
  constexpr int kLaneK = kStepK / 4;                // ... and of a lane
  constexpr int kWords = V * (int)sizeof(T) / 4;
  constexpr int kCols = 16 * V;
  // steps in flight, by the registers that hold them
  constexpr int kHeld = NB * kLaneK * kWords + 4 * MT;
  constexpr int U = kHeld <= 24 ? 4 : 2;
  constexpr int kLd = kCols + 4;
  __shared__ float part[kFewWaves][16 * MT][kLd];
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int grp = lane >> 4;
  // a last, incomplete vector is the one that ends with the row of W: its
  // columns are then computed twice, alike, those before the block's first
  // for nothing
  const int32_t n0 = (int32_t)blockIdx.x * kCols;
  const int32_t at = min(n0 + V * (lane & 15), g.n - V);

  struct Step {
    FewVec<T, V> w[NB][kLaneK];
    u32x4_t x[MT];
  };
  // a lane's place in W's first step and in x; few_serves keeps W's offsets
  // below 2^31
  const uint32_t w_at =
      (uint32_t)(((int64_t)grp * kLaneK * g.ldb + at) * (int)sizeof(T));
  const uint32_t w_step = (uint32_t)(kStepK * g.ldb * (int)sizeof(T));
  const T *x_at[MT];
#pragma unroll
  for (int m = 0; m < MT; ++m)
    x_at[m] = g.a[0] + (int64_t)min(16 * m + (lane & 15), g.m - 1) * g.lda +
              grp * kLaneK;
  auto load = [&](int32_t step, Step &s) {
    const uint32_t o = w_at + (uint32_t)step * w_step;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < kLaneK; ++i)
        few_load<kWords>(reinterpret_cast<const char *>(
                             g.b[b] + (int64_t)i * g.ldb) + o,
                         s.w[b][i].d);
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const T *p = x_at[m] + step * kStepK;
      if constexpr (sizeof(T) == 2)
        s.x[m] = *reinterpret_cast<const u32x4_u2 *>(p);
      else
        s.x[m] = *reinterpret_cast<const u32x4_u4 *>(p);
    }
  };
  // the last, incomplete step: zeros on both sides past the end of k
  auto load_rest = [&](int32_t step, Step &s) {
    const int32_t k = step * kStepK + grp * kLaneK;
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < kLaneK; ++i) {
        if (k + i < g.k)
          few_load<kWords>(g.b[b] + (int64_t)(k + i) * g.ldb + at,
                           s.w[b][i].d);
        else
#pragma unroll
          for (int q = 0; q < kWords; ++q) s.w[b][i].d[q] = 0;
      }
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      const T *p = x_at[m] + step * kStepK;
      u32x4_t v = {0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < kLaneK; ++i)
        if (k + i < g.k) {
          if constexpr (sizeof(T) == 2)
            v[i / 2] |= (uint32_t)reinterpret_cast<const uint16_t *>(p)[i]
                        << (16 * (i & 1));
          else
            v[i] = reinterpret_cast<const uint32_t *>(p)[i];
        }
      s.x[m] = v;
    }
  };
  f32x4_t acc[NB][MT][V];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int v = 0; v < V; ++v) acc[b][m][v] = f32x4_t(0.0f);
  auto multiply = [&](const Step &s) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if constexpr (sizeof(T) == 2) {
          u32x4_t w;
#pragma unroll
          for (int p = 0; p < 4; ++p)
            w[p] = __builtin_amdgcn_perm(s.w[b][2 * p + 1].d[v / 2],
                                         s.w[b][2 * p].d[v / 2],
                                         v & 1 ? 0x07060302u : 0x05040100u);
#pragma unroll
          for (int m = 0; m < MT; ++m)
            acc[b][m][v] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                __builtin_bit_cast(bf16x8_t, s.x[m]),
                __builtin_bit_cast(bf16x8_t, w), acc[b][m][v], 0, 0, 0);
        } else {
#pragma unroll
          for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              acc[b][m][v] = __builtin_amdgcn_mfma_f32_16x16x4f32(
                  __uint_as_float(s.x[m][i]),
                  __uint_as_float(s.w[b][i].d[v]), acc[b][m][v], 0, 0, 0);
        }
      }
  };

  // Whole steps, wave after wave.  Rounds of U steps keep U of them on their
  // way without a branch between (the compiler would wait for every load at
  // one); then the steps that fill no round.
  const int32_t steps = g.k / kStepK;
  const int32_t rounds = steps / (U * kFewWaves);
  Step held[U];
  int32_t s = wave;
  if (rounds > 0) {
#pragma unroll
    for (int u = 0; u < U; ++u) load(s + u * kFewWaves, held[u]);
    for (int32_t r = 1; r < rounds; ++r) {
      s += U * kFewWaves;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        multiply(held[u]);
        load(s + u * kFewWaves, held[u]);
      }
    }
    s += U * kFewWaves;
#pragma unroll
    for (int u = 0; u < U; ++u) multiply(held[u]);
  }
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (s + u * kFewWaves < steps) load(s + u * kFewWaves, held[u]);
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (s + u * kFewWaves < steps) multiply(held[u]);
  if (g.k % kStepK && wave == steps % kFewWaves) {
    load_rest(steps, held[0]);
    multiply(held[0]);
  }

  // sums of the waves, one product after the other
  constexpr int kItems = 16 * MT * kCols / kVec;
  constexpr int kPer = (kItems + kFewNT - 1) / kFewNT;
  f32x8_t out[kPer][NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    if (b) __syncthreads();
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int v = 0; v < V; ++v)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (at + v >= n0)
            part[wave][16 * m + 4 * grp + r][at - n0 + v] = acc[b][m][v][r];
    __syncthreads();
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int it = (int)threadIdx.x + j * kFewNT;
      if (it < kItems) {
        const int row = it / (kCols / kVec), c = it % (kCols / kVec) * kVec;
        f32x8_t t = f32x8_t(0.0f);
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w)
#pragma unroll
          for (int i = 0; i < kVec; ++i) t[i] += part[w][row][c + i];
        out[j][b] = t;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < kPer; ++j) {
    const int it = (int)threadIdx.x + j * kFewNT;
    const int row = it / (kCols / kVec);
    const int32_t col = n0 + it % (kCols / kVec) * kVec;
    if (it < kItems && row < g.m && col < g.n)
      epi.at(epi.open(row, col, g.n), 0, out[j]);
  }
}

template <class T, int V, int MT, int NB, class Epi>
void few_launch(const GemmArgs<T> &g, const Epi &epi, hipStream_t st) {
  const int32_t blocks = (g.n + 16 * V - 1) / (16 * V);
  hipLaunchKernelGGL((k_few<T, V, MT, NB, Epi>), dim3((unsigned)blocks),
                     dim3(kFewNT), 0, st, g, epi);
}

// Few rows, and not too long a sum: a CU draws 64-byte pieces of W's rows at
// 20 bytes a nanosecond, whatever is in flight, so a block takes about 2.4 us
// + 3.7 ns a row of W (bfloat16), while the tile kernel with its sum split
// over blocks and joined in a second launch takes 8.5 to 9.5 us up to 16 MB of
// weights.  The two met at k = 1500 (4 rows: 1024 x 4096 in 6.6 against
// 9.3 us, 2048 x 4096 in 10.5 against 9.6) and at 1000 with 32 rows (1024 x
// 4096: 7.9 against 9.4 us; 2048 x 4096: 13.1 against 12.0).
template <class T>
bool few_serves(const GemmArgs<T> &g, int products) {
  return g.m <= kFewRows && g.n >= 4 &&
         (int64_t)g.k * (int)sizeof(T) * products * (g.m <= 16 ? 2 : 3) <=
             6144;
}

template <class T, int NB, class Epi>
void few(const GemmArgs<T> &g, const Epi &epi, hipStream_t st) {
  // whole 128-byte pieces where that leaves every CU a block
  const bool wide = g.n >= 64 * kCus;
#define EZSP_FEW(MT)                       \
  do {                                     \
    if (wide)                              \
      few_launch<T, 4, MT, NB>(g, epi, st); \
    else                                   \
      few_launch<T, 2, MT, NB>(g, epi, st); \
    return;                                \
  } while (0)
  if (g.m <= 16) EZSP_FEW(1);
  if (g.m <= 32) EZSP_FEW(2);
  EZSP_FEW(4);
#undef EZSP_FEW
}

}  // namespace
}  // namespace ezsp
