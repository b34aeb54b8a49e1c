// ezsp_narrow.h -- the backward pass of a product over many rows with few
// columns, in one pass over the rows.
//
// For rows of tens or hundreds of values the gradients are bound by memory:
// forming dz, writing it and reading it twice (for dx and for dW) moves three
// times the bytes of the inputs.  Here a block keeps the weights in LDS and
// the sums of dW in registers, and takes 64 rows at a time:
//   dz of the rows' next kCols columns in registers, from dy and what the
//     forward pass saved, with the bias's sums on the way, then into LDS;
//   dx += dz W^T   (16 x 16 x 32 matrix instructions, k along a row of dz);
//   dW += x^T dz   (32 x 32 x 16, k along the rows, through transposing LDS
//     reads of the same tile),
// while the next columns' inputs are on their way into registers.  Each input
// is read once and dx written once; a block's sums go to the workspace at its
// end and are added over the blocks in order.
#pragma once

#include "ezsp_gemm.h"

namespace ezsp {
namespace {

constexpr int kNarrowNT = 256;
constexpr int kNarrowRows = 64;
constexpr int32_t kNarrowParts = 1024;  // blocks at most

// LDS rows of BYTES bytes in 16-byte pieces; piece p of row r lies at
// p ^ narrow_swz(r), so that 16 rows at one piece, and 4 consecutive rows at
// one 64-byte run, each meet every bank once.
template <int BYTES>
__device__ __forceinline__ int narrow_swz(int r) {
  if constexpr (BYTES >= 256) return ((r & 3) << 2) | ((r >> 2) & 3);
  if constexpr (BYTES == 128) return (((r >> 1) & 1) << 2) | ((r >> 2) & 3);
  return (r >> 2) & 3;
}

// Rows of BYTES bytes in LDS with that exchange.  A lane's place in a
// fragment is a byte offset computed once; steps along the row flip or add
// constant bits of it.
typedef __attribute__((address_space(3))) char lds_char;

template <int BYTES>
struct NarrowTile {
  static __device__ __forceinline__ uint32_t piece(int r, int p) {
    return r * BYTES + ((p ^ narrow_swz<BYTES>(r)) << 4);
  }
  // 64-byte run j of the row from the lane's place in run 0
  static __device__ __forceinline__ uint32_t run(uint32_t at, int j) {
    if constexpr (BYTES >= 256) return (at ^ ((j & 3) << 6)) + (j >> 2) * 256;
    return at ^ (j << 6);
  }
  // k along the row: lane l's piece l / 16 of row l % 16
  static __device__ __forceinline__ uint32_t along_at(int lane) {
    return piece(lane & 15, lane >> 4);
  }
  static __device__ __forceinline__ bf16x8_t along(const lds_char *t,
                                                   uint32_t at, int row0,
                                                   int j) {
    typedef __attribute__((address_space(3))) const bf16x8_t *ptr;
    return *(ptr)(t + run(at, j) + row0 * BYTES);
  }
  // k across 16 rows: lane l's eight rows 8 (l / 32) + 0 .. 7 of column
  // l % 32, read four rows at a time (rows 4 on: one piece bit flipped)
  static __device__ __forceinline__ uint32_t across_at(int lane) {
    return piece(8 * (lane >> 5) + ((lane & 15) >> 2),
                 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1)) +
           8 * (lane & 1);
  }
  static __device__ __forceinline__ bf16x8_t across(lds_char *t, uint32_t at,
                                                    int row0, int j) {
    typedef __attribute__((address_space(3))) s16x4_t *ptr;
    lds_char *p = t + row0 * BYTES;
    const uint32_t o = run(at, j);
    const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(p + o));
    const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (ptr)(p + (o ^ 16) + 4 * BYTES));
    return __builtin_bit_cast(
        bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
  static __device__ __forceinline__ void put(lds_char *t, int r, int p,
                                             bf16x8_t v) {
    typedef __attribute__((address_space(3))) bf16x8_t *ptr;
    *(ptr)(t + piece(r, p)) = v;
  }
};

template <class T>
struct NarrowArgs {
  const T *x, *w[2];
  int64_t ldx;
  int32_t n, d_in, d_out;
  T *dx;  // nullable
  int64_t lddx;
  T *dw[2];     // nullable
  float *db[2];   // nullable
  float *part;  // [block][product][d_in + 1][d_out]: dW, then db's row
};

// DT: 32-column tiles of x; CH chunks of COLS columns of dz per product, NB
// products.  Op gives dz: raw() loads a row's columns, value() computes.
// Waves a SIMD is to hold, by the accumulators of a lane.
constexpr int narrow_waves(int nb, int dt, int cols, int ch) {
  const int regs = ch * ((nb * cols / 32 + 3) / 4) * dt * 16 + ch * nb * 8;
  return regs <= 32 ? 3 : regs <= 72 ? 2 : 1;
}

template <class Op, int NB, int DT, int COLS, int CH>
__global__ __launch_bounds__(kNarrowNT, narrow_waves(NB, DT, COLS, CH))
void k_narrow_bwd(NarrowArgs<__bf16> g, Op op) {
  constexpr int kDzBytes = NB * COLS * 2;       // a row of the dz tile
  constexpr int kWBytes = NB * COLS * CH * 2;   // a row of W: all of dz's
  constexpr int kXBytes = DT * 64;
  constexpr int kGroups = COLS / kVec;          // threads along a row
  constexpr int kStep = kNarrowNT / kGroups;    // rows of one load
  constexpr int kLoads = kNarrowRows / kStep;
  constexpr int kXGroups = DT * 4;
  constexpr int kXLoads = kNarrowRows * kXGroups / kNarrowNT;
  constexpr int kTiles = NB * COLS / 32;        // dW column tiles of a chunk
  constexpr int kPerWave = (kTiles + 3) / 4;
  typedef NarrowTile<kDzBytes> Dz;
  typedef NarrowTile<kWBytes> W;
  typedef NarrowTile<kXBytes> X;
  __shared__ __attribute__((aligned(256))) char
      lds[DT * 32 * kWBytes + kNarrowRows * (kDzBytes + kXBytes)];
  lds_char *wt = (lds_char *)lds, *dzt = wt + DT * 32 * kWBytes;
  lds_char *xt = dzt + kNarrowRows * kDzBytes;

  const int tid = threadIdx.x, lane = tid & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  // W, zero past its ends
  for (int i = tid; i < DT * 32 * (kWBytes / 16); i += kNarrowNT) {
    const int r = i / (kWBytes / 16), p = i % (kWBytes / 16);
    const int b = p / (COLS * CH / kVec), c = p % (COLS * CH / kVec) * kVec;
    W::put(wt, r, p,
           __builtin_convertvector(load8(g.w[b] + (int64_t)r * g.d_out + c,
                                         r < g.d_in ? g.d_out - c : 0),
                                   bf16x8_t));
  }

  const uint32_t dz_along = Dz::along_at(lane), w_along = W::along_at(lane);
  const uint32_t x_across = X::across_at(lane);
  // the wave's column tiles: every fourth from its own on
  const uint32_t dz_across =
      Dz::across_at(lane) ^ ((kTiles > 1 ? wave : 0) << 6);
  const int cg = tid % kGroups * kVec, r_in = tid / kGroups;
  const int xc = tid % kXGroups * kVec, xr = tid / kXGroups;
  f32x8_t sum[CH][NB];
  f32x16_t dw[CH][kPerWave][DT];
#pragma unroll
  for (int c = 0; c < CH; ++c) {
#pragma unroll
    for (int b = 0; b < NB; ++b) sum[c][b] = f32x8_t(0.0f);
#pragma unroll
    for (int j = 0; j < kPerWave; ++j)
#pragma unroll
      for (int i = 0; i < DT; ++i) dw[c][j][i] = f32x16_t(0.0f);
  }

  typename Op::Raw raw[kLoads];
  Vec8<__bf16> xraw[kXLoads];
  const Span x_span = span_of(xc, g.d_in);
  auto load_dz = [&](int64_t r0, int c) {
    const Span sp = span_of(c * COLS + cg, g.d_out);
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
      raw[i] = op.raw(r0 + r_in + i * kStep, g.n, g.d_out, sp);
  };
  auto load_x = [&](int64_t r0) {
#pragma unroll
    for (int i = 0; i < kXLoads; ++i) {
      int32_t back;
      xraw[i] = raw8(g.x + span_at(r0 + xr + i * (kNarrowNT / kXGroups),
                                           g.ldx, g.n, g.d_in, x_span, back));
    }
  };

  const int64_t stride = (int64_t)gridDim.x * kNarrowRows;
  int64_t r0 = (int64_t)blockIdx.x * kNarrowRows;
  load_x(r0);
  load_dz(r0, 0);
  for (; r0 < g.n; r0 += stride) {
    f32x4_t dx[2 * DT];
#pragma unroll
    for (int i = 0; i < 2 * DT; ++i) dx[i] = f32x4_t(0.0f);
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      __syncthreads();  // the tiles of the step before have been read
      if (c == 0) {
#pragma unroll
        for (int i = 0; i < kXLoads; ++i)
        {
          const int64_t row = r0 + xr + i * (kNarrowNT / kXGroups);
          int32_t back;
          span_at(row, g.ldx, g.n, g.d_in, x_span, back);
          X::put(xt, xr + i * (kNarrowNT / kXGroups), xc / kVec,
                 settle(xraw[i], x_span.off + back,
                        row < g.n ? x_span.cnt : 0));
        }
      }
      const Span sp = span_of(c * COLS + cg, g.d_out);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        f32x8_t v[NB];
        op.value(raw[i], r0 + r_in + i * kStep, g.n, g.d_out, sp, v);
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          sum[c][b] += v[b];
          Dz::put(dzt, r_in + i * kStep, (b * COLS + cg) / kVec,
                  __builtin_convertvector(v[b], bf16x8_t));
        }
        __builtin_amdgcn_sched_barrier(0);  // one load's values at a time
      }
      if (c + 1 < CH) {
        load_dz(r0, c + 1);
      } else if (r0 + stride < g.n) {
        load_x(r0 + stride);
        load_dz(r0 + stride, 0);
      }
      __syncthreads();
      // dx: the wave's 16 rows, all columns of x
      if (g.dx) {
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int s = 0; s < COLS / 32; ++s) {
            const bf16x8_t z =
                Dz::along(dzt, dz_along, wave * 16, b * (COLS / 32) + s);
#pragma unroll
            for (int i = 0; i < 2 * DT; ++i)
              dx[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                  W::along(wt, w_along, i * 16, (b * CH + c) * (COLS / 32) + s),
                  z, dx[i], 0, 0, 0);
          }
      }
      // dW: the wave's column tiles, all rows
#pragma unroll
      for (int s = 0; s < kNarrowRows / 16; ++s) {
        bf16x8_t xf[DT];
#pragma unroll
        for (int i = 0; i < DT; ++i)
          xf[i] = X::across(xt, x_across, 16 * s, i);
#pragma unroll
        for (int j = 0; j < kPerWave; ++j) {
          const int tile = wave + 4 * j;
          if (tile < kTiles) {
            const bf16x8_t z =
                Dz::across(dzt, dz_across, 16 * s, 4 * j);
#pragma unroll
            for (int i = 0; i < DT; ++i)
              dw[c][j][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                  z, xf[i], dw[c][j][i], 0, 0, 0);
          }
        }
      }
    }
    if (g.dx) {
      const int64_t row = r0 + wave * 16 + (lane & 15);
      if (row < g.n) {
        __bf16 *o = g.dx + row * g.lddx;
#pragma unroll
        for (int i = 0; i < 2 * DT; ++i) {
          const int col = i * 16 + 4 * (lane >> 4);
          typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
          typedef bf16x4_t bf16x4_u __attribute__((aligned(2)));
          const bf16x4_t v = __builtin_convertvector(dx[i], bf16x4_t);
          if (col + 4 <= g.d_in) {
            *reinterpret_cast<bf16x4_u *>(o + col) = v;
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (col + e < g.d_in) o[col + e] = v[e];
          }
        }
      }
    }
  }

  // this block's sums: its parts, or the results where it is alone
  const int64_t mat = (int64_t)g.d_in * g.d_out, plane = mat + g.d_out;
  const bool alone = gridDim.x == 1;
  float *part = g.part + (int64_t)blockIdx.x * NB * plane;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int j = 0; j < kPerWave; ++j) {
      const int tile = wave + 4 * j;
      const int b = tile / (COLS / 32);
      const int col0 = c * COLS + tile % (COLS / 32) * 32;
      if (tile < kTiles) {
#pragma unroll
        for (int i = 0; i < DT; ++i) {
          const int d = i * 32 + (lane & 31);
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int col = col0 + 8 * (r >> 2) + 4 * (lane >> 5) + (r & 3);
            const int64_t at = (int64_t)d * g.d_out + col;
            if (d < g.d_in && col < g.d_out) {
              if (!alone)
                part[b * plane + at] = dw[c][j][i][r];
              else if (g.dw[b])
                g.dw[b][at] = (__bf16)dw[c][j][i][r];
            }
          }
        }
      }
    }
  // db: over the block's row groups, through LDS
  float *red =  // [kStep][COLS], over the tiles
      reinterpret_cast<float *>(lds + DT * 32 * kWBytes);
  static_assert(kStep * COLS * 4 <= kNarrowRows * (kDzBytes + kXBytes),
                "the sums fit the tiles");
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kVec; ++i) red[r_in * COLS + cg + i] = sum[c][b][i];
      __syncthreads();
      const int col = c * COLS + tid;
      if (tid < COLS && col < g.d_out) {
        float t = 0.0f;
        for (int r = 0; r < kStep; ++r) t += red[r * COLS + tid];
        if (!alone)
          part[b * plane + mat + col] = t;
        else if (g.db[b])
          g.db[b][col] = t;
      }
    }
}

// Adds the blocks' sums in order: part[block][product][d_in + 1][d_out].
constexpr int kNJoinCols = 32;
constexpr int kNJoinNT = 1024;
template <class T, int NB>
__global__ __launch_bounds__(kNJoinNT) void k_narrow_join(
    const float *__restrict__ part, int32_t parts, int32_t d_in,
    int32_t d_out, T *dw0, T *dw1, float *db0, float *db1) {
  constexpr int kSlices = kNJoinNT / kNJoinCols;
  __shared__ float sl[kSlices][kNJoinCols];
  const int64_t plane = (int64_t)(d_in + 1) * d_out, len = NB * plane;
  const int c = threadIdx.x % kNJoinCols, s = threadIdx.x / kNJoinCols;
  const int64_t at = (int64_t)blockIdx.x * kNJoinCols + c;
  float v = 0.0f;
  if (at < len) {
#pragma unroll 8
    for (int32_t p = s; p < parts; p += kSlices) v += part[p * len + at];
  }
  sl[s][c] = v;
  __syncthreads();
  if (s == 0 && at < len) {
    v = 0.0f;
#pragma unroll
    for (int t = 0; t < kSlices; ++t) v += sl[t][c];
    const int b = at >= plane;
    const int64_t e = at - b * plane, mat = (int64_t)d_in * d_out;
    T *dw = b ? dw1 : dw0;
    float *db = b ? db1 : db0;
    if (e < mat) {
      if (dw) dw[e] = (T)v;
    } else if (db) {
      db[e - mat] = v;
    }
  }
}

template <class T, int NB>
void narrow_join(const NarrowArgs<T> &g, int32_t blocks, hipStream_t st) {
  if (blocks == 1 || (!g.dw[0] && !g.dw[1] && !g.db[0] && !g.db[1])) return;
  const int64_t len = (int64_t)NB * (g.d_in + 1) * g.d_out;
  hipLaunchKernelGGL((k_narrow_join<T, NB>),
                     dim3((unsigned)((len + kNJoinCols - 1) / kNJoinCols)),
                     dim3(kNJoinNT), 0, st, g.part, blocks, g.d_in, g.d_out,
                     g.dw[0], g.dw[1], g.db[0], g.db[1]);
}

// Whether a block's registers and LDS hold the weights and their sums:
// tiles of 32 columns of x times chunks of dz.  (The loads of rows shorter
// than a vector need a vector's worth of rows.)
inline bool narrow_fits(int64_t n, int64_t d_in, int64_t d_out,
                        int products) {
  const int64_t dt = d_in <= 32 ? 1 : d_in <= 64 ? 2 : 4;
  const int64_t ch = d_out <= 128 ? 1 : d_out <= 256 ? 2 : 4;
  return n >= kVec && d_in <= 128 && d_out <= 512 && dt * ch * products <= 8 &&
         ch * products <= 4;
}

inline size_t narrow_part_bytes(int64_t n, int64_t d_in, int64_t d_out,
                                int products) {
  const int64_t parts = std::min<int64_t>(
      (n + kNarrowRows - 1) / kNarrowRows, kNarrowParts);
  return (size_t)(parts * products * (d_in + 1) * d_out * 4);
}

// The most that any shape up to this one takes which the one-pass kernels
// accept (fp32's are among bfloat16's), so that a workspace does not shrink
// where they start or cease to serve.
inline size_t narrow_room(int64_t n, int64_t d_in, int64_t d_out,
                          int products) {
  size_t most = 0;
  for (int64_t k = 32; k <= 128; k *= 2)
    for (int64_t m = 128; m <= 512; m *= 2)
      if (narrow_fits(kVec, k, m, products))
        most = std::max(most, narrow_part_bytes(n, std::min(d_in, k),
                                                std::min(d_out, m),
                                                products));
  return most;
}

template <class Op, int NB, int DT, int COLS, int CH>
void narrow_launch(const NarrowArgs<__bf16> &g, const Op &op, hipStream_t st) {
  static const int64_t slots = [] {
    int per_cu = 0;
    if (hipOccupancyMaxActiveBlocksPerMultiprocessor(
            &per_cu, (const void *)k_narrow_bwd<Op, NB, DT, COLS, CH>,
            kNarrowNT, 0) != hipSuccess ||
        per_cu < 1)
      per_cu = 1;
    return std::min<int64_t>((int64_t)per_cu * kCus, kNarrowParts);
  }();
  const int32_t blocks = (int32_t)std::min<int64_t>(
      ((int64_t)g.n + kNarrowRows - 1) / kNarrowRows, slots);
  hipLaunchKernelGGL((k_narrow_bwd<Op, NB, DT, COLS, CH>),
                     dim3((unsigned)blocks), dim3(kNarrowNT), 0, st, g, op);
  narrow_join<__bf16, NB>(g, blocks, st);
}

template <class Op, int NB>
void narrow(const NarrowArgs<__bf16> &g, const Op &op, hipStream_t st) {
#define EZSP_NARROW(DT, COLS, CH)                                         \
  do {                                                                    \
    if constexpr (DT * CH * NB <= 8 && CH * NB <= 4)                      \
      narrow_launch<Op, NB, DT, COLS, CH>(g, op, st);                     \
    return;                                                               \
  } while (0)
#define EZSP_NARROW_D(DT)                       \
  do {                                          \
    if (g.d_out <= 32) EZSP_NARROW(DT, 32, 1);  \
    if (g.d_out <= 64) EZSP_NARROW(DT, 64, 1);  \
    if (g.d_out <= 128) EZSP_NARROW(DT, 128, 1); \
    if (g.d_out <= 256) EZSP_NARROW(DT, 128, 2); \
    EZSP_NARROW(DT, 128, 4);                    \
  } while (0)
  if (g.d_in <= 32) EZSP_NARROW_D(1);
  if (g.d_in <= 64) EZSP_NARROW_D(2);
  EZSP_NARROW_D(4);
#undef EZSP_NARROW_D
#undef EZSP_NARROW
}

}  // namespace
}  // namespace ezsp
