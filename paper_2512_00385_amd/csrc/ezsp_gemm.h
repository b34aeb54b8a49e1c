// ezsp_gemm.h -- the matrix products behind the dense operators, on the
// matrix cores:  D[m][n] = sum over k of A(m, k) B(k, n), fp32 accumulators,
// with an epilogue applied to each element before its only store.
//
// Layouts.  Either operand may be contiguous along k ("K-major": rows of x,
// rows of dz, and weights [d_in][d_out] seen from dx = dz W^T) or along its
// own index (weights in y = x W, both operands of dW = x^T dz).  Both come
// into LDS as they lie in memory, 128 bytes of k at a time (64 bfloat16, 32
// fp32 values):
//   K-major  rows of 128 bytes, read as 16-byte pieces along k; piece p of
//            row r sits at p ^ (r / 2 mod 8): two rows fill the 64 banks
//            once, and 16 rows read without a conflict (with r mod 8 every
//            second access was one);
//   else     one line per k, read through ds_read_b64_tr_b16, which hands
//            every lane four consecutive k of its own column (fp32: four
//            separate reads).  A line's 64-byte pieces are exchanged by the
//            low bits of k for the same reason.
// The matrix instruction is v_mfma_f32_32x32x16_bf16 (fp32: four
// v_mfma_f32_32x32x2_f32 over a 16-byte piece each) in transposed form:
// its rows are n, its columns m, so that a lane's accumulators are runs of
// four neighbouring columns of D.
#pragma once

#include <algorithm>

#include "ezsp_dense.h"

namespace ezsp {
namespace {

// How the two B matrices of an operator enter.
enum : int {
  kPlain = 0,  // D = A B0
  kDual = 1,   // D0 = A B0 and D1 = A B1, both n wide, in one pass over A
  kSeq = 2,    // D = A0 B0 + A1 B1, the two as one longer sum
};

template <class T>
struct GemmArgs {
  const T *a[2];
  const T *b[2];
  int64_t lda, ldb;
  int32_t m, n, k;  // k of one (A, B) pair
  // what is stored of each operand: its own index and k.  Beyond m, n and k
  // where it is padded (a workspace matrix; k with zeros), else those (0).
  int32_t ra, rb, ka, kb;
  int32_t tiles_m, tiles_n;
  int32_t splits;   // the sum over k in this many parts
  int32_t kt_split; // LDS tiles of k per part
  bool to_parts;    // the parts go to the workspace
};

// Lines that read as zero, for pieces past the end of k.
static __device__ __attribute__((aligned(16))) const uint32_t kZeroLine[4] = {
    0, 0, 0, 0};

// Copies 16 bytes a lane from memory into LDS past the registers: lane l's
// go to lds + 16 l.  Written as instructions because the compiler makes every
// LDS read after such a copy wait for it, also when it fills another buffer;
// they write no register, and copies_landed() before the barrier is the wait
// that the reads need.  The address is base + off, or a full one per lane.
__device__ __forceinline__ uint32_t lds_addr(const void *lds) {
  return (uint32_t)(uintptr_t)(
      (const __attribute__((address_space(3))) void *)lds);
}
// A pointer that is the same in every lane, where the compiler can't tell.
__device__ __forceinline__ const void *uniform(const void *p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v);
  const uint32_t hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return reinterpret_cast<const void *>(((uint64_t)hi << 32) | lo);
}
__device__ __forceinline__ void copy_to_lds16(const void *base, uint32_t off,
                                              uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %0\n\ts_nop 0\n\t"
      "global_load_lds_dwordx4 %1, %2"
      :
      : "s"(lds), "v"(off), "s"(uniform(base))
      : "memory", "m0");
}
__device__ __forceinline__ void copy_to_lds16(const void *src, uint32_t lds) {
  asm volatile(
      "s_mov_b32 m0, %0\n\ts_nop 0\n\t"
      "global_load_lds_dwordx4 %1, off"
      :
      : "s"(lds), "v"(src)
      : "memory", "m0");
}

// Waits for this wave's copies into LDS (a barrier alone orders LDS accesses,
// not these).
__device__ __forceinline__ void copies_landed() {
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
}

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef short s16x8_t __attribute__((ext_vector_type(8)));

constexpr int64_t kCus = 256;    // of an MI355X
// row distances that keep a tile's offsets in 32 bits
constexpr int64_t kFastLd = (int64_t)1 << 21;
constexpr int kLineBytes = 128;  // bytes of k in an LDS tile

// One operand's LDS tile: R rows (its own index) by 128 bytes of k.
template <class T, int R, bool KMAJOR, int NT, bool FAST>
struct Tile {
  static constexpr int kPer = 16 / (int)sizeof(T);           // a piece
  static constexpr int kK = kLineBytes / (int)sizeof(T);      // k of a tile
  static constexpr int kBytes = R * kLineBytes;
  static constexpr int kCh = R * 8 / NT;  // pieces a thread moves
  static constexpr int kLine = R / kPer;  // pieces of a line (not K-major)
  static_assert(R * 8 % NT == 0, "whole pieces");
  // exchange of a line's 64-byte pieces
  static __device__ __forceinline__ int line_swz(int k) {
    if constexpr (sizeof(T) == 2) {
      if constexpr (R >= 128) return (k & 3) << 2;
      if constexpr (R == 64) return ((k >> 1) & 1) << 2;
    }
    return 0;
  }

  uint32_t off[kCh];              // bytes from the tile's first element
  u32x4_t reg[FAST ? 1 : kCh];
  int32_t first, edge;            // !FAST: first row; rows left if not R
  int32_t left;                   // k left of the step in reg
  bool slow, raw;                 // no vector fits a line; reg as loaded

  // where piece i of this thread comes from: (row, k) of its first element
  static __device__ __forceinline__ void place(int i, int &r, int &k) {
    const int c = i * NT + (int)threadIdx.x;
    if constexpr (KMAJOR) {
      r = c >> 3;
      k = ((c & 7) ^ ((r >> 1) & 7)) * kPer;
    } else {
      k = c / kLine;
      r = ((c % kLine) ^ line_swz(k)) * kPer;
    }
  }

  // A tile of rows row0 .. row0 + R - 1 out of rows.  Rows past the end
  // repeat the last one: they only feed elements of D that do not exist.
  // Without FAST a piece of a line that ends inside it is loaded as the
  // line's last kPer values and shifted into place by put().
  __device__ __forceinline__ void init(int32_t row0, int32_t rows,
                                       int64_t ld) {
    const int32_t left = rows - row0;
    first = row0;
    edge = left < R ? left : 0;
    slow = !FAST && (ld >= kFastLd || (!KMAJOR && rows < kPer));
    raw = false;
#pragma unroll
    for (int i = 0; i < kCh; ++i) {
      int r, k;
      place(i, r, k);
      if constexpr (KMAJOR) {
        r = min(r, left - 1);
        off[i] = (uint32_t)(((int64_t)r * ld + k) * (int)sizeof(T));
      } else {
        r = min(r, left - kPer) + (FAST ? 0 : row0);
        off[i] = (uint32_t)(((int64_t)k * ld + r) * (int)sizeof(T));
      }
    }
  }

  // How far back a K-major piece of the last step starts, in elements, so
  // that it ends with the table at the latest (its last row ends after `left`
  // more k).
  __device__ __forceinline__ int32_t tail_back(int i, int32_t rows,
                                               int64_t ld) const {
    int r, k;
    place(i, r, k);
    r = min(r, rows - first - 1);
    const int64_t over = (int64_t)(r - (rows - first - 1)) * ld + k + kPer -
                         left;
    return over > 0 ? (int32_t)over : 0;
  }

  // Starts bringing in the tile whose first element is p; k_left counts the
  // k that exist from there on.
  __device__ __forceinline__ void fetch(const T *p, int64_t ld, int32_t rows,
                                        int32_t k_left, char *lds) {
    if constexpr (FAST) {
      const uint32_t dst = __builtin_amdgcn_readfirstlane(
          lds_addr(lds) + (threadIdx.x / kWave) * (kWave * 16));
      if (k_left >= kK) {
#pragma unroll
        for (int i = 0; i < kCh; ++i)
          copy_to_lds16(p, off[i], dst + i * NT * 16);
      } else {
#pragma unroll
        for (int i = 0; i < kCh; ++i) {
          int r, k;
          place(i, r, k);
          const char *src = reinterpret_cast<const char *>(p) + off[i];
          copy_to_lds16(k < k_left ? src
                                   : reinterpret_cast<const char *>(kZeroLine),
                        dst + i * NT * 16);
        }
      }
    } else if (k_left >= kK && !slow) {
      const char *src = static_cast<const char *>(
          uniform(KMAJOR ? p : p - first));
#pragma unroll
      for (int i = 0; i < kCh; ++i) {
        if constexpr (sizeof(T) == 2)
          reg[i] = *reinterpret_cast<const u32x4_u2 *>(src + off[i]);
        else
          reg[i] = *reinterpret_cast<const u32x4_u4 *>(src + off[i]);
      }
      raw = true;
      left = kK;
    } else if (!slow &&
               (!KMAJOR || (int64_t)(rows - 1) * ld + k_left >= kPer)) {
      // a last, incomplete step: pieces that would pass the table's end are
      // taken from further back and shifted, lines past it repeat the last
      // one; put() zeroes what lies past the end of k
      left = k_left;
      raw = true;
#pragma unroll
      for (int i = 0; i < kCh; ++i) {
        int r, k;
        place(i, r, k);
        const T *q;
        if constexpr (KMAJOR) {
          r = min(r, rows - first - 1);
          q = p + (int64_t)r * ld + k - tail_back(i, rows, ld);
        } else {
          q = p - first + (int64_t)min(k, k_left - 1) * ld +
              min(first + r, rows - kPer);
        }
        if constexpr (sizeof(T) == 2)
          reg[i] = *reinterpret_cast<const u32x4_u2 *>(q);
        else
          reg[i] = *reinterpret_cast<const u32x4_u4 *>(q);
      }
    } else {
      const int32_t rows_left = rows - first;
#pragma unroll
      for (int i = 0; i < kCh; ++i) {
        int r, k;
        place(i, r, k);
        const T *q = KMAJOR ? p + (int64_t)r * ld + k : p + (int64_t)k * ld + r;
        const int32_t along = KMAJOR ? k_left - k : rows_left - r;
        const bool live = KMAJOR ? r < rows_left : k < k_left;
        const int32_t cnt = live ? along : 0;
        u32x4_t v = {0, 0, 0, 0};
        if (cnt >= kPer) {
          if constexpr (sizeof(T) == 2)
            v = *reinterpret_cast<const u32x4_u2 *>(q);
          else
            v = *reinterpret_cast<const u32x4_u4 *>(q);
        } else if (cnt > 0) {
          if constexpr (sizeof(T) == 2) {
            const uint16_t *h = reinterpret_cast<const uint16_t *>(q);
#pragma unroll
            for (int e = 0; e < kPer; ++e)
              if (e < cnt) v[e / 2] |= (uint32_t)h[e] << (16 * (e & 1));
          } else {
            const uint32_t *h = reinterpret_cast<const uint32_t *>(q);
#pragma unroll
            for (int e = 0; e < kPer; ++e)
              if (e < cnt) v[e] = h[e];
          }
        }
        reg[i] = v;
      }
      raw = false;
    }
  }

  // Ends it where the pieces went through registers.
  static __device__ __forceinline__ u32x4_t drop(u32x4_t v, int by) {
    uint64_t lo = ((uint64_t)v[1] << 32) | v[0];
    uint64_t hi = ((uint64_t)v[3] << 32) | v[2];
    const int bits = min(by * (int)sizeof(T) * 8, 127);  // > 0
    lo = bits >= 64 ? hi >> (bits & 63) : (lo >> bits) | (hi << (64 - bits));
    hi = bits >= 64 ? 0 : hi >> bits;
    return u32x4_t{(uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi,
                   (uint32_t)(hi >> 32)};
  }
  __device__ __forceinline__ void put(char *lds, int32_t rows, int64_t ld) {
    if constexpr (!FAST) {
#pragma unroll
      for (int i = 0; i < kCh; ++i) {
        u32x4_t v = reg[i];
        if (raw && (left < kK || (!KMAJOR && edge))) {
          int r, k;
          place(i, r, k);
          const int by = KMAJOR ? (left < kK ? tail_back(i, rows, ld) : 0)
                         : edge ? r - min(r, edge - kPer)
                                : 0;
          if (by > 0) v = drop(v, by);
          if (left < kK) {
            const int cnt = KMAJOR ? left - k : k < left ? kPer : 0;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              if constexpr (sizeof(T) == 2)
                v[q] = cnt > 2 * q + 1 ? v[q] : cnt > 2 * q ? v[q] & 0xffffu : 0u;
              else
                v[q] = cnt > q ? v[q] : 0u;
            }
          }
        }
        *reinterpret_cast<u32x4_t *>(lds +
                                     (i * NT + (int)threadIdx.x) * 16) = v;
      }
    }
  }

  // Fragment of rows row0 .. row0 + 31 (row0 a multiple of 32) and k step s:
  // lane l gets piece 2 s + l / 32 of row row0 + l % 32.
  static __device__ __forceinline__ u32x4_t frag(const char *lds, int row0,
                                                 int s, int lane) {
    if constexpr (KMAJOR) {
      const int piece = (2 * s + (lane >> 5)) ^ ((lane >> 1) & 7);
      return *reinterpret_cast<const u32x4_t *>(
          lds + (row0 + (lane & 31)) * kLineBytes + piece * 16);
    } else if constexpr (sizeof(T) == 2) {
      const int q = (lane & 15) >> 2;
      const int k = 16 * s + 8 * (lane >> 5) + q;
      const int byte = (((row0 >> 3) ^ line_swz(q)) << 4) +
                       32 * ((lane >> 4) & 1) + 8 * (lane & 3);
      const char *at = lds + k * (R * 2) + byte;
      typedef __attribute__((address_space(3))) s16x4_t *lds_ptr;
      const s16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)at);
      const s16x4_t hi =
          __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)(at + 4 * R * 2));
      const s16x8_t both =
          __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      return __builtin_bit_cast(u32x4_t, both);
    } else {
      const float *f = reinterpret_cast<const float *>(lds) + row0 +
                       (lane & 31) + (8 * s + 4 * (lane >> 5)) * R;
      u32x4_t v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(f[e * R]);
      return v;
    }
  }
};

template <class T>
__device__ __forceinline__ f32x16_t mma(u32x4_t n_frag, u32x4_t m_frag,
                                        f32x16_t acc) {
  if constexpr (sizeof(T) == 2) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(
        __builtin_bit_cast(bf16x8_t, n_frag),
        __builtin_bit_cast(bf16x8_t, m_frag), acc, 0, 0, 0);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      acc = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(n_frag[e]),
                                                 __uint_as_float(m_frag[e]),
                                                 acc, 0, 0, 0);
    return acc;
  }
}

// Block of WM x WN waves on a tile of BM x BN of D (kDual: BN / 2 columns of
// each product side by side).
template <class T_, int BM_, int BN_, int WM_, int WN_, bool AK_, bool BK_,
          int MODE_, bool FAST_>
struct Shape {
  typedef T_ T;
  static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_, MODE = MODE_;
  static constexpr bool AK = AK_, BK = BK_, FAST = FAST_;
  static constexpr int NT = WM * WN * kWave;
  static constexpr int TM = BM / WM / 32, TN = BN / WN / 32;  // of a wave
  static constexpr int NB = MODE == kDual ? 2 : 1;
  static constexpr int CN = BN / NB;   // columns of D of a tile
  static constexpr int WC = TN * 32 / NB;  // ... and of a wave
  typedef Tile<T, BM, AK, NT, FAST> TileA;
  typedef Tile<T, CN, BK, NT, FAST> TileB;
  static constexpr int kK = TileA::kK;
  static constexpr int kStage = (BM + BN) * kLineBytes;
  static_assert(MODE != kDual || TN % 2 == 0, "both products in a wave");
  // epilogue: 32 rows of a wave's columns
  static constexpr int kOutLd = TN * 32 + 4;
  static constexpr int kOut = 32 * kOutLd * 4;
  // waves whose part fits one stage; the others' lie past both
  static constexpr int kFit = kStage / kOut < WM * WN ? kStage / kOut : WM * WN;
  static constexpr int kLds = 2 * kStage + (WM * WN - kFit) * kOut;
  // waves a SIMD is to hold: those of the blocks that LDS lets in
  static constexpr int kWaves = 160 * 1024 / kLds * WM * WN / 4;
};

// Logical tile of block b out of total: XCD x takes the x-th contiguous run
// (blocks are dealt to the XCDs in turn), and inside it tiles go in bands of
// kBand tile rows, so that a band's A rows and the B columns it meets stay in
// that XCD's L2.
constexpr int kBand = 8;
__device__ __forceinline__ void tile_of(int32_t b, int32_t total,
                                        int32_t tiles_m, int32_t tiles_n,
                                        int32_t &tm, int32_t &tn, int32_t &sp) {
  const int32_t per = total / kXcd, extra = total % kXcd;
  const int32_t x = b % kXcd, j = b / kXcd;
  int32_t t = x * per + min(x, extra) + j;
  const int32_t tiles = tiles_m * tiles_n;
  sp = t / tiles;
  t -= sp * tiles;
  const int32_t band = t / (kBand * tiles_n);
  const int32_t rows = min(kBand, tiles_m - band * kBand);
  const int32_t in = t - band * kBand * tiles_n;
  tm = band * kBand + in % rows;
  tn = in / rows;
}

// A block takes tiles of D gridDim.x apart and keeps one pipeline running
// across them.  Its steps are LDS tiles of k; while one is multiplied,
//  - the next one lies in LDS or lands there (FAST: two steps ahead, issued as
//    soon as its stage is free; else one, by way of registers),
//  - each quarter's fragments are read while the quarter before is
//    multiplied, the next step's first ones during the last quarter, so that
//    the barrier between two steps has multiplications to hide behind.
// During an epilogue the next tile's first step is on its way.
template <class S, class Epi>
__global__ __launch_bounds__(S::NT, S::kWaves) void k_gemm(
    GemmArgs<typename S::T> g, Epi epi) {
  typedef typename S::T T;
  __shared__ __attribute__((aligned(16))) char stages[S::kLds];
  const int lane = threadIdx.x & (kWave - 1);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const int wm = wave / S::WN, wn = wave % S::WN;
  const int32_t total = g.tiles_m * g.tiles_n * g.splits;
  const int32_t kt1 = (g.k + S::kK - 1) / S::kK;  // steps of one pair
  const int32_t kt_all = S::MODE == kSeq ? 2 * kt1 : kt1;

  // the tile and step to fetch next
  typename S::TileA ta;
  typename S::TileB tb[S::NB];
  int32_t f_blk = blockIdx.x, m0 = 0, n0 = 0, f_t = 0, f_end = 0;
  auto open = [&] {
    int32_t tm, tn, sp;
    tile_of(f_blk, total, g.tiles_m, g.tiles_n, tm, tn, sp);
    m0 = tm * S::BM;
    n0 = tn * S::CN;
    f_t = sp * g.kt_split;
    f_end = min(kt_all, f_t + g.kt_split);
    ta.init(m0, g.ra, g.lda);
#pragma unroll
    for (int p = 0; p < S::NB; ++p) tb[p].init(n0, g.rb, g.ldb);
  };
  // After a tile's last step, the block's next tile.  A step that goes by way
  // of registers is finished by put() with what init() and fetch() noted of
  // its tile, so there the next one opens after that.
  auto advance = [&] {
    if (f_t < f_end) return;
    f_blk += gridDim.x;
    if (f_blk < total) open();
  };
  auto fetch = [&](char *st) {
    if (f_blk >= total) return;
    const bool second = S::MODE == kSeq && f_t >= kt1;
    const int32_t k0 = (second ? f_t - kt1 : f_t) * S::kK;
    const T *a = second ? g.a[1] : g.a[0];
    ta.fetch(S::AK ? a + (int64_t)m0 * g.lda + k0
                   : a + (int64_t)k0 * g.lda + m0,
             g.lda, g.ra, g.ka - k0, st);
#pragma unroll
    for (int p = 0; p < S::NB; ++p) {
      const T *b = (second || p) ? g.b[1] : g.b[0];
      tb[p].fetch(S::BK ? b + (int64_t)n0 * g.ldb + k0
                        : b + (int64_t)k0 * g.ldb + n0,
                  g.ldb, g.rb, g.kb - k0,
                  st + S::TileA::kBytes + p * S::TileB::kBytes);
    }
    ++f_t;
    if (S::FAST) advance();
  };
  // every fetch() has its put() before the next one
  auto put = [&](char *st) {
    if (S::FAST) return;
    ta.put(st, g.ra, g.lda);
#pragma unroll
    for (int p = 0; p < S::NB; ++p)
      tb[p].put(st + S::TileA::kBytes + p * S::TileB::kBytes, g.rb, g.ldb);
    advance();
  };

  f32x16_t acc[S::TM][S::TN];
  u32x4_t fa[2][S::TM], fb[2][S::TN];  // fragments of quarters, in turn
  auto frags = [&](const char *st, int s) {
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
      fa[s & 1][i] = S::TileA::frag(st, (wm * S::TM + i) * 32, s, lane);
#pragma unroll
    for (int j = 0; j < S::TN; ++j) {
      const int p = j / (S::TN / S::NB), jj = j % (S::TN / S::NB);
      fb[s & 1][j] =
          S::TileB::frag(st + S::TileA::kBytes + p * S::TileB::kBytes,
                         wn * S::WC + jj * 32, s, lane);
    }
  };
  auto multiply = [&](int s) {
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
#pragma unroll
      for (int j = 0; j < S::TN; ++j)
        acc[i][j] = mma<T>(fb[s & 1][j], fa[s & 1][i], acc[i][j]);
  };

  int32_t blk = blockIdx.x;
  if (blk >= total) return;
  int32_t cur = 0;  // the stage being multiplied
  open();
  fetch(stages);
  put(stages);
  if (S::FAST) fetch(stages + S::kStage);
  copies_landed();
  __syncthreads();
  frags(stages, 0);
  while (true) {
    int32_t tm, tn, tile_sp;
    tile_of(blk, total, g.tiles_m, g.tiles_n, tm, tn, tile_sp);
    const int32_t tile_m0 = tm * S::BM, tile_n0 = tn * S::CN;
    const int32_t steps =
        min(kt_all - tile_sp * g.kt_split, g.kt_split);
    blk += gridDim.x;
    const bool more = blk < total;
#pragma unroll
    for (int i = 0; i < S::TM; ++i)
#pragma unroll
      for (int j = 0; j < S::TN; ++j) acc[i][j] = f32x16_t(0.0f);
    for (int32_t t = 0; t < steps; ++t) {
      char *here = stages + cur, *next = stages + (S::kStage - cur);
      const bool ahead = t + 1 < steps || more;
      if (!S::FAST && ahead) fetch(next);
#pragma unroll
      for (int s = 0; s < 3; ++s) {
        frags(here, s + 1);
        __builtin_amdgcn_sched_barrier(0);
        multiply(s);
      }
      if (!S::FAST && ahead) put(next);
      copies_landed();
      __syncthreads();
      if (S::FAST && t + 1 < steps) fetch(here);
      frags(next, 0);  // (of no use after a block's last step)
      __builtin_amdgcn_sched_barrier(0);
      multiply(3);
      cur = S::kStage - cur;
    }

    // epilogue: 32 rows at a time through the wave's own part of LDS (the
    // stage just read, and what lies past both), so that each lane ends up
    // with kVec neighbouring columns of a row
    float *out = reinterpret_cast<float *>(
        stages + (wave < S::kFit ? S::kStage - cur + wave * S::kOut
                                 : 2 * S::kStage + (wave - S::kFit) * S::kOut));
    constexpr int kLanes = S::WC / kVec;  // lanes of a row
    const int32_t col = tile_n0 + wn * S::WC + (lane % kLanes) * kVec;
    const int32_t row0 = tile_m0 + wm * S::TM * 32 + lane / kLanes;
    const bool in_n = col < g.n;
    const typename Epi::Lane view = epi.open(row0, in_n ? col : 0, g.n);
#pragma unroll
    for (int i = 0; i < S::TM; ++i) {
#pragma unroll
      for (int j = 0; j < S::TN; ++j)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          f32x4_t v;
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] = acc[i][j][4 * q + e];
          *reinterpret_cast<f32x4_t *>(out + (lane & 31) * S::kOutLd + j * 32 +
                                       8 * q + 4 * (lane >> 5)) = v;
        }
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int pass = 0; pass < 32 * kLanes / kWave; ++pass) {
        const int down = i * 32 + pass * (kWave / kLanes);
        const float *src =
            out + (pass * (kWave / kLanes) + lane / kLanes) * S::kOutLd +
            (lane % kLanes) * kVec;
        f32x8_t v[S::NB];
#pragma unroll
        for (int p = 0; p < S::NB; ++p) {
          const f32x4_t lo =
              *reinterpret_cast<const f32x4_t *>(src + p * S::WC);
          const f32x4_t hi =
              *reinterpret_cast<const f32x4_t *>(src + p * S::WC + 4);
          v[p] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
        if (row0 + down < g.m && in_n) {
          if (!g.to_parts)
            epi.at(view, down, v);
          else
            epi.partial(tile_sp, g.m, g.n, row0 + down, col, v);
        }
      }
      __builtin_amdgcn_wave_barrier();
    }
    if (!more) break;
    __syncthreads();  // the other stage is free again
    if (S::FAST) fetch(stages + (S::kStage - cur));
  }
}

// The parts of a split sum, added in order, through the epilogue.  kJoinAhead
// parts are loaded at once, and with SL > 1 a block's SL slices of 64 threads
// take every SL-th part and meet in LDS: one load after the other, the
// latencies would cost more than the product they end.
constexpr int kJoinAhead = 8;
constexpr int kJoinSlices = 16;
template <int NB, int SL, class Epi>
__global__ __launch_bounds__(64 * SL) void k_gemm_join(int32_t splits,
                                                       int32_t m, int32_t n,
                                                       Epi epi) {
  __shared__ f32x4_t meet[SL > 1 ? SL : 1][SL > 1 ? 2 * NB : 1][64];
  const int32_t per_row = (n + kVec - 1) / kVec;
  const int64_t items = (int64_t)m * per_row;
  const int64_t next = (int64_t)NB * m * n;  // from part to part
  const int lane = threadIdx.x % 64, slice = threadIdx.x / 64;
  // (a block's threads take the same number of steps)
  for (int64_t i0 = (int64_t)blockIdx.x * 64; i0 < items;
       i0 += (int64_t)gridDim.x * 64) {
    const int64_t it = i0 + lane;
    const int32_t row = (int32_t)(it / per_row);
    const int32_t col = (int32_t)(it % per_row) * kVec;
    const int32_t cnt = it < items ? n - col : 0;
    f32x8_t v[NB];
#pragma unroll
    for (int p = 0; p < NB; ++p) {
      const float *src = epi.part + ((int64_t)p * m + row) * n + col;
      f32x8_t sum = f32x8_t(0.0f);
      int32_t s = slice;
      if (cnt >= kVec) {
        for (; s + (kJoinAhead - 1) * SL < splits; s += kJoinAhead * SL) {
          f32x8_t t[kJoinAhead];
#pragma unroll
          for (int q = 0; q < kJoinAhead; ++q)
            t[q] =
                *reinterpret_cast<const f32x8_u *>(src + (s + q * SL) * next);
#pragma unroll
          for (int q = 0; q < kJoinAhead; ++q) sum += t[q];
        }
      }
      for (; s < splits; s += SL) sum += load8(src + s * next, cnt);
      v[p] = sum;
    }
    if constexpr (SL > 1) {
      __syncthreads();
#pragma unroll
      for (int p = 0; p < NB; ++p) {
        meet[slice][2 * p][lane] =
            __builtin_shufflevector(v[p], v[p], 0, 1, 2, 3);
        meet[slice][2 * p + 1][lane] =
            __builtin_shufflevector(v[p], v[p], 4, 5, 6, 7);
      }
      __syncthreads();
      if (slice) continue;
#pragma unroll
      for (int p = 0; p < NB; ++p) {
        f32x4_t lo = meet[0][2 * p][lane], hi = meet[0][2 * p + 1][lane];
#pragma unroll
        for (int t = 1; t < SL; ++t) {
          lo += meet[t][2 * p][lane];
          hi += meet[t][2 * p + 1][lane];
        }
        v[p] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
      }
    }
    if (cnt > 0) epi.at(epi.open(row, col, n), 0, v);
  }
}

// --- epilogues --------------------------------------------------------------
// open() gives a lane's view of kVec columns from col on, from a first row
// on: the bias and where its results go; at() applies the epilogue `down` rows
// further (uniform, so its addresses cost one addition).
template <int NB>
struct EpiParts {
  float *part;  // [split][product][m][n]
  __device__ __forceinline__ void partial(int32_t sp, int32_t m, int32_t n,
                                          int32_t row, int32_t col,
                                          const f32x8_t *v) const {
#pragma unroll
    for (int p = 0; p < NB; ++p)
      store8(part + (((int64_t)sp * NB + p) * m + row) * n + col, v[p],
             n - col);
  }
};

// y = act(acc + bias) + residual, z = acc + bias
struct EpiLinear : EpiParts<1> {
  const float *bias;
  const void *res;
  int64_t ldr;
  void *y;
  int64_t ldy;
  void *z;
  int64_t ldz;
  int32_t type, type_y, act;
  void shift(int64_t rows) {  // rows of D further on
    auto on = [&](const void *p, int64_t ld, int t) {
      return p ? (char *)p + rows * ld * (int64_t)type_bytes(t) : nullptr;
    };
    res = on(res, ldr, type_y);
    y = on(y, ldy, type_y);
    z = on(z, ldz, type);
  }
  struct Lane {
    f32x8_t bias;
    int64_t y, z, res;  // elements
    int32_t cnt;
  };
  __device__ __forceinline__ Lane open(int64_t row, int32_t col,
                                       int32_t n) const {
    Lane l;
    l.cnt = n - col;
    l.bias = bias ? load8(bias + col, l.cnt) : f32x8_t(0.0f);
    l.y = row * ldy + col;
    l.z = row * ldz + col;
    l.res = row * ldr + col;
    return l;
  }
  __device__ __forceinline__ void at(const Lane &l, int64_t down,
                                     f32x8_t *v) const {
    v[0] += l.bias;
    if (z) store8_t(z, l.z + down * ldz, type, v[0], l.cnt);
    f32x8_t o = act8(v[0], act);
    if (res) o += load8_t(res, l.res + down * ldr, type_y, l.cnt);
    store8_t(y, l.y + down * ldy, type_y, o, l.cnt);
  }
};

// h = act(acc0 + bias0) * (acc1 + bias1), and the two sums
template <class T>
struct EpiGated : EpiParts<2> {
  const float *bias[2];
  T *h, *gate, *up;
  int64_t ldh, lds;
  int32_t act;
  void shift(int64_t rows) {
    h += rows * ldh;
    if (gate) gate += rows * lds;
    if (up) up += rows * lds;
  }
  struct Lane {
    f32x8_t bias[2];
    int64_t h, s;
    int32_t cnt;
  };
  __device__ __forceinline__ Lane open(int64_t row, int32_t col,
                                       int32_t n) const {
    Lane l;
    l.cnt = n - col;
#pragma unroll
    for (int p = 0; p < 2; ++p)
      l.bias[p] = bias[p] ? load8(bias[p] + col, l.cnt) : f32x8_t(0.0f);
    l.h = row * ldh + col;
    l.s = row * lds + col;
    return l;
  }
  __device__ __forceinline__ void at(const Lane &l, int64_t down,
                                     f32x8_t *v) const {
    v[0] += l.bias[0];
    v[1] += l.bias[1];
    if (gate) store8(gate + l.s + down * lds, v[0], l.cnt);
    if (up) store8(up + l.s + down * lds, v[1], l.cnt);
    store8(h + l.h + down * ldh, act8(v[0], act) * v[1], l.cnt);
  }
};

// one or two plain results
template <class T, int NB>
struct EpiStore : EpiParts<NB> {
  T *out[NB];
  int64_t ld;
  void shift(int64_t rows) {
    for (T *&o : out)
      if (o) o += rows * ld;
  }
  struct Lane {
    int64_t at;
    int32_t cnt;
  };
  __device__ __forceinline__ Lane open(int64_t row, int32_t col,
                                       int32_t n) const {
    return {row * ld + col, n - col};
  }
  __device__ __forceinline__ void at(const Lane &l, int64_t down,
                                     f32x8_t *v) const {
#pragma unroll
    for (int p = 0; p < NB; ++p)
      if (out[p]) store8(out[p] + l.at + down * ld, v[p], l.cnt);
  }
};

// --- launch -----------------------------------------------------------------
inline bool fast_operand(const void *p, int64_t ld, int32_t contiguous,
                         int32_t bytes) {
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && ld * bytes % 16 == 0 &&
         contiguous * bytes % 16 == 0 && ld < kFastLd;
}

template <class S, class Epi>
void gemm_join(int32_t splits, int32_t m, int32_t n, const Epi &epi,
               hipStream_t st) {
  const int64_t items = (int64_t)m * ((n + kVec - 1) / kVec);
  const dim3 grid(
      (unsigned)std::min<int64_t>((items + 63) / 64, (int64_t)1 << 18));
  if (splits >= 2 * kJoinSlices)
    hipLaunchKernelGGL((k_gemm_join<S::NB, kJoinSlices, Epi>), grid,
                       dim3(64 * kJoinSlices), 0, st, splits, m, n, epi);
  else
    hipLaunchKernelGGL((k_gemm_join<S::NB, 1, Epi>), grid, dim3(64), 0, st,
                       splits, m, n, epi);
}

// parts_only: the sum's parts stay in epi.part, however many (a longer sum's
// share); returns their number.
template <class S, class Epi>
int32_t gemm_launch(GemmArgs<typename S::T> g, const Epi &epi, int32_t splits,
                    bool parts_only, hipStream_t st) {
  g.tiles_m = (g.m + S::BM - 1) / S::BM;
  g.tiles_n = (g.n + S::CN - 1) / S::CN;
  const int32_t kt = (g.k + S::kK - 1) / S::kK * (S::MODE == kSeq ? 2 : 1);
  g.kt_split = (kt + splits - 1) / splits;
  g.splits = (kt + g.kt_split - 1) / g.kt_split;  // no empty part
  g.to_parts = parts_only || g.splits > 1;
  const int64_t total = (int64_t)g.tiles_m * g.tiles_n * g.splits;
  // as many blocks as the chip holds at once
  static const int64_t slots = [] {
    int per_cu = 0;
    if (hipOccupancyMaxActiveBlocksPerMultiprocessor(
            &per_cu, (const void *)k_gemm<S, Epi>, S::NT, 0) != hipSuccess ||
        per_cu < 1)
      per_cu = 1;
    return (int64_t)per_cu * kCus;
  }();
  hipLaunchKernelGGL((k_gemm<S, Epi>),
                     dim3((unsigned)std::min<int64_t>(total, slots)),
                     dim3(S::NT), 0, st, g, epi);
  if (g.splits > 1 && !parts_only)
    gemm_join<S>(g.splits, g.m, g.n, epi, st);
  return g.splits;
}

// How a product is cut: its sum over k in `splits` parts, and the microseconds
// that takes by the model below.
struct Plan {
  int32_t splits;
  double us;
};

// The chip takes a launch's blocks in rounds of as many as its CUs hold.  A
// step brings (BM + BN) lines of 128 bytes from L2, which gives a CU 55 bytes
// a nanosecond when it holds one block and 69 when it holds more (17.7 TB/s in
// all), and multiplies for 1.47 us per 256 x 256 tile in bfloat16, 0.95 per
// 128 x 64 in fp32; the longer of the two counts.  So bfloat16 tiles of 128 x
// 128 are bound by L2 (0.6 us a step alone, 0.94 for two) and only those of
// 256 x 256 by the matrix cores.  Parts cost a second launch and 0.3 us a
// megabyte.  (512 x 4096 -> 4096: 44.5 us in one part, 33.6 in two, 31.1 in
// four, 42.3 in eight; 1024 x 1024 -> 1024: 12.9, 14.8 and 16.9 in one, two
// and four.)
//
// With 32 rows or fewer the weights' bytes are what takes time: 512 blocks of
// at least four steps (one token, 4096 -> 4096: 20.2 us in 4 parts, 13.5 in
// 8, 12.0 in 16).
template <class S>
Plan gemm_plan(const GemmArgs<typename S::T> &g, size_t part_bytes) {
  constexpr double kFetch = (S::BM + S::BN) * kLineBytes * 1e-3;  // KB
  constexpr double kMul = sizeof(typename S::T) == 4
                              ? 0.95 * S::BM * S::BN / (128 * 64)
                              : 1.47 * S::BM * S::BN / (256 * 256);
  constexpr int64_t per_cu = 160 * 1024 / S::kLds;
  constexpr double one = std::max(kFetch / 55.0, kMul);
  constexpr double full = per_cu * std::max(kFetch / 69.0, kMul);
  const int64_t tiles = (int64_t)((g.m + S::BM - 1) / S::BM) *
                        ((g.n + S::CN - 1) / S::CN);
  const int64_t kt = ((int64_t)g.k + S::kK - 1) / S::kK *
                     (S::MODE == kSeq ? 2 : 1);
  const double mat = 4.0 * g.m * g.n * S::NB;  // bytes of a part
  const int64_t fit = (int64_t)((double)part_bytes / mat);
  if (S::BM == 32) {
    int64_t s = std::min<int64_t>(2 * kCus / std::max<int64_t>(tiles, 1),
                                  kt / 4);
    s = std::max<int64_t>(std::min(s, fit), 1);
    return {(int32_t)s, 0.0};
  }
  Plan best = {1, 0.0};
  for (int64_t s = 1; s <= 512; s += std::max<int64_t>(s / 4, 1)) {
    if (s > 1 && (s > fit || s > kt / 4)) break;
    const int64_t work = tiles * s, slots = per_cu * kCus;
    const int64_t rest = work % slots;
    const double round = (double)(work / slots) * full +
                         (rest == 0      ? 0.0
                          : rest <= kCus ? one
                                         : full * ((rest + kCus - 1) / kCus) /
                                               per_cu);
    const double us = round * (double)((kt + s - 1) / s) +
                      (s > 1 ? 4.0 + 0.3e-6 * mat * (double)s : 0.0);
    if (s == 1 || us < best.us) best = {(int32_t)s, us};
  }
  return best;
}

// Tile of the block by the shape of D; f gets its Shape and the splits.
template <class T, bool AK, bool BK, int MODE, bool FAST, class F>
void gemm_shape(const GemmArgs<T> &g, size_t part_bytes, F f) {
#define EZSP_SHAPE(BM, BN, WM, WN) \
  Shape<T, BM, BN, WM, WN, AK, BK, MODE, FAST>
#define EZSP_GEMM(BM, BN, WM, WN)                                         \
  do {                                                                    \
    typedef EZSP_SHAPE(BM, BN, WM, WN) S;                                 \
    f(S{}, gemm_plan<S>(g, part_bytes).splits);                           \
    return;                                                               \
  } while (0)
  constexpr int kB = MODE == kDual ? 2 : 1;
  if (g.m <= 32) EZSP_GEMM(32, 128, 1, kB == 2 ? 2 : 4);
  if (g.n <= 32) EZSP_GEMM(128, 32 * kB, 4, 1);
  // fp32 is bound by its matrix instructions at any tile, so the tile is the
  // one that wastes the fewest (20,011 x 515: 785 tiles of 128 x 128 in two
  // rounds of 512, at 53 %; 1413 of 128 x 64 at 82 %)
  if constexpr (sizeof(T) == 4) {
    if constexpr (MODE == kDual)
      EZSP_GEMM(128, 64, 4, 1);
    else
      EZSP_GEMM(128, 64, 2, 2);
  }
  if (g.n * kB <= 64) EZSP_GEMM(128, 64, 4, 1);
  if constexpr (FAST && sizeof(T) == 2) {
    typedef EZSP_SHAPE(256, 256, 2, 4) L;
    typedef EZSP_SHAPE(128, 128, 2, 2) M;
    if (gemm_plan<L>(g, part_bytes).us < gemm_plan<M>(g, part_bytes).us)
      EZSP_GEMM(256, 256, 2, 4);
  }
  EZSP_GEMM(128, 128, 2, 2);
#undef EZSP_GEMM
#undef EZSP_SHAPE
}

// --- packing ----------------------------------------------------------------
// Rows [rows][cols] at any alignment into rows of ldp (a multiple of kVec)
// values, zero past cols.
template <class T>
__global__ __launch_bounds__(256) void k_pack(const T *__restrict__ src,
                                              int64_t ld, int32_t rows,
                                              int32_t cols,
                                              T *__restrict__ dst,
                                              int64_t ldp) {
  const int32_t per_row = (int32_t)(ldp / kVec);
  const int64_t items = (int64_t)rows * per_row;
  for (int64_t it = (int64_t)blockIdx.x * 256 + threadIdx.x; it < items;
       it += (int64_t)gridDim.x * 256) {
    const int32_t row = (int32_t)(it / per_row);
    const int32_t col = (int32_t)(it % per_row) * kVec;
    store8(dst + row * ldp + col, load8(src + row * ld + col, cols - col),
           kVec);
  }
}

template <class T>
void pack_launch(const T *src, int64_t ld, int32_t rows, int32_t cols, T *dst,
                 hipStream_t st) {
  const int64_t ldp = pad_row(cols);
  const int64_t items = (int64_t)rows * (ldp / kVec);
  hipLaunchKernelGGL(k_pack<T>,
                     dim3((unsigned)std::min<int64_t>((items + 255) / 256,
                                                      1 << 14)),
                     dim3(256), 0, st, src, ld, rows, cols, dst, ldp);
}

// D = A B through epi, whose parts lie in the part_bytes at epi.part.
//
// Operands at 16-byte alignment go past the registers into LDS, others
// through them, at half the rate in products that fill the chip.  There an
// unaligned operand is first packed into the same workspace, W whole and the
// long one in chunks of rows.  A copy of W costs next to nothing (20,000 x 512
// -> 515: 33 us for 45; 300,000 x 256 -> 100: 73 for 91).  One of the long
// operand costs 2 k e bytes a row, which 2 n k multiplications repay by n, the
// columns of all B together.  Products of 1.2e11 operations, rows three values
// longer than k, packed for unpacked, us:
//                        n = 256        384          512          1024
//   bf16, k = 64      1187 (1157)  1046 (1110)  1021 (1141)   947 (1075)
//        200           662  (645)   550  (597)   578  (628)   500  (555)
//        512           419  (384)   382  (360)   308  (379)   253  (339)
//   gated, k = 200     546  (568)   478  (522)   456  (550)   409  (485)
//   x^T dz with dx, k = 200
//                     1719 (1018)  1308  (926)   924  (905)   764  (905)
//   gated, 200        1708 (1067)               857  (883)   753  (932)
//   fp32 (a sixth of the operations), k = 512
//                      261  (225)                222  (202)   195  (200)
//   ... x^T dz with dx
//                      848  (540)                440  (517)   422  (510)
// So 512 columns, and forward 384 where k is short.
// Below kPackFlops the two differ by up to 6 us either way (4000 x 515 -> 515,
// bf16: 24 us packed, 25 as it lies, backward 48 and 53; fp32 57 and 52).
constexpr double kPackFlops = 4e9;
constexpr int32_t kPackN = 512;
constexpr int32_t kPackShortN = 384, kPackShortK = 256;
inline bool pack_pays(bool forward, int64_t k, int64_t n) {
  return n >= (forward && k <= kPackShortK ? kPackShortN : kPackN);
}

template <class T, bool AK, bool BK, int MODE, class Epi>
void gemm(GemmArgs<T> g, Epi epi, size_t part_bytes, hipStream_t st) {
  constexpr int32_t e = (int32_t)sizeof(T);
  constexpr int kB = MODE == kPlain ? 1 : 2;  // B matrices
  if (!g.ra) g.ra = g.m;
  if (!g.rb) g.rb = g.n;
  if (!g.ka) g.ka = g.k;
  if (!g.kb) g.kb = g.k;
  bool fast_a = fast_operand(g.a[0], g.lda, AK ? g.ka : g.ra, e);
  bool fast_b = fast_operand(g.b[0], g.ldb, BK ? g.kb : g.rb, e);
  if (MODE == kSeq)
    fast_a = fast_a && fast_operand(g.a[1], g.lda, AK ? g.ka : g.ra, e);
  if (MODE != kPlain)
    fast_b = fast_b && fast_operand(g.b[1], g.ldb, BK ? g.kb : g.rb, e);

  char *space = reinterpret_cast<char *>(epi.part);
  size_t room = part_bytes & ~(size_t)255;
  const double flops = 2.0 * g.m * g.n * (double)g.k * kB;
  if ((!fast_a || !fast_b) && flops >= kPackFlops &&
      (fast_a || (MODE != kSeq && pack_pays(AK, g.k, (int64_t)g.n * kB)))) {
    const int64_t b_rows = BK ? g.n : g.k, b_cols = BK ? g.k : g.n;
    const size_t b_bytes =
        fast_b ? 0 : (size_t)(b_rows * pad_row(b_cols)) * e * kB;
    if (b_bytes <= room / 2) {
      if (!fast_b) {
        room = (room - b_bytes) & ~(size_t)255;
        T *dst = reinterpret_cast<T *>(space + room);
        for (int p = 0; p < kB; ++p) {
          pack_launch(g.b[p], g.ldb, (int32_t)b_rows, (int32_t)b_cols,
                      dst + p * b_rows * pad_row(b_cols), st);
          g.b[p] = dst + p * b_rows * pad_row(b_cols);
        }
        g.ldb = pad_row(b_cols);
        (BK ? g.kb : g.rb) = (int32_t)g.ldb;
        fast_b = true;
      }
      // rows of A at a time that fit half of the room
      const int64_t a_rows = AK ? g.m : g.k, a_cols = AK ? g.k : g.m;
      const int64_t a_row = pad_row(a_cols) * e;
      const int64_t fit = (int64_t)(room / 2) / a_row / 256 * 256;
      if (!fast_a && (fit >= a_rows || fit >= 8192)) {
        const int64_t chunk = std::min(fit, a_rows);
        room = (room - (size_t)(chunk * a_row)) & ~(size_t)255;
        T *dst = reinterpret_cast<T *>(space + room);
        const T *src = g.a[0];
        const int64_t ld = g.lda;
        GemmArgs<T> c = g;
        c.a[0] = c.a[1] = dst;
        c.lda = pad_row(a_cols);
        (AK ? c.ka : c.ra) = (int32_t)c.lda;
        if (AK) {
          for (int64_t r = 0; r < a_rows; r += chunk) {
            c.m = c.ra = (int32_t)std::min(chunk, a_rows - r);
            pack_launch(src + r * ld, ld, c.m, (int32_t)a_cols, dst, st);
            gemm_shape<T, AK, BK, MODE, true>(c, room, [&](auto s, int32_t sp) {
              gemm_launch<decltype(s)>(c, epi, sp, false, st);
            });
            epi.shift(c.m);
          }
          return;
        }
        // chunks of the sum: their parts side by side, joined at the end
        gemm_shape<T, AK, BK, MODE, true>(g, room, [&](auto s, int32_t sp) {
          typedef decltype(s) S;
          const int64_t chunks = (a_rows + chunk - 1) / chunk;
          const size_t one = (size_t)g.m * g.n * S::NB * 4;
          const int64_t all = std::max<int64_t>(sp, chunks);
          const int64_t each = std::max<int64_t>(all / chunks, 1);
          if (room / one < (size_t)(each * chunks)) return;  // as they lie
          Epi at = epi;
          int32_t parts = 0;
          for (int64_t r = 0; r < a_rows; r += chunk) {
            c.k = c.ka = c.kb = (int32_t)std::min(chunk, a_rows - r);
            pack_launch(src + r * ld, ld, c.k, (int32_t)a_cols, dst, st);
            for (int p = 0; p < kB; ++p) c.b[p] = g.b[p] + r * g.ldb;
            at.part = epi.part + parts * (one / 4);
            parts += gemm_launch<S>(c, at, (int32_t)each, true, st);
          }
          gemm_join<S>(parts, g.m, g.n, epi, st);
          fast_a = true;
        });
        if (fast_a) return;
      }
    }
  }
  auto whole = [&](auto s, int32_t sp) {
    gemm_launch<decltype(s)>(g, epi, sp, false, st);
  };
  if (fast_a && fast_b)
    gemm_shape<T, AK, BK, MODE, true>(g, room, whole);
  else
    gemm_shape<T, AK, BK, MODE, false>(g, room, whole);
}

// --- gradients before their products ---------------------------------------
// Op::at gives the gradients of NB pre-activations at kVec neighbouring
// columns of a row, Op::put stores them; the column sums (the biases'
// gradients) are kept in registers over a block's rows, in fp32 and before
// any rounding, and joined over the block: part[p] is product p's row of m,
// stride from block row to block row, or the result itself where one block
// row takes all rows.
constexpr int kPrepNT = 256;
constexpr int kPrepCols = 16;                    // column groups of a block
constexpr int kPrepRows = kPrepNT / kPrepCols;   // rows of a step
constexpr int32_t kPrepParts = 512;

template <int NB, class Op>
__global__ __launch_bounds__(kPrepNT) void k_prep(Op op, int32_t n, int32_t m,
                                                  float *part0, float *part1,
                                                  int64_t stride) {
  __shared__ float red[kPrepNT / kWave][kPrepCols][kVec];
  const int cg = threadIdx.x % kPrepCols, rg = threadIdx.x / kPrepCols;
  const int32_t col = ((int32_t)blockIdx.x * kPrepCols + cg) * kVec;
  f32x8_t sum[NB];
#pragma unroll
  for (int p = 0; p < NB; ++p) sum[p] = f32x8_t(0.0f);
  if (col < m) {
    for (int64_t row = (int64_t)blockIdx.y * kPrepRows + rg; row < n;
         row += (int64_t)gridDim.y * kPrepRows) {
      f32x8_t v[NB];
      op.at(row, col, m - col, v);
      op.put(row, col, m - col, v);
#pragma unroll
      for (int p = 0; p < NB; ++p) sum[p] += v[p];
    }
  }
  if (!part0 && !part1) return;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
#pragma unroll
  for (int p = 0; p < NB; ++p) {
    float *part = p ? part1 : part0;
#pragma unroll
    for (int i = 0; i < kVec; ++i) {
      sum[p][i] += __shfl_xor(sum[p][i], 16, kWave);
      sum[p][i] += __shfl_xor(sum[p][i], 32, kWave);
      if (lane < kPrepCols) red[wave][cg][i] = sum[p][i];
    }
    __syncthreads();
    if (threadIdx.x < kPrepCols * kVec) {
      const int c = threadIdx.x / kVec, i = threadIdx.x % kVec;
      const int32_t at = ((int32_t)blockIdx.x * kPrepCols + c) * kVec + i;
      float t = 0.0f;
#pragma unroll
      for (int w = 0; w < kPrepNT / kWave; ++w) t += red[w][c][i];
      if (at < m && part) part[blockIdx.y * stride + at] = t;
    }
    __syncthreads();
  }
}

inline int32_t prep_parts(int64_t n) {
  return (int32_t)std::min<int64_t>((n + kPrepRows - 1) / kPrepRows,
                                    kPrepParts);
}

template <int NB, class Op>
void prep_launch(const Op &op, int32_t n, int32_t m, float *part,
                 float *db0, float *db1, hipStream_t st) {
  const bool sums = db0 || db1;
  // a few steps of one block row cost less than a second launch
  const int32_t parts = n <= 4 * kPrepRows && sums ? 1 : prep_parts(n);
  const bool join = sums && parts > 1;
  const int32_t bx = (m + kPrepCols * kVec - 1) / (kPrepCols * kVec);
  hipLaunchKernelGGL((k_prep<NB, Op>), dim3((unsigned)bx, (unsigned)parts),
                     dim3(kPrepNT), 0, st, op, n, m, join ? part : db0,
                     join ? part + m : db1, (int64_t)NB * m);
  if (join) join_rows(part, parts, NB * m, db0, db1, m, st);
}

// Bytes for the parts of a split product of m x n results: every part of a
// small product, at most 128 MiB (the splits then follow).  Grows with each
// argument.
inline size_t gemm_part_bytes(int64_t k, int64_t m, int64_t n, int products) {
  const int64_t parts = std::min<int64_t>(512, (k + 127) / 128 * products);
  const double want = 4.0 * (double)parts * (double)m * (double)n * products;
  return (size_t)std::min<double>(want, (double)((size_t)128 << 20)) + 256;
}

// Bytes that let a backward pass keep an aligned copy of x in half of them,
// where that is worth making, at most 256 MiB a product (x then goes in
// chunks).  Whether x is aligned is not known yet.
inline size_t gemm_pack_bytes(int64_t n, int64_t d_in, int64_t d_out,
                              int type, int products) {
  const double flops = 2.0 * (double)n * (double)d_in * (double)d_out *
                       products;
  if (flops < kPackFlops || !pack_pays(false, n, d_out * products)) return 0;
  const double want = 2.0 * (double)(n + 256) * (double)pad_row(d_in) *
                      (double)type_bytes(type);
  return (size_t)std::min<double>(
             want, (double)products * (double)((size_t)256 << 20)) + 512;
}

// The same for a forward product.  A sum of fewer than eight steps in either
// type is not split, and for so few columns W alone is packed, into the half
// of the space.
inline size_t gemm_fwd_bytes(int64_t n, int64_t d_in, int64_t d_out,
                             int products) {
  constexpr int64_t kUnsplit = 7 * kLineBytes / (int64_t)sizeof(float);
  const size_t parts = gemm_part_bytes(d_in, n, d_out, products);
  if (d_in > kUnsplit || pack_pays(true, d_in, d_out * products))
    return parts;
  const size_t w = (size_t)(products * d_in * pad_row(d_out)) * sizeof(float);
  return std::min(parts, 2 * w + 1024);
}

}  // namespace
}  // namespace ezsp
