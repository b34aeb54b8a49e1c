// ezsp_attn.h -- the kernels of cross attention, forward and backward:
//
//   S_ij = scale q_i . k_j + b_j, P_ij = exp(S_ij - lse_i), o_i = sum P_ij v_j
//   D_i = do_i . o_i, dS_ij = P_ij (do_i . v_j - D_i)
//   dq_i = scale sum dS_ij k_j, dk_j = scale sum dS_ij q_i, dv_j = sum P_ij do_i
//
// All three kernels have one form.  A block owns some columns (rows of q
// forward and for dq, keys for dk and dv), whose operands and sums stay in
// registers, and streams the other side, the lines, through LDS in tiles of
// R.  A product of two operands over d_head has the lines as its rows,
//   X[line][column] = sum over d of line[d] column[d],
// by v_mfma_f32_16x16x32_bf16 (fp32: v_mfma_f32_16x16x4_f32), so that a lane
// holds one column, lane % 16, and the lines 4 (lane / 16) + 0..3 of
// each 16: sums and maxima over the lines are sums over a lane's registers
// and two exchanges.  The second product, over the lines,
//   Y[d][column] = sum over lines of line[d] X[line][column],
// takes X as it stands: its k is the lines in the order in which a lane holds
// those of two tiles of 16, and the line tile is read across
// (ds_read_b64_tr_b16: four lines of a column of d a lane) in that order.  So
// no X goes through LDS.
//
// Heads that share a head of k and v are columns of the same block: column c
// of a cloud is row c / group of q, head c % group of the group.
//
// What bounds them, measured on one MI355X.  Short heads in bfloat16: vector
// instructions, since each score takes an exponential (a quarter of the rate),
// a fused product, an addition and half a conversion (forward of 1,265,474 x
// 613, 4 heads of 32: 1.75 million cycles, in 0.79 of them vector instructions
// issue, in 0.24 the matrix cores are busy; 736 us at the full clock, 870 at
// that of a chip that has rested).  Long heads: the matrix cores, at 0.7 of a
// large library product's rate where rows and keys are many (400,000 x 3000:
// heads of 128 and 64 at 890 to 920 TFLOP/s; gradients 820 to 1040), less where
// clouds are small and uneven.  fp32: its matrix instructions (busy in 0.63 to
// 0.69 of the cycles in gradients of 20,011 x 3511 in eleven clouds).  One row:
// latency (8192 keys, 32 heads on 8 of 128: 16 us, 13 and 4 in the kernels, 2.5
// TB/s: one of a block's waves has columns, and its two tiles of keys come one
// after the other).
#pragma once

#include <math.h>

#include <algorithm>
#include <type_traits>

#include "ezsp_dense.h"

namespace ezsp {
namespace {

typedef short s16x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));
typedef bf16x4_t bf16x4_u __attribute__((aligned(2)));
typedef f32x4_t f32x4_u __attribute__((aligned(4)));
typedef __attribute__((address_space(3))) char lds_byte;

// d_head comes in blocks of 16, B of them, in lines of this length.
constexpr int width_of(int b) { return b <= 2 ? 32 : b <= 4 ? 64 : 128; }

constexpr int kAttnNT = 256;
constexpr int kAttnWaves = kAttnNT / kWave;
constexpr float kLog2e = 1.44269504f, kLn2 = 0.69314718f;
constexpr float kBiasMask = 268435456.0f;  // 2^28: a mask, as -inf is

// Operands of a lane.  LineFrag: eight lines of a column of d, the second
// product's.  The first product's k is d, up to 16 B: bfloat16 takes 32 of it
// a step, eight to a lane; fp32 four values a lane and step, of the 4 B that
// are the lane's (any order of k does, if both operands have it).
template <class T, int B>
struct FragsOf;
template <int B>
struct FragsOf<__bf16, B> {
  typedef bf16x8_t Along, Line;
  static constexpr int kSteps = (B + 1) / 2, kEach = 8;
  static __device__ __forceinline__ int d(int step, int g) {
    return 32 * step + 8 * g;
  }
};
template <int B>
struct FragsOf<float, B> {
  typedef f32x4_t Along;
  typedef f32x8_t Line;
  static constexpr int kSteps = B, kEach = 4;
  static __device__ __forceinline__ int d(int step, int g) {
    return 4 * (B * g + step);
  }
};
template <class T>
using frag_t = typename FragsOf<T, 1>::Line;

__device__ __forceinline__ f32x4_t mma16(bf16x8_t a, bf16x8_t b, f32x4_t c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4_t mma16(f32x4_t a, f32x4_t b, f32x4_t c) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}
__device__ __forceinline__ f32x4_t mma16(f32x8_t a, f32x8_t b, f32x4_t c) {
#pragma unroll
  for (int e = 0; e < 8; ++e)
    c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[e], b[e], c, 0, 0, 0);
  return c;
}

// eight fp32 values as an operand: the one rounding of P and dS
template <class T>
__device__ __forceinline__ frag_t<T> to_frag(f32x4_t lo, f32x4_t hi) {
  const f32x8_t v = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  return __builtin_convertvector(v, frag_t<T>);
}

// cnt (at most 8) elements from p on, the rest 0
__device__ __forceinline__ bf16x8_t load_frag(const __bf16 *p, int cnt) {
  if (cnt >= 8) return *reinterpret_cast<const bf16x8_u *>(p);
  bf16x8_t r;
#pragma unroll
  for (int i = 0; i < 8; ++i) r[i] = i < cnt ? p[i] : (__bf16)0.0f;
  return r;
}
__device__ __forceinline__ f32x8_t load_frag(const float *p, int cnt) {
  return load8(p, cnt);
}
// a step's piece of a row of dh values, or zeros
template <int B>
__device__ __forceinline__ bf16x8_t load_along(const __bf16 *p, int step,
                                               int g, int dh) {
  const int d = FragsOf<__bf16, B>::d(step, g);
  return load_frag(p + d, dh - d);
}
template <int B>
__device__ __forceinline__ f32x4_t load_along(const float *p, int step, int g,
                                              int dh) {
  const int d = FragsOf<float, B>::d(step, g);
  if (d + 4 <= dh) return *reinterpret_cast<const f32x4_u *>(p + d);
  f32x4_t r = {0, 0, 0, 0};
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (d + i < dh) r[i] = p[d + i];
  return r;
}

// the first cnt (at most 4) of v to p
__device__ __forceinline__ void store4(__bf16 *p, f32x4_t v, int cnt) {
  const bf16x4_t b = __builtin_convertvector(v, bf16x4_t);
  if (cnt >= 4) {
    *reinterpret_cast<bf16x4_u *>(p) = b;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < cnt) p[i] = b[i];
  }
}
__device__ __forceinline__ void store4(float *p, f32x4_t v, int cnt) {
  if (cnt >= 4) {
    *reinterpret_cast<f32x4_u *>(p) = v;
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < cnt) p[i] = v[i];
  }
}

// Lines of D elements, a power of two, in LDS, placed so that 16 lines read
// along, or four groups of four read across, have all banks once (16 pieces of
// 16 bytes).  Lines of 256 bytes and more lie an odd number of pieces apart, the
// pieces of shorter ones are exchanged by the line's number.  (Exchanged, the
// pieces of long lines took two dozen registers for their addresses, which are
// offsets of one otherwise: backward of 16,384 x 12,288 in eight clouds, 16
// heads of 128 on 4: 970 us, 1066 exchanged.  Short lines apart: nothing,
// 1,265,474 x 613, 4 of 32 2282 us and 2271.)  What the banks make of it, in
// short kernels of one access each, against the 4 cycles of an instruction of
// 64 pieces in a row: bfloat16 across and put meet none twice, along takes 8 in
// every layout, so its lanes are not served 16 in turn; fp32 across takes the
// least (half as much again for lines of 32 elements), along and put twice it.
template <class T, int D>
struct Lines {
  static constexpr int kPieces = D * (int)sizeof(T) / 16;
  static constexpr bool kApart = kPieces >= 16;
  static constexpr bool kHalf = sizeof(T) == 2;
  static constexpr int kBytes = 16 * (kPieces + (kApart ? kHalf ? 2 : 1 : 0));
  static constexpr int kPer = kApart ? 1 : 16 / kPieces;
  static __device__ __forceinline__ uint32_t at(int line, int piece) {
    if constexpr (kApart) {
      if constexpr (kHalf) piece += line >> 3 & 1;
    } else {
      int by = line / kPer;
      if constexpr (kHalf) by = 2 * by | (by & kPieces - 1) / (kPieces / 2);
      piece ^= by & (kPieces - 1);
    }
    return (uint32_t)(line * kBytes + piece * 16);
  }
  // step i of a line's d, up to 16 B
  template <int B>
  static __device__ __forceinline__ typename FragsOf<T, B>::Along along(
      const char *t, int line, int i, int g) {
    const int piece = FragsOf<T, B>::d(i, g) * (int)sizeof(T) / 16;
    return *reinterpret_cast<const typename FragsOf<T, B>::Along *>(
        t + at(line, piece));
  }
  // d 16 b + lane % 16 of the lines first + 4 (lane / 16) + 0..3 and of
  // those 16 further on (whose pieces are exchanged alike)
  static __device__ __forceinline__ frag_t<T> across(const char *t, int first,
                                                     int b, int lane) {
    const int g = lane >> 4, i = lane & 15;
    if constexpr (sizeof(T) == 2) {
      const int line = first + 4 * g + (i >> 2);
      const uint32_t o = at(line, 2 * b + ((i & 3) >> 1)) + 8 * (i & 1);
      typedef __attribute__((address_space(3))) s16x4_t *ptr;
      const s16x4_t lo =
          __builtin_amdgcn_ds_read_tr16_b64_v4i16((ptr)(lds_byte *)(t + o));
      const s16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          (ptr)(lds_byte *)(t + o + 16 * kBytes));
      return __builtin_bit_cast(
          bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    } else {
      f32x8_t v;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int line = first + 16 * (j / 4) + 4 * g + j % 4;
        v[j] = *reinterpret_cast<const float *>(
            t + at(line, 4 * b + (i >> 2)) + 4 * (i & 3));
      }
      return v;
    }
  }
  template <int B>
  static __device__ __forceinline__ void put_along(
      char *t, int line, int i, int g, typename FragsOf<T, B>::Along v) {
    const int piece = FragsOf<T, B>::d(i, g) * (int)sizeof(T) / 16;
    *reinterpret_cast<typename FragsOf<T, B>::Along *>(t + at(line, piece)) =
        v;
  }
  static __device__ __forceinline__ void put(char *t, int line, int q,
                                             bf16x8_t v) {
    *reinterpret_cast<bf16x8_t *>(t + at(line, q)) = v;
  }
  static __device__ __forceinline__ void put(char *t, int line, int q,
                                             f32x8_t v) {
    *reinterpret_cast<f32x4_t *>(t + at(line, 2 * q)) =
        __builtin_shufflevector(v, v, 0, 1, 2, 3);
    *reinterpret_cast<f32x4_t *>(t + at(line, 2 * q + 1)) =
        __builtin_shufflevector(v, v, 4, 5, 6, 7);
  }
};

// A block's part of the way from memory to a tile of R lines: each thread
// moves kCh pieces of eight elements through its registers, always the same
// ones of a line, kStep lines apart.
template <class T, int D, int R>
struct Mover {
  static constexpr int kOcts = D / 8;
  static constexpr int kCh = R * kOcts / kAttnNT;
  static constexpr int kStep = kAttnNT / kOcts;
  static_assert(R * kOcts % kAttnNT == 0, "whole pieces");
  frag_t<T> reg[kCh];
  static __device__ __forceinline__ int line() {
    return (int)threadIdx.x / kOcts;
  }
  static __device__ __forceinline__ int d() {
    return (int)threadIdx.x % kOcts * 8;
  }
  // at(ch): the piece's first element; live(ch): it is read, else zeros.
  // cnt elements of it exist.
  template <class P, class F>
  __device__ __forceinline__ void load(P at, F live, int cnt) {
#pragma unroll
    for (int ch = 0; ch < kCh; ++ch) {
#pragma unroll
      for (int i = 0; i < 8; ++i) reg[ch][i] = (T)0.0f;
      if (cnt > 0 && live(ch)) reg[ch] = load_frag(at(ch), cnt);
    }
  }
  __device__ __forceinline__ void put(char *t) const {
#pragma unroll
    for (int ch = 0; ch < kCh; ++ch)
      Lines<T, D>::put(t, line() + ch * kStep, d() / 8, reg[ch]);
  }
};

struct Attn {
  const void *q, *k, *v;
  int64_t ldq, ldk, ldv;
  int32_t nq, nk, heads, kv_heads, group, dh;
  uint32_t group_inv;             // ceil(2^32 / group), group > 1
  const int32_t *q_off, *k_off;   // nullable
  int32_t clouds;                 // 1 without offsets, else n_clouds + 2
  const float *bias;              // nullable
  float scale, c;                 // c = scale log2(e)
  float inv_scale;
  int32_t tiles;                  // of columns
  int32_t stripe;                 // XCDs that share heads in a batch
  int32_t splits, chunk;          // parts of the lines at most, lines of one
  void *out;
  int64_t ldo;
  float *lse;                     // forward: nullable
  // backward
  const void *dout;
  int64_t lddo;
  float *delta;                   // D, heads * nq: workspace
  void *dq, *dk, *dv;
  int64_t lddq, lddk, lddv;
  float *part;                    // workspace: sums of splits
};

// What the kernels take of a call.
inline Attn attn_of(const AttnArgs &a) {
  Attn g = {};
  g.q = a.q;
  g.ldq = a.ldq;
  g.nq = a.nq;
  g.k = a.k;
  g.ldk = a.ldk;
  g.v = a.v;
  g.ldv = a.ldv;
  g.nk = a.nk;
  g.heads = a.heads;
  g.kv_heads = a.kv_heads;
  g.group = a.heads / a.kv_heads;
  g.dh = a.dh;
  g.group_inv = (uint32_t)((((uint64_t)1 << 32) + g.group - 1) / g.group);
  g.q_off = a.q_off;
  g.k_off = a.k_off;
  g.clouds = a.q_off ? a.n_clouds + 2 : 1;
  g.bias = a.bias;
  g.scale = a.scale;
  g.c = a.scale * kLog2e;
  g.inv_scale = 1.0f / a.scale;
  g.splits = 1;
  g.stripe = kXcd;
  while (g.stripe > 1 && g.kv_heads % (2 * kXcd / g.stripe) == 0)
    g.stripe /= 2;
  g.out = a.out;
  g.ldo = a.ldo;
  g.lse = a.lse;
  g.dout = a.dout;
  g.lddo = a.lddo;
  g.delta = a.delta;
  g.dq = a.dq;
  g.lddq = a.lddq;
  g.dk = a.dk;
  g.lddk = a.lddk;
  g.dv = a.dv;
  g.lddv = a.lddv;
  g.part = a.part;
  return g;
}

constexpr int kMaxSplits = 64;  // a lane of the join each
constexpr int64_t kPartFloats = (int64_t)64 << 20;  // of the parts' sums
constexpr int64_t kLeastLines = 32;                 // of a part: a tile's
constexpr int64_t kCus = 256;                       // of an MI355X

// The parts of a call's lines: `cols` columns of each head of k in blocks of
// `per`, `lines` in all, at least `least` to a part, `floats` of sums from
// each part.  The time of s parts, in lines of a block at full speed:
//   - of one cloud, the rounds in which `slots` blocks at once take them;
//   - of a batch, whose lines fall on its clouds as nobody here knows, all of
//     the work spread evenly, and a long cloud's part at its end;
//   - 8 or 16 bytes of sums a column and d written and read at some 4 TB/s,
//     next to a line's 4 to 8 operations at 850 (fp32 110) TFLOP/s: 400 to 600
//     (50) lines a block and part, less for blocks with few columns;
//   - 5 lines a part for the join's one look after the other.
// bfloat16 needs two blocks a CU for its full speed, fp32, bound by its matrix
// instructions, one.  A batch's parts have one length, so that a long cloud has
// more of them, up to twice a mean one's.  (Backward of 16,384 x 12,288 in
// eight clouds of one to six lengths, 16 heads of 128 on 4, three drawings: 966,
// 1058 and 1017 us, 1172, 1342 and 1344 with each cloud whole; 20,011 x 3511 in
// eleven, 6 heads of 40 in fp32: 346, 338 and 344, and 446, 508 and 516.  With
// up to four times a mean one's nothing changes.)  attn_reserve
// counts with at most 2 lines / kLeastLines parts.
template <class T>
void plan_parts(Attn &g, int64_t cols, int64_t per, int64_t lines,
                int64_t least, int64_t floats) {
  const bool batch = g.q_off != nullptr;
  const int64_t clouds = batch ? g.clouds - 2 : 1;
  const double full = (double)cols / (double)((cols + per - 1) / per * per);
  const double part = (sizeof(T) == 2 ? batch ? 600.0 : 400.0 : 50.0) * full;
  const double slots = (double)(sizeof(T) == 2 ? 2 * kCus : kCus);
  // (of a batch the clouds' last blocks, half empty)
  const double blocks = (double)((cols + per - 1) / per * g.kv_heads +
                                 (batch ? clouds * g.kv_heads / 2 : 0));
  const double mean = (double)lines / (double)clouds;
  const int64_t most = std::max<int64_t>(
      1, std::min<int64_t>(kMaxSplits, std::min(lines / clouds / least,
                                                kPartFloats / floats)));
  int64_t best = 1;
  double shortest = 0.0;
  for (int64_t s = 1; s <= most; ++s) {
    const double rounds = ceil(blocks * s / slots);
    const double time =
        (batch ? mean * (blocks / slots + 1.6 / s) : mean * rounds / s) +
        (s > 1 ? part * blocks * s / slots + 5.0 * s : 0.0);
    if (s == 1 || time < 0.95 * shortest) {
      best = s;
      shortest = time;
    }
  }
  g.splits = (int32_t)best;
  if (batch && best > 1)
    g.splits = (int32_t)std::min<int64_t>(
        2 * best, std::min<int64_t>(kMaxSplits, kPartFloats / floats));
  g.chunk = (int32_t)((lines + clouds * best - 1) / (clouds * best));
}

// Whether blocks of `wide` columns, too few for the chip, fill it where their
// lines come in parts, so that waves need not have 16 columns alone, for which
// each tile is read from LDS twice as often.  Parts of 1024 lines; no more than
// a sixteenth of such a block's columns beyond those of halves of it; not for
// batches in fp32, whose clouds end in half empty blocks of more matrix
// instructions.  (Gradients of keys, by waves of 16 and of 32 columns:
// 1,265,474 x 613, 4 heads of 32: 2014 and 1418 us; 400,000 x 3000, 8 of 128:
// 17.5 and 11.8 ms; 20,000 x 613, 8 of 64: 111 and 90; 100,000 x 100, 8 of 64:
// 141 and 130; of 100 keys, 256 blocks with parts: 568 and 603; fp32, 100,000 x
// 2000, 8 of 64: 10.3 and 7.7 ms; 100,000 x 2400 in eight clouds, 8 of 48: 956
// and 1220.  2000 rows to 100,000 keys each, 8 heads of 64: forward 910 and 507,
// dq 1064 and 722.)
template <class T>
bool parts_fill(const Attn &g, int64_t cols, int64_t wide, int64_t lines) {
  if (g.q_off && sizeof(T) == 4) return false;
  const int64_t clouds = g.q_off ? g.clouds - 2 : 1;
  const int64_t blocks = (cols + wide - 1) / wide;
  const int64_t half = (2 * cols + wide - 1) / wide;  // halves of them
  return blocks * 32 <= half * 17 &&
         blocks * g.kv_heads *
                 std::min<int64_t>(kMaxSplits, lines / clouds / 1024) >=
             2 * kCus;
}

// Cloud s of the call's: its rows and keys.  With offsets the rows before
// the first and behind the last are clouds of their own, without the other
// side, so that every row is some cloud's.
struct Cloud {
  int32_t q0, q1, k0, k1;
};
__device__ __forceinline__ int32_t edge(const int32_t *off, int32_t clouds,
                                        int32_t s, int32_t n) {
  if (s <= 0) return 0;
  if (s >= clouds) return n;
  return min(max(off[s - 1], 0), n);
}
template <bool KEYS>  // the columns are keys
__device__ __forceinline__ Cloud cloud_of(const Attn &a, int32_t s) {
  if (!a.q_off) return {0, a.nq, 0, a.nk};
  Cloud c = {edge(a.q_off, a.clouds, s, a.nq),
             edge(a.q_off, a.clouds, s + 1, a.nq),
             edge(a.k_off, a.clouds, s, a.nk),
             edge(a.k_off, a.clouds, s + 1, a.nk)};
  if (s == 0 || s == a.clouds - 1) {
    if (KEYS)
      c.q1 = c.q0;
    else
      c.k1 = c.k0;
  }
  return c;
}
// Tiles of `per` columns are numbered so that cloud s, whose first column is
// f_s, has the tiles from floor(f_s / per) + s on: as many as it can need,
// and the numbers can be told without a sum over the clouds.  This is the
// cloud of a tile, by 64 lanes looking at once.
__device__ __forceinline__ int32_t find_cloud(const int32_t *off,
                                              int32_t clouds, int32_t n,
                                              int32_t group, int32_t per,
                                              int32_t tile) {
  int32_t lo = 0, hi = clouds;
  while (hi - lo > 1) {
    const int32_t step = (hi - lo + kWave - 1) / kWave;
    const int32_t s = lo + (int32_t)(threadIdx.x % kWave) * step;
    const bool before =
        s < hi && edge(off, clouds, s, n) * group / per + s <= tile;
    const int32_t cnt = max(__popcll(__ballot(before)), 1);
    lo += (cnt - 1) * step;
    hi = min(hi, lo + step);
  }
  return lo;
}

// bias / scale of a key, as the sums of q k start: a key that is not there or
// is masked has -inf.
__device__ __forceinline__ float start_of(const Attn &a, int32_t key,
                                          int32_t end) {
  if (key >= end) return -INFINITY;
  if (!a.bias) return 0.0f;
  const float s = a.bias[key] * a.inv_scale;
  return s <= -kBiasMask ? -INFINITY : s;
}

// The columns of a lane: rows of q, or keys.
struct Column {
  int32_t row, head;   // head of the group; row < 0: none
};
__device__ __forceinline__ Column q_column(const Attn &a, const Cloud &cl,
                                           int32_t c) {
  const int32_t len = (cl.q1 - cl.q0) * a.group;
  if (c >= len) return {-1, 0};
  // c / group by the product with ceil(2^32 / group), which is one too large
  // at most (c < 2^31)
  int32_t r = c;
  if (a.group > 1) {
    r = (int32_t)(((uint64_t)(uint32_t)c * a.group_inv) >> 32);
    if ((uint32_t)r * (uint32_t)a.group > (uint32_t)c) --r;
  }
  return {cl.q0 + r, c - r * a.group};
}

constexpr int kFewUnits = 32;  // in order: some XCDs would have none

// A launch has fewer than 2^32 threads along x, so that more than kGridRow
// blocks come in rows (whole rounds of the XCDs); those behind the last do
// nothing.
constexpr unsigned kGridRow = 1u << 23;
inline dim3 grid_of(unsigned blocks) {
  if (blocks <= kGridRow) return dim3(blocks);
  return dim3(kGridRow, (blocks + kGridRow - 1) / kGridRow);
}
__device__ __forceinline__ uint32_t block_number() {
  return blockIdx.y * gridDim.x + blockIdx.x;
}

// The block's columns and part.  Without clouds in runs for each XCD (as
// xcd_block), the parts of a tile after each other.  In a batch the tiles' work
// is their clouds': the XCDs come in groups of `stripe`, each group has some of
// the heads whole, and its XCDs take their tiles in turn, so that each has its
// share of every cloud and a head's lines pass through few L2s (backward of
// 16,384 x 12,288 in eight clouds, 16 heads of 128 on 4, three drawings: 966,
// 1058 and 1017 us, in runs 971, 1107 and 1062, with all tiles in turn over all
// XCDs 1005, 1083 and 1079).  And all tiles have their first
// part before any has its second, so that the parts which a cloud has not end
// together: in a row they fell on the same CUs each time and left the work to
// the others (dq of 20,011 x 3511 in eleven clouds, two of them in two parts of
// four: 377 us, whole 153).
__device__ __forceinline__ bool unit_of(const Attn &a, int32_t &tile,
                                        int32_t &kvh, int32_t &split) {
  const int32_t units = a.tiles * a.kv_heads;
  const uint32_t block = block_number();
  const int32_t x = (int32_t)(block % kXcd), j = (int32_t)(block / kXcd);
  int32_t u;
  if (!a.q_off) {
    const int32_t per = (units * a.splits + kXcd - 1) / kXcd;
    if (j >= per) return false;
    const int32_t b = x * per + j;
    u = b / a.splits;
    split = b % a.splits;
  } else if (units < kFewUnits) {
    u = (int32_t)block % units;
    split = (int32_t)block / units;
  } else {
    const int32_t per = (units + kXcd - 1) / kXcd;
    split = j / per;
    const int32_t each = units / (kXcd / a.stripe);
    const int32_t v = j % per * a.stripe + x % a.stripe;
    u = v < each ? x / a.stripe * each + v : units;
  }
  tile = u % a.tiles;
  kvh = u / a.tiles;
  return u < units && split < a.splits;
}
inline unsigned attn_grid(const Attn &a) {
  const int64_t units = (int64_t)a.tiles * a.kv_heads;
  if (!a.q_off) return xcd_grid(units * a.splits);
  return (units < kFewUnits ? (unsigned)units : xcd_grid(units)) *
         (unsigned)a.splits;
}

// Parts that so many lines of a cloud come in.
__device__ __forceinline__ int32_t parts_of(const Attn &a, int32_t lines) {
  if (a.splits == 1 || lines <= a.chunk) return 1;
  return min(a.splits, (lines - 1) / a.chunk + 1);
}
// The cloud of a row or key, for the kernels that add the parts.
__device__ __forceinline__ int32_t cloud_at(const int32_t *off,
                                            int32_t clouds, int32_t n,
                                            int32_t row) {
  int32_t lo = 0, hi = clouds;
  while (off && hi - lo > 1) {
    const int32_t mid = lo + (hi - lo) / 2;
    if (edge(off, clouds, mid, n) <= row)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// Part `split` of the lines [first, last), whole tiles of R.
template <int R>
__device__ __forceinline__ void part_of(int32_t first, int32_t last,
                                        int32_t split, int32_t splits,
                                        int32_t &begin, int32_t &end) {
  const int32_t tiles = (max(last - first, 0) + R - 1) / R;
  const int32_t each = (tiles + splits - 1) / splits;
  begin = first + min(split * each, tiles) * R;
  end = min(last, first + min((split + 1) * each, tiles) * R);
}

// The keys of a head on their way to LDS: tiles of R from `first` to `end`,
// k, v and what the scores start from.
template <class T, int D, int R>
struct KeyStream {
  typedef Mover<T, D, R> M;
  static_assert(R <= kWave, "the first wave fetches a tile's starts");
  M k, v;
  const T *kp, *vp;     // this thread's piece of the next tile
  int32_t key, end;     // the next tile's first key
  int cnt;
  float start;
  bool seen;            // a key that is there and not masked
  __device__ __forceinline__ KeyStream(const Attn &a, int32_t kvh,
                                       int32_t first, int32_t end)
      : key(first), end(end), seen(false) {
    const int64_t at = (int64_t)kvh * a.dh + M::d();
    const int64_t row = first + M::line();
    kp = static_cast<const T *>(a.k) + row * a.ldk + at;
    vp = static_cast<const T *>(a.v) + row * a.ldv + at;
    cnt = a.dh - M::d();
  }
  __device__ __forceinline__ void load(const Attn &a) {
    uint32_t live = 0;
#pragma unroll
    for (int ch = 0; ch < M::kCh; ++ch)
      if (start_of(a, key + M::line() + ch * M::kStep, end) != -INFINITY)
        live |= 1u << ch;
    auto is = [&](int ch) { return (live >> ch & 1) != 0; };
    k.load([&](int ch) { return kp + (int64_t)(ch * M::kStep) * a.ldk; }, is,
           cnt);
    v.load([&](int ch) { return vp + (int64_t)(ch * M::kStep) * a.ldv; }, is,
           cnt);
    if (threadIdx.x < R) {
      start = start_of(a, key + (int)threadIdx.x, end);
      seen |= start != -INFINITY;
    }
    key += R;
    kp += R * a.ldk;
    vp += R * a.ldv;
  }
  __device__ __forceinline__ void put(char *tk, char *tv, float *starts) const {
    k.put(tk);
    v.put(tv);
    if (threadIdx.x < R) starts[threadIdx.x] = start;
  }
};

// What the sums of a score start from, and what is added to the finished sum:
// bfloat16 scores start from the key's term, which costs nothing; in fp32 the
// roundings of each step would then be those of the larger sum, and it is
// added once.
template <class T>
__device__ __forceinline__ f32x4_t sums_from(f32x4_t start) {
  return sizeof(T) == 2 ? start : f32x4_t{0, 0, 0, 0};
}
template <class T>
__device__ __forceinline__ f32x4_t sums_done(f32x4_t s, f32x4_t start) {
  return sizeof(T) == 2 ? s : s + start;
}

__device__ __forceinline__ float lanes16_max(float v) {
  v = fmaxf(v, __shfl_xor(v, 16, kWave));
  return fmaxf(v, __shfl_xor(v, 32, kWave));
}
__device__ __forceinline__ float lanes16_sum(float v) {
  v += __shfl_xor(v, 16, kWave);
  return v + __shfl_xor(v, 32, kWave);
}

// --- forward -----------------------------------------------------------------

// Groups of 16 columns a wave and keys a tile: as the registers of two waves a
// SIMD hold, of three with short heads, whose exponentials are the work
// (1,265,474 x 613 with a bias, 4 heads of 32: 3 groups of columns 765 us, 4
// 831, 2 780, without one 722, 764 and 706; 400,000 x 3000, 8 of 32: 1817, 1932
// and 1863; 100,000 x 2000, 8 of 48: 451, 493 and 462; of 64: 4 groups 501, 3
// 555).  With few columns, unless parts of their keys fill the chip, one group
// (of wide heads with tiles that leave LDS for three blocks a CU: 64 rows to
// 2000 keys each, 8 heads of 128: 105 us with tiles of 32, 113 with 64).
template <class T, int B>
struct ForwardShape {
  static constexpr bool kBf = sizeof(T) == 2;
  static constexpr int kGroups =
      kBf ? (B <= 3 ? 3 : B == 4 ? 4 : 2) : (B <= 4 ? 2 : 1);
  static constexpr int kKeys = B <= 2 || (kBf && B > 4) ? 64 : 32;
  static constexpr int kFewKeys = B <= 2 || (kBf && B <= 4) ? 64 : 32;
};

constexpr float kGrown = 4096.0f;

// P = 2^(S c - mc) of a lane's scores as operands, and its sum over them
// before they are rounded.
template <class T, int RT>
__device__ __forceinline__ float powers(const f32x4_t (&s)[RT], float c,
                                        float mc, frag_t<T> (&p)[RT / 2]) {
  float sum = 0.0f;
#pragma unroll
  for (int t = 0; t < RT; t += 2) {
    f32x4_t e[2];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        e[h][r] =
            __builtin_amdgcn_exp2f(__builtin_fmaf(s[t + h][r], c, -mc));
        sum += e[h][r];
      }
    p[t / 2] = to_frag<T>(e[0], e[1]);
  }
  return sum;
}

// NC groups of 16 columns a wave; tiles of R keys.  The running maximum m and
// sum l of a column are those of scores before `scale`.  splits > 1: each
// takes a part of the cloud's keys and leaves its sums to k_attn_join.
template <class T, int B, int NC, int R, int W = 2>
__global__ __launch_bounds__(kAttnNT, W) void k_attn_fwd(Attn a) {
  constexpr int D = width_of(B);
  typedef Lines<T, D> L;
  typedef FragsOf<T, B> F;
  typedef typename F::Along Along;
  constexpr int kCols = kAttnWaves * 16 * NC;
  constexpr int kTile = R * L::kBytes;
  constexpr int kDb = B, kDs = F::kSteps, kRt = R / 16;
  __shared__ __attribute__((aligned(16))) char lds[2][2][kTile];
  __shared__ __attribute__((aligned(16))) float start[2][R];
  __shared__ bool any_key;
  int32_t tile, kvh, split;
  if (!unit_of(a, tile, kvh, split)) return;
  const int32_t cloud =
      a.q_off ? find_cloud(a.q_off, a.clouds, a.nq, a.group, kCols, tile) : 0;
  const Cloud cl = cloud_of<false>(a, cloud);
  const int32_t base =
      (a.q_off ? cl.q0 * a.group / kCols + cloud : 0);
  const int32_t first = (tile - base) * kCols;
  if (first < 0 || first >= (cl.q1 - cl.q0) * a.group) return;
  const int32_t parts = parts_of(a, cl.k1 - cl.k0);
  if (split >= parts) return;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int g = lane >> 4;
  const int32_t dh = a.dh;

  Column col[NC];
  Along qf[NC][kDs];
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    col[n] = q_column(a, cl, first + (wave * NC + n) * 16 + (lane & 15));
    const bool live = col[n].row >= 0;
    const T *qp = static_cast<const T *>(a.q) +
                  (live ? col[n].row * a.ldq +
                              (int64_t)(kvh * a.group + col[n].head) * dh
                        : 0);
#pragma unroll
    for (int s = 0; s < kDs; ++s)
      qf[n][s] = load_along<B>(qp, s, g, live ? dh : 0);
  }
  f32x4_t o[NC][kDb];
  float m[NC], l[NC];
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    m[n] = -1e30f;
    l[n] = 0.0f;
#pragma unroll
    for (int i = 0; i < kDb; ++i) o[n][i] = f32x4_t{0, 0, 0, 0};
  }

  // a wave without columns fetches keys for the others
  const bool busy =
      first + wave * NC * 16 < (cl.q1 - cl.q0) * a.group;
  int32_t k_begin, k_end;
  part_of<R>(cl.k0, cl.k1, split, parts, k_begin, k_end);
  KeyStream<T, D, R> keys(a, kvh, k_begin, k_end);
  if (k_begin < k_end) {
    keys.load(a);
    keys.put(lds[0][0], lds[0][1], start[0]);
  }
  int at = 0;
  for (int32_t k0 = k_begin; k0 < k_end; k0 += R, at ^= 1) {
    __syncthreads();  // the tile is there, the other one has been read
    const bool more = k0 + R < k_end;
    if (more) keys.load(a);
    const char *tk = lds[at][0], *tv = lds[at][1];
    if (busy) {
      f32x4_t s[NC][kRt];
      float tile_sum[NC] = {};
#pragma unroll
      for (int t = 0; t < kRt; ++t) {
        const f32x4_t b0 =
            *reinterpret_cast<const f32x4_t *>(&start[at][16 * t + 4 * g]);
#pragma unroll
        for (int n = 0; n < NC; ++n) s[n][t] = sums_from<T>(b0);
#pragma unroll
        for (int i = 0; i < kDs; ++i) {
          const Along kf =
              L::template along<B>(tk, 16 * t + (lane & 15), i, g);
#pragma unroll
          for (int n = 0; n < NC; ++n) s[n][t] = mma16(kf, qf[n][i], s[n][t]);
        }
#pragma unroll
        for (int n = 0; n < NC; ++n) s[n][t] = sums_done<T>(s[n][t], b0);
      }
      // With the maximum met so far P may exceed 1; a column whose sums over
      // this tile stay below kGrown needs no new one, and few do after the
      // first tile.  (What a column does is its own affair, so that results do
      // not depend on the rows that share a wave.)
      frag_t<T> p[NC][kRt / 2];
      const bool first_tile = k0 == k_begin;
      bool fits = !first_tile;
      if (fits) {
        bool small = true;
#pragma unroll
        for (int n = 0; n < NC; ++n) {
          const float sum = powers<T, kRt>(s[n], a.c, m[n] * a.c, p[n]);
          small &= sum <= kGrown;  // (not so for NaN)
          tile_sum[n] = sum;
        }
        fits = __ballot(!small) == 0;
      }
      if (!fits) {
#pragma unroll
        for (int n = 0; n < NC; ++n) {
          float top = s[n][0][0];
#pragma unroll
          for (int t = 0; t < kRt; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) top = fmaxf(top, s[n][t][r]);
          const float over = first_tile || !(tile_sum[n] <= kGrown);
          top = lanes16_max(over) > 0.0f ? fmaxf(lanes16_max(top), m[n]) : m[n];
          const float mc = top * a.c;
          // (not a fused product: 0 where the maximum stays, also the first)
          const float alpha = __builtin_amdgcn_exp2f(m[n] * a.c - mc);
          m[n] = top;
          tile_sum[n] = powers<T, kRt>(s[n], a.c, mc, p[n]);
          l[n] *= alpha;
#pragma unroll
          for (int i = 0; i < kDb; ++i) o[n][i] *= alpha;
        }
      }
#pragma unroll
      for (int n = 0; n < NC; ++n) l[n] += tile_sum[n];
#pragma unroll
      for (int t = 0; t < kRt; t += 2)
#pragma unroll
        for (int i = 0; i < kDb; ++i) {
          const frag_t<T> vf = L::across(tv, 16 * t, i, lane);
#pragma unroll
          for (int n = 0; n < NC; ++n) o[n][i] = mma16(vf, p[n][t / 2], o[n][i]);
        }
    }
    if (more) keys.put(lds[at ^ 1][0], lds[at ^ 1][1], start[at ^ 1]);
  }

  // without a key there is no result, whatever q holds
  if (wave == 0) {
    const bool any = __ballot(keys.seen) != 0;
    if (lane == 0) any_key = any;
  }
  __syncthreads();
  const bool none = !any_key;
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    const float sum = none ? 0.0f : lanes16_sum(l[n]);
    if (none) {
      m[n] = -1e30f;
#pragma unroll
      for (int i = 0; i < kDb; ++i) o[n][i] = f32x4_t{0, 0, 0, 0};
    }
    if (col[n].row < 0) continue;
    const int32_t head = kvh * a.group + col[n].head;
    if (parts > 1) {
      // (row by row: head, then d)
      const int64_t cols = (int64_t)a.nq * a.heads;
      const int64_t c = (int64_t)col[n].row * a.heads + head;
      float *po = a.part + ((int64_t)split * cols + c) * D;
#pragma unroll
      for (int i = 0; i < kDb; ++i)
        *reinterpret_cast<f32x4_t *>(po + 16 * i + 4 * g) = o[n][i];
      if (g == 0) {
        float *pm = a.part + (int64_t)a.splits * cols * D +
                    ((int64_t)split * cols + c) * 2;
        pm[0] = m[n] * a.c;
        pm[1] = sum;
      }
      continue;
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    T *op = static_cast<T *>(a.out) + col[n].row * a.ldo + (int64_t)head * dh;
#pragma unroll
    for (int i = 0; i < kDb; ++i) {
      const int d = 16 * i + 4 * g;
      if (d < dh) store4(op + d, o[n][i] * inv, dh - d);
    }
    if (a.lse && g == 0)
      a.lse[(int64_t)head * a.nq + col[n].row] =
          sum == 0.0f ? -INFINITY
                      : (m[n] * a.c + __builtin_amdgcn_logf(sum)) * kLn2;
  }
}

// What a column's parts come to: o / l and lse.
template <class T>
__device__ __forceinline__ void put_out(const Attn &a, int64_t c, int d,
                                        f32x4_t o, float m, float l) {
  const int32_t head = (int32_t)(c % a.heads);
  const int64_t row = c / a.heads;
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  if (d < a.dh)
    store4(static_cast<T *>(a.out) + row * a.ldo + (int64_t)head * a.dh + d,
           o * inv, a.dh - d);
  if (a.lse && d == 0)
    a.lse[(int64_t)head * a.nq + row] =
        l == 0.0f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// Adds the parts of a column, relative to the largest of their maxima: D / 4
// lanes for a column, or for few columns of many parts (WIDE) a block, whose
// groups of so many lanes take parts side by side.
constexpr int kWideSplits = 8;
template <class T, int D, bool WIDE>
__global__ __launch_bounds__(kAttnNT) void k_attn_join(Attn a) {
  constexpr int kLanes = D / 4, kRows = kAttnNT / kLanes;
  constexpr int kStep = WIDE ? kRows : 1;
  __shared__ f32x4_t so[WIDE ? kRows : 1][kLanes];
  __shared__ float sl[WIDE ? kRows : 1];
  const int64_t cols = (int64_t)a.nq * a.heads;
  const int tid = threadIdx.x, group = tid / kLanes, d = tid % kLanes * 4;
  const int64_t c =
      WIDE ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * kRows + group;
  if (c >= cols) return;
  const Cloud cl = cloud_of<false>(
      a, cloud_at(a.q_off, a.clouds, a.nq, (int32_t)(c / a.heads)));
  const int32_t parts = parts_of(a, cl.k1 - cl.k0);
  if (parts == 1) return;  // that one gave the results
  const float *pm = a.part + (int64_t)a.splits * cols * D + c * 2;
  float m = -INFINITY;
  if constexpr (WIDE) {
    // (kMaxSplits lanes look at one part each)
    if (tid % kWave < parts) m = pm[(int64_t)(tid % kWave) * cols * 2];
#pragma unroll
    for (int off = kWave / 2; off > 0; off >>= 1)
      m = fmaxf(m, __shfl_xor(m, off, kWave));
  } else {
    for (int32_t s = 0; s < parts; ++s)
      m = fmaxf(m, pm[(int64_t)s * cols * 2]);
  }
  f32x4_t o = {0, 0, 0, 0};
  float l = 0.0f;
#pragma unroll 4
  for (int32_t s = WIDE ? group : 0; s < parts; s += kStep) {
    const float f = __builtin_amdgcn_exp2f(pm[(int64_t)s * cols * 2] - m);
    l = __builtin_fmaf(pm[(int64_t)s * cols * 2 + 1], f, l);
    o += f * *reinterpret_cast<const f32x4_t *>(
                 a.part + ((int64_t)s * cols + c) * D + d);
  }
  if constexpr (WIDE) {
    so[group][tid % kLanes] = o;
    if (d == 0) sl[group] = l;
    __syncthreads();
    if (group) return;
    l = sl[0];
#pragma unroll
    for (int s = 1; s < kRows; ++s) {
      o += so[s][tid];
      l += sl[s];
    }
  }
  put_out<T>(a, c, d, o, m, l);
}

// --- backward ----------------------------------------------------------------

// Groups of 16 columns a wave: as the registers of two waves a SIMD hold, half
// of them where the blocks would leave CUs idle, in parts too.  Keys a tile for
// dq, rows a tile for dk and dv: the rows of q that pass a key block come from
// further away than keys, longer tiles cover their latency.  (Backward of
// 100,000 x 2000, 8 heads of 64: 1573 us with tiles of 64 rows, 1545 of 128;
// 1,265,474 x 613, 4 of 32: 2361 and 2282; fp32, 200,000 x 1000, 4 of 32: 3329
// and 3249.)  kKept: k_attn_dkv's v in LDS.
template <class T, int B>
struct BackwardShape {
  static constexpr bool kBf = sizeof(T) == 2;
  static constexpr int kGroups = kBf || B <= 4 ? 2 : 1;
  static constexpr int kKeys = B <= 2 ? 64 : 32;
  static constexpr int kRows = B <= 2 || (kBf && B <= 4) ? 128 : 32;
  static constexpr bool kKept = kBf && B > 4;
};

// What lane group g has of D = dout . out of a row and head.  Both kernels
// that need it add in this order and then over the groups, g ^ 1 first.
template <class T, int B>
__device__ __forceinline__ float delta_of(const T *dout, const T *out, int g,
                                          int dh) {
  typedef FragsOf<T, B> F;
  float sum = 0.0f;
#pragma unroll
  for (int s = 0; s < F::kSteps; ++s) {
    const typename F::Along x = load_along<B>(dout, s, g, dh);
    const typename F::Along y = load_along<B>(out, s, g, dh);
#pragma unroll
    for (int e = 0; e < F::kEach; ++e)
      sum = __builtin_fmaf((float)x[e], (float)y[e], sum);
  }
  return sum;
}

// D of every row and head, four lanes each, where k_attn_dq does not run.
constexpr int64_t kDeltaGrid = (int64_t)1 << 20;  // blocks of its launch
template <class T, int B>
__global__ __launch_bounds__(kAttnNT) void k_attn_delta(Attn a) {
  constexpr int kPer = kAttnNT / 4;
  const int64_t cols = (int64_t)a.nq * a.heads;
  for (int64_t c0 = (int64_t)blockIdx.x * kPer; c0 < cols;
       c0 += (int64_t)gridDim.x * kPer) {
    const int64_t at = c0 + threadIdx.x / 4;
    const int64_t c = min(at, cols - 1);
    const int64_t row = c / a.heads;
    const int32_t head = (int32_t)(c % a.heads);
    float sum = delta_of<T, B>(
        static_cast<const T *>(a.dout) + row * a.lddo + (int64_t)head * a.dh,
        static_cast<const T *>(a.out) + row * a.ldo + (int64_t)head * a.dh,
        threadIdx.x % 4, a.dh);
    sum += __shfl_xor(sum, 1, kWave);
    sum += __shfl_xor(sum, 2, kWave);
    if (threadIdx.x % 4 == 0 && at < cols)
      a.delta[(int64_t)head * a.nq + row] = sum;
  }
}

// lse of a row in base 2, +inf where it has no keys: P is 0 there
__device__ __forceinline__ float lse2_of(float lse) {
  return lse == -INFINITY ? INFINITY : lse * kLog2e;
}

// dq: columns are rows of q, lines are keys.  It leaves D for k_attn_dkv.
template <class T, int B, int NC, int R, int W = 2>
__global__ __launch_bounds__(kAttnNT, W) void k_attn_dq(Attn a) {
  constexpr int D = width_of(B);
  typedef Lines<T, D> L;
  typedef FragsOf<T, B> F;
  typedef typename F::Along Along;
  constexpr int kCols = kAttnWaves * 16 * NC;
  constexpr int kTile = R * L::kBytes;
  constexpr int kDb = B, kDs = F::kSteps;
  __shared__ __attribute__((aligned(16))) char lds[2][2][kTile];
  __shared__ __attribute__((aligned(16))) float start[2][R];
  int32_t tile, kvh, split;
  if (!unit_of(a, tile, kvh, split)) return;
  const int32_t cloud =
      a.q_off ? find_cloud(a.q_off, a.clouds, a.nq, a.group, kCols, tile) : 0;
  const Cloud cl = cloud_of<false>(a, cloud);
  const int32_t base =
      (a.q_off ? cl.q0 * a.group / kCols + cloud : 0);
  const int32_t first = (tile - base) * kCols;
  if (first < 0 || first >= (cl.q1 - cl.q0) * a.group) return;
  const int32_t parts = parts_of(a, cl.k1 - cl.k0);
  if (split >= parts) return;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int g = lane >> 4;
  const int32_t dh = a.dh;

  Column col[NC];
  Along qf[NC][kDs], gf[NC][kDs];
  float lse2[NC], delta[NC];
  f32x4_t dq[NC][kDb];
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    col[n] = q_column(a, cl, first + (wave * NC + n) * 16 + (lane & 15));
    const bool live = col[n].row >= 0;
    const int32_t head = kvh * a.group + col[n].head;
    const int64_t row = live ? col[n].row : 0;
    const T *qp = static_cast<const T *>(a.q) + row * a.ldq +
                  (int64_t)head * dh;
    const T *gp = static_cast<const T *>(a.dout) + row * a.lddo +
                  (int64_t)head * dh;
#pragma unroll
    for (int s = 0; s < kDs; ++s) {
      qf[n][s] = load_along<B>(qp, s, g, live ? dh : 0);
      gf[n][s] = load_along<B>(gp, s, g, live ? dh : 0);
    }
    const int64_t c = (int64_t)head * a.nq + row;
    lse2[n] = live ? lse2_of(a.lse[c]) : INFINITY;
    delta[n] = lanes16_sum(delta_of<T, B>(
        gp, static_cast<const T *>(a.out) + row * a.ldo + (int64_t)head * dh,
        g, live ? dh : 0));
    // for the gradients of k
    if (live && split == 0 && g == 0) a.delta[c] = delta[n];
#pragma unroll
    for (int i = 0; i < kDb; ++i) dq[n][i] = f32x4_t{0, 0, 0, 0};
  }

  // a wave without columns fetches keys for the others
  const bool busy =
      first + wave * NC * 16 < (cl.q1 - cl.q0) * a.group;
  int32_t k_begin, k_end;
  part_of<R>(cl.k0, cl.k1, split, parts, k_begin, k_end);
  KeyStream<T, D, R> keys(a, kvh, k_begin, k_end);
  if (k_begin < k_end) {
    keys.load(a);
    keys.put(lds[0][0], lds[0][1], start[0]);
  }
  int at = 0;
  for (int32_t k0 = k_begin; k0 < k_end; k0 += R, at ^= 1) {
    __syncthreads();  // the tile is there, the other one has been read
    const bool more = k0 + R < k_end;
    if (more) keys.load(a);
    const char *tk = lds[at][0], *tv = lds[at][1];
#pragma unroll
    for (int t = 0; t < R / 16; t += 2) {
      if (!busy || (t && k0 + 16 * t >= k_end)) break;
      f32x4_t s[NC][2], dp[NC][2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4_t b0 = *reinterpret_cast<const f32x4_t *>(
            &start[at][16 * (t + h) + 4 * g]);
#pragma unroll
        for (int n = 0; n < NC; ++n) {
          s[n][h] = sums_from<T>(b0);
          dp[n][h] = f32x4_t{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < kDs; ++i) {
          const int line = 16 * (t + h) + (lane & 15);
          const Along kf = L::template along<B>(tk, line, i, g);
          const Along vf = L::template along<B>(tv, line, i, g);
#pragma unroll
          for (int n = 0; n < NC; ++n) {
            s[n][h] = mma16(kf, qf[n][i], s[n][h]);
            dp[n][h] = mma16(vf, gf[n][i], dp[n][h]);
          }
        }
#pragma unroll
        for (int n = 0; n < NC; ++n) s[n][h] = sums_done<T>(s[n][h], b0);
      }
      __builtin_amdgcn_sched_barrier(0);  // as in k_attn_dkv
      frag_t<T> ds[NC];
#pragma unroll
      for (int n = 0; n < NC; ++n) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r)
            s[n][h][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(
                             s[n][h][r], a.c, -lse2[n])) *
                         (dp[n][h][r] - delta[n]);
        ds[n] = to_frag<T>(s[n][0], s[n][1]);
      }
#pragma unroll
      for (int i = 0; i < kDb; ++i) {
        const frag_t<T> kf = L::across(tk, 16 * t, i, lane);
#pragma unroll
        for (int n = 0; n < NC; ++n) dq[n][i] = mma16(kf, ds[n], dq[n][i]);
      }
    }
    if (more) keys.put(lds[at ^ 1][0], lds[at ^ 1][1], start[at ^ 1]);
  }
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    if (col[n].row < 0) continue;
    const int32_t head = kvh * a.group + col[n].head;
    T *op = static_cast<T *>(a.dq) + col[n].row * a.lddq + (int64_t)head * dh;
#pragma unroll
    for (int i = 0; i < kDb; ++i) {
      const int d = 16 * i + 4 * g;
      // (a row without keys has none, whatever dout holds)
      const f32x4_t v =
          lse2[n] == INFINITY ? f32x4_t{0, 0, 0, 0} : dq[n][i] * a.scale;
      if (parts > 1)
        *reinterpret_cast<f32x4_t *>(
            a.part +
            (((int64_t)split * a.nq + col[n].row) * a.heads + head) * D + d) =
            v;
      else if (d < dh)
        store4(op + d, v, dh - d);
    }
  }
}

// dk and dv: columns are keys, lines are the rows of q of every head that
// shares them, column by column of the forward pass.  splits > 1: each takes
// a part of the lines and leaves fp32 sums to k_attn_join_kv.
// KEPT: the columns' v lie in LDS, read again for each tile, where registers
// for them would leave no room for more columns a wave.
template <class T, int B, int NC, int R, bool KEPT = false, int W = 2>
__global__ __launch_bounds__(kAttnNT, W) void k_attn_dkv(Attn a) {
  constexpr int D = width_of(B);
  typedef Lines<T, D> L;
  typedef FragsOf<T, B> F;
  typedef typename F::Along Along;
  constexpr int kCols = kAttnWaves * 16 * NC;
  constexpr int kTile = R * L::kBytes;
  constexpr int kDb = B, kDs = F::kSteps;
  __shared__ __attribute__((aligned(16))) char lds[2][2][kTile];
  __shared__ __attribute__((aligned(16))) float stats[2][2][R];
  __shared__ __attribute__((aligned(16))) char kept[KEPT ? kCols * L::kBytes
                                                         : 16];
  int32_t tile, kvh, split;
  if (!unit_of(a, tile, kvh, split)) return;
  const int32_t cloud =
      a.k_off ? find_cloud(a.k_off, a.clouds, a.nk, 1, kCols, tile) : 0;
  const Cloud cl = cloud_of<true>(a, cloud);
  const int32_t base = (a.k_off ? cl.k0 / kCols + cloud : 0);
  const int32_t first = cl.k0 + (tile - base) * kCols;
  if (first < cl.k0 || first >= cl.k1) return;
  const int32_t lines = max(cl.q1 - cl.q0, 0) * a.group;
  const int32_t parts = parts_of(a, lines);
  if (split >= parts) return;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  const int g = lane >> 4;
  const int32_t dh = a.dh;

  int32_t key[NC];
  float start[NC];
  Along kf[NC][kDs], vf[KEPT ? 1 : NC][KEPT ? 1 : kDs];
  const int line16 = lane & 15;
  f32x4_t dk[NC][kDb], dv[NC][kDb];
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    key[n] = first + (wave * NC + n) * 16 + (lane & 15);
    start[n] = start_of(a, key[n], cl.k1);
    const bool live = start[n] != -INFINITY;
    const int64_t row = live ? key[n] : 0;
    const T *kp = static_cast<const T *>(a.k) + row * a.ldk +
                  (int64_t)kvh * dh;
    const T *vp = static_cast<const T *>(a.v) + row * a.ldv +
                  (int64_t)kvh * dh;
#pragma unroll
    for (int s = 0; s < kDs; ++s) {
      kf[n][s] = load_along<B>(kp, s, g, live ? dh : 0);
      const Along v = load_along<B>(vp, s, g, live ? dh : 0);
      // (read by the lanes of this wave alone, which are ordered)
      if constexpr (KEPT)
        L::template put_along<B>(kept, (wave * NC + n) * 16 + line16, s, g, v);
      else
        vf[n][s] = v;
    }
#pragma unroll
    for (int i = 0; i < kDb; ++i)
      dk[n][i] = dv[n][i] = f32x4_t{0, 0, 0, 0};
  }

  // this split's lines
  const bool busy = first + wave * NC * 16 < cl.k1;
  int32_t l_begin, l_end;
  part_of<R>(0, lines, split, parts, l_begin, l_end);

  typedef Mover<T, D, R> M;
  M mq, mg;
  float st_lse = 0.0f, st_delta = 0.0f;
  auto load = [&](int32_t l0) {
    int64_t at[M::kCh];
    int32_t row[M::kCh];
#pragma unroll
    for (int ch = 0; ch < M::kCh; ++ch) {
      const int32_t l = l0 + M::line() + ch * M::kStep;
      const Column c = q_column(a, cl, min(l, lines - 1));
      row[ch] = l < l_end ? c.row : -1;
      at[ch] = (int64_t)(kvh * a.group + c.head) * dh + M::d();
    }
    auto is = [&](int ch) { return row[ch] >= 0; };
    const T *q = static_cast<const T *>(a.q);
    const T *dout = static_cast<const T *>(a.dout);
    mq.load([&](int ch) { return q + row[ch] * a.ldq + at[ch]; }, is,
            dh - M::d());
    mg.load([&](int ch) { return dout + row[ch] * a.lddo + at[ch]; }, is,
            dh - M::d());
    if (tid < R) {
      st_lse = INFINITY;
      st_delta = 0.0f;
      if (l0 + tid < l_end) {
        const Column c = q_column(a, cl, l0 + tid);
        const int64_t at = (int64_t)(kvh * a.group + c.head) * a.nq + c.row;
        st_lse = lse2_of(a.lse[at]);
        st_delta = a.delta[at];
      }
    }
  };
  auto put = [&](int at) {
    mq.put(lds[at][0]);
    mg.put(lds[at][1]);
    if (tid < R) {
      stats[at][0][tid] = st_lse;
      stats[at][1][tid] = st_delta;
    }
  };
  if (l_begin < l_end) {
    load(l_begin);
    put(0);
  }
  int at = 0;
  for (int32_t l0 = l_begin; l0 < l_end; l0 += R, at ^= 1) {
    __syncthreads();  // the tile is there, the other one has been read
    const bool more = l0 + R < l_end;
    if (more) load(l0 + R);
    const char *tq = lds[at][0], *tg = lds[at][1];
#pragma unroll
    for (int t = 0; t < R / 16; t += 2) {
      if (!busy || (t && l0 + 16 * t >= l_end)) break;
      f32x4_t s[NC][2], dp[NC][2];
      f32x4_t lse2[2], delta[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        lse2[h] = *reinterpret_cast<const f32x4_t *>(
            &stats[at][0][16 * (t + h) + 4 * g]);
        delta[h] = *reinterpret_cast<const f32x4_t *>(
            &stats[at][1][16 * (t + h) + 4 * g]);
#pragma unroll
        for (int n = 0; n < NC; ++n) {
          s[n][h] = sums_from<T>(f32x4_t(start[n]));
          dp[n][h] = f32x4_t{0, 0, 0, 0};
        }
#pragma unroll
        for (int i = 0; i < kDs; ++i) {
          const int line = 16 * (t + h) + line16;
          const Along qf = L::template along<B>(tq, line, i, g);
          Along gf;
          if constexpr (!KEPT) gf = L::template along<B>(tg, line, i, g);
#pragma unroll
          for (int n = 0; n < NC; ++n) {
            s[n][h] = mma16(qf, kf[n][i], s[n][h]);
            if constexpr (!KEPT)
              dp[n][h] = mma16(gf, vf[n][i], dp[n][h]);
          }
        }
#pragma unroll
        for (int n = 0; n < NC; ++n)
          s[n][h] = sums_done<T>(s[n][h], f32x4_t(start[n]));
      }
      if constexpr (KEPT) {
#pragma unroll
        for (int i = 0; i < kDs; ++i) {
          Along gf[2];
#pragma unroll
          for (int h = 0; h < 2; ++h)
            gf[h] = L::template along<B>(tg, 16 * (t + h) + line16, i, g);
#pragma unroll
          for (int n = 0; n < NC; ++n) {
            const Along v = L::template along<B>(
                kept, (wave * NC + n) * 16 + line16, i, g);
#pragma unroll
            for (int h = 0; h < 2; ++h) dp[n][h] = mma16(gf[h], v, dp[n][h]);
          }
        }
      }
      // the lines for the products that follow are read behind the scores, not
      // among them, whose registers they would take (16,384 x 12,288 in
      // eight clouds, 16 heads of 128 on 4, three drawings: 966, 1058 and 1017
      // us, 997, 1094 and 1055 without this)
      __builtin_amdgcn_sched_barrier(0);
      frag_t<T> p[NC], ds[NC];
#pragma unroll
      for (int n = 0; n < NC; ++n) {
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            s[n][h][r] = __builtin_amdgcn_exp2f(
                __builtin_fmaf(s[n][h][r], a.c, -lse2[h][r]));
            dp[n][h][r] = s[n][h][r] * (dp[n][h][r] - delta[h][r]);
          }
        p[n] = to_frag<T>(s[n][0], s[n][1]);
        ds[n] = to_frag<T>(dp[n][0], dp[n][1]);
      }
#pragma unroll
      for (int i = 0; i < kDb; ++i) {
        const frag_t<T> gf = L::across(tg, 16 * t, i, lane);
        const frag_t<T> qf = L::across(tq, 16 * t, i, lane);
#pragma unroll
        for (int n = 0; n < NC; ++n) {
          dv[n][i] = mma16(gf, p[n], dv[n][i]);
          dk[n][i] = mma16(qf, ds[n], dk[n][i]);
        }
      }
    }
    if (more) put(at ^ 1);
  }
#pragma unroll
  for (int n = 0; n < NC; ++n) {
    if (key[n] >= cl.k1) continue;
    if (start[n] == -INFINITY)  // masked
#pragma unroll
      for (int i = 0; i < kDb; ++i) dk[n][i] = dv[n][i] = f32x4_t{0, 0, 0, 0};
    if (parts > 1) {
      // (key by key: head, dk before dv, d)
      float *p = a.part +
                 (((int64_t)split * a.nk + key[n]) * a.kv_heads + kvh) * 2 * D;
#pragma unroll
      for (int i = 0; i < kDb; ++i) {
        *reinterpret_cast<f32x4_t *>(p + 16 * i + 4 * g) = dk[n][i];
        *reinterpret_cast<f32x4_t *>(p + D + 16 * i + 4 * g) = dv[n][i];
      }
      continue;
    }
#pragma unroll
    for (int i = 0; i < kDb; ++i) {
      const int d = 16 * i + 4 * g;
      if (d >= dh) continue;
      if (a.dk)
        store4(static_cast<T *>(a.dk) + key[n] * a.lddk + (int64_t)kvh * dh + d,
               dk[n][i] * a.scale, dh - d);
      if (a.dv)
        store4(static_cast<T *>(a.dv) + key[n] * a.lddv + (int64_t)kvh * dh + d,
               dv[n][i], dh - d);
    }
  }
}

// Adds the splits of dq in their order, D / 4 lanes a row and head.
template <class T, int D>
__global__ __launch_bounds__(kAttnNT) void k_attn_join_q(Attn a) {
  constexpr int kLanes = D / 4;
  const int64_t cols = (int64_t)a.nq * a.heads;
  const int64_t c = ((int64_t)blockIdx.x * kAttnNT + threadIdx.x) / kLanes;
  if (c >= cols) return;
  const int d = (threadIdx.x % kLanes) * 4;
  if (d >= a.dh) return;
  const Cloud cl = cloud_of<false>(
      a, cloud_at(a.q_off, a.clouds, a.nq, (int32_t)(c / a.heads)));
  const int32_t parts = parts_of(a, cl.k1 - cl.k0);
  if (parts == 1) return;  // that one gave the results
  f32x4_t sum = {0, 0, 0, 0};
#pragma unroll 8
  for (int32_t s = 0; s < parts; ++s)
    sum += *reinterpret_cast<const f32x4_t *>(
        a.part + ((int64_t)s * cols + c) * D + d);
  store4(static_cast<T *>(a.dq) + c / a.heads * a.lddq +
             c % a.heads * a.dh + d,
         sum, a.dh - d);
}

// Adds the splits of dk and dv in their order, D / 4 lanes a key and head.
template <class T, int D>
__global__ __launch_bounds__(kAttnNT) void k_attn_join_kv(Attn a) {
  constexpr int kLanes = D / 4;
  const int64_t cols = (int64_t)a.nk * a.kv_heads;
  const int64_t c = ((int64_t)blockIdx.x * kAttnNT + threadIdx.x) / kLanes;
  if (c >= cols) return;
  const int d = (threadIdx.x % kLanes) * 4;
  if (d >= a.dh) return;
  const Cloud cl = cloud_of<true>(
      a, cloud_at(a.k_off, a.clouds, a.nk, (int32_t)(c / a.kv_heads)));
  const int32_t parts = parts_of(a, max(cl.q1 - cl.q0, 0) * a.group);
  if (parts == 1) return;  // that one gave the results
  f32x4_t dk = {0, 0, 0, 0}, dv = {0, 0, 0, 0};
#pragma unroll 8
  for (int32_t s = 0; s < parts; ++s) {
    const float *p = a.part + ((int64_t)s * cols + c) * 2 * D + d;
    dk += *reinterpret_cast<const f32x4_t *>(p);
    dv += *reinterpret_cast<const f32x4_t *>(p + D);
  }
  const int64_t key = c / a.kv_heads;
  const int64_t at = c % a.kv_heads * a.dh + d;
  if (a.dk)
    store4(static_cast<T *>(a.dk) + key * a.lddk + at, dk * a.scale, a.dh - d);
  if (a.dv)
    store4(static_cast<T *>(a.dv) + key * a.lddv + at, dv, a.dh - d);
}

}  // namespace
}  // namespace ezsp
