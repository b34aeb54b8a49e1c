// ezsp_logp.hip -- log probabilities of given classes, entropy and the
// largest scores over the rows of a matrix, and the gradient.
//
//   m = max x, s = sum e^(x - m), t = sum e^(x - m) (x - m)
//   lse = m + log s, log p_j = x_j - m - log s, entropy = log s - t / s
//   backward: dx_j = g (1[j = id] - p_j) - h p_j (x_j - lse + entropy)
//
// Bound by memory: the scores are read once (backward: read and written
// once).  Rows of up to 4096 scores stay in the registers of a group of
// lanes; longer ones are streamed by a block with a running maximum, in parts
// if there are few of them, which a second kernel joins.  The largest scores
// are found one after the other among registers.  Of a long row each thread
// knows its own largest; the largest of as many lanes bound the row's from
// below, so that the few threads with scores above list them, and a wave sorts
// the list.  Only where more than a wave's are alike they are found one after
// the other, the thread that gave its largest up looking again.  Equal scores
// go to the smaller class everywhere, so results do not depend on how a row is
// divided.
//
// Measured on one MI355X: 1,265,474 x 19 fp32 with entropy and two classes 31
// us (4.4 TB/s of read and written bytes; vector instructions issue in 0.8 of
// the cycles), the gradient of 4096 x 50,001 bfloat16 with entropy 175 us (4.7
// TB/s), one row of 65,536 bfloat16 with eight classes 13 us, of which the
// second launch takes 4.
#include <float.h>

#include <algorithm>

#include "ezsp_rows.h"

namespace ezsp {

namespace {

constexpr int64_t kLogpGrid = (int64_t)1 << 22;  // blocks of a launch

// v of the lane whose number differs in the bit `by`, a constant where it is
// inlined: moves within a row of 16 lanes (4: the quad reversed, then the half
// row), exchanges of rows beyond.  A search is made of dozens of these, one
// after the other, and through LDS each takes its latency (one row of 65,536
// with eight classes: 17.7 us that way, 15.2 so).
__device__ __forceinline__ int32_t lane_xor(int32_t v, int by) {
  typedef unsigned u32x2 __attribute__((ext_vector_type(2)));
  const int lane = threadIdx.x % kWave;
  switch (by) {
    case 1:
      return __builtin_amdgcn_mov_dpp(v, 0xB1, 0xf, 0xf, true);
    case 2:
      return __builtin_amdgcn_mov_dpp(v, 0x4E, 0xf, 0xf, true);
    case 4:
      return __builtin_amdgcn_mov_dpp(
          __builtin_amdgcn_mov_dpp(v, 0x1B, 0xf, 0xf, true), 0x141, 0xf, 0xf,
          true);
    case 8:
      return __builtin_amdgcn_mov_dpp(v, 0x128, 0xf, 0xf, true);
    case 16: {
      const u32x2 r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
      return (int32_t)(lane & 16 ? r[0] : r[1]);
    }
    default: {
      const u32x2 r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
      return (int32_t)(lane & 32 ? r[0] : r[1]);
    }
  }
}
__device__ __forceinline__ float lane_xor(float v, int by) {
  return __builtin_bit_cast(float,
                            lane_xor(__builtin_bit_cast(int32_t, v), by));
}
// as group_sum
template <int G, int N>
__device__ __forceinline__ void lanes_sum(float (&v)[N], float *red) {
#pragma unroll
  for (int off = (G < kWave ? G : kWave) / 2; off > 0; off >>= 1)
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] += lane_xor(v[i], off);
  if constexpr (G > kWave) across_waves<G>(v, red);
}
template <int G>
__device__ __forceinline__ float lanes_max(float v) {
#pragma unroll
  for (int off = (G < kWave ? G : kWave) / 2; off > 0; off >>= 1)
    v = fmaxf(v, lane_xor(v, off));
  return v;
}

// What a row's scores come to: relative to the maximum m (0 where every score
// is -inf), the sum s of the exponentials and their mean's numerator t.
struct RowSum {
  float m, s, t;
};

// e^(x - m) and its product with x - m; -inf gives 0 and 0.
__device__ __forceinline__ void term(float x, float m, float &s, float &t) {
  const float z = x - m;
  const float e = exp_f(z);
  s += e;
  t = __builtin_fmaf(e, fmaxf(z, -1e30f), t);
}

// Sums relative to m as sums relative to `to`, which is not smaller.
__device__ __forceinline__ void shift(RowSum &r, float to) {
  const float by = fmaxf(r.m - to, -1e30f);  // (-inf: s and t are 0)
  const float f = exp_f(by);
  r.t = f * __builtin_fmaf(r.s, by, r.t);
  r.s *= f;
  r.m = to;
}

struct LogpOut {
  const int32_t *ids;
  float *logp, *lse, *entropy;
  int32_t top;
  int32_t *top_ids;
  float *top_logp;
};

// The row's results; at = its class's score (0 without one).
__device__ __forceinline__ void put_row(const LogpOut &o, int64_t row,
                                        RowSum r, int32_t id, int32_t v,
                                        float at, float log_s) {
  const bool none = r.s == 0.0f;  // every score -inf
  if (o.logp)
    o.logp[row] = id < 0 || id >= v ? 0.0f
                  : none            ? -INFINITY
                                    : (at - r.m) - log_s;
  if (o.lse) o.lse[row] = none ? -INFINITY : r.m + log_s;
  if (o.entropy) o.entropy[row] = none ? 0.0f : log_s - r.t / r.s;
}
__device__ __forceinline__ void put_top(const LogpOut &o, int64_t row, int k,
                                        float val, int32_t id, float m,
                                        float log_s) {
  const bool none = val == -INFINITY;
  o.top_ids[row * o.top + k] = none ? -1 : id;
  o.top_logp[row * o.top + k] = none ? -INFINITY : (val - m) - log_s;
}

// The better of two candidates: the larger score, the smaller place.
__device__ __forceinline__ void better(float &val, int32_t &at, float val2,
                                       int32_t at2) {
  if (val2 > val || (val2 == val && at2 < at)) {
    val = val2;
    at = at2;
  }
}
template <int G>
__device__ __forceinline__ void lanes_best(float &val, int32_t &at) {
#pragma unroll
  for (int off = G / 2; off > 0; off >>= 1) {
    const float v2 = lane_xor(val, off);
    const int32_t a2 = lane_xor(at, off);
    better(val, at, v2, a2);
  }
}

constexpr int32_t kNowhere = 0x7fffffff;

// The 64 candidates of a wave in order, the best in lane 0 (bitonic).
__device__ __forceinline__ void lanes_sort(float &val, int32_t &at) {
  const int lane = threadIdx.x % kWave;
#pragma unroll
  for (int run = 2; run <= kWave; run <<= 1)
#pragma unroll
    for (int by = run / 2; by > 0; by >>= 1) {
      const float v2 = lane_xor(val, by);
      const int32_t a2 = lane_xor(at, by);
      const bool second = v2 > val || (v2 == val && a2 < at);  // is better
      // the lower lane of a pair takes the better one in runs that fall
      if (second == (((lane & run) == 0) == ((lane & by) == 0))) {
        val = v2;
        at = a2;
      }
    }
}

// fewer are found sooner one after the other (50,000 x 500 bfloat16 with four:
// 47 us, listed 54; 20,000 x 2000 with five: 94 and 71)
constexpr int kListTop = 5;

// Rows held in registers.  red: as group_sum, twice that for the candidates.
// LIST, of groups from a wave on: the largest scores as of a long row, below
// (50,000 x 1000 with 32: 82 us, 397 one after the other; in a kernel of its
// own, whose registers the others would pay for).
template <class T, int G, int NV, bool LIST = false>
__global__ __launch_bounds__(norm_nt(G)) void k_logp_rows(
    const T *__restrict__ x, int64_t ldx, int64_t n, int32_t v, LogpOut o) {
  constexpr int kRows = norm_nt(G) / G;
  constexpr int kW = G > kWave ? G / kWave : 1;
  __shared__ float red[2 * norm_nt(G) / kWave];
  __shared__ int32_t red_at[norm_nt(G) / kWave];
  static_assert(!LIST || G >= kWave, "a wave sorts a list");
  constexpr int kLists = LIST ? kRows : 1;
  __shared__ float list[kLists][kWave];
  __shared__ int32_t list_at[kLists][kWave];
  __shared__ int32_t found[kLists];
  const int gl = threadIdx.x % G;
  for (int64_t r0 = (int64_t)blockIdx.x * kRows; r0 < n;
       r0 += (int64_t)gridDim.x * kRows) {
    const int64_t row = r0 + threadIdx.x / G;
    const bool live = row < n;
    const T *xr = x + (live ? row : 0) * ldx;
    const int32_t id = o.ids && live ? o.ids[row] : -1;
    f32x8_t a[NV];
    float m[1] = {-INFINITY};
#pragma unroll
    for (int j = 0; j < NV; ++j) {
      const int c = (gl + G * j) * kVec;
      a[j] = load8(xr + c, live ? v - c : 0);
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        a[j][i] = c + i < v ? a[j][i] : -INFINITY;
        m[0] = fmaxf(m[0], a[j][i]);
      }
    }
    // (the maximum of the lanes)
    m[0] = lanes_max<G>(m[0]);
    if constexpr (G > kWave) {
      __syncthreads();
      if (threadIdx.x % kWave == 0) red[threadIdx.x / kWave] = m[0];
      __syncthreads();
      m[0] = red[0];
#pragma unroll
      for (int w = 1; w < kW; ++w) m[0] = fmaxf(m[0], red[w]);
    }
    RowSum r;
    r.m = m[0] == -INFINITY ? 0.0f : m[0];
    float st[2] = {0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < NV; ++j)
#pragma unroll
      for (int i = 0; i < kVec; ++i) term(a[j][i], r.m, st[0], st[1]);
    lanes_sum<G>(st, red);
    r.s = st[0];
    r.t = st[1];
    const float log_s = logf(r.s);
    if (gl == 0 && live)
      put_row(o, row, r, id, v,
              id >= 0 && id < v ? (float)xr[id] : 0.0f, log_s);
    if constexpr (LIST) {
      const int own = threadIdx.x / G;
      float mine = -INFINITY;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < kVec; ++i) mine = fmaxf(mine, a[j][i]);
      float bound = mine;
      int32_t order = gl;
      lanes_sort(bound, order);
      bound = __shfl(bound, o.top - 1, kWave);
      if (gl == 0) found[own] = 0;
      __syncthreads();  // (and what red held has been read)
      if (G > kWave && gl % kWave == 0) red[gl / kWave] = bound;
      __syncthreads();
      if constexpr (G > kWave)
#pragma unroll
        for (int w = 0; w < kW; ++w) bound = fmaxf(bound, red[w]);
      if (mine >= bound && bound > -INFINITY)
#pragma unroll
        for (int j = 0; j < NV; ++j)
#pragma unroll
          for (int i = 0; i < kVec; ++i)
            if (a[j][i] >= bound) {
              const int32_t k = atomicAdd(&found[own], 1);
              if (k < kWave) {
                list[own][k] = a[j][i];
                list_at[own][k] = (gl + G * j) * kVec + i;
              }
            }
      __syncthreads();
      const int32_t listed = found[own];
      if (listed >= o.top && listed <= kWave) {
        if (gl < kWave) {
          float val = gl < listed ? list[own][gl] : -INFINITY;
          int32_t at = gl < listed ? list_at[own][gl] : kNowhere;
          lanes_sort(val, at);
          if (gl < o.top && live) put_top(o, row, gl, val, at, r.m, log_s);
        }
        continue;
      }
    }
    for (int k = 0; k < o.top; ++k) {
      float val = -INFINITY;
      int32_t at = kNowhere;
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < kVec; ++i)
          if (a[j][i] > val) {
            val = a[j][i];
            at = (gl + G * j) * kVec + i;
          }
      lanes_best<(G < kWave ? G : kWave)>(val, at);
      if constexpr (G > kWave) {
        __syncthreads();
        if (threadIdx.x % kWave == 0) {
          red[threadIdx.x / kWave] = val;
          red_at[threadIdx.x / kWave] = at;
        }
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kW; ++w) better(val, at, red[w], red_at[w]);
      }
      // what is given leaves the row
#pragma unroll
      for (int j = 0; j < NV; ++j)
#pragma unroll
        for (int i = 0; i < kVec; ++i)
          if ((gl + G * j) * kVec + i == at) a[j][i] = -INFINITY;
      if (gl == 0 && live) put_top(o, row, k, val, at, r.m, log_s);
    }
  }
}

constexpr int kLongVecs = 4;    // vectors a thread loads at once
constexpr int kMaxParts = 64;   // a wave joins them

// One part of a long row, `per` vectors of it, by a block.  Without parts
// (parts == 1) it gives the row's results, else the sums and its largest
// scores to the workspace: 3 floats and 2 * top words a part.
template <class T, int kLongNT>
__global__ __launch_bounds__(kLongNT) void k_logp_long(
    const T *__restrict__ x, int64_t ldx, int64_t n, int32_t v, int32_t parts,
    int32_t per, LogpOut o, float *__restrict__ ws) {
  constexpr int kWaves = kLongNT / kWave;
  __shared__ float red[2 * kWaves];
  __shared__ float best[kLongNT];
  __shared__ int32_t best_at[kLongNT];
  __shared__ float least;
  __shared__ int32_t found;
  const int32_t vecs = (v + kVec - 1) / kVec;
  const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
  for (int64_t item = blockIdx.x; item < n * parts; item += gridDim.x) {
    const int64_t row = item / parts;
    const int32_t part = (int32_t)(item % parts);
    const int32_t first = part * per, last = min(first + per, vecs);
    const T *xr = x + row * ldx;
    RowSum r = {-FLT_MAX, 0.0f, 0.0f};
    float top_val = -INFINITY;  // this thread's largest, and its vector
    int32_t top_at = kNowhere;
    for (int32_t w0 = first + tid; w0 < last; w0 += kLongNT * kLongVecs) {
      f32x8_t a[kLongVecs];
#pragma unroll
      for (int j = 0; j < kLongVecs; ++j) {
        const int32_t w = w0 + j * kLongNT;
        const int cnt = w < last ? min(v - w * kVec, kVec) : 0;
        a[j] = load8(xr + (int64_t)min(w, last - 1) * kVec, cnt);
        if (cnt < kVec)
#pragma unroll
          for (int i = 0; i < kVec; ++i)
            if (i >= cnt) a[j][i] = -INFINITY;
      }
      float m = r.m;
#pragma unroll
      for (int j = 0; j < kLongVecs; ++j) {
        float vm = a[j][0];
#pragma unroll
        for (int i = 1; i < kVec; ++i) vm = fmaxf(vm, a[j][i]);
        if (vm > top_val) {
          top_val = vm;
          top_at = w0 + j * kLongNT;
        }
        m = fmaxf(m, vm);
      }
      if (m > r.m) shift(r, m);
#pragma unroll
      for (int j = 0; j < kLongVecs; ++j)
#pragma unroll
        for (int i = 0; i < kVec; ++i) term(a[j][i], r.m, r.s, r.t);
    }
    // the block's sums, relative to its largest
    float m = lanes_max<kWave>(r.m);
    __syncthreads();  // what the arrays held has been read
    if (lane == 0) red[wave] = m;
    best[tid] = top_val;
    best_at[tid] = top_at;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kWaves; ++w) m = fmaxf(m, red[w]);
    shift(r, m);
    float st[2] = {r.s, r.t};
    lanes_sum<kLongNT>(st, red);
    r.s = st[0];
    r.t = st[1];
    const float log_s = logf(r.s);
    float *out = ws + item * (3 + 2 * o.top);
    if (tid == 0) {
      if (parts == 1) {
        const int32_t id = o.ids ? o.ids[row] : -1;
        put_row(o, row, r, id, v,
                id >= 0 && id < v ? (float)xr[id] : 0.0f, log_s);
      } else {
        out[0] = r.m;
        out[1] = r.s;
        out[2] = r.t;
      }
    }
    if (!o.top) continue;
    // the first wave keeps every thread's largest, kWaves a lane
    float val[kWaves];
    int32_t at[kWaves];
    if (wave == 0) {
      float lane_best = -INFINITY;
#pragma unroll
      for (int s = 0; s < kWaves; ++s) {
        val[s] = best[s * kWave + lane];
        at[s] = best_at[s * kWave + lane];
        lane_best = fmaxf(lane_best, val[s]);
      }
      // as many scores as are asked for are no smaller than the largest ones
      // of as many lanes
      int32_t order = lane;
      lanes_sort(lane_best, order);
      if (lane == o.top - 1) least = lane_best;
      if (lane == 0) found = 0;
    }
    __syncthreads();
    // the few threads that have such scores list them
    const float bound = least;
    if (top_val >= bound && bound > -INFINITY)
      for (int32_t w0 = first + tid; w0 < last; w0 += kLongNT * kLongVecs) {
        f32x8_t a[kLongVecs];
        int cnt[kLongVecs];
#pragma unroll
        for (int j = 0; j < kLongVecs; ++j) {
          const int32_t w = w0 + j * kLongNT;
          cnt[j] = w < last ? min(v - w * kVec, kVec) : 0;
          a[j] = load8(xr + (int64_t)min(w, last - 1) * kVec, cnt[j]);
        }
#pragma unroll
        for (int j = 0; j < kLongVecs; ++j)
#pragma unroll
          for (int i = 0; i < kVec; ++i)
            if (i < cnt[j] && a[j][i] >= bound) {
              const int32_t k = atomicAdd(&found, 1);
              if (k < kWave) {
                best[k] = a[j][i];
                best_at[k] = (w0 + j * kLongNT) * kVec + i;
              }
            }
      }
    __syncthreads();
    const int32_t listed = found;
    if (wave) continue;
    if (listed >= o.top && listed <= kWave) {
      // (they come in any order and leave sorted)
      float bv = lane < listed ? best[lane] : -INFINITY;
      int32_t bi = lane < listed ? best_at[lane] : kNowhere;
      lanes_sort(bv, bi);
      if (lane < o.top) {
        if (parts == 1) {
          put_top(o, row, lane, bv, bi, r.m, log_s);
        } else {
          out[3 + lane] = bv;
          reinterpret_cast<int32_t *>(out)[3 + o.top + lane] = bi;
        }
      }
      continue;
    }
    // too many alike (or -inf among them): one after the other
    float had = INFINITY;  // the score given last, and its place
    int32_t had_at = -1;
    for (int k = 0; k < o.top; ++k) {
      float bv = -INFINITY;
      int32_t bw = kNowhere;
#pragma unroll
      for (int s = 0; s < kWaves; ++s) better(bv, bw, val[s], at[s]);
      lanes_best<kWave>(bv, bw);
      int32_t id = kNowhere;
      if (bw != kNowhere) {
        // the first of the vector's scores that is it and was not given
        const int32_t c = bw * kVec + lane;
        const bool is = lane < kVec && c < v && (float)xr[c] == bv &&
                        (bv < had || c > had_at);
        id = bw * kVec + (int32_t)__ffsll(__ballot(is)) - 1;
        had = bv;
        had_at = id;
        // its thread's next largest, by the whole wave
        const int32_t owner = (bw - first) % kLongNT;
        float nv = -INFINITY;
        int32_t nw = kNowhere;
        for (int32_t w = first + owner + lane * kLongNT; w < last;
             w += kWave * kLongNT) {
          const int cnt = min(v - w * kVec, kVec);
          const f32x8_t a = load8(xr + (int64_t)w * kVec, cnt);
#pragma unroll
          for (int i = 0; i < kVec; ++i)
            if (i < cnt && a[i] > nv &&
                (a[i] < had || (a[i] == had && w * kVec + i > had_at))) {
              nv = a[i];
              nw = w;
            }
        }
        lanes_best<kWave>(nv, nw);
#pragma unroll
        for (int s = 0; s < kWaves; ++s)
          if (owner == s * kWave + lane) {
            val[s] = nv;
            at[s] = nw;
          }
      }
      if (lane == 0) {
        if (parts == 1) {
          put_top(o, row, k, bv, id, r.m, log_s);
        } else {
          out[3 + k] = bv;
          reinterpret_cast<int32_t *>(out)[3 + o.top + k] = id;
        }
      }
    }
  }
}

// The parts of a row, a lane each: the sums, and the lists of largest scores
// merged from their heads.
template <class T>
__global__ __launch_bounds__(kWave) void k_logp_join(
    const T *__restrict__ x, int64_t ldx, int64_t n, int32_t v, int32_t parts,
    LogpOut o, const float *__restrict__ ws) {
  const int lane = threadIdx.x;
  for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
    const float *in = ws + (row * parts + lane) * (3 + 2 * o.top);
    const bool live = lane < parts;
    RowSum r = {-FLT_MAX, 0.0f, 0.0f};
    if (live) r = {in[0], in[1], in[2]};
    float m = lanes_max<kWave>(r.m);
    shift(r, m);
    float st[2] = {r.s, r.t};
    lanes_sum<kWave>(st, nullptr);
    r.s = st[0];
    r.t = st[1];
    const float log_s = logf(r.s);
    if (lane == 0) {
      const int32_t id = o.ids ? o.ids[row] : -1;
      put_row(o, row, r, id, v,
              id >= 0 && id < v ? (float)x[row * ldx + id] : 0.0f, log_s);
    }
    if (parts * o.top <= kWave) {
      // every list at once
      float val = -INFINITY;
      int32_t at = kNowhere;
      if (lane < parts * o.top) {
        const float *list =
            ws + (row * parts + lane / o.top) * (3 + 2 * o.top) + 3 +
            lane % o.top;
        val = list[0];
        at = reinterpret_cast<const int32_t *>(list)[o.top];
      }
      lanes_sort(val, at);
      if (lane < o.top) put_top(o, row, lane, val, at, r.m, log_s);
      continue;
    }
    int32_t head = 0;
    for (int k = 0; k < o.top; ++k) {
      float val = -INFINITY;
      int32_t at = kNowhere;
      if (live && head < o.top) {
        val = in[3 + head];
        at = reinterpret_cast<const int32_t *>(in)[3 + o.top + head];
      }
      const int32_t mine = at;
      lanes_best<kWave>(val, at);
      if (at != kNowhere && mine == at) ++head;
      if (lane == 0) put_top(o, row, k, val, at, r.m, log_s);
    }
  }
}

// --- gradient ----------------------------------------------------------------

constexpr int kGradNT = 256;
constexpr int kGradVecs = 4;  // vectors a thread and step
constexpr int64_t kGradGrid = (int64_t)1 << 20;

template <class T>
__global__ __launch_bounds__(kGradNT) void k_logp_grad(
    const T *x, int64_t ldx, int64_t n, int32_t v, int32_t vecs,
    const float *__restrict__ dlogp, const int32_t *__restrict__ ids,
    const float *__restrict__ lse, const float *__restrict__ ent,
    const float *__restrict__ dent, T *dx, int64_t lddx) {
  constexpr int64_t kSpan = (int64_t)kGradNT * kGradVecs;
  const int64_t total = n * vecs;
  const double inv = 1.0 / (double)vecs;
  for (int64_t i0 = (int64_t)blockIdx.x * kSpan; i0 < total;
       i0 += (int64_t)gridDim.x * kSpan) {
    int64_t row[kGradVecs];
    int32_t col[kGradVecs];
    f32x8_t a[kGradVecs];
#pragma unroll
    for (int j = 0; j < kGradVecs; ++j) {
      const int64_t at = i0 + j * kGradNT + threadIdx.x;
      // (exact as a double, the row off by one at most)
      row[j] = (int64_t)((double)at * inv);
      int64_t w = at - row[j] * vecs;
      if (w < 0) {
        --row[j];
        w += vecs;
      } else if (w >= vecs) {
        ++row[j];
        w -= vecs;
      }
      col[j] = (int32_t)w * kVec;
      if (at >= total) row[j] = -1;
      if (row[j] >= 0) a[j] = load8(x + row[j] * ldx + col[j], v - col[j]);
    }
#pragma unroll
    for (int j = 0; j < kGradVecs; ++j) {
      if (row[j] < 0) break;
      const float l = lse[row[j]];
      const int32_t id = ids ? ids[row[j]] : -1;
      const bool has = id >= 0 && id < v;
      const float g = has ? dlogp[row[j]] : 0.0f;
      const float h = ent ? dent[row[j]] : 0.0f;
      const float hh = ent ? ent[row[j]] : 0.0f;
      f32x8_t out;
#pragma unroll
      for (int i = 0; i < kVec; ++i) {
        const float z = a[j][i] - l;
        const float p = exp_f(z);
        // (p is 0 from z = -150 on: a bound below keeps h z finite)
        const float f = __builtin_fmaf(h, fmaxf(z, -256.0f) + hh, g);
        out[i] = __builtin_fmaf(-p, f, col[j] + i == id ? g : 0.0f);
        if (l == -INFINITY) out[i] = 0.0f;
      }
      store8(dx + row[j] * lddx + col[j], out, v - col[j]);
    }
  }
}

template <class T, int G, int NV>
void rows(const LogpArgs &a, const LogpOut &o, hipStream_t st) {
  const int64_t per = norm_nt(G) / G;
  auto kernel = k_logp_rows<T, G, NV>;
  if constexpr (G >= kWave)
    if (o.top >= kListTop) kernel = k_logp_rows<T, G, NV, true>;
  hipLaunchKernelGGL(kernel,
                     dim3((unsigned)std::min<int64_t>((a.n + per - 1) / per,
                                                      kLogpGrid)),
                     dim3(norm_nt(G)), 0, st, static_cast<const T *>(a.x),
                     a.ldx, a.n, a.v, o);
}

// Beyond it a streamed row is faster (4096 x 8192 fp32: 23 us, 26 in registers).
constexpr int32_t kRowsMaxV = 4096;
constexpr int64_t kCus = 256;  // of an MI355X

// Threads that take a long row: many rows keep the chip busy in blocks of 256,
// whose waves wait less for each other (4096 x 50,001 bfloat16: 109 us, 123 in
// blocks of 512; 700 rows with five classes 41 and 46), few rows are over
// sooner in larger ones (200 rows with eight classes: 21.1 us in blocks of 512,
// 24.8 of 256, 26.4 of 1024).
bool many_rows(int64_t n) { return n >= 2 * kCus; }

// Parts of a long row: as many as give every CU a block, each of at least 8K
// scores (one row of 40,000 with eight classes: 13.3 us, 16.8 whole; of 300,000
// 16.2, in parts of 16K 18.2), but no more than eight while these stay below
// 24K: the join sorts up to 64 scores of all parts at once (131,072 with eight
// classes: 12.9 us in eight parts, 15.7 in sixteen), and not two, for which the
// second launch takes longer than they save (20,000: 12.7 us whole, 13.4).  The
// rule was set with eight classes and does not read their number.  With none to
// four, which the join would sort from more parts, it is within 0.6 us of the
// best of 1, 4, 8, 16 and 24 parts up to 131,072 scores; at 196,608, the last row
// of eight parts, sixteen are sooner (none 7.9 us and 9.6, four 12.7 and 16.5,
// eight 15.7 and 17.3); and with more than eight the join takes them one after
// the other, so that few or no parts are sooner (65,536 with sixteen: 13.3 us in
// four, 19.8; 40,000 with 32: 17.9 whole, 27.3).
int32_t parts_of(int64_t n, int32_t v) {
  int64_t most = std::min<int64_t>(kMaxParts, v / 8192);
  if (most > 8 && v / 8 <= 24576) most = 8;
  if (most < 3) most = 1;
  return (int32_t)std::max<int64_t>(
      1, std::min<int64_t>(most, (kCus + n - 1) / n));
}

template <class T, int NT>
void long_rows(const LogpArgs &a, const LogpOut &o, hipStream_t st) {
  const int32_t vecs = (a.v + kVec - 1) / kVec;
  const int32_t parts = parts_of(a.n, a.v);
  const int32_t per = (vecs + parts - 1) / parts;
  hipLaunchKernelGGL((k_logp_long<T, NT>),
                     dim3((unsigned)std::min<int64_t>(a.n * parts, kLogpGrid)),
                     dim3(NT), 0, st, static_cast<const T *>(a.x), a.ldx, a.n,
                     a.v, parts, per, o, a.part);
  if (parts > 1)
    hipLaunchKernelGGL(k_logp_join<T>,
                       dim3((unsigned)std::min<int64_t>(a.n, kLogpGrid)),
                       dim3(kWave), 0, st, static_cast<const T *>(a.x), a.ldx,
                       a.n, a.v, parts, o, a.part);
}

template <class T>
void forward(const LogpArgs &a, hipStream_t st) {
  const LogpOut o = {a.ids, a.logp, a.lse, a.entropy,
                     a.top, a.top_ids, a.top_logp};
  if (a.v > kRowsMaxV)
    return many_rows(a.n) ? long_rows<T, 256>(a, o, st)
                          : long_rows<T, 512>(a, o, st);
  const int32_t chunks = (a.v + kVec - 1) / kVec;
  // (a lane has short rows to itself: no exchanges, and no lanes without
  // scores; 1,265,474 x 19 with two classes 31.6 us, 43 by four lanes)
  if (chunks <= 1) return rows<T, 1, 1>(a, o, st);
  if (chunks <= 2) return rows<T, 1, 2>(a, o, st);
  if (chunks <= 3) return rows<T, 1, 3>(a, o, st);
  if (chunks <= 4) return rows<T, 1, 4>(a, o, st);
  if (chunks <= 8) return rows<T, 8, 1>(a, o, st);
  if (chunks <= 16) return rows<T, 16, 1>(a, o, st);
  if (chunks <= 32) return rows<T, 32, 1>(a, o, st);
  if (chunks <= 64) return rows<T, 64, 1>(a, o, st);
  if (chunks <= 128) return rows<T, 64, 2>(a, o, st);
  if (chunks <= 256) return rows<T, 256, 1>(a, o, st);
  rows<T, 256, 2>(a, o, st);
}

template <class T>
void gradient(const LogpArgs &a, hipStream_t st) {
  const int32_t vecs = (a.v + kVec - 1) / kVec;
  const int64_t span = (int64_t)kGradNT * kGradVecs;
  hipLaunchKernelGGL(k_logp_grad<T>,
                     dim3((unsigned)std::min<int64_t>(
                         (a.n * vecs + span - 1) / span, kGradGrid)),
                     dim3(kGradNT), 0, st, static_cast<const T *>(a.x), a.ldx,
                     a.n, a.v, vecs, a.dlogp, a.ids, a.lse, a.entropy, a.dent,
                     static_cast<T *>(a.dx), a.lddx);
}

}  // namespace

void logp_reserve(Arena &ar, int32_t v, int32_t top, LogpArgs *a) {
  // (n rows in parts_of(n, v) > 1 parts are fewer than kCus + n, n < kCus)
  const int64_t most = v > kRowsMaxV ? 2 * kCus : 0;
  a->part = ar.take<float>((size_t)most * (3 + 2 * (size_t)top));
}

int logp_fwd_run(const LogpArgs &a, hipStream_t st) {
  prof_begin("log_probs", st);
  if (a.type == EZSP_TYPE_BF16)
    forward<__bf16>(a, st);
  else
    forward<float>(a, st);
  prof_end(st);
  const int rc = check_hip(hipGetLastError(), "log probs launch");
  prof_bytes("log_probs", (double)a.n * ((double)a.v * type_bytes(a.type) +
                                         8.0 * a.top));
  return rc;
}

int logp_bwd_run(const LogpArgs &a, hipStream_t st) {
  prof_begin("log_probs", st);
  if (a.type == EZSP_TYPE_BF16)
    gradient<__bf16>(a, st);
  else
    gradient<float>(a, st);
  prof_end(st);
  const int rc = check_hip(hipGetLastError(), "log probs gradient launch");
  prof_bytes("log_probs", 2.0 * (double)a.n * a.v * type_bytes(a.type));
  return rc;
}

}  // namespace ezsp
