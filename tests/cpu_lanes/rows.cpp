// rows.cpp -- layer norm and the one-pass backward of few columns on the CPU:
// tables in allocations that end with their last row, so that a load past a
// table is an error under a sanitizer.  What they load of a row's neighbours
// is NaN where it is padding; integer results are compared for equality, the
// norm's within a bound.  Prints a line per case; exits 1 if one differs.
#include "lanes.h"

#include <stdio.h>

#include <random>

#include "../../paper_2512_00385_amd/csrc/ezsp_narrow_f32.h"
#include "../../paper_2512_00385_amd/csrc/ezsp_norm.hip"

namespace ezsp {
void prof_begin(const char *, hipStream_t) {}
void prof_end(hipStream_t) {}
void prof_bytes(const char *, double) {}
int check_hip(hipError_t, const char *) { return 0; }
}  // namespace ezsp
extern "C" hipError_t hipGetLastError() { return hipSuccess; }

using namespace ezsp;

namespace {

std::mt19937 rng(1);

// n rows of d values ld apart, the last one ending with the allocation
template <class T>
struct Table {
  int32_t n, d;
  int64_t ld, len;
  std::unique_ptr<T[]> at;
  Table(int32_t n, int32_t d, int64_t ld, int spread)
      : n(n), d(d), ld(ld), len((n - 1) * ld + d), at(new T[len]) {
    for (int64_t i = 0; i < len; ++i)
      at[i] = (T)(i % ld < d ? (float)((int)(rng() % (2 * spread + 1)) - spread)
                             : NAN);
  }
  double get(int32_t i, int32_t j) const {
    return (double)(float)at[i * ld + j];
  }
};

int report(const char *name, size_t bytes, int32_t n, int32_t k, int32_t m,
           int64_t pad, int64_t bad) {
  printf("%s %s %d x %d -> %d, pad %lld: %lld wrong\n", name,
         bytes == 2 ? "bf16" : "fp32", n, k, m, (long long)pad,
         (long long)bad);
  fflush(stdout);
  return bad != 0;
}

// dz is dy: what the operators' own structures load, without an activation
struct PlainBf16 {
  const __bf16 *dy;
  int64_t ld;
  struct Raw {
    Vec8<__bf16> dy;
  };
  Raw raw(int64_t row, int32_t n, int32_t d, Span s) const {
    int32_t back;
    return {raw8(dy + span_at(row, ld, n, d, s, back))};
  }
  void value(const Raw &r, int64_t row, int32_t n, int32_t d, Span s,
             f32x8_t *v) const {
    int32_t back;
    span_at(row, ld, n, d, s, back);
    v[0] = __builtin_convertvector(
        settle(r.dy, s.off + back, row < n ? s.cnt : 0), f32x8_t);
  }
};
struct PlainF32 {
  const float *dy;
  int64_t ld;
  struct Raw {
    f32x4_t dy;
  };
  Raw raw(int64_t row, int32_t n, int32_t d, SpanOf<4> s) const {
    int32_t back;
    return {raw4(dy + span_at(row, ld, n, d, s, back))};
  }
  void value(const Raw &r, int64_t row, int32_t n, int32_t d, SpanOf<4> s,
             f32x4_t *v) const {
    int32_t back;
    span_at(row, ld, n, d, s, back);
    v[0] = settle4(r.dy, s.off + back, row < n ? s.cnt : 0);
  }
};

template <class T, class Op, class Kernel>
int narrow_case(int32_t n, int32_t k, int32_t m, int64_t pad, unsigned blocks,
                Kernel kernel) {
  const Table<T> x(n, k, k + pad, 2), dy(n, m, m + pad, 2), w(k, m, m, 2);
  Table<T> dx(n, k, k, 0), dw(k, m, m, 0);
  const int64_t plane = (int64_t)(k + 1) * m;
  std::unique_ptr<float[]> db(new float[m]), part(new float[blocks * plane]);
  NarrowArgs<T> g = {};
  g.x = x.at.get();
  g.w[0] = g.w[1] = w.at.get();
  g.ldx = x.ld;
  g.n = n;
  g.d_in = k;
  g.d_out = m;
  g.dx = dx.at.get();
  g.lddx = k;
  g.dw[0] = dw.at.get();
  g.db[0] = db.get();
  g.part = part.get();
  Op op;
  op.dy = dy.at.get();
  op.ld = dy.ld;
  lanes::launch(blocks, kNarrowNT, [=] { kernel(g, op); });
  int64_t bad = 0;
  for (int32_t i = 0; i < n; ++i)
    for (int32_t q = 0; q < k; ++q) {
      double s = 0.0;
      for (int32_t j = 0; j < m; ++j) s += dy.get(i, j) * w.get(q, j);
      bad += (double)(float)(T)(float)s != dx.get(i, q);
    }
  for (int32_t q = 0; q <= k; ++q)
    for (int32_t j = 0; j < m; ++j) {
      double s = 0.0, got = 0.0;
      for (int32_t i = 0; i < n; ++i)
        s += (q < k ? x.get(i, q) : 1.0) * dy.get(i, j);
      if (blocks > 1) {
        for (unsigned b = 0; b < blocks; ++b)
          got += part[b * plane + (int64_t)q * m + j];
      } else {
        got = q < k ? dw.get(q, j) : (double)db[j];
        if (q < k) s = (double)(float)(T)(float)s;
      }
      bad += s != got;
    }
  return report("one-pass backward", sizeof(T), n, k, m, pad, bad);
}

template <int DT, int COLS, int CH>
int narrow_bf16(int32_t n, int32_t k, int32_t m, int64_t pad,
                unsigned blocks) {
  return narrow_case<__bf16, PlainBf16>(
      n, k, m, pad, blocks, [](NarrowArgs<__bf16> g, PlainBf16 op) {
        k_narrow_bwd<PlainBf16, 1, DT, COLS, CH>(g, op);
      });
}
template <int DT, int CT>
int narrow_f32(int32_t n, int32_t k, int32_t m, int64_t pad,
               unsigned blocks) {
  return narrow_case<float, PlainF32>(
      n, k, m, pad, blocks, [](NarrowArgs<float> g, PlainF32 op) {
        k_narrow_bwd_f32<PlainF32, 1, DT, CT>(g, op);
      });
}

template <class T, int G, int NV>
int norm_case(int32_t n, int32_t d, int64_t pad, unsigned blocks) {
  Table<T> x(n, d, d + pad, 9);
  const Table<T> dy(n, d, d + pad, 3), dres(n, d, d + pad, 3);
  Table<T> y(n, d, d, 0), dx(n, d, d, 0);
  const Table<float> w(1, d, d, 2), b(1, d, d, 2);
  std::unique_ptr<float[]> mean(new float[n]), rstd(new float[n]),
      part(new float[blocks * 2 * d]);
  T *xp = x.at.get(), *yp = y.at.get(), *dxp = dx.at.get();
  const T *dyp = dy.at.get(), *rp = dres.at.get();
  const float *wp = w.at.get(), *bp = b.at.get();
  float *mp = mean.get(), *sp = rstd.get(), *pp = part.get();
  const int64_t ld = d + pad;
  lanes::launch(blocks, norm_nt(G), [=] {
    k_norm_fwd<T, T, G, NV>(xp, ld, n, d, wp, bp, 1.0f, yp, d, mp, sp);
  });
  lanes::launch(blocks, norm_nt(G), [=] {
    k_norm_bwd<T, T, G, NV>(dyp, ld, xp, ld, n, d, wp, mp, sp, rp, ld, dxp, d,
                            pp, pp + d);
  });
  int64_t bad = 0;
  const double ulp = sizeof(T) == 2 ? 1.0 / 128 : 1e-4;
  auto off = [&](double got, double ref) {
    bad += !(fabs(got - ref) <= ulp * (1.0 + fabs(ref)));
  };
  std::vector<double> dw(d), db(d);
  for (int32_t i = 0; i < n; ++i) {
    double m = 0.0, v = 0.0, s0 = 0.0, s1 = 0.0;
    for (int32_t j = 0; j < d; ++j) m += x.get(i, j) / d;
    for (int32_t j = 0; j < d; ++j) v += pow(x.get(i, j) - m, 2) / d;
    const double r = 1.0 / sqrt(v + 1.0);
    off(mean[i], m);
    off(rstd[i], r);
    for (int32_t j = 0; j < d; ++j) {
      const double h = (x.get(i, j) - m) * r, g = dy.get(i, j) * w.get(0, j);
      off(y.get(i, j), h * w.get(0, j) + b.get(0, j));
      s0 += g / d;
      s1 += g * h / d;
      dw[j] += dy.get(i, j) * h;
      db[j] += dy.get(i, j);
    }
    for (int32_t j = 0; j < d; ++j) {
      const double h = (x.get(i, j) - m) * r, g = dy.get(i, j) * w.get(0, j);
      off(dx.get(i, j), (g - s0 - h * s1) * r + dres.get(i, j));
    }
  }
  for (int32_t j = 0; j < d; ++j) {
    double gw = 0.0, gb = 0.0;
    for (unsigned k = 0; k < blocks; ++k) {
      gw += part[k * 2 * d + j];
      gb += part[k * 2 * d + d + j];
    }
    bad += !(fabs(gw - dw[j]) <= 1e-4 * n) + !(gb == db[j]);
  }
  return report("layer norm", sizeof(T), n, d, d, pad, bad);
}

}  // namespace

int main() {
  int bad = 0;
  for (int64_t pad : {0, 1, 9}) {
    // rows shorter than a vector, as few as they may be; several steps
    bad += narrow_bf16<1, 32, 1>(8, 1, 1, pad, 1);
    bad += narrow_bf16<1, 32, 1>(150, 3, 5, pad, 1);
    bad += narrow_bf16<1, 64, 1>(130, 31, 33, pad, 2);
    bad += narrow_bf16<2, 128, 1>(70, 40, 100, pad, 1);
    bad += narrow_bf16<1, 128, 2>(66, 9, 130, pad, 1);
    bad += narrow_f32<1, 1>(8, 1, 1, pad, 1);
    bad += narrow_f32<1, 1>(150, 3, 5, pad, 2);
    bad += narrow_f32<2, 4>(130, 17, 63, pad, 1);
    // tables of less than a vector, rows shorter than one, ragged ones
    bad += norm_case<__bf16, 1, 1>(1, 1, pad, 1);
    bad += norm_case<float, 1, 1>(7, 1, pad, 1);
    bad += norm_case<__bf16, 1, 1>(300, 3, pad, 1);
    bad += norm_case<float, 1, 1>(9, 7, pad, 1);
    bad += norm_case<float, 2, 1>(5, 9, pad, 1);
    bad += norm_case<__bf16, 16, 1>(40, 65, pad, 2);
    bad += norm_case<float, 64, 2>(9, 600, pad, 2);
    bad += norm_case<__bf16, 256, 1>(3, 1031, pad, 2);
  }
  return bad != 0;
}
