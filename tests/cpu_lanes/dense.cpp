// dense.cpp -- k_few and the tile kernel's form for unaligned operands on the
// CPU: operands in allocations of their exact size, integer values, results
// compared for equality.  Prints a line per case; exits 1 if one differs.
#include "lanes.h"

#include <stdio.h>

#include <random>

#include "../../paper_2512_00385_amd/csrc/ezsp_few.h"

using namespace ezsp;

namespace {

template <class T>
struct Case {
  int32_t n, k, m;
  int64_t ldx;
  std::unique_ptr<T[]> x, w[2], y[2];
  std::vector<float> bias;

  // x: n rows ldx apart, the last one ending with the allocation
  Case(int32_t n, int32_t k, int32_t m, int64_t ldx)
      : n(n), k(k), m(m), ldx(ldx), bias(m) {
    std::mt19937 g(n + k + m);
    auto draw = [&] { return (float)((int)(g() % 5) - 2); };
    const int64_t len = (n - 1) * ldx + k;
    x.reset(new T[len]);
    for (int64_t i = 0; i < len; ++i)
      x[i] = (T)(i % ldx < k ? draw() : NAN);
    for (int p = 0; p < 2; ++p) {
      w[p].reset(new T[(int64_t)k * m]);
      for (int64_t i = 0; i < (int64_t)k * m; ++i) w[p][i] = (T)draw();
      y[p].reset(new T[(int64_t)n * m]);
    }
    for (float &b : bias) b = draw();
  }
  GemmArgs<T> args() const {
    GemmArgs<T> g = {};
    g.a[0] = g.a[1] = x.get();
    g.b[0] = w[0].get();
    g.b[1] = w[1].get();
    g.lda = ldx;
    g.ldb = m;
    g.m = n;
    g.n = m;
    g.k = k;
    return g;
  }
  EpiLinear linear() const {
    EpiLinear e = {};
    e.bias = bias.data();
    e.y = y[0].get();
    e.ldy = m;
    e.type = e.type_y = sizeof(T) == 2 ? EZSP_TYPE_BF16 : EZSP_TYPE_F32;
    e.act = EZSP_ACT_NONE;
    return e;
  }
  EpiStore<T, 2> both() const {
    EpiStore<T, 2> e = {};
    e.out[0] = y[0].get();
    e.out[1] = y[1].get();
    e.ld = m;
    return e;
  }
  // products p < np against sums in 64 bits; 0 if equal
  int differ(const char *name, int np, bool with_bias) const {
    int64_t bad = 0;
    for (int p = 0; p < np; ++p)
      for (int32_t i = 0; i < n; ++i)
        for (int32_t j = 0; j < m; ++j) {
          double s = with_bias ? bias[j] : 0.0;
          for (int32_t q = 0; q < k; ++q)
            s += (double)(float)x[i * ldx + q] *
                 (double)(float)w[p][(int64_t)q * m + j];
          bad += (float)(T)(float)s != (float)y[p][(int64_t)i * m + j];
        }
    printf("%s %s %d x %d -> %d, rows %lld apart: %lld wrong\n", name,
           sizeof(T) == 2 ? "bf16" : "fp32", n, k, m, (long long)ldx,
           (long long)bad);
    fflush(stdout);
    return bad != 0;
  }
};

template <class T, int V, int MT>
int few_case(int32_t n, int32_t k, int32_t m, int64_t ldx) {
  Case<T> c(n, k, m, ldx);
  const GemmArgs<T> g = c.args();
  const EpiLinear e = c.linear();
  lanes::launch((m + 16 * V - 1) / (16 * V), kFewNT,
                [=] { k_few<T, V, MT, 1, EpiLinear>(g, e); });
  return c.differ("few", 1, true);
}

// `blocks` blocks take all tiles of the shape.
template <class S, class Epi>
void tiles(GemmArgs<typename S::T> g, const Epi &e, unsigned blocks) {
  g.ra = g.m;
  g.rb = g.n;
  g.ka = g.kb = g.k;
  g.tiles_m = (g.m + S::BM - 1) / S::BM;
  g.tiles_n = (g.n + S::CN - 1) / S::CN;
  g.splits = 1;
  g.kt_split = (g.k + S::kK - 1) / S::kK;
  lanes::launch(blocks, S::NT, [=] { k_gemm<S, Epi>(g, e); });
}

template <class T, int BM, int BN, int WM, int WN>
int tile_case(int32_t n, int32_t k, int32_t m, int64_t ldx, unsigned blocks) {
  Case<T> c(n, k, m, ldx);
  tiles<Shape<T, BM, BN, WM, WN, true, false, kPlain, false>>(
      c.args(), c.linear(), blocks);
  return c.differ("tiles", 1, true);
}

template <class T, int BM, int BN, int WM, int WN>
int dual_case(int32_t n, int32_t k, int32_t m, int64_t ldx, unsigned blocks) {
  Case<T> c(n, k, m, ldx);
  tiles<Shape<T, BM, BN, WM, WN, true, false, kDual, false>>(
      c.args(), c.both(), blocks);
  return c.differ("dual tiles", 2, false);
}

// the weights' gradient: x^T dz, x [k][n] and dz [k][m], both in lines of k
template <class T, int BM, int BN, int WM, int WN>
int lines_case(int32_t n, int32_t k, int32_t m, unsigned blocks) {
  Case<T> c(n, k, m, k);
  std::unique_ptr<T[]> xt(new T[(int64_t)n * k]);
  for (int32_t i = 0; i < n; ++i)
    for (int32_t q = 0; q < k; ++q) xt[(int64_t)q * n + i] = c.x[i * k + q];
  GemmArgs<T> g = c.args();
  g.a[0] = g.a[1] = xt.get();
  g.lda = n;
  tiles<Shape<T, BM, BN, WM, WN, false, false, kPlain, false>>(g, c.linear(),
                                                               blocks);
  return c.differ("tiles of lines", 1, true);
}

// dx = dz W^T: both along k
template <class T, int BM, int BN, int WM, int WN>
int along_case(int32_t n, int32_t k, int32_t m, int64_t ldx,
               unsigned blocks) {
  Case<T> c(n, k, m, ldx);
  std::unique_ptr<T[]> wt(new T[(int64_t)k * m]);
  for (int32_t q = 0; q < k; ++q)
    for (int32_t j = 0; j < m; ++j)
      wt[(int64_t)j * k + q] = c.w[0][(int64_t)q * m + j];
  GemmArgs<T> g = c.args();
  g.b[0] = g.b[1] = wt.get();
  g.ldb = k;
  tiles<Shape<T, BM, BN, WM, WN, true, true, kPlain, false>>(g, c.linear(),
                                                             blocks);
  return c.differ("tiles along k", 1, true);
}

}  // namespace

int main(int argc, char **argv) {
  int bad = 0;
  const bool few = argc > 1 && !strcmp(argv[1], "few");
  if (few) {
    // columns that leave 1 to V - 1 for the last block, and none
    for (int32_t m : {4, 31, 32, 33, 65}) {
      bad += few_case<__bf16, 2, 1>(3, 70, m, 70);
      bad += few_case<float, 2, 1>(3, 37, m, 40);
    }
    for (int32_t m : {63, 65, 66, 67}) {
      bad += few_case<__bf16, 4, 1>(2, 33, m, 35);
      bad += few_case<float, 4, 2>(20, 17, m, 17);
    }
  } else {
    bad += tile_case<__bf16, 128, 128, 2, 2>(300, 100, 100, 100, 1);
    bad += tile_case<__bf16, 128, 64, 4, 1>(270, 65, 61, 67, 2);
    bad += tile_case<float, 128, 64, 2, 2>(300, 33, 70, 35, 2);
    bad += tile_case<__bf16, 32, 128, 1, 4>(7, 130, 300, 131, 1);
    bad += dual_case<__bf16, 128, 128, 2, 2>(260, 33, 130, 33, 1);
    bad += dual_case<float, 128, 64, 4, 1>(150, 24, 70, 25, 1);
    bad += lines_case<__bf16, 128, 128, 2, 2>(130, 70, 257, 1);
    bad += lines_case<float, 128, 64, 2, 2>(130, 35, 67, 1);
    bad += along_case<__bf16, 128, 64, 4, 1>(300, 42, 61, 43, 1);
    bad += along_case<float, 128, 64, 2, 2>(140, 101, 67, 101, 1);
  }
  return bad != 0;
}
