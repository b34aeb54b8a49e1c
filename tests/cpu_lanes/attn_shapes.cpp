// attn_shapes.cpp -- cross attention's kernels on the CPU in the tile shapes
// that the library launches (ForwardShape, BackwardShape), few columns' and
// many columns': operands in allocations of their exact size, uneven clouds,
// shared heads, masked keys, lines in parts.  Values are whole numbers with q
// and k on different places of d, so S = 0, P = 1 and every sum is exact.
// Prints a line per case; exits 1 if one differs.  PART (0 to 4) says which
// shapes this program holds.
#include "lanes.h"

#include <stdio.h>

#include <random>

namespace lanes {
inline uint64_t ballot(bool v) {
  Wave &w = wave();
  w.a[lane()][0] = v;
  wave_meets();
  uint64_t r = 0;
  for (int i = 0; i < kWaveLanes; ++i) r |= (uint64_t)w.a[i][0] << i;
  wave_meets();
  return r;
}
}  // namespace lanes
#define __ballot(v) lanes::ballot(v)
#define __popcll(v) __builtin_popcountll(v)
#define __builtin_amdgcn_logf log2f

#include "../../paper_2512_00385_amd/csrc/ezsp_attn.h"

using namespace ezsp;

namespace {

constexpr double kScale = 0.25;

template <class T>
struct Table {
  int64_t ld;
  std::unique_ptr<T[]> v;
  // rows ld apart, the last one ending with the allocation; of each head's dh
  // places those with d % 2 == zero hold 0, the others -1, 0 or 1; NaN between
  // rows, and everywhere without a generator
  Table(int rows, int cols, int dh, int pad, std::mt19937 *g, int zero = -1)
      : ld(cols + pad) {
    const int64_t len = (int64_t)(rows - 1) * ld + cols;
    v.reset(new T[len]);
    for (int64_t i = 0; i < len; ++i) {
      const int c = (int)(i % ld);
      float x = NAN;
      if (c < cols && g)
        x = c % dh % 2 == zero ? 0.0f : (float)((int)((*g)() % 3) - 1);
      v[i] = (T)x;
    }
  }
  double at(int r, int c) const { return (double)(float)v[r * ld + c]; }
};

struct Batch {
  std::vector<int> q_off, k_off;  // of the clouds; empty: one
  int nq, nk;
};

template <class T, int B, bool FEW>
bool run(int heads, int kv_heads, int dh, const Batch &s, int splits) {
  typedef ForwardShape<T, B> F;
  typedef BackwardShape<T, B> W;
  constexpr int D = width_of(B);
  constexpr int NF = FEW ? 1 : F::kGroups, RF = FEW ? F::kFewKeys : F::kKeys;
  constexpr int NB = FEW ? 1 : W::kGroups;
  constexpr bool kKept = !FEW && W::kKept;
  std::mt19937 gen(s.nq * 7 + s.nk + dh);
  const int wq = heads * dh, wk = kv_heads * dh;
  Table<T> q(s.nq, wq, dh, 3, &gen, 1), k(s.nk, wk, dh, 1, &gen, 0),
      v(s.nk, wk, dh, 0, &gen), dout(s.nq, wq, dh, 0, &gen),
      given(s.nq, wq, dh, 5, &gen), out(s.nq, wq, dh, 2, nullptr),
      dq(s.nq, wq, dh, 0, nullptr), dk(s.nk, wk, dh, 5, nullptr),
      dv(s.nk, wk, dh, 0, nullptr);
  std::vector<float> bias(s.nk), lse((size_t)heads * s.nq, NAN),
      delta((size_t)heads * s.nq, NAN);
  for (int j = 0; j < s.nk; ++j)
    if (j % 7 == 3) {  // what a masked key holds enters nowhere
      bias[j] = -INFINITY;
      for (int c = 0; c < wk; ++c) k.v[j * k.ld + c] = v.v[j * v.ld + c] = NAN;
    }
  const bool one = s.q_off.empty();
  const int clouds = one ? 1 : (int)s.q_off.size() - 1;
  std::vector<float> part((size_t)splits *
                          std::max(s.nq * heads * (D + 2),
                                   s.nk * kv_heads * 2 * D));
  AttnArgs a = {};
  a.q = q.v.get(), a.ldq = q.ld, a.nq = s.nq;
  a.k = k.v.get(), a.ldk = k.ld, a.v = v.v.get(), a.ldv = v.ld, a.nk = s.nk;
  a.heads = heads, a.kv_heads = kv_heads, a.dh = dh;
  if (!one) a.q_off = s.q_off.data(), a.k_off = s.k_off.data();
  a.n_clouds = clouds;
  a.bias = bias.data();
  a.scale = (float)kScale;
  a.out = out.v.get(), a.ldo = out.ld, a.lse = lse.data();
  a.dout = dout.v.get(), a.lddo = dout.ld;
  a.dq = dq.v.get(), a.lddq = dq.ld, a.dk = dk.v.get(), a.lddk = dk.ld;
  a.dv = dv.v.get(), a.lddv = dv.ld;
  a.delta = delta.data(), a.part = part.data();

  Attn g = attn_of(a);
  const int cols = s.nq * g.group;
  auto tiles = [&](int n, int per) {
    return one ? (n + per - 1) / per : n / per + g.clouds;
  };
  auto blocks = [&](int64_t lanes) {
    return (unsigned)((lanes + kAttnNT - 1) / kAttnNT);
  };
  g.splits = splits;
  g.chunk = s.nk / splits / 2 + 1;  // (some clouds come in one part)
  g.tiles = tiles(cols, kAttnWaves * 16 * NF);
  lanes::launch(attn_grid(g), kAttnNT, [g] { k_attn_fwd<T, B, NF, RF>(g); });
  if (splits > 1)
    lanes::launch(blocks((int64_t)s.nq * heads * (D / 4)), kAttnNT,
                  [g] { k_attn_join<T, D, false>(g); });
  const std::vector<float> got_lse = lse;
  for (float &l : lse) l = l == -INFINITY ? l : 0.0f;  // says P = 1
  g.out = given.v.get(), g.ldo = given.ld;
  g.tiles = tiles(cols, kAttnWaves * 16 * NB);
  lanes::launch(attn_grid(g), kAttnNT,
                [g] { k_attn_dq<T, B, NB, W::kKeys>(g); });
  if (splits > 1)
    lanes::launch(blocks((int64_t)s.nq * heads * (D / 4)), kAttnNT,
                  [g] { k_attn_join_q<T, D>(g); });
  g.tiles = tiles(s.nk, kAttnWaves * 16 * NB);
  g.chunk = s.nq * g.group / splits / 2 + 1;
  lanes::launch(attn_grid(g), kAttnNT,
                [g] { k_attn_dkv<T, B, NB, W::kRows, kKept>(g); });
  if (splits > 1)
    lanes::launch(blocks((int64_t)s.nk * kv_heads * (D / 4)), kAttnNT,
                  [g] { k_attn_join_kv<T, D>(g); });

  // the sums, cloud by cloud; rows of none have no keys
  std::vector<int> qc(s.nq, -1), kc(s.nk, -1);
  for (int c = 0; c < clouds; ++c) {
    for (int i = one ? 0 : s.q_off[c]; i < (one ? s.nq : s.q_off[c + 1]); ++i)
      qc[i] = c;
    for (int j = one ? 0 : s.k_off[c]; j < (one ? s.nk : s.k_off[c + 1]); ++j)
      kc[j] = c;
  }
  std::vector<double> rdk(s.nk * wk), rdv(s.nk * wk);
  int wrong = 0;
  auto same = [&](double got, double ref) {  // one rounding to the type
    if (got != (double)(float)(T)(float)ref) ++wrong;
  };
  for (int i = 0; i < s.nq; ++i)
    for (int h = 0; h < heads; ++h) {
      const int kh = h / g.group;
      std::vector<double> total(dh), rq(dh);
      double along = 0;
      int n = 0;
      for (int d = 0; d < dh; ++d)
        along += dout.at(i, h * dh + d) * given.at(i, h * dh + d);
      for (int j = 0; j < s.nk; ++j) {
        if (kc[j] < 0 || kc[j] != qc[i] || bias[j] == -INFINITY) continue;
        ++n;
        double dp = 0;
        for (int d = 0; d < dh; ++d)
          dp += dout.at(i, h * dh + d) * v.at(j, kh * dh + d);
        for (int d = 0; d < dh; ++d) {
          const int ck = j * wk + kh * dh + d;
          total[d] += v.at(j, kh * dh + d);
          rq[d] += kScale * (dp - along) * k.at(j, kh * dh + d);
          rdk[ck] += kScale * (dp - along) * q.at(i, h * dh + d);
          rdv[ck] += dout.at(i, h * dh + d);
        }
      }
      const double half = sizeof(T) == 2 ? 0x1p-8 : 0x1p-24;
      for (int d = 0; d < dh; ++d) {
        const double ref = n ? total[d] / n : 0.0;
        if (!(fabs(out.at(i, h * dh + d) - ref) <=
              1.01 * (half + 0x1p-23) * fabs(ref)))
          ++wrong;
        same(dq.at(i, h * dh + d), rq[d]);
      }
      const float l = got_lse[(size_t)h * s.nq + i];
      if (n ? !(fabs(l - log((double)n)) <= 5 * 0x1p-24 * log((double)n))
            : l != -INFINITY)
        ++wrong;
    }
  for (int j = 0; j < s.nk; ++j)
    for (int c = 0; c < wk; ++c) {
      same(dk.at(j, c), rdk[j * wk + c]);
      same(dv.at(j, c), rdv[j * wk + c]);
    }
  printf("%s %s, %d x %d, %d / %d heads of %d, %d clouds, %d parts: %d wrong\n",
         sizeof(T) == 2 ? "bf16" : "fp32", FEW ? "few columns" : "many columns",
         s.nq, s.nk, heads, kv_heads, dh, clouds, splits, wrong);
  fflush(stdout);
  return wrong == 0;
}

template <class T, int B>
bool shape() {
  // a cloud that is longer than a tile on both sides, single rows and keys,
  // empty ones; rows and keys of none in front and behind
  const Batch uneven = {{1, 3, 3, 100, 101, 103}, {2, 2, 40, 178, 179, 181},
                        104, 183};
  const Batch whole = {{}, {}, 97, 131};
  bool ok = run<T, B, false>(2, 1, 16 * B, uneven, 2);
  ok &= run<T, B, false>(1, 1, 16 * B - 5, whole, 3);
  ok &= run<T, B, true>(2, 2, 16 * B - 9, uneven, 1);
  return ok;
}

}  // namespace

int main() {
  bool ok = true;
#if PART == 0
  ok &= shape<__bf16, 1>() & shape<__bf16, 2>() & shape<__bf16, 3>();
#elif PART == 1
  ok &= shape<__bf16, 4>() & shape<__bf16, 5>();
#elif PART == 2
  ok &= shape<__bf16, 6>() & shape<__bf16, 8>();
#elif PART == 3
  ok &= shape<float, 1>() & shape<float, 2>() & shape<float, 3>();
#else
  ok &= shape<float, 4>() & shape<float, 5>() & shape<float, 6>() &
        shape<float, 8>();
#endif
  return ok ? 0 : 1;
}
