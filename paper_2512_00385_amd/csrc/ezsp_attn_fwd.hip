// ezsp_attn_fwd.hip -- cross attention, forward: which kernel takes a call.
#include "ezsp_attn.h"

namespace ezsp {
namespace {

template <class T, int B, int NC, int R>
void launch(Attn g, hipStream_t st) {
  constexpr int kCols = kAttnWaves * 16 * NC;
  const int64_t cols = (int64_t)g.nq * g.group;
  g.tiles = (int32_t)(g.q_off ? cols / kCols + g.clouds
                              : (cols + kCols - 1) / kCols);
  // few columns leave the chip empty: the keys in parts of two tiles or more
  static_assert(R >= kLeastLines, "as attn_reserve counts");
  plan_parts<T>(g, cols, kCols, g.nk, R,
                (int64_t)g.nq * g.heads * (width_of(B) + 2));
  hipLaunchKernelGGL((k_attn_fwd<T, B, NC, R>),
                     grid_of(attn_grid(g)), dim3(kAttnNT), 0, st, g);
  if (g.splits == 1) return;
  constexpr int D = width_of(B), kPer = kAttnNT / (D / 4);
  const int64_t joined = (int64_t)g.nq * g.heads;
  if (g.splits > kWideSplits)
    hipLaunchKernelGGL((k_attn_join<T, D, true>), dim3((unsigned)joined),
                       dim3(kAttnNT), 0, st, g);
  else
    hipLaunchKernelGGL((k_attn_join<T, D, false>),
                       dim3((unsigned)((joined + kPer - 1) / kPer)),
                       dim3(kAttnNT), 0, st, g);
}

template <class T, int B>
void by_columns(const Attn &g, hipStream_t st) {
  typedef ForwardShape<T, B> S;
  constexpr int N = S::kGroups;
  const int64_t cols = (int64_t)g.nq * g.group * g.kv_heads;
  if (cols < 256 * kAttnWaves * 16 &&
      !parts_fill<T>(g, (int64_t)g.nq * g.group, kAttnWaves * 16 * N, g.nk))
    launch<T, B, 1, S::kFewKeys>(g, st);
  else
    launch<T, B, N, S::kKeys>(g, st);
}

template <class T>
void dispatch(const Attn &g, hipStream_t st) {
  if (g.dh <= 16) return by_columns<T, 1>(g, st);
  if (g.dh <= 32) return by_columns<T, 2>(g, st);
  if (g.dh <= 48) return by_columns<T, 3>(g, st);
  if (g.dh <= 64) return by_columns<T, 4>(g, st);
  if (g.dh <= 80) return by_columns<T, 5>(g, st);
  if (g.dh <= 96) return by_columns<T, 6>(g, st);
  by_columns<T, 8>(g, st);
}

}  // namespace

void attn_reserve(Arena &ar, int64_t nq, int64_t nk, int64_t heads,
                  int64_t kv_heads, int64_t dh, bool bwd, AttnArgs *a) {
  const int64_t d = width_of((int)((dh + 15) / 16));
  // As many parts of the sums as plan_parts may choose, up to kPartFloats; a
  // size that grows with every argument.  (Calls of so many columns that they
  // come in one part have kPartFloats too, as smaller ones use it.)
  const auto floats = [](int64_t part, int64_t parts) {
    return (size_t)std::min(part * parts, kPartFloats);
  };
  const int64_t of_keys = std::min<int64_t>(kMaxSplits, 2 * (nk / kLeastLines));
  if (!bwd) {
    a->part = ar.take<float>(floats(nq * heads * (d + 2), of_keys));
    return;
  }
  a->delta = ar.take<float>((size_t)(nq * heads));
  // dq's and then dk's and dv's, whose lines are the rows of heads / kv_heads
  // heads: the parts of all kv_heads
  const int64_t of_rows = std::min<int64_t>(kMaxSplits * kv_heads,
                                            2 * nq * heads / kLeastLines);
  a->part = ar.take<float>(std::max(floats(nq * heads * d, of_keys),
                                    floats(nk * 2 * d, of_rows)));
}

int attn_fwd_run(const AttnArgs &a, hipStream_t st) {
  const Attn g = attn_of(a);
  prof_begin("cross_attention", st);
  if (a.type == EZSP_TYPE_BF16)
    dispatch<__bf16>(g, st);
  else
    dispatch<float>(g, st);
  prof_end(st);
  const int rc = check_hip(hipGetLastError(), "cross attention launch");
  prof_bytes("cross_attention",
             2.0 * a.dh * type_bytes(a.type) *
                 ((double)a.nq * a.heads + (double)a.nk * a.kv_heads));
  return rc;
}

}  // namespace ezsp
