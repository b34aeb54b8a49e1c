// ezsp_attn_bwd.hip -- cross attention, backward: which kernels take a call.
#include "ezsp_attn.h"

namespace ezsp {
namespace {

template <class T, int B, int NC, int R>
void dq(Attn g, hipStream_t st) {
  constexpr int kCols = kAttnWaves * 16 * NC;
  const int64_t cols = (int64_t)g.nq * g.group;
  g.tiles = (int32_t)(g.q_off ? cols / kCols + g.clouds
                              : (cols + kCols - 1) / kCols);
  static_assert(R >= kLeastLines, "as attn_reserve counts");
  plan_parts<T>(g, cols, kCols, g.nk, R,
                (int64_t)g.nq * g.heads * width_of(B));
  hipLaunchKernelGGL((k_attn_dq<T, B, NC, R>),
                     grid_of(attn_grid(g)), dim3(kAttnNT), 0, st, g);
  if (g.splits > 1) {
    constexpr int D = width_of(B);
    const int64_t lanes = (int64_t)g.nq * g.heads * (D / 4);
    hipLaunchKernelGGL((k_attn_join_q<T, D>),
                       dim3((unsigned)((lanes + kAttnNT - 1) / kAttnNT)),
                       dim3(kAttnNT), 0, st, g);
  }
}

template <class T, int B, int NC, int R, bool KEPT>
void dkv(Attn g, hipStream_t st) {
  constexpr int kCols = kAttnWaves * 16 * NC;
  g.tiles = (int32_t)(g.k_off ? g.nk / kCols + g.clouds
                              : (g.nk + kCols - 1) / kCols);
  static_assert(R >= kLeastLines, "as attn_reserve counts");
  plan_parts<T>(g, g.nk, kCols, (int64_t)g.nq * g.group, R,
                (int64_t)g.nk * g.kv_heads * 2 * width_of(B));
  hipLaunchKernelGGL((k_attn_dkv<T, B, NC, R, KEPT>),
                     grid_of(attn_grid(g)), dim3(kAttnNT), 0, st, g);
  if (g.splits > 1) {
    constexpr int D = width_of(B);
    const int64_t lanes = (int64_t)g.nk * g.kv_heads * (D / 4);
    hipLaunchKernelGGL((k_attn_join_kv<T, D>),
                       dim3((unsigned)((lanes + kAttnNT - 1) / kAttnNT)),
                       dim3(kAttnNT), 0, st, g);
  }
}

template <class T, int B>
void both(const Attn &g, hipStream_t st) {
  typedef BackwardShape<T, B> S;
  constexpr int N = S::kGroups, R = S::kKeys, RQ = S::kRows;
  auto few = [&](int64_t cols, int64_t lines) {
    const int64_t per = kAttnWaves * 16 * 2;
    return (cols + per - 1) / per * g.kv_heads < kCus &&
           !parts_fill<T>(g, cols, per, lines);
  };
  if (g.dq) {
    if (few((int64_t)g.nq * g.group, g.nk))
      dq<T, B, 1, R>(g, st);
    else
      dq<T, B, N, R>(g, st);
  } else {
    const int64_t lanes = (int64_t)g.nq * g.heads * 4;
    hipLaunchKernelGGL((k_attn_delta<T, B>),
                       dim3((unsigned)std::min(
                           (lanes + kAttnNT - 1) / kAttnNT, kDeltaGrid)),
                       dim3(kAttnNT), 0, st, g);
  }
  if (!g.dk && !g.dv) return;
  if (few(g.nk, (int64_t)g.nq * g.group))
    dkv<T, B, 1, RQ, false>(g, st);
  else
    dkv<T, B, N, RQ, S::kKept>(g, st);
}

template <class T>
void dispatch(const Attn &g, hipStream_t st) {
  if (g.dh <= 16) return both<T, 1>(g, st);
  if (g.dh <= 32) return both<T, 2>(g, st);
  if (g.dh <= 48) return both<T, 3>(g, st);
  if (g.dh <= 64) return both<T, 4>(g, st);
  if (g.dh <= 80) return both<T, 5>(g, st);
  if (g.dh <= 96) return both<T, 6>(g, st);
  both<T, 8>(g, st);
}

}  // namespace

int attn_bwd_run(const AttnArgs &a, hipStream_t st) {
  const Attn g = attn_of(a);
  prof_begin("cross_attention", st);
  if (a.type == EZSP_TYPE_BF16)
    dispatch<__bf16>(g, st);
  else
    dispatch<float>(g, st);
  prof_end(st);
  const int rc =
      check_hip(hipGetLastError(), "cross attention gradient launch");
  prof_bytes("cross_attention",
             4.0 * a.dh * type_bytes(a.type) *
                 ((double)a.nq * a.heads + (double)a.nk * a.kv_heads));
  return rc;
}

}  // namespace ezsp
