// ezsp_gated.hip -- the gated feed-forward product
//   g = x Wg + bg,  u = x Wu + bu,  h = act(g) u
// in one kernel (a block holds the same columns of both products, so the
// activation and the product happen on its accumulators), and its gradients
//   dg = dh u act'(g),  du = dh act(g),
//   dx = dg Wg^T + du Wu^T,  dWg = x^T dg,  dWu = x^T du,  db = row sums.
// dg and du are formed once, side by side in one table (in bfloat16 for
// bfloat16 inputs, the matrix cores' operands); dx sums over both in
// one product of twice the length, and both weights' gradients come from one
// pass over x.  Few columns take the one-pass kernel instead.
#include "ezsp_few.h"
#include "ezsp_narrow_f32.h"
#include "ezsp_narrow_fwd.h"

namespace ezsp {

namespace {

template <class T>
struct PrepGated {
  const T *dh, *gate, *up;
  int64_t lddh, lds;
  int32_t act;
  T *dz;  // dg | du, nullable
  int64_t lddz, half;
  __device__ __forceinline__ void at(int64_t row, int32_t col, int32_t cnt,
                                     f32x8_t *v) const {
    const f32x8_t d = load8(dh + row * lddh + col, cnt);
    const f32x8_t g = load8(gate + row * lds + col, cnt);
    const f32x8_t u = load8(up + row * lds + col, cnt);
    f32x8_t a, da;
    act_both8(g, act, a, da);
    v[0] = d * u * da;
    v[1] = d * a;
  }
  __device__ __forceinline__ void put(int64_t row, int32_t col, int32_t cnt,
                                      const f32x8_t *v) const {
    if (!dz) return;
    store8(dz + row * lddz + col, v[0], kVec);  // zeros past the end
    store8(dz + row * lddz + half + col, v[1], kVec);
  }
};

// The same for the one-pass backward: dg and du from registers.
struct NarrowGated {
  const __bf16 *dh, *gate, *up;
  int64_t lddh, lds;
  int32_t act;
  struct Raw {
    Vec8<__bf16> d, g, u;
  };
  __device__ __forceinline__ Raw raw(int64_t row, int32_t n, int32_t d,
                                     Span s) const {
    Raw r;
    int32_t back;
    r.d = raw8(dh + span_at(row, lddh, n, d, s, back));
    const int64_t at = span_at(row, lds, n, d, s, back);
    r.g = raw8(gate + at);
    r.u = raw8(up + at);
    return r;
  }
  __device__ __forceinline__ void value(const Raw &r, int64_t row, int32_t n,
                                        int32_t d, Span s, f32x8_t *v) const {
    const int32_t cnt = row < n ? s.cnt : 0;
    int32_t back;
    span_at(row, lds, n, d, s, back);
    const f32x8_t g =
        __builtin_convertvector(settle(r.g, s.off + back, cnt), f32x8_t);
    const f32x8_t u =
        __builtin_convertvector(settle(r.u, s.off + back, cnt), f32x8_t);
    span_at(row, lddh, n, d, s, back);
    const f32x8_t dv =
        __builtin_convertvector(settle(r.d, s.off + back, cnt), f32x8_t);
    f32x8_t a, da;
    act_both8(g, act, a, da);
    v[0] = dv * u * da;
    v[1] = dv * a;
  }
};

// ... and for fp32, four columns at a time.
struct NarrowGatedF32 {
  const float *dh, *gate, *up;
  int64_t lddh, lds;
  int32_t act;
  struct Raw {
    f32x4_t d, g, u;
  };
  __device__ __forceinline__ Raw raw(int64_t row, int32_t n, int32_t d,
                                     SpanOf<4> s) const {
    Raw r;
    int32_t back;
    r.d = raw4(dh + span_at(row, lddh, n, d, s, back));
    const int64_t at = span_at(row, lds, n, d, s, back);
    r.g = raw4(gate + at);
    r.u = raw4(up + at);
    return r;
  }
  __device__ __forceinline__ void value(const Raw &r, int64_t row, int32_t n,
                                        int32_t d, SpanOf<4> s,
                                        f32x4_t *v) const {
    const int32_t cnt = row < n ? s.cnt : 0;
    int32_t back;
    span_at(row, lds, n, d, s, back);
    const f32x4_t u = settle4(r.u, s.off + back, cnt);
    f32x8_t a, da;
    act_both8(widen4(settle4(r.g, s.off + back, cnt)), act, a, da);
    span_at(row, lddh, n, d, s, back);
    const f32x4_t dv = settle4(r.d, s.off + back, cnt);
    v[0] = dv * u * low4(da);
    v[1] = dv * low4(a);
  }
};

template <class T, class Op>
void backward_narrow(const GatedArgs &a, hipStream_t st) {
  NarrowArgs<T> g = {};
  g.x = static_cast<const T *>(a.x);
  g.w[0] = static_cast<const T *>(a.w_gate);
  g.w[1] = static_cast<const T *>(a.w_up);
  g.ldx = a.ldx;
  g.n = a.n;
  g.d_in = a.d_in;
  g.d_out = a.d_out;
  g.dx = static_cast<T *>(a.dx);
  g.lddx = a.lddx;
  g.part = a.part;
  Op op;
  op.dh = static_cast<const T *>(a.dh);
  op.gate = static_cast<const T *>(a.gate);
  op.up = static_cast<const T *>(a.up);
  op.lddh = a.lddh;
  op.lds = a.lds;
  op.act = act_for(a.act, a.type);
  g.dw[0] = static_cast<T *>(a.dw_gate);
  g.dw[1] = static_cast<T *>(a.dw_up);
  g.db[0] = a.db_gate;
  g.db[1] = a.db_up;
  if constexpr (sizeof(T) == 2)
    narrow<Op, 2>(g, op, st);
  else
    narrow_f32<Op, 2>(g, op, st);
}

template <class T>
void forward(const GatedArgs &a, hipStream_t st) {
  GemmArgs<T> g = {};
  g.a[0] = g.a[1] = static_cast<const T *>(a.x);
  g.b[0] = static_cast<const T *>(a.w_gate);
  g.b[1] = static_cast<const T *>(a.w_up);
  g.lda = a.ldx;
  g.ldb = a.d_out;
  g.m = a.n;
  g.n = a.d_out;
  g.k = a.d_in;
  EpiGated<T> e;
  e.part = a.part;
  e.bias[0] = a.b_gate;
  e.bias[1] = a.b_up;
  e.h = static_cast<T *>(a.h);
  e.ldh = a.ldh;
  e.gate = static_cast<T *>(a.gate);
  e.up = static_cast<T *>(a.up);
  e.lds = a.lds;
  e.act = act_for(a.act, a.type);
  if (few_serves(g, 2))
    few<T, 2>(g, e, st);
  else if (narrow_fwd_serves(g))
    narrow_fwd<T, 2>(g, e, st);
  else
    gemm<T, true, false, kDual>(g, e, a.part_bytes, st);
}

template <class T>
void backward(const GatedArgs &a, hipStream_t st) {
  if (narrow_serves(a.type, a.n, a.d_in, a.d_out, 2)) {
    if constexpr (sizeof(T) == 2)
      backward_narrow<T, NarrowGated>(a, st);
    else
      backward_narrow<T, NarrowGatedF32>(a, st);
    return;
  }
  const int64_t half = pad_row(a.d_out);
  T *dz = static_cast<T *>(a.dz);
  {
    PrepGated<T> p;
    p.dh = static_cast<const T *>(a.dh);
    p.lddh = a.lddh;
    p.gate = static_cast<const T *>(a.gate);
    p.up = static_cast<const T *>(a.up);
    p.lds = a.lds;
    p.act = act_for(a.act, a.type);
    p.dz = a.dx || a.dw_gate || a.dw_up ? dz : nullptr;
    p.lddz = 2 * half;
    p.half = half;
    prep_launch<2>(p, a.n, a.d_out, a.part, a.db_gate, a.db_up, st);
  }
  GemmArgs<T> g = {};
  if (a.dx) {
    g.a[0] = dz;
    g.a[1] = dz + half;
    g.lda = 2 * half;
    g.b[0] = static_cast<const T *>(a.w_gate);
    g.b[1] = static_cast<const T *>(a.w_up);
    g.ldb = a.d_out;
    g.m = a.n;
    g.n = a.d_in;
    g.k = a.d_out;
    g.ka = (int32_t)half;
    EpiStore<T, 1> e;
    e.part = a.part;
    e.out[0] = static_cast<T *>(a.dx);
    e.ld = a.lddx;
    gemm<T, true, true, kSeq>(g, e, a.part_bytes, st);
  }
  if (a.dw_gate || a.dw_up) {
    g = GemmArgs<T>{};
    g.a[0] = g.a[1] = static_cast<const T *>(a.x);
    g.lda = a.ldx;
    g.b[0] = dz;
    g.b[1] = dz + half;
    g.ldb = 2 * half;
    g.m = a.d_in;
    g.n = a.d_out;
    g.k = a.n;
    g.rb = (int32_t)half;
    EpiStore<T, 2> e;
    e.part = a.part;
    e.out[0] = static_cast<T *>(a.dw_gate);
    e.out[1] = static_cast<T *>(a.dw_up);
    e.ld = a.d_out;
    gemm<T, false, false, kDual>(g, e, a.part_bytes, st);
  }
}

}  // namespace

void gated_reserve(Arena &ar, int64_t n, int64_t d_in, int64_t d_out,
                   int32_t type, bool bwd, GatedArgs *a) {
  a->part_bytes = gemm_fwd_bytes(n, d_in, d_out, 2);
  if (bwd) {
    // (sizes may not fall where the one-pass kernel starts to serve)
    const int64_t rows =
        narrow_serves(type, n, d_in, d_out, 2) ? kVec - 1 : n;
    a->part_bytes = std::max(
        std::max(std::max(narrow_room(n, d_in, d_out, 2),
                          gemm_pack_bytes(n, d_in, d_out, type, 2)),
                 (size_t)prep_parts(rows) * 2 * (size_t)d_out * 4),
        std::max(gemm_part_bytes(2 * d_out, rows, d_in, 1),
                 gemm_part_bytes(rows, d_in, d_out, 2)));
    a->dz = ar.take<char>((size_t)rows * 2 * (size_t)pad_row(d_out) *
                          type_bytes(type));
  }
  a->part = reinterpret_cast<float *>(ar.take<char>(a->part_bytes));
}

int gated_fwd_run(const GatedArgs &a, hipStream_t st) {
  prof_begin("gated_ff", st);
  if (a.type == EZSP_TYPE_BF16)
    forward<__bf16>(a, st);
  else
    forward<float>(a, st);
  prof_end(st);
  const double e = (double)type_bytes(a.type);
  prof_bytes("gated_ff", e * ((double)a.n * (a.d_in + a.d_out *
                                             (1.0 + (a.gate ? 2.0 : 0.0))) +
                              2.0 * a.d_in * a.d_out));
  return check_hip(hipGetLastError(), "gated_ff launch");
}

int gated_bwd_run(const GatedArgs &a, hipStream_t st) {
  prof_begin("gated_ff", st);
  if (a.type == EZSP_TYPE_BF16)
    backward<__bf16>(a, st);
  else
    backward<float>(a, st);
  prof_end(st);
  const double e = (double)type_bytes(a.type);
  prof_bytes("gated_ff", e * ((double)a.n * (2.0 * a.d_in + 3.0 * a.d_out) +
                              4.0 * a.d_in * a.d_out));
  return check_hip(hipGetLastError(), "gated_ff backward launch");
}

}  // namespace ezsp
