// ezsp_linear.hip -- y = act(x W + b) + residual and its gradients
//   dz = dy act'(z),  dx = dz W^T,  dW = x^T dz,  db = sum over rows of dz.
// The forward pass is one matrix product with everything else in its
// epilogue.  Backward, dz is formed once (both products read it) with the
// bias's sums on the way; for bfloat16 it is rounded there, also from an fp32
// dy, while db is summed from the unrounded values.  The matrix cores take
// bfloat16 operands alike on both sides: dz in more bits would be a second
// bfloat16 term and twice the products' work, for gradients 0.0017 off in
// place of 0.0023.  Few columns take the one-pass kernel instead.
#include "ezsp_few.h"
#include "ezsp_narrow_f32.h"
#include "ezsp_narrow_fwd.h"

namespace ezsp {

namespace {

template <class T>
struct PrepLinear {
  const void *dy;
  int64_t lddy;
  int32_t type_y;
  const T *z;  // nullable with EZSP_ACT_NONE
  int64_t ldz;
  int32_t act;
  T *dz;       // nullable: dy itself serves
  int64_t lddz;
  __device__ __forceinline__ void at(int64_t row, int32_t col, int32_t cnt,
                                     f32x8_t *v) const {
    v[0] = load8_t(dy, row * lddy + col, type_y, cnt);
    if (act != EZSP_ACT_NONE)
      v[0] *= act_grad8(load8(z + row * ldz + col, cnt), act);
  }
  __device__ __forceinline__ void put(int64_t row, int32_t col, int32_t cnt,
                                      const f32x8_t *v) const {
    if (dz) store8(dz + row * lddz + col, v[0], kVec);  // zeros past the end
  }
};

// The same for the one-pass backward (bfloat16): dz from registers.
template <class TY, bool ACT>
struct NarrowLinear {
  const TY *dy;
  int64_t lddy;
  const __bf16 *z;
  int64_t ldz;
  int32_t act;
  struct Raw {
    Vec8<TY> dy;
    Vec8<__bf16> z[ACT ? 1 : 0];
  };
  __device__ __forceinline__ Raw raw(int64_t row, int32_t n, int32_t d,
                                     Span s) const {
    Raw r;
    int32_t back;
    r.dy = raw8(dy + span_at(row, lddy, n, d, s, back));
    if constexpr (ACT)
      r.z[0] = raw8(z + span_at(row, ldz, n, d, s, back));
    return r;
  }
  __device__ __forceinline__ void value(const Raw &r, int64_t row, int32_t n,
                                        int32_t d, Span s, f32x8_t *v) const {
    const int32_t cnt = row < n ? s.cnt : 0;
    int32_t back;
    span_at(row, lddy, n, d, s, back);
    v[0] = __builtin_convertvector(settle(r.dy, s.off + back, cnt), f32x8_t);
    if constexpr (ACT) {
      span_at(row, ldz, n, d, s, back);
      v[0] *= act_grad8(__builtin_convertvector(
                            settle(r.z[0], s.off + back, cnt), f32x8_t),
                        act);
    }
  }
};

// ... and for fp32, four columns at a time.
template <bool ACT>
struct NarrowLinearF32 {
  const float *dy;
  int64_t lddy;
  const float *z;
  int64_t ldz;
  int32_t act;
  struct Raw {
    f32x4_t dy, z[ACT ? 1 : 0];
  };
  __device__ __forceinline__ Raw raw(int64_t row, int32_t n, int32_t d,
                                     SpanOf<4> s) const {
    Raw r;
    int32_t back;
    r.dy = raw4(dy + span_at(row, lddy, n, d, s, back));
    if constexpr (ACT) r.z[0] = raw4(z + span_at(row, ldz, n, d, s, back));
    return r;
  }
  __device__ __forceinline__ void value(const Raw &r, int64_t row, int32_t n,
                                        int32_t d, SpanOf<4> s,
                                        f32x4_t *v) const {
    const int32_t cnt = row < n ? s.cnt : 0;
    int32_t back;
    span_at(row, lddy, n, d, s, back);
    v[0] = settle4(r.dy, s.off + back, cnt);
    if constexpr (ACT) {
      span_at(row, ldz, n, d, s, back);
      v[0] *= low4(
          act_grad8(widen4(settle4(r.z[0], s.off + back, cnt)), act));
    }
  }
};

template <class T, class Op>
void backward_narrow(const LinearArgs &a, hipStream_t st) {
  NarrowArgs<T> g = {};
  g.x = static_cast<const T *>(a.x);
  g.w[0] = g.w[1] = static_cast<const T *>(a.w);
  g.ldx = a.ldx;
  g.n = a.n;
  g.d_in = a.d_in;
  g.d_out = a.d_out;
  g.dx = static_cast<T *>(a.dx);
  g.lddx = a.lddx;
  g.part = a.part;
  Op op;
  op.dy = static_cast<decltype(op.dy)>(a.dy);
  op.lddy = a.lddy;
  op.z = static_cast<const T *>(a.z);
  op.ldz = a.ldz;
  op.act = act_for(a.act, a.type);
  g.dw[0] = static_cast<T *>(a.dw);
  g.db[0] = a.db;
  if constexpr (sizeof(T) == 2)
    narrow<Op, 1>(g, op, st);
  else
    narrow_f32<Op, 1>(g, op, st);
}

// dz has to be formed unless dy is it already, at an alignment that the
// products take at their full rate
bool needs_dz(const LinearArgs &a) {
  return a.act != EZSP_ACT_NONE || a.type_y != a.type ||
         !fast_operand(a.dy, a.lddy, a.d_out, (int32_t)type_bytes(a.type));
}

template <class T>
void forward(const LinearArgs &a, hipStream_t st) {
  GemmArgs<T> g = {};
  g.a[0] = static_cast<const T *>(a.x);
  g.b[0] = static_cast<const T *>(a.w);
  g.lda = a.ldx;
  g.ldb = a.d_out;
  g.m = a.n;
  g.n = a.d_out;
  g.k = a.d_in;
  EpiLinear e;
  e.part = a.part;
  e.bias = a.bias;
  e.res = a.res;
  e.ldr = a.ldr;
  e.y = a.y;
  e.ldy = a.ldy;
  e.z = a.z;
  e.ldz = a.ldz;
  e.type = a.type;
  e.type_y = a.type_y;
  e.act = act_for(a.act, a.type_y);
  if (few_serves(g, 1))
    few<T, 1>(g, e, st);
  else if (narrow_fwd_serves(g))
    narrow_fwd<T, 1>(g, e, st);
  else
    gemm<T, true, false, kPlain>(g, e, a.part_bytes, st);
}

template <class T>
void backward(const LinearArgs &a, hipStream_t st) {
  if (narrow_serves(a.type, a.n, a.d_in, a.d_out, 1)) {
    const bool none = a.act == EZSP_ACT_NONE;
    if constexpr (sizeof(T) == 4)
      none ? backward_narrow<T, NarrowLinearF32<false>>(a, st)
           : backward_narrow<T, NarrowLinearF32<true>>(a, st);
    else if (a.type_y == EZSP_TYPE_F32)
      none ? backward_narrow<T, NarrowLinear<float, false>>(a, st)
           : backward_narrow<T, NarrowLinear<float, true>>(a, st);
    else
      none ? backward_narrow<T, NarrowLinear<__bf16, false>>(a, st)
           : backward_narrow<T, NarrowLinear<__bf16, true>>(a, st);
    return;
  }
  const bool form = needs_dz(a) && (a.dx || a.dw);
  const T *dz = static_cast<const T *>(a.dy);
  int64_t lddz = a.lddy;
  if (form || a.db) {
    PrepLinear<T> p;
    p.dy = a.dy;
    p.lddy = a.lddy;
    p.type_y = a.type_y;
    p.z = static_cast<const T *>(a.z);
    p.ldz = a.ldz;
    p.act = act_for(a.act, a.type);
    p.dz = form ? static_cast<T *>(a.dz) : nullptr;
    p.lddz = pad_row(a.d_out);
    prep_launch<1>(p, a.n, a.d_out, a.part, a.db, nullptr, st);
  }
  if (form) {
    dz = static_cast<const T *>(a.dz);
    lddz = pad_row(a.d_out);
  }
  EpiStore<T, 1> e;
  e.part = a.part;
  GemmArgs<T> g = {};
  if (a.dx) {
    g.a[0] = dz;
    g.lda = lddz;
    g.b[0] = static_cast<const T *>(a.w);
    g.ldb = a.d_out;
    g.m = a.n;
    g.n = a.d_in;
    g.k = a.d_out;
    if (form) g.ka = (int32_t)lddz;
    e.out[0] = static_cast<T *>(a.dx);
    e.ld = a.lddx;
    gemm<T, true, true, kPlain>(g, e, a.part_bytes, st);
  }
  if (a.dw) {
    g = GemmArgs<T>{};
    g.a[0] = static_cast<const T *>(a.x);
    g.lda = a.ldx;
    g.b[0] = dz;
    g.ldb = lddz;
    g.m = a.d_in;
    g.n = a.d_out;
    g.k = a.n;
    if (form) g.rb = (int32_t)lddz;
    e.out[0] = static_cast<T *>(a.dw);
    e.ld = a.d_out;
    gemm<T, false, false, kPlain>(g, e, a.part_bytes, st);
  }
}

}  // namespace

void linear_reserve(Arena &ar, int64_t n, int64_t d_in, int64_t d_out,
                    int32_t type, bool bwd, LinearArgs *a) {
  a->part_bytes = gemm_fwd_bytes(n, d_in, d_out, 1);
  if (bwd) {
    // the one-pass kernel needs its parts alone, but sizes may not fall where
    // it starts to serve
    const int64_t rows =
        narrow_serves(type, n, d_in, d_out, 1) ? kVec - 1 : n;
    a->part_bytes = std::max(
        std::max(std::max(narrow_room(n, d_in, d_out, 1),
                          gemm_pack_bytes(n, d_in, d_out, type, 1)),
                 (size_t)prep_parts(rows) * (size_t)d_out * 4),
        std::max(gemm_part_bytes(d_out, rows, d_in, 1),
                 gemm_part_bytes(rows, d_in, d_out, 1)));
    a->dz = ar.take<char>((size_t)rows * (size_t)pad_row(d_out) *
                          type_bytes(type));
  }
  a->part = reinterpret_cast<float *>(ar.take<char>(a->part_bytes));
}

int linear_fwd_run(const LinearArgs &a, hipStream_t st) {
  prof_begin("linear", st);
  if (a.type == EZSP_TYPE_BF16)
    forward<__bf16>(a, st);
  else
    forward<float>(a, st);
  prof_end(st);
  const double e = (double)type_bytes(a.type), y = (double)type_bytes(a.type_y);
  prof_bytes("linear", (double)a.n * (a.d_in * e + a.d_out *
                                      (y + (a.res ? y : 0.0) +
                                       (a.z ? e : 0.0))) +
                           (double)a.d_in * a.d_out * e);
  return check_hip(hipGetLastError(), "linear launch");
}

int linear_bwd_run(const LinearArgs &a, hipStream_t st) {
  prof_begin("linear", st);
  if (a.type == EZSP_TYPE_BF16)
    backward<__bf16>(a, st);
  else
    backward<float>(a, st);
  prof_end(st);
  const double e = (double)type_bytes(a.type), y = (double)type_bytes(a.type_y);
  prof_bytes("linear", (double)a.n * (a.d_in * 2 * e + a.d_out *
                                      (y + (a.z ? e : 0.0))) +
                           2.0 * a.d_in * a.d_out * e);
  return check_hip(hipGetLastError(), "linear backward launch");
}

}  // namespace ezsp
