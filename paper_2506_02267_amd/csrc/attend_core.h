// The step that the attention kernels share: 32 keys against 32 QT queries of one wave, products on the
// 32x32x16 bf16 matrix instructions, everything between them in registers.
//
// Scores are taken transposed, S^T = K Q^T: a lane then holds one query (column l % 32) and, where the
// tile's rows are keys in the order pi(8j + 4h + i) = 16h + 4j + i, the 16 consecutive keys
// 16h .. 16h + 15 of it (h = l / 32), register r being key 16h + r.  Those registers, rounded to
// bf16, are the operand of O^T = V^T P^T as they stand, against 16 consecutive keys of a feature: one
// or two 16-byte loads where V lies by feature.  No lane exchanges but the joining of the two
// halves' maxima.
//
// The softmax's reference m is raised only where a weight would pass 2^RAISE, and then to where the
// largest is 2^ROOM or a little more: any reference gives the same quotient, the sums are fp32, and raising
// it is rare after a query's first keys.  The room is for weights in fp16, whose least step is 2^-24: 2^-30 of
// the largest weight.  A query's references are its own scores' alone, whatever its neighbours in the wave do.
// For weights in bf16 the largest is then 2^ROOM itself and not rounded, where it weighs most (error of 32
// sequences of 203 - 4000 tokens 0.0021 of the outputs, of which their own rounding 0.0016; with whole numbers
// as references 0.0023).  For fp16 weights, whose rounding counts for little, references are whole
// numbers, so that it does not depend on where they stand.
//
// Values may come with a scale 2^lv of their own for each block of keys.  What is multiplied is then a weight
// times 2^lv, against m; the weights' sum l has a reference of its own, n, since scales lie further apart
// than fp32's powers of two reach (m is kept as what it lies above n).  A block's part of it comes from the same
// exponentials, 2^(c s + lv - m): times 2^-lv 2^(m - n) = inv d.  A block whose products are all below 2^(m - FLOOR), or
// whose values are zeros (lv = -inf), adds nothing to the features, its weights being zeros in fp16; its
// exponentials are taken against its own largest score, for the sum alone.
//
// References past 2^20 are numbers that fp32 rounds to the size of an exponent and more, c s in the fused multiply-add
// is not rounded: their difference may then be anything, infinite weights included.  Such rows' scores are taken
// against the block's own largest one first, which leaves differences that are exact, of scores as fp32 rounds them.
#pragma once

#include <float.h>

#include "common.h"

namespace tav2 {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;

constexpr float RAISE = 14.f, ROOM = 6.f, FLOOR = 32.f, FAR = 0x1p20f;

__device__ __forceinline__ f32x16 mfma32(const f16x8& a, const f16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t pack2h(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){a, b}, f16x2));
}

// Row of a 32-key tile that lane l % 32 = m loads, so that register r is key 16h + r.
__device__ __forceinline__ int key_row(int m) { return 16 * ((m >> 2) & 1) + 4 * (m >> 3) + (m & 3); }

// What a wave keeps of 32 QT queries: O^T unnormalised (D / 32 tiles of 32 features), the
// reference m (powers of two; -FLT_MAX: no key yet, finite so that no difference is a NaN) and the
// sum l of this lane half's weights.
template <int D, int QT>
struct AttState {
  f32x16 o[D / 32][QT];
  float m[QT], l[QT];
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      m[q] = -FLT_MAX;
      l[q] = 0.f;
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][q][r] = 0.f;
    }
  }
};

// Which keys a lane's queries see: positions below hi that are at least lo or below sinks.
template <int QT>
struct AttSeen {
  int hi[QT], lo[QT];
  int sinks;
};

// With scaled values: n refers to the weights, n + m to the products, d = 2^m.
template <int D, int QT>
struct AttScaledState : AttState<D, QT> {
  float n[QT], d[QT];
  __device__ __forceinline__ void clear() {
    AttState<D, QT>::clear();
#pragma unroll
    for (int q = 0; q < QT; ++q) {
      this->m[q] = 0.f;
      n[q] = -FLT_MAX;
      d[q] = 1.f;
    }
  }
};

// What a block's values are to be multiplied by: nothing, or 2^lv = 1 / inv.
struct AttNoScale {};
struct AttScale {
  float lv, inv;
};

// Scores of keys that are not seen become -inf; returns the largest of the others, of both halves.
template <int QT, int NB>
__device__ __forceinline__ float att_mask(f32x16 (&s)[NB], int q, bool masked, const AttSeen<QT>& seen, int key0) {
  if (masked) {
    // against register numbers: nothing for each key is left to be prepared where nothing is masked
    const int hi = seen.hi[q] - key0, lo = seen.lo[q] - key0, sinks = seen.sinks - key0;
#pragma unroll
    for (int u = 0; u < NB; ++u)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int k = 32 * u + r;
        s[u][r] = k < hi && (k >= lo || k < sinks) ? s[u][r] : -INFINITY;
      }
  }
  float top = s[0][0];
#pragma unroll
  for (int r = 1; r < 16 * NB; ++r) top = vmax(top, s[r / 16][r % 16]);
  return xmax32(top);
}

// s becomes 2^(c s + b); returns the sum.
template <int NB>
__device__ __forceinline__ float att_exp(f32x16 (&s)[NB], float c, float b) {
  float sum = 0.f;
#pragma unroll
  for (int r = 0; r < 16 * NB; ++r) {
    const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r / 16][r % 16], c, b));
    s[r / 16][r % 16] = p;
    sum += p;
  }
  return sum;
}

// A largest score as a power of two, a number by itself: with the product fused into the subtractions that follow, a
// reference would not be what it is compared with.
__device__ __forceinline__ float att_top(float raw, float c) {
#pragma clang fp contract(off)
  return raw * c;
}
// Whether a reference is that large (the first one, of no key yet, is not), and whether one of the wave's may be: seldom,
// so the branch is laid out apart.
__device__ __forceinline__ bool att_far(float m) { return m > FAR || (m < -FAR && m > -FLT_MAX); }
__device__ __forceinline__ bool att_any_far(float m) { return __builtin_expect(__any(__builtin_fabsf(m) > FAR), false); }
// What a far row's scores are taken against, `raw` the block's largest one.
__device__ __forceinline__ float att_own(bool far, float raw) { return far && raw > -FLT_MAX ? raw : 0.f; }

// s: this lane's scores of query tile q against NB blocks of 32 keys; c s (c > 0) are powers of two; key0:
// position of the first key.  Leaves in s the weights (times the values' scale), against m.
template <int D, int QT, int NB>
__device__ __forceinline__ void att_softmax(AttState<D, QT>& st, int q, f32x16 (&s)[NB], float c, AttNoScale,
                                            bool masked, const AttSeen<QT>& seen, int key0) {
  const float raw = att_mask(s, q, masked, seen, key0), top = att_top(raw, c);
  if (__any(top - st.m[q] > RAISE)) {
    const float m = top - st.m[q] > RAISE ? top - ROOM : st.m[q];
    const float f = __builtin_amdgcn_exp2f(st.m[q] - m);
    st.m[q] = m;
    st.l[q] *= f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) st.o[d][q][r] *= f;
  }
  float b = -st.m[q];
  if (att_any_far(st.m[q])) {
    const bool far = att_far(st.m[q]);
    const float own = att_own(far, raw);
    b = far ? top - st.m[q] : b;
#pragma unroll
    for (int r = 0; r < 16 * NB; ++r) s[r / 16][r % 16] -= own;
  }
  st.l[q] += att_exp(s, c, b);
}

// Where a block's largest score `top` passes the references, those that it does not: m, n and d, and the factors
// of the features and of the sum so far.
__device__ __forceinline__ void att_raise(float top, float lv, float& m, float& n, float& d, float* of, float* lf) {
  const float n1 = top - n > RAISE ? __builtin_floorf(top) - ROOM : n;
  const float down = vmax(n - n1, -0x1p100f);   // (finite, from the first one on)
  const float t = top - n1, m0 = m + down;
  const float m1 = t + (lv - m0) > RAISE ? __builtin_floorf(t + lv) - ROOM : m0;
  *of = __builtin_amdgcn_exp2f(m0 - m1);
  *lf = __builtin_amdgcn_exp2f(down);
  d = __builtin_amdgcn_exp2f(m1);
  m = m1;
  n = n1;
}
__device__ __forceinline__ bool att_passes(float top, float lv, float m, float n) {
  const float t = top - n;
  return t > RAISE || t + (lv - m) > RAISE;   // (the first may be infinite, the second then a NaN)
}

// The exponentials' offset b, the factor e of their sum, and what the scores are taken against first (`raw` is the block's
// largest one, `top` the same as a power of two).  Returns whether that is anything but zero for some row.  Far rows are
// looked for with the other exception: with a test of their own 1000 candidates of one history took 40.6 us for 38.6.
__device__ __forceinline__ bool att_offset(float raw, float top, AttScale v, float m, float n, float d, float* b, float* e,
                                           float* own) {
  *b = v.lv - (n + m);
  *e = v.inv * d;
  *own = 0.f;
  const bool low = top + *b < -FLOOR;
  bool some_far = false;
  if (__any(low || __builtin_fabsf(n) > FAR)) {
    // (a score of 2^20 and more is itself rounded by 2^-24 of it: further below then.  Nothing seen: the
    // exponentials are zeros whatever they are taken against)
    const bool some = top > -FLT_MAX;
    const float bl = some ? -FLOOR - top - __builtin_fabsf(top) * 0x1p-22f : 0.f;
    const float el = some ? __builtin_amdgcn_exp2f(-bl - n) : 0.f;
    *b = low ? bl : *b;
    *e = low ? el : *e;
    const bool far = att_far(n);
    some_far = __any(far);
    if (some_far) {
      const float t = top - n, bt = t + (v.lv - m);
      *own = att_own(far, raw);
      *b = !far ? *b : bt < -FLOOR ? -FLOOR : bt;
      *e = !far ? *e : bt < -FLOOR ? __builtin_amdgcn_exp2f(t + FLOOR) : v.inv * d;
    }
  }
  return some_far;
}

template <int D, int QT, int NB>
__device__ __forceinline__ void att_softmax(AttScaledState<D, QT>& st, int q, f32x16 (&s)[NB], float c, AttScale v,
                                            bool masked, const AttSeen<QT>& seen, int key0) {
  const float raw = att_mask(s, q, masked, seen, key0), top = att_top(raw, c);
  if (__any(att_passes(top, v.lv, st.m[q], st.n[q]))) {
    float of, lf;
    att_raise(top, v.lv, st.m[q], st.n[q], st.d[q], &of, &lf);
    st.l[q] *= lf;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) st.o[d][q][r] *= of;
  }
  float b, e, own;
  if (att_offset(raw, top, v, st.m[q], st.n[q], st.d[q], &b, &e, &own)) {
#pragma unroll
    for (int r = 0; r < 16 * NB; ++r) s[r / 16][r % 16] -= own;
  }
  st.l[q] = __builtin_fmaf(att_exp(s, c, b), e, st.l[q]);
}

// 16 weights as the operands of two products, which take both in one type: bf16 where the values are bf16 (a
// weight is off by at most 2^-8, as each value may be already; fp16 would not hold the values), fp16 (2^-11)
// where they are codes.
__device__ __forceinline__ void att_operands(const f32x16& p, bf16x8 (&f)[2]) {
#pragma unroll
  for (int t = 0; t < 2; ++t)
    f[t] = as_bf16x8(make_uint4(pack2(p[8 * t], p[8 * t + 1]), pack2(p[8 * t + 2], p[8 * t + 3]),
                                pack2(p[8 * t + 4], p[8 * t + 5]), pack2(p[8 * t + 6], p[8 * t + 7])));
}
__device__ __forceinline__ void att_operands(const f32x16& p, f16x8 (&f)[2]) {
#pragma unroll
  for (int t = 0; t < 2; ++t)
    f[t] = __builtin_bit_cast(
        f16x8, make_uint4(pack2h(p[8 * t], p[8 * t + 1]), pack2h(p[8 * t + 2], p[8 * t + 3]),
                          pack2h(p[8 * t + 4], p[8 * t + 5]), pack2h(p[8 * t + 6], p[8 * t + 7])));
}

// NB blocks of 32 keys.  keys(u, kf) sets kf[t]: operand of block u's key row's features h D / 2 + 8t ..; qf the
// queries' likewise; values(u, vf) sets vf[d][t]: feature 32 d + l % 32, keys 16h + 8t .. of block u; c: a
// lane's queries' factors.
template <class V, int NB, int D, int QT, class State, class Keys, class Values, class Scale>
__device__ __forceinline__ void att_step(State& st, Keys keys, Values values, const V (&qf)[QT][D / 16],
                                         const float (&c)[QT], Scale scale, bool masked,
                                         const AttSeen<QT>& seen, int key0) {
  f32x16 s[QT][NB];
#pragma unroll
  for (int u = 0; u < NB; ++u) {
    V kf[D / 16];
    keys(u, kf);
#pragma unroll
    for (int q = 0; q < QT; ++q) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[q][u][r] = 0.f;
#pragma unroll
      for (int t = 0; t < D / 16; ++t) s[q][u] = mfma32(kf[t], qf[q][t], s[q][u]);
    }
  }
  V pf[QT][NB][2];
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    att_softmax(st, q, s[q], c[q], scale, masked, seen, key0);
#pragma unroll
    for (int u = 0; u < NB; ++u) att_operands(s[q][u], pf[q][u]);
  }
#pragma unroll
  for (int u = 0; u < NB; ++u) {
    V vf[D / 32][2];
    values(u, vf);
#pragma unroll
    for (int q = 0; q < QT; ++q)
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int t = 0; t < 2; ++t) st.o[d][q] = mfma32(vf[d][t], pf[q][u][t], st.o[d][q]);
  }
}

}  // namespace tav2
