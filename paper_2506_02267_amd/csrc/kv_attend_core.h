// Attention over the cache's pages: what the kernels share, from a page's codes to a tile's state.
#pragma once

#include <algorithm>

#include "attend_core.h"
#include "internal.h"
#include "kv_common.h"
#include "token_source.h"

namespace tav2 {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Workgroups that a launch is divided into, about (two to a CU).  New actions of 64 users, us: 35.5 with
// 512, 37.0 with 768, 34.3 with 1024, 44.1 with 4096; 64 sequences of 8192 tokens each 27.5, 28.5, 28.9, 38.0.
constexpr int SHARES = 512;
// Pages to a share, at most (a longer one ends later than the rest).  8 copies each of 16 histories, us: 102 with
// 16, 86 with 32, 80 with 64; 64 sequences of 16384 tokens, 8 heads, 200, 195 and 191.
constexpr int SHARE_MOST = 64;

// The pages that a tile's queries see: [0, sink) and [first, last), counted through.
struct PageList {
  int sink, first, last;
  __device__ __forceinline__ int count() const { return sink + (last > first ? last - first : 0); }
  __device__ __forceinline__ int at(int i) const { return i < sink ? i : first + i - sink; }
};

// For queries at positions lo .. hi of a sequence of len tokens.
__device__ __forceinline__ PageList pages_seen(int len, int64_t lo, int64_t hi, int window, int sinks) {
  PageList p;
  const int64_t top = hi + 1 < len ? hi + 1 : len;
  p.last = top > 0 ? int((top + KVP - 1) / KVP) : 0;
  const int64_t low = window > 0 && lo - window + 1 > 0 ? lo - window + 1 : 0;
  p.first = int(low / KVP);
  const int s = int((int64_t(sinks) + KVP - 1) / KVP);
  p.sink = window > 0 ? min(min(s, p.first), p.last) : 0;
  return p;
}

// Codes as fp16: a byte biased to 0 .. 255 is 1024 and that much as the low bits of 0x6400.
__device__ __forceinline__ uint32_t codes2h(uint32_t biased, uint32_t sel) {
  const uint32_t w = __builtin_amdgcn_perm(0x64646464u, biased, sel);
  const f16x2 x = __builtin_bit_cast(f16x2, w) - (f16x2){(_Float16)1152.f, (_Float16)1152.f};
  return __builtin_bit_cast(uint32_t, x);
}
__device__ __forceinline__ f16x8 codes8h(uint32_t x, uint32_t y) {
  x ^= 0x80808080u;
  y ^= 0x80808080u;
  return __builtin_bit_cast(f16x8, make_uint4(codes2h(x, 0x04010400u), codes2h(x, 0x04030402u),
                                              codes2h(y, 0x04010400u), codes2h(y, 0x04030402u)));
}

// Places of a row's 16-byte pieces in LDS, xor'ed: the rows that 8 or 16 neighbouring lanes read
// (key_row: 0 .. 3, 16 .. 19, 4 .. 7, 20 .. 23, and on; features: one after the other) lie in
// different banks.
template <int D>
__device__ __forceinline__ int swz_key(int r) {
  const int b0 = r & 1, b1 = (r >> 1) & 1, b2 = (r >> 2) & 1, b4 = (r >> 4) & 1;
  return D == 32 ? b4 : D == 64 ? (b1 ^ b2) | b4 << 1 : (b0 ^ b2) | b1 << 1 | b4 << 2;
}
__device__ __forceinline__ int swz_feature(int d) { return ((d >> 2) & 1) | (((d >> 1) ^ (d >> 3)) & 1) << 1; }

// 8 bf16 values of which the first n are kept and the others (whatever they hold) become zeros: by
// selects, so that the loads before it stay together.
__device__ __forceinline__ u32x4 first_of8(u32x4 w, int n) {
#pragma unroll
  for (int e = 0; e < 4; ++e) w[e] &= n > 2 * e + 1 ? 0xFFFFFFFFu : n > 2 * e ? 0xFFFFu : 0u;
  return w;
}

// 8 bf16 values times f (a power of two) as fp16.
__device__ __forceinline__ f16x8 scaled8h(const u32x4& x, float f) {
  uint32_t y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e)
    y[e] = pack2h(__uint_as_float(x[e] << 16) * f, __uint_as_float(x[e] & 0xFFFF0000u) * f);
  return __builtin_bit_cast(f16x8, make_uint4(y[0], y[1], y[2], y[3]));
}
__device__ __forceinline__ float max8(const u32x4& x, float m) {
#pragma unroll
  for (int e = 0; e < 4; ++e)
    m = fmaxf(m, fmaxf(__builtin_fabsf(__uint_as_float(x[e] << 16)),
                       __builtin_fabsf(__uint_as_float(x[e] & 0xFFFF0000u))));
  return m;
}
// The power of two that takes top into [2^TO, 2^(TO + 1)), as a factor and back (tops below 2^-86 like
// 2^-86: both stay normal numbers).  Queries and keys go as high as fp16 has room for, the open block's values to
// where codes are: next to a page's products theirs then begin as high, and their small weights keep as
// many bits.
template <int TO>
__device__ __forceinline__ void into_half(float top, float* f, float* back) {
  uint32_t ex = __float_as_uint(top) >> 23;
  ex = ex < 41 ? 41 : ex > 254 ? 254 : ex;
  *f = __uint_as_float((254 + TO - ex) << 23);
  *back = __uint_as_float((ex - TO) << 23);
}
constexpr int TO_TOP = 14, TO_CODES = 6;

// The scale of an open block's values; of zeros none.
__device__ __forceinline__ AttScale tail_scale(float top, float back, float f) {
  return AttScale{top > 0.f ? __builtin_amdgcn_logf(back) : -INFINITY, f};
}

// 2^(x / 2), to be taken twice: a weight of 2^-127 and less may belong to a value as large beside the others.
__device__ __forceinline__ float half_factor(float x) { return __builtin_amdgcn_exp2f(0.5f * x); }

// A score's factor: the scale times the keys' (k), and the power of two (e) that takes the query's and the
// scale's back, apart, since their product alone may leave fp32's range.  One that leaves it with the keys
// (queries of zeros, tiny scales) is no zero, by which a masked -inf would become a NaN, and not
// infinite, by which a zero would: scores are below 2^38, so 2^-126 adds at most 2^-88 to an exponent that is
// nearer to zero still.
__device__ __forceinline__ float score_factor(float k, int e) {
  return __builtin_amdgcn_fmed3f(__builtin_amdgcn_ldexpf(k, e), FLT_MIN, FLT_MAX);
}

// A wave's pages: every fourth entry of the share from c0 + wave on.
template <int D>
struct Feed {
  // the next 64, one a lane: number (-1: released, or the open block), key scale, and the value
  // scale as a power of two and reciprocal.  Read once, so that no page waits for a chain of
  // small loads.
  int ids;
  float kss, lvs, invs;
  u32x4 rk[D / 16], rv[D / 16];   // a page's codes as they lie

  template <class A, class J>
  __device__ __forceinline__ void look_up(const A& a, const J& j, int base) {
    const int full = j.len / KVP, i = base + 4 * (threadIdx.x % WAVE);
    const int b = i < j.c1 ? j.list.at(i) : full;
    ids = b < full ? j.table[b] : -1;
    if (ids >= a.c.pages) ids = -1;
    const int64_t at = kv_unit(a.c, a.layer, ids < 0 ? 0 : ids, j.h);
    const float vs = a.c.v_scale[at];
    kss = a.c.k_scale[at];
    lvs = __builtin_amdgcn_logf(vs);
    invs = __builtin_amdgcn_rcpf(vs);
  }
  __device__ __forceinline__ int page(int t) const { return __builtin_amdgcn_readlane(ids, t); }
  static __device__ __forceinline__ float lane_f(float v, int t) {
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), t));
  }
  template <class A, class J>
  __device__ __forceinline__ void load(const A& a, const J& j, int page) {
    const int lane = threadIdx.x % WAVE;
    const int64_t at = kv_unit(a.c, a.layer, page < 0 ? 0 : page, j.h) * KVP * D;
    const u32x4* kp = reinterpret_cast<const u32x4*>(a.c.k + at) + lane;
    const u32x4* vp = reinterpret_cast<const u32x4*>(a.c.v + at) + lane;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      rk[i] = kp[i * WAVE];
      rv[i] = vp[i * WAVE];
    }
  }
  // Factors of entry t.  Scale 1 may be a block of zeros, whose scale counts as none.
  __device__ __forceinline__ void factors(int t, float* ks, AttScale* v) const {
    *ks = lane_f(kss, t);
    v->lv = lane_f(lvs, t);
    v->inv = lane_f(invs, t);
    if (v->lv == 0.f) {
      uint32_t any = 0;
#pragma unroll
      for (int e = 0; e < D / 16; ++e) any |= rv[e].x | rv[e].y | rv[e].z | rv[e].w;
      if (!__any(any != 0)) v->lv = -INFINITY;
    }
  }
  // The page into the wave's part of LDS: keys' pieces from 0, features' from 4 D (KC and VC pieces a
  // row).  A wave's LDS operations are done in order; the barriers keep the compiler to it.
  static constexpr int KC = D / 16, VC = KVP / 16;
  __device__ __forceinline__ void put(u32x4* my) const {
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int e = 0; e < D / 16; ++e) {
      const int i = e * WAVE + threadIdx.x % WAVE, kr = i / KC, vr = i / VC;
      my[kr * KC + ((i % KC) ^ swz_key<D>(kr))] = rk[e];
      my[4 * D + vr * VC + ((i % VC) ^ swz_feature(vr))] = rv[e];
    }
    __builtin_amdgcn_wave_barrier();
  }
};

// 32 QT query rows of job j.  The arguments' type says, by row_seen and tile_seen, which positions a row and all
// rows of the tile see, and whether the result is one of several parts.
template <int D, int QT, class A, class J>
__device__ __forceinline__ void attend_rows(const A& a, const J& j) {
  constexpr int KB = D / 2;   // bytes of a key's codes per lane
  // a wave's page on its way, then its state
  constexpr int STAGE = QT * D / 32 * 4 * WAVE;   // 16-byte pieces; a page has 8 D of them
  static_assert(STAGE >= 8 * D, "a page fits");
  __shared__ u32x4 stage[4][STAGE];
  __shared__ float mm[4][QT][2][WAVE];
  const tav2_kv& c = a.c;
  const int G = j.G, h = j.h, len = j.len, rows = j.rows, row0 = j.row0, full = len / KVP;
  const int64_t q0 = j.q0;
  const int lane = threadIdx.x % WAVE, m = lane % 32, half = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);   // (scalar page arithmetic)
  u32x4* const my = stage[wave];
  Feed<D> feed;
  feed.look_up(a, j, j.c0 + wave);
  int page = feed.page(0);
  feed.load(a, j, page);

  // this lane's queries: operands, and what they see
  f16x8 qf[QT][D / 16];
  int cq[QT];   // powers of two
  AttSeen<QT> seen;
  seen.sinks = tile_sinks(a, j);
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    const int row = min(row0 + 32 * q + m, rows - 1);
    const int i = row / G, g = row % G;
    const bf16_t* p = static_cast<const bf16_t*>(a.q.q) + (q0 + i) * a.q.ld + (h * G + g) * D + half * KB;
    u32x4 w[D / 16];
    float top = 0.f, f, back;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) w[t] = *reinterpret_cast<const u32x4*>(p + 8 * t);
#pragma unroll
    for (int t = 0; t < D / 16; ++t) top = max8(w[t], top);
    into_half<TO_TOP>(xmax32(top), &f, &back);
#pragma unroll
    for (int t = 0; t < D / 16; ++t) qf[q][t] = scaled8h(w[t], f);
    cq[q] = a.scale_e + __builtin_amdgcn_frexp_expf(back) - 1;
    row_seen(a, j, row, &seen.hi[q], &seen.lo[q]);
  }
  // a page is seen whole by all of them where it ends by the first's last key and starts at the last's
  // first one (or lies among the sinks)
  int64_t all_hi, all_lo;
  tile_seen(a, j, &all_hi, &all_lo);
  auto part_seen = [&](int b) {
    return int64_t(b + 1) * KVP > all_hi ||
           (int64_t(b) * KVP < all_lo && int64_t(b + 1) * KVP > seen.sinks);
  };

  AttScaledState<D, QT> st;
  st.clear();
  bool open = false;
  int i = j.c0 + wave, t = 0;
  auto visit = [&]() {
    if (t == WAVE) {
      t = 0;
      feed.look_up(a, j, i);
      page = feed.page(0);
      feed.load(a, j, page);
    }
    const int b = j.list.at(i);
    open |= i < j.c1 && b >= full;
    const int next = t + 1 < WAVE ? feed.page(t + 1) : -1;
    const bool masked = part_seen(b);
    float ks, cs[QT];
    AttScale vs;
    feed.factors(t, &ks, &vs);
#pragma unroll
    for (int q = 0; q < QT; ++q) cs[q] = score_factor(a.scale * ks, cq[q]);
    feed.put(my);
    feed.load(a, j, next);
    if (page >= 0) {
      // Both halves of a page at once where the registers suffice: one look at the references for 64 keys.  One
      // history of 16384 tokens, us: 64 candidates 13.3 for 14.0, 200: 17.3 for 17.9, 400: 29.2 for 27.9 (fewer waves
      // fit), 500: 24.9 for 26.3.
      constexpr int NB = QT == 1 && D <= 64 ? 2 : 1;
#pragma unroll 1
      for (int u0 = 0; u0 < 2; u0 += NB) {
        auto keys = [&](int e, f16x8(&kf)[D / 16]) {
          const int u = u0 + e;
          const int kr = 32 * u + key_row(m);
#pragma unroll
          for (int t = 0; t < D / 32; ++t) {
            const u32x4 w = my[kr * Feed<D>::KC + ((half * (D / 32) + t) ^ swz_key<D>(key_row(m)))];
            kf[2 * t] = codes8h(w.x, w.y);
            kf[2 * t + 1] = codes8h(w.z, w.w);
          }
        };
        auto values = [&](int e, f16x8(&vf)[D / 32][2]) {
          const int u = u0 + e;
#pragma unroll
          for (int d = 0; d < D / 32; ++d) {
            const int vr = 32 * d + m;
            const u32x4 w = my[4 * D + vr * Feed<D>::VC + ((2 * u + half) ^ swz_feature(m))];
            vf[d][0] = codes8h(w.x, w.y);
            vf[d][1] = codes8h(w.z, w.w);
          }
        };
        att_step<f16x8, NB, D, QT>(st, keys, values, qf, cs, vs, masked, seen,
                                   b * KVP + 32 * u0 + 16 * half);
      }
    }
    page = next;
    ++t;
    i += 4;
  };
  // With 64 rows of 32 features a wave without a page passes once, with page -1: the state then lies in one set
  // of registers, with no copies to another at each page's end (16 histories, 1000 candidates each, 295 us for 326).
  // Elsewhere such waves go on at once (64 features, 1000 candidates of one history 39.0 us for 39.3).
  if constexpr (QT > 1 && D == 32) {
    do visit(); while (i < j.c1);
  } else {
    while (i < j.c1) visit();
  }
  if (open) {   // the open block, in bf16: scaled into fp16's range; what lies behind the last token is
                // taken as zeros
    const int64_t tail = kv_tail(c, a.layer, j.s, h);
    const bool masked = part_seen(full);
#pragma unroll 1
    for (int u = 0; u < 2; ++u) {
      const int kr = 32 * u + key_row(m), k0 = 32 * u + 16 * half, held = len - full * KVP;
      float kt = 0.f, vt = 0.f, f, back, cs[QT];
      auto raw_key = [&](int t) {
        return first_of8(*reinterpret_cast<const u32x4*>(c.k_tail + tail + kr * D + half * KB + 8 * t),
                         kr < held ? 8 : 0);
      };
      auto raw_value = [&](int d, int t) {
        return first_of8(*reinterpret_cast<const u32x4*>(c.v_tail + tail + (32 * d + m) * KVP + k0 + 8 * t),
                         held - k0 - 8 * t);
      };
      // (read twice, the second time from the cache: the scales come first, and the registers do not
      // hold it all)
#pragma unroll
      for (int t = 0; t < D / 16; ++t) kt = max8(raw_key(t), kt);
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int t = 0; t < 2; ++t) vt = max8(raw_value(d, t), vt);
      __builtin_amdgcn_wave_barrier();
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) {
        kt = fmaxf(kt, __shfl_xor(kt, o, WAVE));
        vt = fmaxf(vt, __shfl_xor(vt, o, WAVE));
      }
      into_half<TO_TOP>(kt, &f, &back);
      float fv, backv;
      into_half<TO_CODES>(vt, &fv, &backv);
#pragma unroll
      for (int q = 0; q < QT; ++q) cs[q] = score_factor(a.scale * back, cq[q]);
      auto keys = [&](int, f16x8(&kf)[D / 16]) {
#pragma unroll
        for (int t = 0; t < D / 16; ++t) kf[t] = scaled8h(raw_key(t), f);
      };
      auto values = [&](int, f16x8(&vf)[D / 32][2]) {
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
          for (int t = 0; t < 2; ++t) vf[d][t] = scaled8h(raw_value(d, t), fv);
      };
      att_step<f16x8, 1, D, QT>(st, keys, values, qf, cs, tail_scale(vt, backv, fv), masked, seen,
                                full * KVP + k0);
    }
  }

  __builtin_amdgcn_wave_barrier();
  // the four waves' states meet in LDS, features against the weights' reference as their sums are; wave w
  // then joins registers 4w .. 4w + 3 of each tile (in the order of the waves), features 8w + 4 half .. of it
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    mm[wave][q][0][lane] = st.n[q];
    mm[wave][q][1][lane] = xsum32(st.l[q]);
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        my[((q * (D / 32) + d) * 4 + j) * WAVE + lane] = __builtin_bit_cast(
            u32x4, (f32x4){st.o[d][q][4 * j], st.o[d][q][4 * j + 1], st.o[d][q][4 * j + 2],
                           st.o[d][q][4 * j + 3]} * st.d[q]);
  }
  __syncthreads();
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    const int row = row0 + 32 * q + m;
    if (row >= rows) continue;
    float M = -FLT_MAX, l = 0.f, f[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) M = vmax(M, mm[w][q][0][lane]);
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      f[w] = half_factor(mm[w][q][0][lane] - M);
      l += mm[w][q][1][lane] * f[w] * f[w];
    }
    const int64_t at = (q0 + row / G) * a.q.heads + h * G + row % G;
    const int64_t part = int64_t(j.split) * a.q.total * a.q.heads + at;
    const bool some = l > 0.f || l != l;   // nothing seen: zeros
    const float inv = a.parts() ? 1.f : some ? 1.f / l : 0.f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d) {
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const f32x4 x = __builtin_bit_cast(
            f32x4, stage[w][((q * (D / 32) + d) * 4 + wave) * WAVE + lane]);
        o.x = __builtin_fmaf(x.x * f[w], f[w], o.x);
        o.y = __builtin_fmaf(x.y * f[w], f[w], o.y);
        o.z = __builtin_fmaf(x.z * f[w], f[w], o.z);
        o.w = __builtin_fmaf(x.w * f[w], f[w], o.w);
      }
      const int feature = 32 * d + 8 * wave + 4 * half;
      if (a.parts())
        *reinterpret_cast<float4*>(a.part_o + part * D + feature) = o;
      else
        *reinterpret_cast<uint2*>(a.out + at * D + feature) =
            make_uint2(pack2(o.x * inv, o.y * inv), pack2(o.z * inv, o.w * inv));
    }
    if (wave == 0 && half == 0) {
      if (a.parts()) {
        a.part_ml[2 * part] = M;
        a.part_ml[2 * part + 1] = l;
      } else if (a.lse) {
        a.lse[at] = some ? (M + __builtin_amdgcn_logf(l)) * LN2 : -INFINITY;
      }
    }
  }
}

// At most 16 query rows of a wave, on the 16x16x32 instructions, a page's 64 keys at once.  S^T comes in four tiles
// of 16 keys, in the order that makes a lane's 16 scores its quarter's 16 consecutive keys
// (16 g + 4 i + r in register r of tile i, g = l / 16), again the operand of O^T = V^T P^T as they
// stand.  A lane's row is l % 16.
template <int D>
struct Tile16 {
  static constexpr int F = D / 4;    // features of a lane's quarter
  static constexpr int NK = D / 32;  // products over the features
  static constexpr int ND = D / 16;  // tiles of O^T
  f16x8 qf[NK];
  int cq;                            // a power of two
  int lo, all_hi, all_lo, sinks;     // what the row sees (besides hi, which a caller keeps), and what all rows do
  f32x4 o[ND];
  float ref, wref, ratio, sum;       // (m, n, d, l of attend_core.h: ref is above wref)

  // The row's query, at its first feature.
  __device__ __forceinline__ void query(const bf16_t* p, int scale_e) {
    u32x4 w[NK];
    float top = 0.f, f, back;
#pragma unroll
    for (int t = 0; t < NK; ++t)
      w[t] = *reinterpret_cast<const u32x4*>(p + int(threadIdx.x) % WAVE / 16 * F + 8 * t);
#pragma unroll
    for (int t = 0; t < NK; ++t) top = max8(w[t], top);
    into_half<TO_TOP>(xmax32(xmax16(top)), &f, &back);
#pragma unroll
    for (int t = 0; t < NK; ++t) qf[t] = scaled8h(w[t], f);
    cq = scale_e + __builtin_amdgcn_frexp_expf(back) - 1;
  }
  // The rows see the positions below hi that are at least lo or among the sinks.
  __device__ __forceinline__ void sees(int hi, int lo_, int sinks_) {
    lo = lo_;
    sinks = sinks_;
    all_hi = hi;   // from the last one's first key to the first's last
    all_lo = lo;
#pragma unroll
    for (int x = 8; x >= 1; x >>= 1) {
      all_hi = min(all_hi, __shfl_xor(all_hi, x, WAVE));
      all_lo = max(all_lo, __shfl_xor(all_lo, x, WAVE));
    }
    all_hi = __builtin_amdgcn_readfirstlane(all_hi);
    all_lo = __builtin_amdgcn_readfirstlane(all_lo);
  }
  __device__ __forceinline__ void clear() {
    ref = 0.f;
    wref = -FLT_MAX;
    ratio = 1.f;
    sum = 0.f;
#pragma unroll
    for (int d = 0; d < ND; ++d) o[d] = (f32x4){0.f, 0.f, 0.f, 0.f};
  }

  // One page: keys(i, kf) sets the operands of S^T's tile i, values(d, vf) those of O^T's tile d.
  template <class Keys, class Values>
  __device__ __forceinline__ void step(Keys keys, Values values, float cs, AttScale vs, int key0, const int& hi) {
    const int g = int(threadIdx.x) % WAVE / 16;
    f32x4 s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f16x8 kf[NK];
      keys(i, kf);
      s[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < NK; ++t) s[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[t], qf[t], s[i], 0, 0, 0);
    }
    if (key0 + KVP > all_hi || (key0 < all_lo && key0 + KVP > sinks)) {
      const int k0 = key0 + 16 * g, hi_ = hi - k0, lo_ = lo - k0, sinks_ = sinks - k0;
#pragma unroll
      for (int r = 0; r < 16; ++r)
        s[r / 4][r % 4] = r < hi_ && (r >= lo_ || r < sinks_) ? s[r / 4][r % 4] : -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = vmax(top, s[r / 4][r % 4]);
    const float raw = xmax32(xmax16(top));
    top = att_top(raw, cs);
    if (__any(att_passes(top, vs.lv, ref, wref))) {
      float of, lf;
      att_raise(top, vs.lv, ref, wref, ratio, &of, &lf);
      sum *= lf;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] *= of;
    }
    float b, e, own;
    if (att_offset(raw, top, vs, ref, wref, ratio, &b, &e, &own)) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r / 4][r % 4] -= own;
    }
    float part = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r / 4][r % 4], cs, b));
      s[r / 4][r % 4] = x;
      part += x;
    }
    sum = __builtin_fmaf(part, e, sum);
    f16x8 pf[2];
#pragma unroll
    for (int t = 0; t < 2; ++t)
      pf[t] = __builtin_bit_cast(
          f16x8, make_uint4(pack2h(s[2 * t][0], s[2 * t][1]), pack2h(s[2 * t][2], s[2 * t][3]),
                            pack2h(s[2 * t + 1][0], s[2 * t + 1][1]),
                            pack2h(s[2 * t + 1][2], s[2 * t + 1][3])));
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      f16x8 vf[2];
      values(d, vf);
#pragma unroll
      for (int t = 0; t < 2; ++t)
        o[d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf[t], pf[t], o[d], 0, 0, 0);
    }
  }
  // The key of tile 0 that this lane's row of the operand is (+ 4 i: of tile i).
  static __device__ __forceinline__ int key() {
    const int m = int(threadIdx.x) % 16;
    return 16 * (m / 4) + m % 4;
  }

  // The open block of a sequence of `full` pages, in bf16 (as in attend_rows).
  __device__ __forceinline__ void open_block(const tav2_kv& c, int layer, int of, int h, int full, float scale,
                                             const int& hi) {
    const int m = int(threadIdx.x) % 16, g = int(threadIdx.x) % WAVE / 16, krow = key();
    const int64_t tail = kv_tail(c, layer, of, h);
    const int held = kv_len(c, of) - full * KVP;
    float kt = 0.f, vt = 0.f, fk, backk, fv, backv;
    auto raw_key = [&](int i, int t) {
      return first_of8(*reinterpret_cast<const u32x4*>(c.k_tail + tail + (krow + 4 * i) * D + g * F + 8 * t),
                       krow + 4 * i < held ? 8 : 0);
    };
    auto raw_value = [&](int d, int t) {
      return first_of8(*reinterpret_cast<const u32x4*>(c.v_tail + tail + (16 * d + m) * KVP + 16 * g + 8 * t),
                       held - 16 * g - 8 * t);
    };
    // (read twice, as there)
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < NK; ++t) kt = max8(raw_key(i, t), kt);
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int t = 0; t < 2; ++t) vt = max8(raw_value(d, t), vt);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int x = 32; x >= 1; x >>= 1) {
      kt = fmaxf(kt, __shfl_xor(kt, x, WAVE));
      vt = fmaxf(vt, __shfl_xor(vt, x, WAVE));
    }
    into_half<TO_TOP>(kt, &fk, &backk);
    into_half<TO_CODES>(vt, &fv, &backv);
    auto keys = [&](int i, f16x8(&kf)[NK]) {
#pragma unroll
      for (int t = 0; t < NK; ++t) kf[t] = scaled8h(raw_key(i, t), fk);
    };
    auto values = [&](int d, f16x8(&vf)[2]) {
#pragma unroll
      for (int t = 0; t < 2; ++t) vf[t] = scaled8h(raw_value(d, t), fv);
    };
    step(keys, values, score_factor(scale * backk, cq), tail_scale(vt, backv, fv), full * KVP, hi);
  }
};

// At most 16 query rows of a workgroup, whose four waves take the share's pages in turn.  A lane's row is
// query qi's head g_row of its kv head.  feed has been asked for the share's first pages; stage and mm are the workgroup's
// LDS: a wave's page on its way, then its state.  open_blocks(f) calls f(sequence) for the open blocks that are this
// wave's; finish(M, l, tile) gets a row's reference and sum, and tile(d) its features 16 d + 4 g .. + 3.
template <int D, class A, class J, class Open, class Finish>
__device__ __forceinline__ void attend16(const A& a, const J& j, Feed<D>& feed, int page, u32x4 (&stage)[4][8 * D],
                                         float (&mm)[4][2][16], int64_t qi, int g_row, int& hi, int lo, Open open_blocks,
                                         Finish finish) {
  using T = Tile16<D>;
  constexpr int NK = T::NK, ND = T::ND;
  const tav2_kv& c = a.c;
  const int lane = threadIdx.x % WAVE, m = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int full = j.len / KVP;
  u32x4* const my = stage[wave];
  T st;
  st.sees(hi, lo, tile_sinks(a, j));
  st.query(static_cast<const bf16_t*>(a.q.q) + qi * a.q.ld + (j.h * j.G + g_row) * D, a.scale_e);
  st.clear();
  const int krow = T::key();
  for (int i = j.c0 + wave, t = 0; i < j.c1; i += 4, ++t) {
    if (t == WAVE) {
      t = 0;
      feed.look_up(a, j, i);
      page = feed.page(0);
      feed.load(a, j, page);
    }
    const int b = j.list.at(i);
    const int next = t + 1 < WAVE ? feed.page(t + 1) : -1;
    float ks;
    AttScale vs;
    feed.factors(t, &ks, &vs);
    feed.put(my);
    feed.load(a, j, next);
    if (page >= 0) {
      auto keys = [&](int i, f16x8(&kf)[NK]) {
        const int kr = krow + 4 * i;
        if constexpr (D == 32) {   // 8 bytes: half a piece
          const uint2 w = reinterpret_cast<const uint2*>(my)[2 * (kr * 2 + ((g / 2) ^ swz_key<D>(kr))) + g % 2];
          kf[0] = codes8h(w.x, w.y);
        } else {
#pragma unroll
          for (int p = 0; p < D / 64; ++p) {
            const u32x4 w = my[kr * Feed<D>::KC + ((g * (D / 64) + p) ^ swz_key<D>(kr))];
            kf[2 * p] = codes8h(w.x, w.y);
            kf[2 * p + 1] = codes8h(w.z, w.w);
          }
        }
      };
      auto values = [&](int d, f16x8(&vf)[2]) {
        const int vr = 16 * d + m;
        const u32x4 w = my[4 * D + vr * Feed<D>::VC + (g ^ swz_feature(m))];
        vf[0] = codes8h(w.x, w.y);
        vf[1] = codes8h(w.z, w.w);
      };
      st.step(keys, values, score_factor(a.scale * ks, st.cq), vs, b * KVP, hi);
    }
    page = next;
  }
  open_blocks([&](int of) { st.open_block(c, a.layer, of, j.h, full, a.scale, hi); });

  // the four waves' states meet in LDS; wave w joins every fourth tile of O^T, in the order of the waves
  __builtin_amdgcn_wave_barrier();
  const float sum = xsum32(xsum16(st.sum));
  if (g == 0) {
    mm[wave][0][m] = st.wref;
    mm[wave][1][m] = sum;
  }
#pragma unroll
  for (int d = 0; d < ND; ++d) my[d * WAVE + lane] = __builtin_bit_cast(u32x4, st.o[d] * st.ratio);
  __syncthreads();
  float M = -FLT_MAX, l = 0.f, f[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) M = vmax(M, mm[w][0][m]);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    f[w] = half_factor(mm[w][0][m] - M);
    l += mm[w][1][m] * f[w] * f[w];
  }
  finish(M, l, [&](int d) {
    f32x4 x = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) x += __builtin_bit_cast(f32x4, stage[w][d * WAVE + lane]) * f[w] * f[w];
    return x;
  });
}

}  // namespace tav2
