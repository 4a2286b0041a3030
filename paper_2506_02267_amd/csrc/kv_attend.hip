// Attention over the paged 8-bit cache: every head's queries of a sequence against its codes.
//
// A workgroup takes 32 QT queries of one kv head (the heads that share it count as queries) and a
// share of the pages they see; its four waves take the pages in turn, each turning a page's codes
// into matrix operands in its own registers, once for all 32 QT queries, and meet in LDS at
// the end.  A wave reads a page as it lies, a kilobyte a load, into registers (the next page's
// loads are in flight while this one is multiplied), and passes it through its own part of LDS,
// where a lane then reads its operands: half a key's codes, and 16 keys of one feature of V^T.  (Each
// lane reading its operands from the page itself took 115 cycles of the address path a load: 44 us
// for 64 users' new actions.)
// Operands are fp16, which holds codes exactly and the weights to 11 bits; a query is scaled by a
// power of two first so that its largest feature lies in [2^14, 2^15) (features below 2^-28 of
// that lose bits that fp32 sums would lose as well).  A page's key scale multiplies the fp32
// scores, its value scale enters the weights as a power of two added to the exponent.  Where queries are
// few, the pages are split over more workgroups, whose partial results a second launch joins
// in a fixed order.
#include <algorithm>

#include "attend_core.h"
#include "internal.h"
#include "kv_common.h"
#include "token_source.h"

namespace tav2 {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

struct AttendArgs {
  tav2_kv c;
  int layer;
  tav2_kv_queries q;
  bool causal;
  float scale;
  bf16_t* out;
  float* lse;        // nullable
  float* part_o;     // [splits, total, heads, D], with splits > 1
  float* part_ml;    // [splits, total, heads, 2]: reference and sum
  int tiles;         // query tiles per (sequence, kv head)
  int splits, chunk; // shares of a sequence's pages, and pages to a share
  int units;         // (sequence, kv head, split) groups, padded to a multiple of 8
};

constexpr int SHARES = 2048;   // workgroups that a launch is divided into, about

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

// 8 bf16 values times f (a power of two) as fp16.
__device__ __forceinline__ f16x8 scaled8h(const uint4& w, float f) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
  uint32_t y[4];
#pragma unroll
  for (int e = 0; e < 4; ++e)
    y[e] = pack2h(__uint_as_float(x[e] << 16) * f, __uint_as_float(x[e] & 0xFFFF0000u) * f);
  return __builtin_bit_cast(f16x8, make_uint4(y[0], y[1], y[2], y[3]));
}
__device__ __forceinline__ float max8(const uint4& w, float m) {
  const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    m = fmaxf(m, fmaxf(__builtin_fabsf(__uint_as_float(x[e] << 16)),
                       __builtin_fabsf(__uint_as_float(x[e] & 0xFFFF0000u))));
  return m;
}
// The power of two that takes top into [2^14, 2^15), as a factor and back (tops below 2^-86 like
// 2^-86: the factor back is a weight's, and sums of those over it stay finite).
__device__ __forceinline__ void into_half(float top, float* f, float* back) {
  uint32_t ex = __float_as_uint(top) >> 23;
  ex = ex < 41 ? 41 : ex > 254 ? 254 : ex;
  *f = __uint_as_float((268 - ex) << 23);
  *back = __uint_as_float((ex - 14) << 23);
}

template <int D, int QT>
__global__ __launch_bounds__(256, 2) void kv_attend_kernel(AttendArgs a) {
  constexpr int KB = D / 2;   // bytes of a key's codes per lane
  // a wave's page on its way, then its state
  constexpr int STAGE = QT * D / 32 * 4 * WAVE;   // 16-byte pieces; a page has 8 D of them
  static_assert(STAGE >= 8 * D, "a page fits");
  __shared__ u32x4 stage[4][STAGE];
  __shared__ float mm[4][QT][2][WAVE];
  const tav2_kv& c = a.c;
  const int H = c.kv_heads, G = a.q.heads / H;
  // units (which share K and V) on one XCD: a unit's query tiles are 8 apart, and so on
  const int unit = int(blockIdx.x % unsigned(a.units));
  const int tile = int(blockIdx.x / unsigned(a.units));
  const int split = unit % a.splits, sh = unit / a.splits;
  const int s = sh / H, h = sh % H;
  if (s >= c.num_seqs) return;
  const int64_t q0 = a.q.offset[s];
  int64_t nq = a.q.offset[s + 1] - q0;
  nq = nq < 0 ? 0 : nq > a.q.max_count ? a.q.max_count : nq;
  if (q0 < 0 || q0 + nq > a.q.total) return;
  const int rows = int(nq) * G, row0 = tile * 32 * QT;
  if (row0 >= rows) return;
  const int len = kv_len(c, s);
  const int lane = threadIdx.x % WAVE, m = lane % 32, half = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);   // (scalar page arithmetic)

  // which pages, and which of them this wave takes: every fourth of the workgroup's share
  const int64_t first_pos = a.causal ? int64_t(len) - nq : len;
  const int last_row = min(row0 + 32 * QT, rows) - 1;
  const int64_t lo_pos = a.causal ? first_pos + row0 / G : first_pos;
  const int64_t hi_pos = a.causal ? first_pos + last_row / G : first_pos;
  const PageList list = pages_seen(len, lo_pos, hi_pos, a.q.window, a.q.sinks);
  const int n = list.count();
  // shares of one size, so that a long sequence has more of them (larger ones where it is
  // longer than the host's estimate)
  const int chunk = max(a.chunk, (n + a.splits - 1) / a.splits);
  if (a.splits > 1 && split * chunk >= n) {   // an empty share: no sum, and kv_merge reads no more of it
    const int row = row0 + int(threadIdx.x);
    if (threadIdx.x < 32 * QT && row < rows) {
      const int64_t part = int64_t(split) * a.q.total * a.q.heads + (q0 + row / G) * a.q.heads +
                           h * G + row % G;
      a.part_ml[2 * part] = -FLT_MAX;
      a.part_ml[2 * part + 1] = 0.f;
    }
    return;
  }
  const int i0 = split * chunk + wave, i1 = min(n, (split + 1) * chunk);
  const int full = len / KVP;
  const int32_t* table = c.table + int64_t(s) * c.max_blocks;
  // this wave's next 64 pages, one a lane: number (-1: released, or the open block), key scale, and
  // the value scale as a power of two and reciprocal.  Read once, so that no page waits for
  // a chain of small loads.
  int ids = -1;
  float kss = 1.f, lvs = 0.f, invs = 1.f;
  auto look_up = [&](int base) {
    const int i = base + 4 * lane;
    const int b = i < i1 ? list.at(i) : full;
    ids = b < full ? table[b] : -1;
    if (ids >= c.pages) ids = -1;
    if (ids < 0) return;
    const int64_t at = kv_unit(c, a.layer, ids, h);
    const float vs = c.v_scale[at];
    kss = c.k_scale[at];
    lvs = __builtin_amdgcn_logf(vs);
    invs = __builtin_amdgcn_rcpf(vs);
  };
  auto lane_f = [](float v, int t) {
    return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), t));
  };
  u32x4 rk[D / 16], rv[D / 16];   // a page's codes as they lie
  auto load = [&](int page) {
    const int64_t at = kv_unit(c, a.layer, page < 0 ? 0 : page, h) * KVP * D;
    const u32x4* kp = reinterpret_cast<const u32x4*>(c.k + at) + lane;
    const u32x4* vp = reinterpret_cast<const u32x4*>(c.v + at) + lane;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) {
      rk[i] = kp[i * WAVE];
      rv[i] = vp[i * WAVE];
    }
  };
  u32x4* const my = stage[wave];
  constexpr int KC = D / 16, VC = KVP / 16;   // pieces of a key, and of a feature's 64 keys
  look_up(i0);
  int page = __builtin_amdgcn_readlane(ids, 0);
  load(page);

  // this lane's queries: operands, and what they see
  f16x8 qf[QT][D / 16];
  float cq[QT];
  AttSeen<QT> seen;
  seen.sinks = a.q.sinks;
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    const int row = min(row0 + 32 * q + m, rows - 1);
    const int i = row / G, g = row % G;
    const bf16_t* p = static_cast<const bf16_t*>(a.q.q) + (q0 + i) * a.q.ld + (h * G + g) * D + half * KB;
    uint4 w[D / 16];
    float top = 0.f, f, back;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) w[t] = *reinterpret_cast<const uint4*>(p + 8 * t);
#pragma unroll
    for (int t = 0; t < D / 16; ++t) top = max8(w[t], top);
    into_half(xmax32(top), &f, &back);
#pragma unroll
    for (int t = 0; t < D / 16; ++t) qf[q][t] = scaled8h(w[t], f);
    cq[q] = a.scale * LOG2E * back;
    const int64_t pos = a.causal ? first_pos + i : first_pos;
    const int64_t end = pos + 1 < len ? pos + 1 : len;
    seen.hi[q] = int(end > 0 ? end : 0);
    const int64_t low = pos - a.q.window + 1;
    seen.lo[q] = a.q.window > 0 && low > 0 ? int(low) : 0;
  }
  // a page is seen whole by all of them where it ends by the first's last key and starts at the last's
  // first one (or lies among the sinks)
  const int64_t all_hi = lo_pos + 1 < len ? lo_pos + 1 : len;
  const int64_t all_lo = a.q.window > 0 ? hi_pos - a.q.window + 1 : 0;
  auto part_seen = [&](int b) {
    return int64_t(b + 1) * KVP > all_hi ||
           (int64_t(b) * KVP < all_lo && int64_t(b + 1) * KVP > a.q.sinks);
  };

  AttState<D, QT> st;
  st.clear();
  bool open = false;
  for (int i = i0, t = 0; i < i1; i += 4, ++t) {
    if (t == WAVE) {
      t = 0;
      look_up(i);
      page = __builtin_amdgcn_readlane(ids, 0);
      load(page);
    }
    const int b = list.at(i);
    open |= b >= full;
    const int next = t + 1 < WAVE ? __builtin_amdgcn_readlane(ids, t + 1) : -1;
    const bool masked = part_seen(b);
    const float ks = lane_f(kss, t);
    float lv = lane_f(lvs, t), inv = lane_f(invs, t), cs[QT];
#pragma unroll
    for (int q = 0; q < QT; ++q) cs[q] = cq[q] * ks;
    if (lv == 0.f) {   // scale 1: a block of zeros, perhaps: taken as if at the smallest
                       // scale, so that its weights do not raise the reference over small values
      uint32_t any = 0;
#pragma unroll
      for (int e = 0; e < D / 16; ++e) any |= rv[e].x | rv[e].y | rv[e].z | rv[e].w;
      if (!__any(any != 0)) {
        lv = -100.f;
        inv = 0x1p100f;
      }
    }
    // (a wave's LDS operations are done in order; the barriers keep the compiler to it)
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int e = 0; e < D / 16; ++e) {
      const int i = e * WAVE + lane, kr = i / KC, vr = i / VC;
      my[kr * KC + ((i % KC) ^ swz_key<D>(kr))] = rk[e];
      my[4 * D + vr * VC + ((i % VC) ^ swz_feature(vr))] = rv[e];
    }
    __builtin_amdgcn_wave_barrier();
    load(next);
    if (page >= 0) {
#pragma unroll 1   // (both halves at once take too many registers)
      for (int u = 0; u < 2; ++u) {
        auto keys = [&](f16x8(&kf)[D / 16]) {
          const int kr = 32 * u + key_row(m);
#pragma unroll
          for (int t = 0; t < D / 32; ++t) {
            const u32x4 w = my[kr * KC + ((half * (D / 32) + t) ^ swz_key<D>(key_row(m)))];
            kf[2 * t] = codes8h(w.x, w.y);
            kf[2 * t + 1] = codes8h(w.z, w.w);
          }
        };
        auto values = [&](f16x8(&vf)[D / 32][2]) {
#pragma unroll
          for (int d = 0; d < D / 32; ++d) {
            const int vr = 32 * d + m;
            const u32x4 w = my[4 * D + vr * VC + ((2 * u + half) ^ swz_feature(m))];
            vf[d][0] = codes8h(w.x, w.y);
            vf[d][1] = codes8h(w.z, w.w);
          }
        };
        att_step<f16x8, D, QT>(st, keys, values, qf, cs, lv, inv, masked, seen,
                               b * KVP + 32 * u + 16 * half);
      }
    }
    page = next;
  }
  if (open) {   // the open block, in bf16: scaled into fp16's range; what lies behind the last token is
                // taken as zeros
    const int64_t tail = kv_tail(c, a.layer, s, h);
    const bool masked = part_seen(full);
#pragma unroll 1
    for (int u = 0; u < 2; ++u) {
      const int kr = 32 * u + key_row(m), k0 = 32 * u + 16 * half, held = len - full * KVP;
      uint4 wk[D / 16], wv[D / 32][2];
      float kt = 0.f, vt = 0.f, f, back, cs[QT];
#pragma unroll
      for (int t = 0; t < D / 16; ++t) {
        wk[t] = make_uint4(0, 0, 0, 0);
        if (kr < held)
          wk[t] = *reinterpret_cast<const uint4*>(c.k_tail + tail + kr * D + half * KB + 8 * t);
        kt = max8(wk[t], kt);
      }
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const uint4 w =
              *reinterpret_cast<const uint4*>(c.v_tail + tail + (32 * d + m) * KVP + k0 + 8 * t);
          uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (k0 + 8 * t + 2 * e >= held) x[e] = 0;
            else if (k0 + 8 * t + 2 * e + 1 >= held) x[e] &= 0xFFFFu;
          }
          wv[d][t] = make_uint4(x[0], x[1], x[2], x[3]);
          vt = max8(wv[d][t], vt);
        }
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) {
        kt = fmaxf(kt, __shfl_xor(kt, o, WAVE));
        vt = fmaxf(vt, __shfl_xor(vt, o, WAVE));
      }
      into_half(kt, &f, &back);
      float fv, backv;
      into_half(vt, &fv, &backv);
#pragma unroll
      for (int q = 0; q < QT; ++q) cs[q] = cq[q] * back;
      auto keys = [&](f16x8(&kf)[D / 16]) {
#pragma unroll
        for (int t = 0; t < D / 16; ++t) kf[t] = scaled8h(wk[t], f);
      };
      auto values = [&](f16x8(&vf)[D / 32][2]) {
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
          for (int t = 0; t < 2; ++t) vf[d][t] = scaled8h(wv[d][t], fv);
      };
      att_step<f16x8, D, QT>(st, keys, values, qf, cs, __builtin_amdgcn_logf(backv), fv, masked,
                             seen, full * KVP + k0);
    }
  }

  __builtin_amdgcn_wave_barrier();
  // the four waves' states meet in LDS; wave w then joins registers 4w .. 4w + 3 of each tile (in the
  // order of the waves), features 8w + 4 half .. of it
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    mm[wave][q][0][lane] = st.m[q];
    mm[wave][q][1][lane] = xsum32(st.l[q]);
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        my[((q * (D / 32) + d) * 4 + j) * WAVE + lane] = __builtin_bit_cast(
            u32x4, (f32x4){st.o[d][q][4 * j], st.o[d][q][4 * j + 1], st.o[d][q][4 * j + 2],
                           st.o[d][q][4 * j + 3]});
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
      f[w] = __builtin_amdgcn_exp2f(mm[w][q][0][lane] - M);
      l += mm[w][q][1][lane] * f[w];
    }
    const int64_t at = (q0 + row / G) * a.q.heads + h * G + row % G;
    const int64_t part = int64_t(split) * a.q.total * a.q.heads + at;
    const bool some = l > 0.f || l != l;   // nothing seen: zeros
    const float inv = a.splits > 1 ? 1.f : some ? 1.f / l : 0.f;
#pragma unroll
    for (int d = 0; d < D / 32; ++d) {
      float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const f32x4 x = __builtin_bit_cast(
            f32x4, stage[w][((q * (D / 32) + d) * 4 + wave) * WAVE + lane]);
        o.x = __builtin_fmaf(x.x, f[w], o.x);
        o.y = __builtin_fmaf(x.y, f[w], o.y);
        o.z = __builtin_fmaf(x.z, f[w], o.z);
        o.w = __builtin_fmaf(x.w, f[w], o.w);
      }
      const int feature = 32 * d + 8 * wave + 4 * half;
      if (a.splits > 1)
        *reinterpret_cast<float4*>(a.part_o + part * D + feature) = o;
      else
        *reinterpret_cast<uint2*>(a.out + at * D + feature) =
            make_uint2(pack2(o.x * inv, o.y * inv), pack2(o.z * inv, o.w * inv));
    }
    if (wave == 0 && half == 0) {
      if (a.splits > 1) {
        a.part_ml[2 * part] = M;
        a.part_ml[2 * part + 1] = l;
      } else if (a.lse) {
        a.lse[at] = some ? (M + __builtin_amdgcn_logf(l)) * LN2 : -INFINITY;
      }
    }
  }
}

// A workgroup per (query, head): D features by 256 / D groups of splits, the groups joined in LDS.
template <int D>
__global__ __launch_bounds__(256) void kv_merge_kernel(AttendArgs a) {
  constexpr int NG = 256 / D;
  __shared__ float lo[NG][D], ll[NG];
  const int64_t at = blockIdx.x, n = a.q.total * a.q.heads;
  const int tid = threadIdx.x, f = tid % D, g = tid / D;
  float M = -FLT_MAX;
  for (int s = tid % WAVE; s < a.splits; s += WAVE) M = fmaxf(M, a.part_ml[2 * (s * n + at)]);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, WAVE));
  float l = 0.f, x = 0.f;
#pragma unroll 4
  for (int s = g; s < a.splits; s += NG) {
    const int64_t p = s * n + at;
    const float lp = a.part_ml[2 * p + 1];
    if (lp == 0.f) continue;   // an empty share (its features are not written), or nothing seen
    const float w = __builtin_amdgcn_exp2f(a.part_ml[2 * p] - M);
    l += lp * w;
    x += a.part_o[p * D + f] * w;
  }
  lo[g][f] = x;
  if (f == 0) ll[g] = l;
  __syncthreads();
  if (g) return;
#pragma unroll
  for (int j = 1; j < NG; ++j) {
    x += lo[j][f];
    l += ll[j];
  }
  const bool some = l > 0.f || l != l;
  a.out[at * D + f] = f2bf(some ? x / l : 0.f);
  if (a.lse && f == 0) a.lse[at] = some ? (M + __builtin_amdgcn_logf(l)) * LN2 : -INFINITY;
}

int query_tiles(const tav2_kv& c, const tav2_kv_queries& q) {
  return int64_t(q.max_count) * (q.heads / c.kv_heads) > 32 && c.head_dim <= 64 ? 2 : 1;
}

// Pages that a query tile of the longest sequence sees, by the host's estimate.
int64_t most_pages(const tav2_kv& c, const tav2_kv_queries& q) {
  int64_t tokens = c.max_len;
  if (q.window > 0) tokens = std::min(tokens, int64_t(q.window) + q.max_count + q.sinks + 2 * KVP);
  return std::max<int64_t>(1, cdiv(tokens, KVP));
}

// Pages to a workgroup's share: such that there are workgroups enough to fill the CUs and to even out
// sequences of different lengths, but no share so small that its partial results (4 bytes a feature,
// written and read) come near the pages it reads (2 bytes a feature of 64 tokens).
int share_pages(const tav2_kv& c, const tav2_kv_queries& q) {
  const int64_t rows = int64_t(q.max_count) * (q.heads / c.kv_heads);
  const int64_t seqs = q.total < c.num_seqs ? q.total : c.num_seqs;
  const int64_t tile = 32 * query_tiles(c, q);
  const int64_t groups = seqs * c.kv_heads * cdiv(rows, tile);
  const int64_t least = std::max<int64_t>(4, std::min<int64_t>(rows, tile) / 2);
  return int(std::max<int64_t>(least, cdiv(groups * most_pages(c, q), SHARES)));
}
int key_splits(const tav2_kv& c, const tav2_kv_queries& q) {
  return int(cdiv(most_pages(c, q), share_pages(c, q)));
}

}  // namespace

int64_t kv_attend_groups(const tav2_kv& c, const tav2_kv_queries& q) {
  const int64_t rows = int64_t(q.max_count) * (q.heads / c.kv_heads);
  const int64_t units = (int64_t(c.num_seqs) * c.kv_heads * key_splits(c, q) + 7) / 8 * 8;
  return units * cdiv(rows, 32 * query_tiles(c, q));
}

size_t kv_attend_bytes(const tav2_kv& c, const tav2_kv_queries& q) {
  const int splits = key_splits(c, q);
  if (splits == 1) return 0;
  return align_up(size_t(splits) * size_t(q.total) * q.heads * (c.head_dim + 2) * 4, 256);
}

hipError_t launch_kv_attend(const tav2_kv& c, int layer, const tav2_kv_queries& q, bool causal,
                            void* out, float* lse, void* ws, hipStream_t st) {
  AttendArgs a{};
  a.c = c;
  a.layer = layer;
  a.q = q;
  a.causal = causal;
  a.scale = q.scale > 0.f ? q.scale : 1.f / sqrtf(float(c.head_dim));
  a.out = static_cast<bf16_t*>(out);
  a.lse = lse;
  const int QT = query_tiles(c, q);
  a.splits = key_splits(c, q);
  a.chunk = share_pages(c, q);
  a.tiles = int(cdiv(int64_t(q.max_count) * (q.heads / c.kv_heads), 32 * QT));
  a.units = int((int64_t(c.num_seqs) * c.kv_heads * a.splits + 7) / 8 * 8);
  a.part_o = static_cast<float*>(ws);
  if (a.splits > 1) a.part_ml = a.part_o + size_t(a.splits) * q.total * q.heads * c.head_dim;
  const unsigned grid = unsigned(a.units) * unsigned(a.tiles);
  {
    ProfScope prof("kv_attend", st);
    if (c.head_dim == 32) {
      if (QT == 1) kv_attend_kernel<32, 1><<<grid, 256, 0, st>>>(a);
      else kv_attend_kernel<32, 2><<<grid, 256, 0, st>>>(a);
    } else if (c.head_dim == 64) {
      if (QT == 1) kv_attend_kernel<64, 1><<<grid, 256, 0, st>>>(a);
      else kv_attend_kernel<64, 2><<<grid, 256, 0, st>>>(a);
    } else {
      kv_attend_kernel<128, 1><<<grid, 256, 0, st>>>(a);
    }
  }
  if (a.splits > 1) {
    ProfScope prof("kv_merge", st);
    const unsigned n = unsigned(q.total * q.heads);
    if (c.head_dim == 32) kv_merge_kernel<32><<<n, 256, 0, st>>>(a);
    else if (c.head_dim == 64) kv_merge_kernel<64><<<n, 256, 0, st>>>(a);
    else kv_merge_kernel<128><<<n, 256, 0, st>>>(a);
  }
  return hipGetLastError();
}

}  // namespace tav2
