// Attention over the paged 8-bit cache: every head's queries of a sequence against its codes.
//
// A workgroup takes 32 QT queries of one kv head (the heads that share it count as queries) and a
// share of the pages they see; its four waves take the pages in turn, each turning a page's codes
// into matrix operands in its own registers, once for all 32 QT queries, and meet in LDS at
// the end.  A wave reads a page as it lies, a kilobyte a load, into registers (the next page's
// loads are in flight while this one is multiplied), and passes it through its own part of LDS,
// where a lane then reads its operands: half a key's codes, and 16 keys of one feature of V^T.  (With
// each lane reading its operands from the page itself, 128 features in a window took 60 us for 50, the
// rest was alike.)
// Operands are fp16, which holds codes exactly and the weights to 11 bits; a query is scaled by a
// power of two first so that its largest feature lies in [2^14, 2^15) (features below 2^-28 of
// that lose bits that fp32 sums would lose as well).  A page's key scale multiplies the fp32
// scores, its value scale enters the weights by its logarithm, added to the exponent.  Where queries are
// few, the pages are split over more workgroups, whose partial results a second launch joins
// in a fixed order.
// One query a sequence is bound by HBM: 64 sequences of 16384 tokens, 8 kv heads, are read at 5.6 TB/s
// with 64 features and 5.7 with 128 (a large copy: 4.7, read and written).  Many queries are bound by the vector
// units, which turn codes into fp16 and scores into weights while the matrix units wait, and the
// reverse: 1000 candidates of one 16384-token history, 4 heads of 64, take 39 us, 13 at a large product's rate.
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
  float scale;       // times log2(e), as scale * 2^scale_e, in [1/2, 1)
  int scale_e;
  bf16_t* out;
  float* lse;        // nullable
  float* part_o;     // [splits, total, heads, D], with splits > 1
  float* part_ml;    // [splits, total, heads, 2]: reference and sum
  int tiles;         // query tiles per (sequence, kv head)
  int splits, chunk; // shares of a sequence's pages, and pages to a share
  int near;          // sequences of a block (my_job)
  int units;         // (sequence, kv head, share) triples, padded
  int group;         // neighbouring sequences whose rows fit one tile together
};

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

// A workgroup's share: `cap` query rows of a kv head of a sequence, entries [c0, c1) of their pages.
struct Job {
  int s, h, split, row0, G, rows;   // rows: the sequence's, (query, head) pairs
  int64_t q0, nq, first_pos;        // its queries, and the first one's position
  int64_t lo_pos, hi_pos;           // positions of this tile's first and last row
  int len, chunk, n, c0, c1;
  PageList list;
  const int32_t* table;
};

__device__ __forceinline__ int64_t query_count(const AttendArgs& a, int s) {
  const int64_t n = a.q.offset[s + 1] - a.q.offset[s];
  return n < 0 ? 0 : n > a.q.max_count ? a.q.max_count : n;
}

// Queries and pages of sequence s; false: none, or out of the arguments' range.
__device__ __forceinline__ bool job_of(const AttendArgs& a, int s, int row0, int cap, Job& j) {
  const tav2_kv& c = a.c;
  j.s = s;
  j.row0 = row0;
  j.G = a.q.heads / c.kv_heads;
  j.q0 = a.q.offset[s];
  j.nq = query_count(a, s);
  if (j.q0 < 0 || j.q0 + j.nq > a.q.total) return false;
  j.rows = int(j.nq) * j.G;
  if (row0 >= j.rows) return false;
  j.len = kv_len(c, s);
  j.first_pos = a.causal ? int64_t(j.len) - j.nq : j.len;
  const int last_row = min(row0 + cap, j.rows) - 1;
  j.lo_pos = a.causal ? j.first_pos + row0 / j.G : j.first_pos;
  j.hi_pos = a.causal ? j.first_pos + last_row / j.G : j.first_pos;
  j.list = pages_seen(j.len, j.lo_pos, j.hi_pos, a.q.window, a.q.sinks);
  j.n = j.list.count();
  // shares of one size, so that a long sequence has more of them (larger ones where it is
  // longer than the host's estimate)
  j.chunk = max(a.chunk, (j.n + a.splits - 1) / a.splits);
  j.table = c.table + int64_t(s) * c.max_blocks;
  return true;
}

// The same for this workgroup, with its split.  An empty share of several leaves a sum of zero and no
// features (kv_merge drops what it reads there).
__device__ __forceinline__ bool my_job(const AttendArgs& a, int cap, Job& j) {
  // Units (sequence, head, share) in the order (share, block of sequences, head), each on one XCD
  // (workgroups go to the 8 in turn) with the block's sequences one after the other, since
  // neighbours may be copies that read the same pages, and so the query tiles of each (8 copies each of 16
  // histories 79 us, with sequences spread over the XCDs 93).  First shares come first, the later
  // ones, which short sequences lack, at the end.
  const int unit = int(blockIdx.x % unsigned(a.units));
  const int tile = int(blockIdx.x / unsigned(a.units));
  const int block = unit / (8 * a.near) * 8 + unit % 8;
  const int blocks = (a.c.num_seqs + a.near - 1) / a.near * a.c.kv_heads;   // of a share
  const int s = block % blocks / a.c.kv_heads * a.near + unit / 8 % a.near;
  j.split = block / blocks;
  if (j.split >= a.splits || s >= a.c.num_seqs || !job_of(a, s, tile * cap, cap, j)) return false;
  j.h = block % a.c.kv_heads;
  j.c0 = j.split * j.chunk;
  j.c1 = min(j.n, j.c0 + j.chunk);
  if (a.splits > 1 && j.c0 >= j.n) {
    const int row = j.row0 + int(threadIdx.x);
    if (int(threadIdx.x) < cap && row < j.rows) {
      const int64_t part = int64_t(j.split) * a.q.total * a.q.heads +
                           (j.q0 + row / j.G) * a.q.heads + j.h * j.G + row % j.G;
      a.part_ml[2 * part] = -FLT_MAX;
      a.part_ml[2 * part + 1] = 0.f;
    }
    return false;
  }
  return true;
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

  __device__ __forceinline__ void look_up(const AttendArgs& a, const Job& j, int base) {
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
  __device__ __forceinline__ void load(const AttendArgs& a, const Job& j, int page) {
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

template <int D, int QT>
__global__ __launch_bounds__(256, 2) void kv_attend_kernel(AttendArgs a) {
  constexpr int KB = D / 2;   // bytes of a key's codes per lane
  // a wave's page on its way, then its state
  constexpr int STAGE = QT * D / 32 * 4 * WAVE;   // 16-byte pieces; a page has 8 D of them
  static_assert(STAGE >= 8 * D, "a page fits");
  __shared__ u32x4 stage[4][STAGE];
  __shared__ float mm[4][QT][2][WAVE];
  const tav2_kv& c = a.c;
  Job j;
  if (!my_job(a, 32 * QT, j)) return;
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
  seen.sinks = a.q.sinks;
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
    const int64_t pos = a.causal ? j.first_pos + i : j.first_pos;
    const int64_t end = pos + 1 < len ? pos + 1 : len;
    seen.hi[q] = int(end > 0 ? end : 0);
    const int64_t low = pos - a.q.window + 1;
    seen.lo[q] = a.q.window > 0 && low > 0 ? int(low) : 0;
  }
  // a page is seen whole by all of them where it ends by the first's last key and starts at the last's
  // first one (or lies among the sinks)
  const int64_t all_hi = j.lo_pos + 1 < len ? j.lo_pos + 1 : len;
  const int64_t all_lo = a.q.window > 0 ? j.hi_pos - a.q.window + 1 : 0;
  auto part_seen = [&](int b) {
    return int64_t(b + 1) * KVP > all_hi ||
           (int64_t(b) * KVP < all_lo && int64_t(b + 1) * KVP > a.q.sinks);
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
    const float inv = a.splits > 1 ? 1.f : some ? 1.f / l : 0.f;
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

// Sequences that hold the same pages in this share (copies of one another) are read once: of a window
// of `a.group` neighbouring sequences, whose rows fit one tile together, the first of each set
// takes the rows of all, and the others leave.  A share may end with the open block, which is each
// sequence's own.  Returns the set as bits of the window (its own alone where the share's first
// page has one holder), 0: leave.
__device__ __forceinline__ uint32_t shared_set(const AttendArgs& a, const Job& j) {
  __shared__ uint32_t differ;
  const int base = j.s / a.group * a.group, me = j.s - base;
  const int full = j.len / KVP, last = j.list.at(j.c1 - 1);
  const bool ends_open = last >= full;
  const int p1 = j.c1 - (ends_open ? 1 : 0);   // the share's pages: [c0, p1)
  int holders = 0;
  if (p1 > j.c0) {
    const int p = j.table[j.list.at(j.c0)];
    if (p >= 0 && p < a.c.pages) holders = a.c.refs[p];
  }
  if (holders < 2) return 1u << me;
  if (threadIdx.x == 0) differ = 0;
  __syncthreads();
  const int k = threadIdx.x / 16;   // 16 threads a candidate
  if (k < a.group && k != me) {
    Job o;
    bool same = base + k < a.c.num_seqs && job_of(a, base + k, 0, 16, o) &&
                o.list.sink == j.list.sink && o.list.first == j.list.first &&
                o.chunk == j.chunk && min(o.n, j.c0 + o.chunk) == j.c1 &&
                (ends_open ? o.len / KVP == full : o.len / KVP > last);
    if (same)
      for (int i = j.c0 + threadIdx.x % 16; i < p1; i += 16)
        same &= o.table[j.list.at(i)] == j.table[j.list.at(i)];
    if (!same) atomicOr(&differ, 1u << k);
  }
  __syncthreads();
  const uint32_t set = ~differ & ((1u << a.group) - 1);
  return (set & ((1u << me) - 1)) ? 0 : set;
}

// At most 16 query rows: on the 16x16x32 instructions, a page's 64 keys at once.  S^T comes in four tiles
// of 16 keys, in the order that makes a lane's 16 scores its quarter's 16 consecutive keys
// (16 g + 4 i + r in register r of tile i, g = l / 16), again the operand of O^T = V^T P^T as they
// stand.  Half the vector work of a 32-row tile: new actions of 64 users (4 rows) 35.4 us for 40.2 with
// that, 8 copies each of 16 histories 79 for 109.  Where rows are few enough, neighbouring sequences share
// a tile over the pages that they have in common (shared_set): the copies take 92 us without.
template <int D>
__global__ __launch_bounds__(256, D <= 64 ? 3 : 2) void kv_attend16_kernel(AttendArgs a) {
  constexpr int F = D / 4;           // features of a lane's quarter
  constexpr int NK = D / 32;         // products over the features
  constexpr int ND = D / 16;         // tiles of O^T
  __shared__ u32x4 stage[4][8 * D];  // a wave's page on its way, then its state (D / 16 x 64)
  __shared__ float mm[4][2][16];
  const tav2_kv& c = a.c;
  Job j;
  if (!my_job(a, 16, j)) return;
  const int lane = threadIdx.x % WAVE, m = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int full = j.len / KVP;
  u32x4* const my = stage[wave];
  Feed<D> feed;
  feed.look_up(a, j, j.c0 + wave);
  int page = feed.page(0);
  feed.load(a, j, page);

  // this lane's row: which (query, head) of which sequence, and what it sees
  int row = min(j.row0 + m, j.rows - 1), count = j.rows - j.row0, slot = j.s;
  uint32_t set = 0;   // sequences taken together, if several
  if (a.group > 1) {
    set = shared_set(a, j);
    if (set == 0) return;
    if (set & (set - 1)) {
      const int base = j.s / a.group * a.group;
      count = 0;
      for (int k = 0; k < a.group; ++k) {
        if (!(set >> k & 1)) continue;
        const int n = int(query_count(a, base + k)) * j.G;
        if (m >= count && m < count + n) {
          slot = base + k;
          row = m - count;
        }
        count += n;
      }
      if (m >= count) row = 0;   // padding: this sequence's first
    }
  }
  const bool valid = m < count;
  const int64_t q0 = a.q.offset[slot];
  const int len = kv_len(c, slot), i_q = row / j.G;
  const int64_t pos = a.causal ? int64_t(len) - query_count(a, slot) + i_q : len;
  const int64_t qi = q0 + i_q, at = qi * a.q.heads + j.h * j.G + row % j.G;
  const int64_t end = pos + 1 < len ? pos + 1 : len, low = pos - a.q.window + 1;
  int hi = int(end > 0 ? end : 0);
  const int lo = a.q.window > 0 && low > 0 ? int(low) : 0;
  int all_hi = hi, all_lo = lo;   // what all rows see: from the last one's first key to the first's last
#pragma unroll
  for (int o = 8; o >= 1; o >>= 1) {
    all_hi = min(all_hi, __shfl_xor(all_hi, o, WAVE));
    all_lo = max(all_lo, __shfl_xor(all_lo, o, WAVE));
  }
  all_hi = __builtin_amdgcn_readfirstlane(all_hi);
  all_lo = __builtin_amdgcn_readfirstlane(all_lo);
  f16x8 qf[NK];
  int cq;   // a power of two
  {
    const bf16_t* p = static_cast<const bf16_t*>(a.q.q) + qi * a.q.ld + (j.h * j.G + row % j.G) * D + g * F;
    u32x4 w[NK];
    float top = 0.f, f, back;
#pragma unroll
    for (int t = 0; t < NK; ++t) w[t] = *reinterpret_cast<const u32x4*>(p + 8 * t);
#pragma unroll
    for (int t = 0; t < NK; ++t) top = max8(w[t], top);
    into_half<TO_TOP>(xmax32(xmax16(top)), &f, &back);
#pragma unroll
    for (int t = 0; t < NK; ++t) qf[t] = scaled8h(w[t], f);
    cq = a.scale_e + __builtin_amdgcn_frexp_expf(back) - 1;
  }

  f32x4 o[ND];
  float ref = -FLT_MAX, wref = -FLT_MAX, ratio = 1.f, sum = 0.f;   // (m, n, d, l of attend_core.h)
#pragma unroll
  for (int d = 0; d < ND; ++d) o[d] = (f32x4){0.f, 0.f, 0.f, 0.f};

  // one page: keys(i, kf) sets the operands of S^T's tile i, values(d, vf) those of O^T's tile d
  auto step = [&](auto keys, auto values, float cs, AttScale vs, int key0) {
    f32x4 s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f16x8 kf[NK];
      keys(i, kf);
      s[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < NK; ++t) s[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kf[t], qf[t], s[i], 0, 0, 0);
    }
    if (key0 + KVP > all_hi || (key0 < all_lo && key0 + KVP > a.q.sinks)) {
      const int k0 = key0 + 16 * g, hi_ = hi - k0, lo_ = lo - k0, sinks = a.q.sinks - k0;
#pragma unroll
      for (int r = 0; r < 16; ++r)
        s[r / 4][r % 4] = r < hi_ && (r >= lo_ || r < sinks) ? s[r / 4][r % 4] : -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int r = 1; r < 16; ++r) top = vmax(top, s[r / 4][r % 4]);
    top = xmax32(xmax16(top)) * cs;
    if (__any(att_passes(top, vs.lv, ref, wref))) {
      float of, lf;
      att_raise(top, vs.lv, ref, wref, ratio, &of, &lf);
      sum *= lf;
#pragma unroll
      for (int d = 0; d < ND; ++d) o[d] *= of;
    }
    float b, e;
    att_offset(top, vs, ref, wref, ratio, &b, &e);
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
  };
  const int krow = 16 * (m / 4) + m % 4;   // + 4 i: the key of tile i that this lane's row is
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
      step(keys, values, score_factor(a.scale * ks, cq), vs, b * KVP);
    }
    page = next;
  }
  // the open block, in bf16 (as in the kernel above): this sequence's, or, of several taken together,
  // each one's, which its own rows alone see, by the waves in turn
  auto open_block = [&](int of) {
    const int64_t tail = kv_tail(c, a.layer, of, j.h);
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
    // (read twice, as above)
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
    step(keys, values, score_factor(a.scale * backk, cq), tail_scale(vt, backv, fv), full * KVP);
  };
  if (j.list.at(j.c1 - 1) >= full) {
    const int mine = hi, base = j.s / a.group * a.group;
    if (set == 0) set = 1u << (j.s - base);
    int turn = j.c1 - 1 - j.c0;   // (the wave whose turn it is takes a single one)
    while (set) {
      const int of = base + __builtin_ctz(set);
      set &= set - 1;
      hi = slot == of ? mine : 0;
      if (turn++ % 4 == wave) open_block(of);
    }
  }

  // the four waves' states meet in LDS; wave w joins every fourth tile of O^T, in the order of the waves
  __builtin_amdgcn_wave_barrier();
  sum = xsum32(xsum16(sum));
  if (g == 0) {
    mm[wave][0][m] = wref;
    mm[wave][1][m] = sum;
  }
#pragma unroll
  for (int d = 0; d < ND; ++d) my[d * WAVE + lane] = __builtin_bit_cast(u32x4, o[d] * ratio);
  __syncthreads();
  if (!valid) return;
  float M = -FLT_MAX, l = 0.f, f[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) M = vmax(M, mm[w][0][m]);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    f[w] = half_factor(mm[w][0][m] - M);
    l += mm[w][1][m] * f[w] * f[w];
  }
  const int64_t part = int64_t(j.split) * a.q.total * a.q.heads + at;
  const bool some = l > 0.f || l != l;
  const float inv = some ? 1.f / l : 0.f;
  for (int d = wave; d < ND; d += 4) {
    f32x4 x = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < 4; ++w) x += __builtin_bit_cast(f32x4, stage[w][d * WAVE + lane]) * f[w] * f[w];
    const int feature = 16 * d + 4 * g;
    if (a.splits > 1)
      *reinterpret_cast<f32x4*>(a.part_o + part * D + feature) = x;
    else
      *reinterpret_cast<uint2*>(a.out + at * D + feature) =
          make_uint2(pack2(x[0] * inv, x[1] * inv), pack2(x[2] * inv, x[3] * inv));
  }
  if (wave == 0 && g == 0) {
    if (a.splits > 1) {
      a.part_ml[2 * part] = M;
      a.part_ml[2 * part + 1] = l;
    } else if (a.lse) {
      a.lse[at] = some ? (M + __builtin_amdgcn_logf(l)) * LN2 : -INFINITY;
    }
  }
}

// A workgroup per (query, head): D features by 256 / D groups of splits, the groups joined in LDS.
// Bound by latency: two dependent reads, 3.2 us for one query of 64 shares.
template <int D>
__global__ __launch_bounds__(256) void kv_merge_kernel(AttendArgs a) {
  constexpr int NG = 256 / D;
  __shared__ float lo[NG][D], ll[NG];
  const int64_t at = blockIdx.x, n = a.q.total * a.q.heads;
  const int tid = threadIdx.x, f = tid % D, g = tid / D;
  // queries of no sequence (their part of the workspace is not written): left as they were
  const int64_t r0 = a.q.offset[0] * a.q.heads, r1 = a.q.offset[a.c.num_seqs] * a.q.heads;
  float M = -FLT_MAX;
  for (int s = tid % WAVE; s < a.splits; s += WAVE) M = fmaxf(M, a.part_ml[2 * (s * n + at)]);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, WAVE));
  float l = 0.f, x = 0.f;
  // An empty share's features are not written: read all the same, so that no load waits for the sum
  // that says so, and dropped.
#pragma unroll 8
  for (int s = g; s < a.splits; s += NG) {
    const int64_t p = s * n + at;
    const float lp = a.part_ml[2 * p + 1], o = a.part_o[p * D + f];
    const float w = half_factor(a.part_ml[2 * p] - M);
    l += lp * w * w;
    x += lp != 0.f ? o * w * w : 0.f;
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
  if (at < r0 || at >= r1) return;
  const bool some = l > 0.f || l != l;
  a.out[at * D + f] = f2bf(some ? x / l : 0.f);
  if (a.lse && f == 0) a.lse[at] = some ? (M + __builtin_amdgcn_logf(l)) * LN2 : -INFINITY;
}

// Pages that a query tile of the longest sequence sees, by the host's estimate.
int64_t most_pages(const tav2_kv& c, const tav2_kv_queries& q) {
  int64_t tokens = std::min<int64_t>(c.max_len, int64_t(c.max_blocks) * KVP + KVP - 1);
  if (q.window > 0) tokens = std::min(tokens, int64_t(q.window) + q.max_count + q.sinks + 2 * KVP);
  return std::max<int64_t>(1, cdiv(tokens, KVP));
}

// Query rows of a workgroup: 16, 32, or, where there are pages enough to fill the CUs with tiles of twice
// the work, 64 (which turn a page's codes into operands once for twice the queries, but start and
// end later; 64 features at most: registers; with 32 the turning is the smaller part).  By the number of 64-row tiles
// times pages; us a call with 32 and 64 rows, 4 heads.  64 features: one history of 16384 tokens, 64 candidates
// (1024) 13.3 and 24.4, 300 (5120) 24.5 and 25.4, 400 (7168) 28.8 and 25.9, 500 (8192) 24.6 and 26.4, 600 (10240)
// 37.5 and 36.1, 800 (13312) 45.1 and 37.5; 8 histories of 4096 - 16384, 64 candidates each (8192) 25.5 and 28.3,
// 100 (16384) 38.5 and 37.8, 500 125 and 119; 16 of them, 1000 each, 473 and 407.  32 features: 800 (13312) 32.4 and
// 30.3, 2000 (32768) 50.3 and 51.6; 8 x 200 (32768) 48.4 and 50.2, 8 x 500 (65536) 88.1 and 90.2; 16 x 1000
// (262144) 309 and 297.
int tile_rows(const tav2_kv& c, const tav2_kv_queries& q) {
  const int64_t rows = int64_t(q.max_count) * (q.heads / c.kv_heads);
  if (rows <= 16) return 16;
  const int64_t seqs = std::min<int64_t>(q.total, c.num_seqs);
  const int64_t work = seqs * c.kv_heads * cdiv(rows, 64) * most_pages(c, q);
  return rows > 32 && c.head_dim <= 64 && work > (c.head_dim == 64 ? 9000 : 100000) ? 64 : 32;
}

// Pages to a workgroup's share: such that there are workgroups enough to fill the CUs and to even out
// sequences of different lengths, but no share so small that its partial results (4 bytes a feature,
// written and read) come near the pages it reads (2 bytes a feature of 64 tokens).
int share_pages(const tav2_kv& c, const tav2_kv_queries& q) {
  const int64_t rows = int64_t(q.max_count) * (q.heads / c.kv_heads);
  const int64_t seqs = q.total < c.num_seqs ? q.total : c.num_seqs;
  const int64_t tile = tile_rows(c, q);
  const int64_t groups = seqs * c.kv_heads * cdiv(rows, tile);
  const int64_t least = std::max<int64_t>(4, std::min<int64_t>(rows, tile) / 2);
  return int(std::max(least, std::min<int64_t>(SHARE_MOST, cdiv(groups * most_pages(c, q), SHARES))));
}
int key_splits(const tav2_kv& c, const tav2_kv_queries& q) {
  return int(cdiv(most_pages(c, q), share_pages(c, q)));
}

int near_seqs(const tav2_kv& c) { return c.num_seqs < 8 ? c.num_seqs : 8; }
int64_t query_units(const tav2_kv& c, int splits) {
  const int near = near_seqs(c);
  return cdiv(splits * cdiv(c.num_seqs, near) * c.kv_heads, 8) * 8 * near;
}

}  // namespace

int64_t kv_attend_groups(const tav2_kv& c, const tav2_kv_queries& q) {
  const int64_t rows = int64_t(q.max_count) * (q.heads / c.kv_heads);
  const int splits = key_splits(c, q);
  return std::max(query_units(c, splits) * cdiv(rows, tile_rows(c, q)),
                  splits > 1 ? q.total * q.heads : 0);
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
  a.scale = frexpf((q.scale > 0.f ? q.scale : 1.f / sqrtf(float(c.head_dim))) * LOG2E, &a.scale_e);
  a.out = static_cast<bf16_t*>(out);
  a.lse = lse;
  const int tile = tile_rows(c, q), rows = q.max_count * (q.heads / c.kv_heads);
  a.splits = key_splits(c, q);
  a.chunk = share_pages(c, q);
  a.tiles = int(cdiv(rows, tile));
  a.group = tile == 16 && a.splits > 1 ? 16 / rows : 1;
  a.near = near_seqs(c);
  a.units = int(query_units(c, a.splits));
  a.part_o = static_cast<float*>(ws);
  if (a.splits > 1) a.part_ml = a.part_o + size_t(a.splits) * q.total * q.heads * c.head_dim;
  const unsigned grid = unsigned(a.units) * unsigned(a.tiles);
  {
    ProfScope prof("kv_attend", st);
    if (c.head_dim == 32) {
      if (tile == 16) kv_attend16_kernel<32><<<grid, 256, 0, st>>>(a);
      else if (tile == 32) kv_attend_kernel<32, 1><<<grid, 256, 0, st>>>(a);
      else kv_attend_kernel<32, 2><<<grid, 256, 0, st>>>(a);
    } else if (c.head_dim == 64) {
      if (tile == 16) kv_attend16_kernel<64><<<grid, 256, 0, st>>>(a);
      else if (tile == 32) kv_attend_kernel<64, 1><<<grid, 256, 0, st>>>(a);
      else kv_attend_kernel<64, 2><<<grid, 256, 0, st>>>(a);
    } else {
      if (tile == 16) kv_attend16_kernel<128><<<grid, 256, 0, st>>>(a);
      else kv_attend_kernel<128, 1><<<grid, 256, 0, st>>>(a);
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
