// Attention over the paged 8-bit cache: every head's queries of a sequence against its codes.
//
// A workgroup takes 32 QT queries of one kv head (the heads that share it count as queries) and a
// share of the pages they see; its four waves take the pages in turn, each turning a page's codes
// into matrix operands in its own registers, once for all 32 QT queries, and meet in LDS at
// the end.  Nothing is staged: a lane's operand of K is half a key's codes, of V^T 16 keys of
// one feature, both read straight from the page.  Codes are exact as bf16; a page's key scale
// multiplies the fp32 scores, its value scale enters the weights as a power of two added to the
// exponent.  Where queries are few, the pages are split over more workgroups, whose partial results
// a second launch joins in a fixed order.
#include <algorithm>

#include "attend_core.h"
#include "internal.h"
#include "kv_common.h"

namespace tav2 {

namespace {

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
  int splits;
  int units;         // (sequence, kv head, split) groups, padded to a multiple of 8
};

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

template <int D, int QT>
__global__ __launch_bounds__(256, D <= 64 ? 2 : 1) void kv_attend_kernel(AttendArgs a) {
  constexpr int KB = D / 2;   // bytes of a key's codes per lane
  __shared__ __align__(16) float mo[2][QT][D / 32][16][WAVE];
  __shared__ float mm[2][QT][2][WAVE];
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
  const int lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
  const int m = lane % 32, half = lane / 32;

  // this lane's queries: operands, and what they see
  bf16x8 qf[QT][D / 16];
  AttSeen<QT> seen;
  seen.sinks = a.q.sinks;
  const int64_t first_pos = a.causal ? int64_t(len) - nq : len;
  const int last_row = min(row0 + 32 * QT, rows) - 1;
  const int64_t lo_pos = a.causal ? first_pos + row0 / G : first_pos;
  const int64_t hi_pos = a.causal ? first_pos + last_row / G : first_pos;
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    const int row = min(row0 + 32 * q + m, rows - 1);
    const int i = row / G, g = row % G;
    const bf16_t* p = static_cast<const bf16_t*>(a.q.q) + (q0 + i) * a.q.ld + (h * G + g) * D + half * KB;
#pragma unroll
    for (int t = 0; t < D / 16; ++t) qf[q][t] = as_bf16x8(*reinterpret_cast<const uint4*>(p + 8 * t));
    const int64_t pos = a.causal ? first_pos + i : first_pos;
    const int64_t top = pos + 1 < len ? pos + 1 : len;
    seen.hi[q] = int(top > 0 ? top : 0);
    const int64_t low = pos - a.q.window + 1;
    seen.lo[q] = a.q.window > 0 && low > 0 ? int(low) : 0;
  }
  // a page is seen whole by all of them where it ends by the first's last key and starts at the last's
  // first one (or lies among the sinks)
  const int64_t all_hi = lo_pos + 1 < len ? lo_pos + 1 : len;
  const int64_t all_lo = a.q.window > 0 ? hi_pos - a.q.window + 1 : 0;

  AttState<D, QT> st;
  st.clear();
  const PageList list = pages_seen(len, lo_pos, hi_pos, a.q.window, a.q.sinks);
  const int n = list.count(), chunk = (n + a.splits - 1) / a.splits;
  const int i1 = min(n, (split + 1) * chunk);
  const int full = len / KVP;
  const int64_t table0 = int64_t(s) * c.max_blocks;
  const float scale = a.scale * LOG2E;
  for (int i = split * chunk + wave; i < i1; i += 4) {
    const int b = list.at(i);
    const bool open = b >= full;   // the tail
    int page = 0;
    if (!open) {
      page = c.table[table0 + b];
      if (page < 0 || page >= c.pages) continue;   // released
    }
    const int64_t at = kv_unit(c, a.layer, page, h);
    const float cs = open ? scale : scale * c.k_scale[at];
    const float vs = open ? 1.f : c.v_scale[at];
    const float lv = open ? 0.f : __builtin_amdgcn_logf(vs), inv = open ? 1.f : 1.f / vs;
    const bool masked = int64_t(b + 1) * KVP > all_hi ||
                        (int64_t(b) * KVP < all_lo && int64_t(b + 1) * KVP > a.q.sinks);
    const int8_t* kp = c.k + at * KVP * D;
    const int8_t* vp = c.v + at * KVP * D;
    const int64_t tail = kv_tail(c, a.layer, s, h);
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      bf16x8 kf[D / 16], vf[D / 32][2];
      const int kr = 32 * u + key_row(m), k0 = 32 * u + 16 * half;
      if (!open) {
#pragma unroll
        for (int t = 0; t < D / 32; ++t) {
          const uint4 w = *reinterpret_cast<const uint4*>(kp + kr * D + half * KB + 16 * t);
          kf[2 * t] = codes8(w.x, w.y);
          kf[2 * t + 1] = codes8(w.z, w.w);
        }
#pragma unroll
        for (int d = 0; d < D / 32; ++d) {
          const uint4 w = *reinterpret_cast<const uint4*>(vp + (32 * d + m) * KVP + k0);
          vf[d][0] = codes8(w.x, w.y);
          vf[d][1] = codes8(w.z, w.w);
        }
      } else {   // bf16; what lies behind the last token is not read as numbers
        const bf16_t* kt = c.k_tail + tail + kr * D + half * KB;
#pragma unroll
        for (int t = 0; t < D / 16; ++t) kf[t] = as_bf16x8(*reinterpret_cast<const uint4*>(kt + 8 * t));
        const int held = len - b * KVP - k0;   // tokens from key k0 on
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            const uint4 w =
                *reinterpret_cast<const uint4*>(c.v_tail + tail + (32 * d + m) * KVP + k0 + 8 * t);
            uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              if (8 * t + 2 * e >= held) x[e] = 0;
              else if (8 * t + 2 * e + 1 >= held) x[e] &= 0xFFFFu;
            }
            vf[d][t] = as_bf16x8(make_uint4(x[0], x[1], x[2], x[3]));
          }
      }
      att_step<D, QT>(st, kf, vf, qf, cs, lv, inv, masked, seen, b * KVP + k0);
    }
  }

  // the four waves' states joined, two at a time: waves 2 and 3 into 0 and 1, then 1 into 0
#pragma unroll
  for (int q = 0; q < QT; ++q) st.l[q] = xsum32(st.l[q]);
#pragma unroll
  for (int step = 2; step >= 1; step /= 2) {
    if (wave >= step && wave < 2 * step) {
#pragma unroll
      for (int q = 0; q < QT; ++q) {
        mm[wave - step][q][0][lane] = st.m[q];
        mm[wave - step][q][1][lane] = st.l[q];
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r) mo[wave - step][q][d][r][lane] = st.o[d][q][r];
      }
    }
    __syncthreads();
    if (wave < step) {
#pragma unroll
      for (int q = 0; q < QT; ++q) {
        const float m2 = mm[wave][q][0][lane], l2 = mm[wave][q][1][lane];
        const float M = m2 > st.m[q] ? m2 : st.m[q];
        const float f1 = __builtin_amdgcn_exp2f(st.m[q] - M), f2 = __builtin_amdgcn_exp2f(m2 - M);
        st.m[q] = M;
        st.l[q] = st.l[q] * f1 + l2 * f2;
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            st.o[d][q][r] = st.o[d][q][r] * f1 + mo[wave][q][d][r][lane] * f2;
      }
    }
    __syncthreads();
  }
  if (wave != 0) return;
#pragma unroll
  for (int q = 0; q < QT; ++q) {
    const int row = row0 + 32 * q + m;
    if (row >= rows) continue;
    const int64_t at = (q0 + row / G) * a.q.heads + h * G + row % G;
    const float l = st.l[q];
    if (a.splits > 1) {
      const int64_t p = int64_t(split) * a.q.total * a.q.heads + at;
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          *reinterpret_cast<float4*>(a.part_o + p * D + 32 * d + 8 * j + 4 * half) =
              make_float4(st.o[d][q][4 * j], st.o[d][q][4 * j + 1], st.o[d][q][4 * j + 2],
                          st.o[d][q][4 * j + 3]);
      if (half == 0) {
        a.part_ml[2 * p] = st.m[q];
        a.part_ml[2 * p + 1] = l;
      }
      continue;
    }
    const float inv = l > 0.f || l != l ? 1.f / l : 0.f;   // nothing seen: zeros
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<uint2*>(a.out + at * D + 32 * d + 8 * j + 4 * half) =
            make_uint2(pack2(st.o[d][q][4 * j] * inv, st.o[d][q][4 * j + 1] * inv),
                       pack2(st.o[d][q][4 * j + 2] * inv, st.o[d][q][4 * j + 3] * inv));
    if (a.lse && half == 0)
      a.lse[at] = l > 0.f || l != l ? (st.m[q] + __builtin_amdgcn_logf(l)) * LN2 : -INFINITY;
  }
}

// One wave per (query, head): the splits' parts in order, a lane two features (D 128), one, or
// half of the lanes one.
__global__ __launch_bounds__(64) void kv_merge_kernel(AttendArgs a, int D) {
  const int64_t at = blockIdx.x, n = a.q.total * a.q.heads;
  const int lane = threadIdx.x;
  float M = -FLT_MAX;
  for (int s = lane; s < a.splits; s += WAVE) M = fmaxf(M, a.part_ml[2 * (s * n + at)]);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) M = fmaxf(M, __shfl_xor(M, o, WAVE));
  float l = 0.f, x0 = 0.f, x1 = 0.f;
  for (int s = 0; s < a.splits; ++s) {
    const int64_t p = s * n + at;
    const float f = __builtin_amdgcn_exp2f(a.part_ml[2 * p] - M);
    l += a.part_ml[2 * p + 1] * f;
    if (lane < D) x0 += a.part_o[p * D + lane] * f;
    if (lane + WAVE < D) x1 += a.part_o[p * D + lane + WAVE] * f;
  }
  const bool some = l > 0.f || l != l;
  const float inv = some ? 1.f / l : 0.f;
  if (lane < D) a.out[at * D + lane] = f2bf(x0 * inv);
  if (lane + WAVE < D) a.out[at * D + lane + WAVE] = f2bf(x1 * inv);
  if (a.lse && lane == 0) a.lse[at] = some ? (M + __builtin_amdgcn_logf(l)) * LN2 : -INFINITY;
}

int query_tiles(const tav2_kv& c, const tav2_kv_queries& q) {
  return int64_t(q.max_count) * (q.heads / c.kv_heads) > 32 && c.head_dim <= 64 ? 2 : 1;
}

// Shares of a sequence's pages: enough workgroups for two per CU, no share below one page
// per wave.
int key_splits(const tav2_kv& c, const tav2_kv_queries& q) {
  const int64_t rows = int64_t(q.max_count) * (q.heads / c.kv_heads);
  const int64_t seqs = q.total < c.num_seqs ? q.total : c.num_seqs;
  const int64_t groups = seqs * c.kv_heads * cdiv(rows, 32 * query_tiles(c, q));
  int64_t tokens = c.max_len;
  if (q.window > 0) tokens = std::min(tokens, int64_t(q.window) + q.max_count + q.sinks + 2 * KVP);
  const int64_t most = std::max<int64_t>(1, tokens / (4 * KVP));
  return int(std::max<int64_t>(1, std::min(most, 512 / std::max<int64_t>(1, groups))));
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
    kv_merge_kernel<<<unsigned(q.total * q.heads), 64, 0, st>>>(a, c.head_dim);
  }
  return hipGetLastError();
}

}  // namespace tav2
