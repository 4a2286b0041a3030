// Attention of many continuations over the one history that they share, and over their own tokens.
//
// Softmax over two sets of keys is joined from each one's largest score, sum and features, so the history
// is taken first: the queries of all members of a group are rows of one tile set over the history's pages (as one
// sequence's queries are in kv_attend), each page read and turned into operands once for 16, 32 or 64 rows of any
// members.  A second launch takes each member's own tokens, joins the shares of its rows, and writes them.
#include "kv_attend_core.h"

namespace tav2 {

namespace {

struct PrefixArgs {
  tav2_kv c;
  int layer;
  tav2_kv_groups g;
  tav2_kv_queries q;
  bool causal;
  float scale;         // times log2(e), as scale * 2^scale_e, in [1/2, 1)
  int scale_e;
  bf16_t* out;
  float* lse;          // nullable
  float* part_o;       // [splits, total, heads, D]
  float* part_ml;      // [splits, total, heads, 2]: reference and sum
  int most_rows;       // rows of a group and kv head, at most
  int tiles;           // row tiles of a group and kv head
  int splits, chunk;   // shares of a prefix's pages, and pages to a share
  int units;           // (share, group, kv head), padded to a multiple of 8
  int own_tiles;       // 16-row tiles of a member and kv head
  __device__ __forceinline__ bool parts() const { return true; }
};

// The members and queries of a group; false: none, or out of the arguments' range.
struct Group {
  int first, n, prefix, len;   // prefix -1 and len 0: none
  int64_t q0, nq;
};
__device__ __forceinline__ bool group_of(const PrefixArgs& a, int g, Group& r) {
  r.first = a.g.offset[g];
  const int end = a.g.offset[g + 1];
  if (r.first < 0 || end > a.c.num_seqs || r.first >= end) return false;
  r.n = min(end - r.first, a.g.max_members);
  r.q0 = a.q.offset[r.first];
  const int64_t q1 = a.q.offset[r.first + r.n];
  if (r.q0 < 0 || q1 < r.q0 || q1 > a.q.total) return false;
  r.nq = q1 - r.q0;
  r.prefix = a.g.prefix[g];
  if (r.prefix >= a.c.num_seqs) r.prefix = -1;
  r.len = r.prefix < 0 ? 0 : kv_len(a.c, r.prefix);
  return true;
}

__device__ __forceinline__ int64_t member_count(const PrefixArgs& a, int s) {
  const int64_t n = a.q.offset[s + 1] - a.q.offset[s];
  return n < 0 ? 0 : n > a.q.max_count ? a.q.max_count : n;
}

// How far behind the prefix query i (of the group's) stands.
__device__ __forceinline__ int64_t place_of(const PrefixArgs& a, const Group& r, int64_t i) {
  const int64_t* off = a.q.offset + r.first;
  const int64_t q = r.q0 + i;
  int m = int(i * r.n / (r.nq > 0 ? r.nq : 1));   // members with as many queries each
  m = min(m, r.n - 1);
  if (!(off[m] <= q && q < off[m + 1])) {
    int lo = 0, hi = r.n - 1;   // the last member that begins at q or before
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (off[mid] <= q) lo = mid; else hi = mid - 1;
    }
    m = lo;
  }
  const int len = kv_len(a.c, r.first + m);
  return a.causal ? len - member_count(a, r.first + m) + (q - off[m]) : len;
}

// A workgroup's share of a prefix: `cap` rows of a kv head, entries [c0, c1) of the pages they see.
struct PrefixJob {
  int s, h, split, row0, G, rows;
  int64_t q0;
  int len, chunk, n, c0, c1;
  PageList list;
  const int32_t* table;
  int lo;            // the first position that row row0 + lane sees
  int all_lo;        // and that all rows of the tile see
};

__device__ __forceinline__ bool prefix_job(const PrefixArgs& a, int cap, PrefixJob& j) {
  // Eight neighbouring workgroups take a tile of eight units, one on each XCD; the units' further tiles follow, so
  // that they find the pages in that XCD's L2.  First shares come first, the later ones, which short
  // prefixes lack, at the end.
  const int unit = int(blockIdx.x / unsigned(8 * a.tiles)) * 8 + int(blockIdx.x % 8);
  const int tile = int(blockIdx.x / 8 % unsigned(a.tiles));
  const int per = a.g.num_groups * a.c.kv_heads;
  j.split = unit / per;
  if (j.split >= a.splits) return false;
  const int g = unit % per / a.c.kv_heads;
  j.h = unit % a.c.kv_heads;
  Group r;
  if (!group_of(a, g, r)) return false;
  j.s = r.prefix;
  j.G = a.q.heads / a.c.kv_heads;
  j.q0 = r.q0;
  const int64_t rows = r.nq * j.G;
  j.rows = int(rows < a.most_rows ? rows : a.most_rows);
  j.row0 = tile * cap;
  if (j.row0 >= j.rows) return false;
  j.len = r.len;
  j.lo = j.all_lo = 0;
  int64_t first = 0;
  if (a.q.window > 0) {
    const int row = min(j.row0 + int(threadIdx.x % WAVE), min(j.row0 + cap, j.rows) - 1);
    const int64_t low = r.len + place_of(a, r, row / j.G) - a.q.window + 1;   // below 2^32 either way
    j.lo = low > 0 ? int(low < r.len ? low : r.len) : 0;
    int least = j.lo, most = j.lo;
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) {
      least = min(least, __shfl_xor(least, o, WAVE));
      most = max(most, __shfl_xor(most, o, WAVE));
    }
    first = __builtin_amdgcn_readfirstlane(least);
    j.all_lo = __builtin_amdgcn_readfirstlane(most);
  }
  j.list.last = (j.len + KVP - 1) / KVP;
  j.list.first = int(first / KVP);
  const int64_t sink_pages = (int64_t(a.q.sinks) + KVP - 1) / KVP;
  j.list.sink = a.q.window > 0 ? min(int(sink_pages < j.list.first ? sink_pages : j.list.first), j.list.last) : 0;
  j.n = j.list.count();
  // shares of one size, so that a long prefix has more of them (larger ones where it is longer
  // than the host's estimate)
  j.chunk = max(a.chunk, (j.n + a.splits - 1) / a.splits);
  j.c0 = j.split * j.chunk;
  j.c1 = min(j.n, j.c0 + j.chunk);
  if (j.c0 >= j.n) {   // an empty share: a sum of zero and no features
    const int row = j.row0 + int(threadIdx.x);
    if (int(threadIdx.x) < cap && row < j.rows) {
      const int64_t part = int64_t(j.split) * a.q.total * a.q.heads +
                           (j.q0 + row / j.G) * a.q.heads + j.h * j.G + row % j.G;
      a.part_ml[2 * part] = -FLT_MAX;
      a.part_ml[2 * part + 1] = 0.f;
    }
    return false;
  }
  j.table = a.c.table + int64_t(j.s) * a.c.max_blocks;
  return true;
}

__device__ __forceinline__ void row_seen(const PrefixArgs& a, const PrefixJob& j, int row, int* hi, int* lo) {
  *hi = j.len;
  *lo = a.q.window > 0 ? __shfl(j.lo, row - j.row0, WAVE) : 0;
}
__device__ __forceinline__ void tile_seen(const PrefixArgs& a, const PrefixJob& j, int64_t* hi, int64_t* lo) {
  *hi = j.len;
  *lo = j.all_lo;
}
__device__ __forceinline__ int tile_sinks(const PrefixArgs& a, const PrefixJob&) { return a.q.sinks; }

template <int D, int QT>
__global__ __launch_bounds__(256, 2) void kv_prefix_kernel(PrefixArgs a) {
  PrefixJob j;
  if (prefix_job(a, 32 * QT, j)) attend_rows<D, QT>(a, j);
}

template <int D>
__global__ __launch_bounds__(256, D <= 64 ? 3 : 2) void kv_prefix16_kernel(PrefixArgs a) {
  constexpr int ND = D / 16;
  __shared__ u32x4 stage[4][8 * D];
  __shared__ float mm[4][2][16];
  PrefixJob j;
  if (!prefix_job(a, 16, j)) return;
  const int lane = threadIdx.x % WAVE, m = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  Feed<D> feed;
  feed.look_up(a, j, j.c0 + wave);
  int page = feed.page(0);
  feed.load(a, j, page);
  const int row = min(j.row0 + m, j.rows - 1);
  const int64_t qi = j.q0 + row / j.G;
  int hi, lo;
  row_seen(a, j, row, &hi, &lo);
  auto open_blocks = [&](auto open_block) {
    if (j.list.at(j.c1 - 1) >= j.len / KVP && (j.c1 - 1 - j.c0) % 4 == wave) open_block(j.s);
  };
  auto finish = [&](float M, float l, auto tile) {
    if (j.row0 + m >= j.rows) return;
    const int64_t part =
        int64_t(j.split) * a.q.total * a.q.heads + qi * a.q.heads + j.h * j.G + row % j.G;
    for (int d = wave; d < ND; d += 4)
      *reinterpret_cast<f32x4*>(a.part_o + part * D + 16 * d + 4 * g) = tile(d);
    if (wave == 0 && g == 0) {
      a.part_ml[2 * part] = M;
      a.part_ml[2 * part + 1] = l;
    }
  };
  attend16<D>(a, j, feed, page, stage, mm, qi, row % j.G, hi, lo, open_blocks, finish);
}

// A member's own tokens, for at most 16 rows of a kv head; positions are counted from its first one.
struct OwnJob {
  int s, h, G, len, c0, c1, sinks;
  PageList list;
  const int32_t* table;
};
__device__ __forceinline__ int tile_sinks(const PrefixArgs& a, const OwnJob& j) { return j.sinks; }

template <int D>
__global__ __launch_bounds__(256, D <= 64 ? 3 : 2) void kv_join_kernel(PrefixArgs a) {
  constexpr int ND = D / 16, Q = D / 4;
  __shared__ u32x4 stage[4][8 * D];
  __shared__ float mm[4][2][16];
  __shared__ f32x4 joined[16][Q];   // the prefix's features, against jm
  __shared__ float jm[16], jl[16];
  const tav2_kv& c = a.c;
  OwnJob j;
  unsigned b = blockIdx.x;
  j.h = int(b % c.kv_heads);
  b /= c.kv_heads;
  const int tile = int(b % a.own_tiles);
  b /= a.own_tiles;
  const int member = int(b % a.g.max_members);
  Group r;
  if (!group_of(a, int(b / a.g.max_members), r) || member >= r.n) return;
  j.s = r.first + member;
  j.G = a.q.heads / c.kv_heads;
  const int64_t q0 = a.q.offset[j.s], most = a.most_rows / j.G;   // queries that the first launch took
  const int64_t nq = member_count(a, j.s);
  if (q0 < r.q0 || q0 + nq > r.q0 + (r.nq < most ? r.nq : most)) return;
  const int rows = int(nq) * j.G, row0 = 16 * tile;
  if (row0 >= rows) return;
  const int tid = threadIdx.x, lane = tid % WAVE, m = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(tid / WAVE);
  const int64_t n = a.q.total * a.q.heads;
  auto at_of = [&](int row) { return (q0 + row / j.G) * a.q.heads + j.h * j.G + row % j.G; };

  // the shares' references and sums: 16 threads a row
  const int R = min(16, rows - row0);
  {
    const int k = tid / 16;
    const int64_t at = at_of(row0 + min(k, R - 1));
    float M = -FLT_MAX, l = 0.f;
    for (int s = tid % 16; s < a.splits; s += 16) M = vmax(M, a.part_ml[2 * (s * n + at)]);
#pragma unroll
    for (int o = 8; o >= 1; o >>= 1) M = vmax(M, __shfl_xor(M, o, WAVE));
    for (int s = tid % 16; s < a.splits; s += 16) {
      const float w = half_factor(a.part_ml[2 * (s * n + at)] - M);
      l += a.part_ml[2 * (s * n + at) + 1] * w * w;
    }
#pragma unroll
    for (int o = 8; o >= 1; o >>= 1) l += __shfl_xor(l, o, WAVE);
    if (tid % 16 == 0) {
      jm[k] = M;
      jl[k] = l;
    }
  }
  __syncthreads();
  // their features: a thread takes four of a row, in every ng-th share
  {
    const int RQ = R * Q, ng = RQ < 256 ? 256 / RQ : 1;
    f32x4* const red = reinterpret_cast<f32x4*>(&stage[0][0]);
    for (int p = tid % (RQ < 256 ? RQ : 256), sg = RQ < 256 ? tid / RQ : 0; p < RQ; p += 256) {
      const int k = p / Q, d = p % Q;
      const int64_t at = at_of(row0 + k);
      f32x4 x = (f32x4){0.f, 0.f, 0.f, 0.f};
      // (an empty share's features are not written: read all the same, so that no load waits for the sum that
      // says so, and dropped)
#pragma unroll 8
      for (int s = sg; s < a.splits; s += ng) {
        const int64_t q = s * n + at;
        const float w = half_factor(a.part_ml[2 * q] - jm[k]);
        const f32x4 o = *reinterpret_cast<const f32x4*>(a.part_o + q * D + 4 * d);
        const bool some = a.part_ml[2 * q + 1] != 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] += some ? o[e] * w * w : 0.f;
      }
      if (sg >= ng) continue;   // (threads that are left over)
      if (ng == 1) joined[k][d] = x;
      else red[sg * RQ + p] = x;
    }
    if (ng > 1) {
      __syncthreads();
      for (int p = tid; p < RQ; p += 256) {
        f32x4 x = red[p];
        for (int sg = 1; sg < ng; ++sg) x += red[sg * RQ + p];
        joined[p / Q][p % Q] = x;
      }
    }
  }
  __syncthreads();

  // the own tokens
  j.len = kv_len(c, j.s);
  const int full = j.len / KVP;
  const int64_t o0 = a.causal ? j.len - nq : j.len;   // the first query's place
  const int row = min(row0 + m, rows - 1), i = row / j.G;
  const int64_t lo_pos = a.causal ? o0 + row0 / j.G : o0;
  const int64_t hi_pos = a.causal ? o0 + (row0 + R - 1) / j.G : o0;
  j.sinks = max(0, a.q.sinks - r.len);
  j.list = pages_seen(j.len, lo_pos, hi_pos, a.q.window, j.sinks);
  const int count = j.list.count();
  const bool open = count > 0 && j.list.at(count - 1) >= full;
  j.c0 = 0;
  j.c1 = count - (open ? 1 : 0);
  j.table = c.table + int64_t(j.s) * c.max_blocks;
  const int64_t pos = a.causal ? o0 + i : o0, low = pos - a.q.window + 1;
  const int64_t end = pos + 1 < j.len ? pos + 1 : j.len;
  int hi = int(end > 0 ? end : 0);
  const int lo = a.q.window > 0 && low > 0 ? int(low) : 0;
  Feed<D> feed = {};
  int page = -1;
  if (j.c1 > 0) {
    feed.look_up(a, j, wave);
    page = feed.page(0);
    feed.load(a, j, page);
  }
  auto open_blocks = [&](auto open_block) {
    if (open && j.c1 % 4 == wave) open_block(j.s);
  };
  auto finish = [&](float M, float l, auto tile) {
    if (row0 + m >= rows) return;
    const int64_t at = at_of(row);
    const float all = vmax(M, jm[m]), f = half_factor(M - all), fp = half_factor(jm[m] - all);
    const float sum = l * f * f + jl[m] * fp * fp;
    const bool some = sum > 0.f || sum != sum;
    const float inv = some ? 1.f / sum : 0.f;
    for (int d = wave; d < ND; d += 4) {
      const f32x4 own = tile(d), pre = joined[m][4 * d + g];
      f32x4 x;
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = (own[e] * f * f + pre[e] * fp * fp) * inv;
      *reinterpret_cast<uint2*>(a.out + at * D + 16 * d + 4 * g) =
          make_uint2(pack2(x[0], x[1]), pack2(x[2], x[3]));
    }
    if (wave == 0 && g == 0 && a.lse)
      a.lse[at] = some ? (all + __builtin_amdgcn_logf(sum)) * LN2 : -INFINITY;
  };
  attend16<D>(a, j, feed, page, stage, mm, q0 + i, row % j.G, hi, lo, open_blocks, finish);
}

// How the work on the prefixes is divided.
struct Plan {
  int64_t rows;        // of a group and kv head
  int64_t pages;       // that a tile of the longest prefix sees, by the host's estimate
  int tile, chunk, splits;
};
Plan plan_of(const tav2_kv& c, const tav2_kv_groups& g, const tav2_kv_queries& q) {
  Plan p;
  const int G = q.heads / c.kv_heads;
  p.rows = std::min<int64_t>(q.total, int64_t(g.max_members) * q.max_count) * G;
  int64_t tokens = std::min<int64_t>(c.max_len, int64_t(c.max_blocks) * KVP + KVP - 1);
  if (q.window > 0)
    tokens = std::min(tokens, int64_t(q.window) + g.max_own + q.sinks + 2 * KVP);
  p.pages = std::max<int64_t>(1, cdiv(tokens, KVP));
  const int64_t work = int64_t(g.num_groups) * c.kv_heads * cdiv(p.rows, 64) * p.pages;
  p.tile = p.rows <= 16 ? 16
           : p.rows > 32 && c.head_dim <= 64 && work > (c.head_dim == 64 ? 9000 : 100000) ? 64 : 32;
  const int64_t tiles = int64_t(g.num_groups) * c.kv_heads * cdiv(p.rows, p.tile);
  const int64_t least = std::max<int64_t>(4, std::min<int64_t>(p.rows, p.tile) / 2);
  p.chunk = int(std::max(least, std::min<int64_t>(SHARE_MOST, cdiv(tiles * p.pages, SHARES))));
  p.splits = int(cdiv(p.pages, p.chunk));
  return p;
}
int64_t prefix_units(const tav2_kv& c, const tav2_kv_groups& g, const Plan& p) {
  return cdiv(int64_t(p.splits) * g.num_groups * c.kv_heads, 8) * 8;
}
int64_t own_tiles(const tav2_kv& c, const tav2_kv_queries& q) {
  return cdiv(int64_t(q.max_count) * (q.heads / c.kv_heads), 16);
}

}  // namespace

// (their product may pass 64 bits)
double kv_prefix_workgroups(const tav2_kv& c, const tav2_kv_groups& g, const tav2_kv_queries& q) {
  const Plan p = plan_of(c, g, q);
  return std::max(double(prefix_units(c, g, p)) * double(cdiv(p.rows, p.tile)),
                  double(g.num_groups) * g.max_members * c.kv_heads * double(own_tiles(c, q)));
}

size_t kv_prefix_bytes(const tav2_kv& c, const tav2_kv_groups& g, const tav2_kv_queries& q) {
  const Plan p = plan_of(c, g, q);
  return align_up(size_t(p.splits) * size_t(q.total) * q.heads * (c.head_dim + 2) * 4, 256);
}

hipError_t launch_kv_prefix(const tav2_kv& c, int layer, const tav2_kv_groups& g,
                            const tav2_kv_queries& q, bool causal, void* out, float* lse, void* ws,
                            hipStream_t st) {
  const Plan p = plan_of(c, g, q);
  PrefixArgs a{};
  a.c = c;
  a.layer = layer;
  a.g = g;
  a.q = q;
  a.causal = causal;
  a.scale = frexpf((q.scale > 0.f ? q.scale : 1.f / sqrtf(float(c.head_dim))) * LOG2E, &a.scale_e);
  a.out = static_cast<bf16_t*>(out);
  a.lse = lse;
  a.part_o = static_cast<float*>(ws);
  a.part_ml = a.part_o + size_t(p.splits) * q.total * q.heads * c.head_dim;
  a.most_rows = int(p.rows);
  a.tiles = int(cdiv(p.rows, p.tile));
  a.splits = p.splits;
  a.chunk = p.chunk;
  a.units = int(prefix_units(c, g, p));
  a.own_tiles = int(own_tiles(c, q));
  {
    ProfScope prof("kv_prefix", st);
    const unsigned grid = unsigned(a.units) * unsigned(a.tiles);
    if (c.head_dim == 32) {
      if (p.tile == 16) kv_prefix16_kernel<32><<<grid, 256, 0, st>>>(a);
      else if (p.tile == 32) kv_prefix_kernel<32, 1><<<grid, 256, 0, st>>>(a);
      else kv_prefix_kernel<32, 2><<<grid, 256, 0, st>>>(a);
    } else if (c.head_dim == 64) {
      if (p.tile == 16) kv_prefix16_kernel<64><<<grid, 256, 0, st>>>(a);
      else if (p.tile == 32) kv_prefix_kernel<64, 1><<<grid, 256, 0, st>>>(a);
      else kv_prefix_kernel<64, 2><<<grid, 256, 0, st>>>(a);
    } else {
      if (p.tile == 16) kv_prefix16_kernel<128><<<grid, 256, 0, st>>>(a);
      else kv_prefix_kernel<128, 1><<<grid, 256, 0, st>>>(a);
    }
  }
  ProfScope prof("kv_join", st);
  const unsigned grid = unsigned(g.num_groups) * unsigned(g.max_members) * unsigned(c.kv_heads) *
                        unsigned(a.own_tiles);
  if (c.head_dim == 32) kv_join_kernel<32><<<grid, 256, 0, st>>>(a);
  else if (c.head_dim == 64) kv_join_kernel<64><<<grid, 256, 0, st>>>(a);
  else kv_join_kernel<128><<<grid, 256, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace tav2
