// Attention of many continuations over the one history that they share, and over their own tokens.
//
// Softmax over two sets of keys is joined from each one's largest score, sum and features, so the history
// is taken first: the queries of all members of a group are rows of one tile set over the history's pages (as one
// sequence's queries are in kv_attend), each page read and turned into operands once for 16, 32 or 64 rows of any
// members.  A second launch takes each member's own tokens, joins the shares of its rows, and writes them.
#include <algorithm>
#include <type_traits>

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
  int32_t* plan;       // pages to a share, as the first launch chose
  int most_rows;       // rows of a group and kv head, at most
  int tile, tiles;     // rows of a tile, and tiles of a group and kv head, at most
  int splits;          // shares of a prefix's pages, at most
  int chunk;           // pages to a share; 0: every workgroup finds it out
  int least, target;   // then: the least, and workgroups that share all pages
  bool fit;            // no more than those
  int seen;            // pages that a row sees at most, by the host's estimate, with a window
  int own_tiles;       // 16-row tiles of a member and kv head
  bool count;          // the second launch has jobs for as many members as there are sequences
  __device__ __forceinline__ bool parts() const { return true; }
};

// The members and queries of a group, and its prefix's length; n 0: none, or out of the arguments' range.
struct Group {
  int first, n, prefix, len;   // prefix -1 and len 0: none
  int64_t q0, nq;
};
// (The reads depend on one another in two steps only: what is out of range is read from somewhere in range, and judged
// afterwards.)
__device__ __forceinline__ Group group_of(const PrefixArgs& a, int g) {
  Group r;
  const int most = a.c.num_seqs;
  const int first = a.g.offset[g], end = a.g.offset[g + 1], prefix = a.g.prefix[g];
  const bool ok = first >= 0 && first < end && end <= most;
  const bool has = prefix >= 0 && prefix < most;
  r.first = ok ? first : 0;
  r.n = ok ? min(end - first, a.g.max_members) : 0;
  r.prefix = has ? prefix : -1;
  r.q0 = a.q.offset[r.first];
  const int64_t q1 = a.q.offset[r.first + r.n];
  const int len = kv_len(a.c, has ? prefix : 0);
  r.len = has ? len : 0;
  r.nq = q1 - r.q0;
  if (r.q0 < 0 || r.nq < 0 || q1 > a.q.total) r.n = 0, r.nq = 0;
  return r;
}
__device__ __forceinline__ int group_rows(const PrefixArgs& a, const Group& r) {
  const int64_t rows = r.nq * (a.q.heads / a.c.kv_heads);
  return int(rows < a.most_rows ? rows : a.most_rows);
}
// Pages that its shares are counted by: those of the prefix; with a window about as many as a row sees.
__device__ __forceinline__ int group_pages(const PrefixArgs& a, int len) {
  const int n = (len + KVP - 1) / KVP;
  return a.q.window > 0 ? min(n, a.seen) : n;
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
  int len, n, c0, c1;
  PageList list;
  const int32_t* table;
  int lo;            // the first position that row row0 + lane sees
  int all_lo;        // and that all rows of the tile see
};

// Sums of v over the lanes up to this one: within sixteen by shifts of 1, 2, 4 and 8 (0x110 + n), then from lane 15 of each
// sixteen to the next (0x142), and from lane 31 to the upper half (0x143).
__device__ __forceinline__ int lanes_upto(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);
  return v;
}

// Every workgroup divides the work by itself, from the groups' lengths, a lane a group: the tiles' pages over the
// target of workgroups in shares of one size, so that long and short prefixes end together.  (In shares by the
// host's estimate of the longest prefix, 64 prefixes of 1024 - 16384 tokens, 16 beams each, took 67 us for 50.)
constexpr int PLAN = 4;   // groups of a lane: at most 64 PLAN groups in all

// Shares of a prefix that `pages` are counted for.
__device__ __forceinline__ int shares_of(const PrefixArgs& a, int pages, int chunk) {
  return min(a.splits, (pages + chunk - 1) / chunk);
}
// Workgroups for a group with T tiles and S shares; where there are tiles, of a multiple of eight pairs (share, head).
__device__ __forceinline__ int group_jobs(const PrefixArgs& a, int T, int S) {
  const int pairs = S * a.c.kv_heads;
  return (a.tiles > 1 ? (pairs + 7) / 8 * 8 : pairs) * T;
}

__device__ __forceinline__ bool prefix_job(const PrefixArgs& a, int cap, PrefixJob& j) {
  const int lane = threadIdx.x % WAVE, H = a.c.kv_heads, G = a.g.num_groups;
  Group my;
  int at = -1, x = 0, T = 0, S = 0, chunk = a.chunk;
  if (chunk == 0) {
    Group r[PLAN];
    int tiles[PLAN], pages[PLAN], most = 0;
    int64_t mine = 0;
#pragma unroll
    for (int e = 0; e < PLAN; ++e) {
      tiles[e] = pages[e] = 0;
      if (64 * e >= G) continue;
      r[e] = group_of(a, min(64 * e + lane, G - 1));
      if (64 * e + lane < G) {
        tiles[e] = (group_rows(a, r[e]) + cap - 1) / cap;
        pages[e] = group_pages(a, r[e].len);
        mine += int64_t(tiles[e]) * pages[e];
        if (tiles[e] > 0) most = max(most, pages[e]);
      }
    }
    // (all groups have fewer than 2^24 tiles of at most 2^20 + 1 pages)
    const int64_t sum = (int64_t(__builtin_amdgcn_readlane(lanes_upto(int(mine >> 24)), 63)) << 24) +
                        __builtin_amdgcn_readlane(lanes_upto(int(mine & 0xFFFFFF)), 63);
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) most = max(most, __shfl_xor(most, o, WAVE));
    most = __builtin_amdgcn_readfirstlane(most);
    // (a multiple of four: the waves of a workgroup take pages in turn)
    const int64_t each = (sum * H + a.target - 1) / a.target;
    chunk = (max(max(a.least, each < most ? int(each) : most), (most + a.splits - 1) / a.splits) + 3) / 4 * 4;
    if (a.fit) {   // larger until all run at once
      while (true) {
        int n = 0;
#pragma unroll
        for (int e = 0; e < PLAN; ++e) n += tiles[e] * shares_of(a, pages[e], chunk);
        n = __builtin_amdgcn_readlane(lanes_upto(n), 63);
        if (n * H <= a.target || chunk >= most) break;
        chunk += 4 + chunk / 128 * 4;
      }
    }
    int before = 0;
#pragma unroll
    for (int e = 0; e < PLAN; ++e) {
      if (64 * e >= G) continue;
      const int shares = shares_of(a, pages[e], chunk), n = group_jobs(a, tiles[e], shares);
      const int upto = before + lanes_upto(n);
      const uint64_t mine = __ballot(int(blockIdx.x) >= upto - n && int(blockIdx.x) < upto);
      if (mine) {
        const int l = __builtin_ctzll(mine);
        at = 64 * e + l;
        x = int(blockIdx.x) - __builtin_amdgcn_readlane(upto - n, l);
        T = __builtin_amdgcn_readlane(tiles[e], l);
        S = __builtin_amdgcn_readlane(shares, l);
        my.first = __builtin_amdgcn_readlane(r[e].first, l);
        my.n = __builtin_amdgcn_readlane(r[e].n, l);
        my.prefix = __builtin_amdgcn_readlane(r[e].prefix, l);
        my.len = __builtin_amdgcn_readlane(r[e].len, l);
        my.q0 = __builtin_amdgcn_readlane(int(r[e].q0), l);   // (below 2^31)
        my.nq = __builtin_amdgcn_readlane(int(r[e].nq), l);
      }
      before = __builtin_amdgcn_readlane(upto, 63);
    }
  } else {
    const int per = group_jobs(a, a.tiles, a.splits);
    at = int(blockIdx.x) / per;
    x = int(blockIdx.x) % per;
    my = group_of(a, min(at, G - 1));
    T = a.tiles;
    S = at < G ? shares_of(a, group_pages(a, my.len), chunk) : 0;   // (the grid may be larger)
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *a.plan = chunk;
  if (at < 0) return false;
  int tile = 0, pair = x;
  if (a.tiles > 1) {
    pair = x / (8 * T) * 8 + x % 8;
    tile = x / 8 % T;
  }
  j.split = pair / H;
  j.h = pair % H;
  if (j.split >= S) return false;
  j.s = my.prefix;
  j.G = a.q.heads / H;
  j.q0 = my.q0;
  j.rows = group_rows(a, my);
  j.row0 = tile * cap;
  if (j.row0 >= j.rows) return false;
  j.len = my.len;
  j.lo = j.all_lo = 0;
  int64_t first = 0;
  if (a.q.window > 0) {
    const int row = min(j.row0 + lane, min(j.row0 + cap, j.rows) - 1);
    const int64_t low = my.len + place_of(a, my, row / j.G) - a.q.window + 1;   // below 2^32 either way
    j.lo = low > 0 ? int(low < my.len ? low : my.len) : 0;
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
  j.c0 = min(j.n, j.split * chunk);
  j.c1 = j.split == S - 1 ? j.n : min(j.n, j.c0 + chunk);   // (more than its share where members are longer than estimated)
  if (j.c0 >= j.c1) {   // an empty share: a sum of zero and no features
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
  bool open;                       // the open block is among what is seen
  int64_t q0, first;               // its first query, and how far behind the prefix that stands
  int rows, row0, R;               // (query, head) pairs of the member; this tile's first, and how many are its
  int shares;                      // of the prefix
};
__device__ __forceinline__ int tile_sinks(const PrefixArgs& a, const OwnJob& j) { return j.sinks; }

// Member x of all groups' members together, from the groups' sizes, a lane a group.
__device__ __forceinline__ bool nth_member(const PrefixArgs& a, int x, int* group, int* member) {
  const int lane = threadIdx.x % WAVE, G = a.g.num_groups;
  int n[PLAN];
#pragma unroll
  for (int e = 0; e < PLAN; ++e) {
    n[e] = 0;
    if (64 * e + lane >= G) continue;
    const int first = a.g.offset[64 * e + lane], end = a.g.offset[64 * e + lane + 1];
    if (first >= 0 && first < end && end <= a.c.num_seqs) n[e] = min(end - first, a.g.max_members);
  }
  int before = 0;
#pragma unroll
  for (int e = 0; e < PLAN; ++e) {
    if (64 * e >= G) continue;
    const int upto = before + lanes_upto(n[e]);
    const uint64_t mine = __ballot(x >= upto - n[e] && x < upto);
    if (mine) {
      const int l = __builtin_ctzll(mine);
      *group = 64 * e + l;
      *member = x - __builtin_amdgcn_readlane(upto - n[e], l);
      return true;
    }
    before = __builtin_amdgcn_readlane(upto, 63);
  }
  return false;
}

// Job number b: (member, group, tile, head), the last one fastest: members that only some groups have come last.  Where
// groups differ so much that their largest sizes come to more than there are sequences, the members are counted instead:
// 12 groups of 3 - 64 members in 4 heads, 397 jobs: 1640 waves instead of nearly twice as many, 21.6 us for 27.
__device__ __forceinline__ bool own_job(const PrefixArgs& a, unsigned b, OwnJob& j) {
  const tav2_kv& c = a.c;
  j.h = int(b % c.kv_heads);
  b /= c.kv_heads;
  const int tile = int(b % a.own_tiles);
  b /= a.own_tiles;
  const int chunk = *a.plan;
  int group, member;
  if (a.count) {
    if (!nth_member(a, int(b), &group, &member)) return false;
  } else {
    member = int(b / a.g.num_groups);
    group = int(b % a.g.num_groups);
    if (member >= a.g.max_members) return false;
  }
  const Group r = group_of(a, group);
  j.s = r.first + min(member, r.n - 1 > 0 ? r.n - 1 : 0);
  j.G = a.q.heads / c.kv_heads;
  j.q0 = a.q.offset[j.s];
  j.len = kv_len(c, j.s);
  const int64_t most = a.most_rows / j.G;   // queries that the first launch took
  const int64_t nq = member_count(a, j.s);
  if (member >= r.n || j.q0 < r.q0 || j.q0 + nq > r.q0 + (r.nq < most ? r.nq : most)) return false;
  j.shares = shares_of(a, group_pages(a, r.len), chunk);
  j.rows = int(nq) * j.G;
  j.row0 = 16 * tile;
  if (j.row0 >= j.rows) return false;
  j.R = min(16, j.rows - j.row0);
  j.first = a.causal ? j.len - nq : j.len;
  const int64_t lo = a.causal ? j.first + j.row0 / j.G : j.first;
  const int64_t hi = a.causal ? j.first + (j.row0 + j.R - 1) / j.G : j.first;
  j.sinks = max(0, a.q.sinks - r.len);
  j.list = pages_seen(j.len, lo, hi, a.q.window, j.sinks);
  const int count = j.list.count();
  j.open = count > 0 && j.list.at(count - 1) >= j.len / KVP;
  j.c0 = 0;
  j.c1 = count - (j.open ? 1 : 0);
  j.table = c.table + int64_t(j.s) * c.max_blocks;
  return true;
}
__device__ __forceinline__ int64_t row_at(const PrefixArgs& a, const OwnJob& j, int row) {
  return (j.q0 + row / j.G) * a.q.heads + j.h * j.G + row % j.G;
}
__device__ __forceinline__ void row_seen(const PrefixArgs& a, const OwnJob& j, int row, int* hi, int* lo) {
  const int64_t pos = a.causal ? j.first + row / j.G : j.first, low = pos - a.q.window + 1;
  const int64_t end = pos + 1 < j.len ? pos + 1 : j.len;
  *hi = int(end > 0 ? end : 0);
  *lo = a.q.window > 0 && low > 0 ? int(low) : 0;
}

// A part of a row's softmax: reference, sum, and features 16 d + 4 g .. against it.
template <int D>
struct Part {
  float M, l;
  f32x4 x[D / 16];
  __device__ __forceinline__ void add(float M2, float l2, const f32x4 (&x2)[D / 16]) {
    const float all = vmax(M, M2), f = half_factor(M - all), f2 = half_factor(M2 - all);
    M = all;
    l = l * f * f + l2 * f2 * f2;
#pragma unroll
    for (int d = 0; d < D / 16; ++d)
#pragma unroll
      for (int e = 0; e < 4; ++e) x[d][e] = x[d][e] * f * f + x2[d][e] * f2 * f2;
  }
};

// An open block for the 16 rows of a wave (tiles as in Tile16), in bf16 as it lies: the scores' products are exact, the
// weights against the block's own largest score enter theirs as the sum of two bf16, 2^-16 of each.  A query's features
// are scaled by the power of two that takes the largest products to 2^20 or so, whatever the keys' size.
template <int D>
struct OpenBlock {
  static constexpr int F = D / 4, NK = D / 32, ND = D / 16;
  u32x4 k[4][NK], v[ND][2];

  // What lies behind the last token is not fetched: the first row and the first tokens stand in its place.
  __device__ __forceinline__ void load(const tav2_kv& c, int layer, int of, int h, int held) {
    const int m = int(threadIdx.x) % 16, g = int(threadIdx.x) % WAVE / 16, krow = Tile16<D>::key();
    const int64_t tail = kv_tail(c, layer, of, h);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bf16_t* const p = c.k_tail + tail + (krow + 4 * i < held ? krow + 4 * i : 0) * D + g * F;
#pragma unroll
      for (int t = 0; t < NK; ++t) k[i][t] = *reinterpret_cast<const u32x4*>(p + 8 * t);
    }
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const bf16_t* const p = c.v_tail + tail + m * KVP + (16 * g + 8 * t < held ? 16 * g + 8 * t : 0);
#pragma unroll
      for (int d = 0; d < ND; ++d) v[d][t] = *reinterpret_cast<const u32x4*>(p + 16 * d * KVP);
    }
  }

  // w: the row's query as it lies.  hi, lo, sinks: what it sees, counted from the block's first token.
  __device__ __forceinline__ void attend(const u32x4 (&w)[NK], const PrefixArgs& a, int held, int hi, int lo, int sinks,
                                         Part<D>& r) {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    const int g = int(threadIdx.x) % WAVE / 16;
    auto most = [](float a, float b) { return vmax(a, b); };
    // the largest magnitudes, as the upper bits of a float
    auto top_of = [&](const u32x4& x, u16x2 t) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        t = __builtin_elementwise_max(t, __builtin_bit_cast(u16x2, x[e] & 0x7FFF7FFFu));
      return t;
    };
    auto both = [](u16x2 t) { return __uint_as_float(uint32_t(t.x > t.y ? t.x : t.y) << 16); };
    u16x2 kt = {0, 0}, qt = {0, 0};
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < NK; ++t) kt = top_of(k[i][t], kt);
#pragma unroll
    for (int t = 0; t < NK; ++t) qt = top_of(w[t], qt);
    const int ek = __builtin_amdgcn_frexp_expf(xmax32(xmax16(steps16(both(kt), 1, most))));
    const int eq = __builtin_amdgcn_frexp_expf(xmax32(xmax16(both(qt))));
    const int to = min(20 - ek, 120);          // the queries' exponent
    bf16x8 q[NK];
#pragma unroll
    for (int t = 0; t < NK; ++t) {
      uint32_t y[4];
#pragma unroll
      for (int e = 0; e < 4; ++e)
        y[e] = pack2(__builtin_amdgcn_ldexpf(__uint_as_float(w[t][e] << 16), to - eq),
                     __builtin_amdgcn_ldexpf(__uint_as_float(w[t][e] & 0xFFFF0000u), to - eq));
      q[t] = as_bf16x8(make_uint4(y[0], y[1], y[2], y[3]));
    }
    f32x4 s[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      s[i] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < NK; ++t)
        s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, k[i][t]), q[t], s[i], 0, 0, 0);
    }
    const float cs = score_factor(a.scale, a.scale_e + eq - to);
    const int k0 = 16 * g, hi_ = min(hi, held) - k0, lo_ = lo - k0, sinks_ = sinks - k0;
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      s[i / 4][i % 4] = i < hi_ && (i >= lo_ || i < sinks_) ? s[i / 4][i % 4] : -INFINITY;
      top = vmax(top, s[i / 4][i % 4]);
    }
    const float raw = xmax32(xmax16(top));
    top = att_top(raw, cs);
    const bool some = top > -INFINITY;
    // a whole number as the reference, as everywhere
    r.M = some ? __builtin_floorf(top) : -FLT_MAX;
    float b = some ? -r.M : 0.f;
    if (att_any_far(r.M)) {   // (large scores: as in attend_core.h)
      const bool far = att_far(r.M);
      const float own = att_own(far, raw);
      b = far ? top - r.M : b;
#pragma unroll
      for (int i = 0; i < 16; ++i) s[i / 4][i % 4] -= own;
    }
    float sum = 0.f;
    uint32_t ph[8], pl[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 2][2 * i % 4], cs, b));
      const float y = __builtin_amdgcn_exp2f(__builtin_fmaf(s[i / 2][2 * i % 4 + 1], cs, b));
      sum += x;
      sum += y;
      ph[i] = pack2(x, y);
      pl[i] = pack2(x - __uint_as_float(ph[i] << 16), y - __uint_as_float(ph[i] & 0xFFFF0000u));
    }
    r.l = xsum32(xsum16(sum));
    // the tokens behind the last one, of the piece that it lies in (and of those that the first one stands in for)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if (held % 8 == 0 || (held > 8 && held / 8 % 2 != t)) continue;
      const int start = 16 * g + 8 * t, n = start < held ? held - start : held < 8 ? 0 : 8;
#pragma unroll
      for (int d = 0; d < ND; ++d) v[d][t] = first_of8(v[d][t], n);
    }
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      r.x[d] = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const bf16x8 vv = __builtin_bit_cast(bf16x8, v[d][t]);
        r.x[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            vv, as_bf16x8(make_uint4(ph[4 * t], ph[4 * t + 1], ph[4 * t + 2], ph[4 * t + 3])), r.x[d], 0, 0, 0);
        r.x[d] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
            vv, as_bf16x8(make_uint4(pl[4 * t], pl[4 * t + 1], pl[4 * t + 2], pl[4 * t + 3])), r.x[d], 0, 0, 0);
      }
    }
  }
};

// The prefix's shares and the own tokens of a job, by one wave, through no LDS, so that as many as registers allow are on
// the way (the launch is a chain of dependent reads), or, where jobs are few or long, by the four of a workgroup: the
// first takes the open block, the others the shares, all of them the pages.  Rows fewer than 16 are repeated over
// the tile, and the repetitions take the shares in turn.
template <int D, int WAVES>
__global__ __launch_bounds__(256, 2) void kv_join_kernel(PrefixArgs a) {
  using T = Tile16<D>;
  constexpr int ND = T::ND, NK = T::NK, KL = D == 128 ? 2 : 1;   // loads of a key's quarter
  const tav2_kv& c = a.c;
  OwnJob j;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  if (!own_job(a, WAVES == 1 ? blockIdx.x * 4 + wave : blockIdx.x, j)) return;
  const int lane = threadIdx.x % WAVE, m = lane % 16, g = lane / 16;
  const int Rp = j.R <= 1 ? 1 : j.R <= 2 ? 2 : j.R <= 4 ? 4 : j.R <= 8 ? 8 : 16;
  const int row = j.row0 + min(m % Rp, j.R - 1);
  const int64_t at = row_at(a, j, row), n = a.q.total * a.q.heads;
  const bf16_t* const q = static_cast<const bf16_t*>(a.q.q) + (j.q0 + row / j.G) * a.q.ld + (j.h * j.G + row % j.G) * D;

  // the open block and the queries are on the way while the prefix's shares are joined (by this wave; where others do
  // that, no registers are held for both)
  const int full = j.len / KVP, held = j.open && (WAVES == 1 || wave == 0) ? j.len - full * KVP : 0;
  OpenBlock<D> open;
  u32x4 w[NK];
  auto fetch = [&]() {
    open.load(c, a.layer, j.s, j.h, held);
#pragma unroll
    for (int t = 0; t < NK; ++t) w[t] = *reinterpret_cast<const u32x4*>(q + g * (D / 4) + 8 * t);
  };
  if (WAVES == 1 && held > 0) fetch();
  int hi, lo;
  row_seen(a, j, row, &hi, &lo);

  // the prefix: references, sums, features
  auto most = [](float a, float b) { return vmax(a, b); };
  auto plus = [](float a, float b) { return a + b; };
  const float2* const ml = reinterpret_cast<const float2*>(a.part_ml) + at;
  Part<D> r;
  r.M = -FLT_MAX;
  r.l = 0.f;
  const bool takes = WAVES == 1 || wave > 0;   // shares, in turn with the other waves that do
  const int turns = WAVES == 1 ? 1 : WAVES - 1, turn = WAVES > 1 && takes ? wave - 1 : 0;
  const int shares = takes ? j.shares : 0, reps = 16 / Rp;
  for (int s = (m / Rp + reps * g) * turns + turn; s < shares; s += 4 * reps * turns) {   // (one, but for very long prefixes)
    const float2 x = ml[s * n];
    const float top = vmax(r.M, x.x), f = half_factor(x.x - top), of = half_factor(r.M - top);
    r.l = r.l * of * of + x.y * f * f;
    r.M = top;
  }
  {
    const float top = xmax32(xmax16(steps16(r.M, Rp, most))), f = half_factor(r.M - top);
    r.l = xsum32(xsum16(steps16(r.l * f * f, Rp, plus)));
    r.M = top;
  }
#pragma unroll
  for (int d = 0; d < ND; ++d) r.x[d] = (f32x4){0.f, 0.f, 0.f, 0.f};
  // (N shares at once, as their loads are what takes the time; past the last one it is read again and dropped)
  auto join = [&](int s0, auto count) {
    constexpr int N = decltype(count)::value;
    float2 x[N];
    f32x4 v[N][ND];
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const int s = s0 + u * reps * turns;
      const int64_t i = min(s, shares - 1) * n;
      x[u] = ml[i];
      if (s >= shares) x[u].y = 0.f;
      const f32x4* const o = reinterpret_cast<const f32x4*>(a.part_o + (i + at) * D) + g;
#pragma unroll
      for (int d = 0; d < ND; ++d) v[u][d] = o[4 * d];   // (an empty share's are not written: read all the same, and dropped)
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const float f = half_factor(x[u].x - r.M);
#pragma unroll
      for (int d = 0; d < ND; ++d)
#pragma unroll
        for (int e = 0; e < 4; ++e) r.x[d][e] += x[u].y != 0.f ? v[u][d][e] * f * f : 0.f;
    }
  };
  constexpr int MOST = WAVES == 1 ? 1 : D <= 64 ? 4 : 2;
  const int step = reps * turns;
  int s0 = m / Rp * turns + turn;
  for (int left = (shares + step - 1) / step; left > 0; left -= MOST, s0 += MOST * step) {
    if (left > 1) join(s0, std::integral_constant<int, MOST>{});
    else join(s0, std::integral_constant<int, 1>{});
  }
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int e = 0; e < 4; ++e) r.x[d][e] = steps16(r.x[d][e], Rp, plus);

  // the own tokens: the open block, then pages as they lie
  if (held > 0) {
    if (WAVES > 1) fetch();
    Part<D> own;
    open.attend(w, a, held, hi - full * KVP, lo - full * KVP, j.sinks - full * KVP, own);
    r.add(own.M, own.l, own.x);
  }
  if (j.c1 > 0) {
    T st;
    st.sees(hi, lo, j.sinks);
    st.query(q, a.scale_e);
    st.clear();
    const int krow = T::key();
    for (int i = WAVES == 1 ? 0 : wave; i < j.c1; i += WAVES) {
      const int b = j.list.at(i), page = __builtin_amdgcn_readfirstlane(j.table[b]);
      if (page < 0 || page >= c.pages) continue;
      const int64_t unit = kv_unit(c, a.layer, page, j.h);
      const float ks = c.k_scale[unit], vs = c.v_scale[unit];
      const int8_t* const kp = c.k + unit * KVP * D;
      const int8_t* const vp = c.v + unit * KVP * D;
      u32x4 kc[4][KL], vc[ND];
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        if constexpr (D == 32) {
          const uint2 x = *reinterpret_cast<const uint2*>(kp + (krow + 4 * t) * D + g * 8);
          kc[t][0] = (u32x4){x.x, x.y, 0, 0};
        } else {
#pragma unroll
          for (int u = 0; u < KL; ++u)
            kc[t][u] = *reinterpret_cast<const u32x4*>(kp + (krow + 4 * t) * D + g * (D / 4) + 16 * u);
        }
      }
      uint32_t any = 0;
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        vc[d] = *reinterpret_cast<const u32x4*>(vp + (16 * d + m) * KVP + 16 * g);
        any |= vc[d].x | vc[d].y | vc[d].z | vc[d].w;
      }
      AttScale v{__builtin_amdgcn_logf(vs), __builtin_amdgcn_rcpf(vs)};
      if (v.lv == 0.f && !__any(any != 0)) v.lv = -INFINITY;   // a block of zeros, whose scale counts as none
      auto keys = [&](int t, f16x8(&kf)[NK]) {
#pragma unroll
        for (int u = 0; u < NK; ++u)
          kf[u] = u % 2 ? codes8h(kc[t][u / 2].z, kc[t][u / 2].w) : codes8h(kc[t][u / 2].x, kc[t][u / 2].y);
      };
      auto values = [&](int d, f16x8(&vf)[2]) {
        vf[0] = codes8h(vc[d].x, vc[d].y);
        vf[1] = codes8h(vc[d].z, vc[d].w);
      };
      st.step(keys, values, score_factor(a.scale * ks, st.cq), v, b * KVP, hi);
    }
#pragma unroll
    for (int d = 0; d < ND; ++d) st.o[d] *= st.ratio;
    r.add(st.wref, xsum32(xsum16(st.sum)), st.o);
  }

  if constexpr (WAVES > 1) {   // the first wave joins the others', in their order
    __shared__ Part<D> parts[WAVES - 1][WAVE];
    if (wave > 0) parts[wave - 1][lane] = r;
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 0; w < WAVES - 1; ++w) r.add(parts[w][lane].M, parts[w][lane].l, parts[w][lane].x);
  }
  if (m >= j.R) return;
  const bool some = r.l > 0.f || r.l != r.l;
  const float inv = some ? 1.f / r.l : 0.f;
#pragma unroll
  for (int d = 0; d < ND; ++d)
    *reinterpret_cast<uint2*>(a.out + at * D + 16 * d + 4 * g) =
        make_uint2(pack2(r.x[d][0] * inv, r.x[d][1] * inv), pack2(r.x[d][2] * inv, r.x[d][3] * inv));
  if (g == 0 && a.lse) a.lse[at] = some ? (r.M + __builtin_amdgcn_logf(r.l)) * LN2 : -INFINITY;
}

constexpr size_t PLAN_BYTES = 256;   // before the parts

int64_t own_tiles(const tav2_kv& c, const tav2_kv_queries& q) {
  return cdiv(int64_t(q.max_count) * (q.heads / c.kv_heads), 16);
}
bool count_members(const tav2_kv& c, const tav2_kv_groups& g) {
  return g.num_groups <= WAVE * PLAN && c.num_seqs < int64_t(g.num_groups) * g.max_members;
}
double own_jobs(const tav2_kv& c, const tav2_kv_groups& g, const tav2_kv_queries& q) {
  const double members = count_members(c, g) ? c.num_seqs : double(g.num_groups) * g.max_members;
  return members * c.kv_heads * double(own_tiles(c, q));
}
// Whether a job is a workgroup's work instead of a wave's: few of them (32 jobs 14.7 us for 18.4, 2048 jobs 67.8 for 64.7), or
// of many pages (8 groups of 16 members with 500 - 2000 tokens 33.2 us for 63.3).
bool join_by_four(const tav2_kv& c, const tav2_kv_groups& g, const tav2_kv_queries& q) {
  return g.max_own > 512 || own_jobs(c, g, q) <= 1024;
}
int pow2_from(int64_t n) {   // the least power of two from n on, up to 16
  int p = 1;
  while (p < 16 && p < n) p *= 2;
  return p;
}

// How the work on the prefixes is divided.
struct Plan {
  int64_t rows;        // of a group and kv head
  int64_t pages;       // that a tile of the longest prefix sees, by the host's estimate
  int64_t grid;
  int tile, tiles, chunk, least, target, splits;
  bool fit;
};
Plan plan_of(const tav2_kv& c, const tav2_kv_groups& g, const tav2_kv_queries& q) {
  Plan p;
  const int G = q.heads / c.kv_heads;
  p.rows = std::min<int64_t>(q.total, int64_t(g.max_members) * q.max_count) * G;
  int64_t tokens = std::min<int64_t>(c.max_len, int64_t(c.max_blocks) * KVP + KVP - 1);
  if (q.window > 0)
    tokens = std::min(tokens, int64_t(q.window) + g.max_own + q.sinks + 2 * KVP);
  p.pages = std::max<int64_t>(1, cdiv(tokens, KVP));
  // Rows of a tile.  64, which read and turn a page once for twice as many, where there are enough pairs of such a tile and a
  // page: groups of 64 rows over 1024 - 16384 tokens, 16 of them (8224 pairs) 30.7 us for 27.6 with 32, 32 of them 42.1
  // for 54.4, 64 of them with 32 features 45.9 for 82.8.
  const double work = double(g.num_groups) * c.kv_heads * cdiv(p.rows, 64) * p.pages;
  p.tile = p.rows <= 16 ? 16
           : p.rows > 48 && c.head_dim <= 64 && work > 12000 ? 64 : 32;
  p.tiles = int(cdiv(p.rows, p.tile));
  // (a product with the pages is below 2^51; more units than 2^30 are refused as too many workgroups)
  const int64_t units = std::min(int64_t(g.num_groups) * c.kv_heads * p.tiles, int64_t(1) << 30);
  // Workgroups: all at once where few tiles' shares can be made larger until they are (48 groups of 64 rows, 96 units: 54.7 us
  // for 70.7), and in turn where a unit would be left whole (32 groups of 256 rows, 256 units: 122 for 177).  What runs at once
  // is two a CU, a little fewer with 32 rows: 64 groups 64.9 us with 512, 70.5 with 448, 75.9 with 768; 16 groups
  // in tiles of 32 27.6 with 448, 32.9 with 512, 33.9 with 256.
  p.fit = units <= 192;
  // A page more for each wave takes about as long as the join of as many shares as it takes at once (0.9 and 0.5 us): shares
  // are of at least the pages for which both come to the least.  (16 rows of one group, 16384 tokens: 4 pages 16.5 us, 8
  // 15.4, 16 16.6; 65536 tokens: 4 - 12 pages 22.7, 16 20.3.)
  const int together = 16 / pow2_from(int64_t(q.max_count) * G) * (join_by_four(c, g, q) ? 3 : 1);
  p.least = int(cdiv(int64_t(sqrt(2.2 / (p.tile == 64 ? 2 : 1) * double(p.pages) / together)), 4)) * 4;
  p.least = std::max(p.least, 4);
  p.target = !p.fit ? 1024 : p.tile == 64 ? 512 : 448;
  // prefixes are a quarter of the longest at least, on average, or shares are larger than they might be
  const bool planned = g.num_groups <= WAVE * PLAN;
  const int64_t chunk = std::max<int64_t>(p.least, cdiv(units * p.pages, (planned ? 4 : 2) * p.target));
  p.chunk = planned ? 0 : int(std::min(chunk, p.pages));
  p.splits = int(cdiv(p.pages, chunk));
  const int64_t pads = p.tiles > 1 ? 8 * int64_t(p.tiles) : 0;
  p.grid = planned ? p.target + units + g.num_groups * pads
                   : g.num_groups * (int64_t(p.splits) * c.kv_heads * p.tiles + pads);
  return p;
}
}  // namespace

// (their product may pass 64 bits)
double kv_prefix_workgroups(const tav2_kv& c, const tav2_kv_groups& g, const tav2_kv_queries& q) {
  const Plan p = plan_of(c, g, q);
  return std::max(double(p.grid), own_jobs(c, g, q));
}

size_t kv_prefix_bytes(const tav2_kv& c, const tav2_kv_groups& g, const tav2_kv_queries& q) {
  const Plan p = plan_of(c, g, q);
  return PLAN_BYTES + align_up(size_t(p.splits) * size_t(q.total) * q.heads * (c.head_dim + 2) * 4, 256);
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
  a.plan = static_cast<int32_t*>(ws);
  a.part_o = reinterpret_cast<float*>(static_cast<char*>(ws) + PLAN_BYTES);
  a.part_ml = a.part_o + size_t(p.splits) * q.total * q.heads * c.head_dim;
  a.most_rows = int(p.rows);
  a.tile = p.tile;
  a.tiles = p.tiles;
  a.splits = p.splits;
  a.chunk = p.chunk;
  a.least = p.least;
  a.target = p.target;
  a.fit = p.fit;
  a.seen = int(p.pages);
  a.own_tiles = int(own_tiles(c, q));
  a.count = count_members(c, g);
  {
    ProfScope prof("kv_prefix", st);
    const unsigned grid = unsigned(p.grid);
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
  const unsigned grid = unsigned(own_jobs(c, g, q));
  if (join_by_four(c, g, q)) {
    if (c.head_dim == 32) kv_join_kernel<32, 4><<<grid, 256, 0, st>>>(a);
    else if (c.head_dim == 64) kv_join_kernel<64, 4><<<grid, 256, 0, st>>>(a);
    else kv_join_kernel<128, 4><<<grid, 256, 0, st>>>(a);
  } else {
    const unsigned n = (grid + 3) / 4;
    if (c.head_dim == 32) kv_join_kernel<32, 1><<<n, 256, 0, st>>>(a);
    else if (c.head_dim == 64) kv_join_kernel<64, 1><<<n, 256, 0, st>>>(a);
    else kv_join_kernel<128, 1><<<n, 256, 0, st>>>(a);
  }
  return hipGetLastError();
}

}  // namespace tav2
