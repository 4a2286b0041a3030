// Reordering of the cache's sequences after beams were selected: members of a group continue one another.
//
// Every member's new state is another's old one, in any order (cycles among them), in place.  The moves of one
// place in a tail or one column of the tables depend only on that place in the group's other
// members, so a workgroup takes the same places of all members of a group: it loads what they are to become into
// registers, waits, and stores.  Nothing is copied aside and a byte is read and written once.
// The counts change by atomics on integers (any order).  The lengths, which the first launch reads, are
// written by a second one.
#include <algorithm>

#include "common.h"
#include "internal.h"
#include "kv_common.h"

namespace tav2 {

namespace {

constexpr int NT = 256;      // threads
constexpr int ONE = 1024;    // where one workgroup takes a group whole
constexpr int HOLD = 8;      // pieces that a thread holds
constexpr int TABLES = 4;    // workgroups a group for the tables

struct Group {
  int first, n, m0;   // its first sequence, members, and the first one's number in parent
};
__device__ __forceinline__ bool group_of(const tav2_kv& c, const tav2_kv_groups& g, int i, Group& r) {
  r.first = g.offset[i];
  const int end = g.offset[i + 1], zero = g.offset[0];
  if (r.first < 0 || end > c.num_seqs || r.first >= end || zero < 0 || zero > r.first) return false;
  r.n = min(end - r.first, g.max_members);
  r.m0 = r.first - zero;
  return true;
}

// What member i continues: itself, another member, or nothing (-1).
__device__ __forceinline__ int source_of(const Group& r, const int32_t* parent, int members, int i) {
  if (r.m0 + i >= members) return i;
  const int p = parent[r.m0 + i];
  return p < 0 ? -1 : p >= r.n ? i : p;
}

// A group's members that change: their places in the group, what they continue (-1: nothing), and the tokens that
// it and they have; alike for all threads after build().
struct Moves {
  int who[TAV2_BEAMS_MAX], from[TAV2_BEAMS_MAX], held[TAV2_BEAMS_MAX], had[TAV2_BEAMS_MAX];
  int n, tokens, blocks;   // how many; the most tokens in an open block that is taken over, and table entries that change
  // (threads: all of the workgroup's.  Members that continue one without an open block are left out where only tails are
  // asked for.)
  __device__ __forceinline__ void build(const tav2_kv& c, const Group& r, const int32_t* parent, int members, int threads,
                                        bool tails) {
    if (threadIdx.x == 0) n = tokens = blocks = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < r.n; i += threads) {
      const int p = source_of(r, parent, members, i);
      if (p == i) continue;
      const int len = p < 0 ? 0 : kv_len(c, r.first + p), old = kv_len(c, r.first + i);
      if (tails && len % KVP == 0) continue;
      const int k = atomicAdd(&n, 1);   // (the order does not matter)
      who[k] = i;
      from[k] = p;
      held[k] = len;
      had[k] = old;
      atomicMax(&tokens, len % KVP);
      atomicMax(&blocks, max(len, old) / KVP);
    }
    __syncthreads();
  }
};

// Places of a tail are 16-byte pieces, the same ones for all members: keys lie by token, values by feature (as many pieces
// of each as the longest open block has).
struct Pieces {
  int D, wide, inverse, keys, values;
  __device__ __forceinline__ Pieces(int D_, int tokens)
      : D(D_), wide((tokens + 7) / 8), inverse(65536 / max(wide, 1) + 1), keys(tokens * (D_ / 8)), values(D_ * wide) {}
  // The first element of key or value piece x, and how many of its eight a member with t tokens takes over.
  __device__ __forceinline__ int key(int x, int t, int* n) const {
    *n = x < t * (D / 8) ? 8 : 0;
    return x * 8;
  }
  __device__ __forceinline__ int value(int x, int t, int* n) const {
    const int f = x * inverse >> 16, part = x - f * wide;   // x / wide: exact below 2^13
    *n = min(8, t - 8 * part);
    return f * KVP + 8 * part;
  }
};

// n elements of v: where fewer than eight, what lies behind them stays.
__device__ __forceinline__ void put_piece(uint16_t* to, const uint4& v, int n) {
  if (n == 8) {
    *reinterpret_cast<uint4*>(to) = v;
    return;
  }
  uint2 w = make_uint2(v.x, v.y);
  if (n & 4) {
    *reinterpret_cast<uint2*>(to) = w;
    to += 4;
    w = make_uint2(v.z, v.w);
  }
  if (n & 2) {
    *reinterpret_cast<uint32_t*>(to) = w.x;
    to += 2;
    w.x = w.y;
  }
  if (n & 1) *to = uint16_t(w.x);
}

// Table entries: HOLD each of `threads` threads at once, from block `first` of every `step` on, and the pages' counts.
__device__ __forceinline__ void move_tables(const tav2_kv& c, const Group& r, const Moves& m, int threads, int shift,
                                            int first, int step) {
  // (place x of all: entry x % 2^shift of member x >> shift)
  const int mask = (1 << shift) - 1;
  for (int b0 = first; b0 < m.blocks; b0 += step) {
    int now[HOLD], was[HOLD];
#pragma unroll
    for (int e = 0; e < HOLD; ++e) {
      const int x = int(threadIdx.x) + e * threads, k = x >> shift, b = b0 + (x & mask);
      now[e] = was[e] = -1;
      if (k >= m.n) continue;
      if (b < m.held[k] / KVP) now[e] = c.table[int64_t(r.first + m.from[k]) * c.max_blocks + b];
      if (b < m.had[k] / KVP) was[e] = c.table[int64_t(r.first + m.who[k]) * c.max_blocks + b];
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < HOLD; ++e) {
      if (now[e] == was[e]) continue;
      const int x = int(threadIdx.x) + e * threads;
      c.table[int64_t(r.first + m.who[x >> shift]) * c.max_blocks + b0 + (x & mask)] = now[e];
      if (now[e] >= 0 && now[e] < c.pages) atomicAdd(c.refs + now[e], 1);
      if (was[e] >= 0 && was[e] < c.pages) atomicSub(c.refs + was[e], 1);
    }
  }
}
// The places of a member that are taken at once, as a power of two.
__device__ __forceinline__ int places_shift(int members, int threads) {
  return 31 - __builtin_clz(threads * HOLD / members);
}

// blockIdx.y: a group.  blockIdx.x: a (layer, head, side) of the tails, and then the tables' share.  blockIdx.z: where the
// others are few, a share of the places.
__global__ __launch_bounds__(NT) void kv_reorder_kernel(tav2_kv c, tav2_kv_groups g,
                                                        const int32_t* __restrict__ parent, int members) {
  __shared__ Moves m;
  Group r;
  if (!group_of(c, g, blockIdx.y, r)) return;
  const int tid = threadIdx.x, D = c.head_dim, H = c.kv_heads;
  const int part = blockIdx.x, tails = 2 * c.layers * H;
  m.build(c, r, parent, members, NT, part < tails);
  if (m.n == 0) return;
  const int shift = places_shift(m.n, NT), per = 1 << shift;
  if (part >= tails) {
    if (blockIdx.z == 0) move_tables(c, r, m, NT, shift, (part - tails) * per, per * TABLES);
    return;
  }
  const bool values = part % 2;
  const int layer = part / 2 / H, h = part / 2 % H;
  uint16_t* const base = (values ? c.v_tail : c.k_tail) + kv_tail(c, layer, r.first, h);
  const int64_t seq = int64_t(H) * KVP * D;   // elements from a sequence's tail to the next one's
  const Pieces pieces(D, m.tokens);
  const int most = values ? pieces.values : pieces.keys;
  for (int b0 = int(blockIdx.z) * per; b0 < most; b0 += per * int(gridDim.z)) {
    uint4 v[HOLD];
    uint16_t* to[HOLD];
    int n[HOLD];
#pragma unroll
    for (int e = 0; e < HOLD; ++e) {
      const int x = tid + e * NT, k = x >> shift, place = b0 + (x & (per - 1));
      n[e] = 0;
      if (k >= m.n || place >= most) continue;
      const int t = m.held[k] % KVP, at = values ? pieces.value(place, t, &n[e]) : pieces.key(place, t, &n[e]);
      to[e] = base + m.who[k] * seq + at;
      if (n[e] > 0) v[e] = *reinterpret_cast<const uint4*>(base + m.from[k] * seq + at);
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < HOLD; ++e)
      if (n[e] > 0) put_piece(to[e], v[e], n[e]);
  }
}

// Groups with little to move: a workgroup a group takes all layers, the tables, and at last the lengths, in one launch.
// The members of a place are neighbouring threads, so that a step never divides them.
__global__ __launch_bounds__(ONE) void kv_reorder_small_kernel(tav2_kv c, tav2_kv_groups g,
                                                              const int32_t* __restrict__ parent, int members) {
  __shared__ Moves m;
  Group r;
  if (!group_of(c, g, blockIdx.x, r)) return;
  m.build(c, r, parent, members, ONE, false);
  if (m.n == 0) return;
  const int tid = threadIdx.x, D = c.head_dim, H = c.kv_heads;
  const int64_t seq = int64_t(H) * KVP * D;
  const Pieces pieces(D, m.tokens);
  const int shift = m.n > 1 ? 32 - __builtin_clz(m.n - 1) : 0;   // members, as a power of two
  const int per = pieces.keys + pieces.values, places = c.layers * H * per;
  if (per > 0)
    for (int x0 = 0; x0 < places << shift; x0 += ONE * HOLD) {
      uint4 v[HOLD];
      uint16_t* to[HOLD];
      int n[HOLD];
#pragma unroll
      for (int e = 0; e < HOLD; ++e) {
        const int x = x0 + tid + e * ONE, k = x & ((1 << shift) - 1), place = x >> shift;
        n[e] = 0;
        if (k >= m.n || place >= places) continue;
        const int unit = place / per, y = place % per, t = m.held[k] % KVP;
        const bool keys = y < pieces.keys;
        const int at = keys ? pieces.key(y, t, &n[e]) : pieces.value(y - pieces.keys, t, &n[e]);
        uint16_t* const base = (keys ? c.k_tail : c.v_tail) + kv_tail(c, unit / H, r.first, unit % H);
        to[e] = base + m.who[k] * seq + at;
        if (n[e] > 0) v[e] = *reinterpret_cast<const uint4*>(base + m.from[k] * seq + at);
      }
      __syncthreads();
#pragma unroll
      for (int e = 0; e < HOLD; ++e)
        if (n[e] > 0) put_piece(to[e], v[e], n[e]);
    }
  const int fit = places_shift(m.n, ONE);
  move_tables(c, r, m, ONE, fit, 0, 1 << fit);
  // (every thread has read the lengths: in build())
  for (int k = tid; k < m.n; k += ONE) {
    c.len[r.first + m.who[k]] = m.held[k];
    c.fresh[r.first + m.who[k]] = 0;
  }
}

// The lengths, a workgroup a group.
__global__ __launch_bounds__(NT) void kv_reorder_lengths(tav2_kv c, tav2_kv_groups g,
                                                         const int32_t* __restrict__ parent, int members) {
  constexpr int EACH = TAV2_BEAMS_MAX / NT;
  Group r;
  if (!group_of(c, g, blockIdx.x, r)) return;
  int len[EACH];
  bool move[EACH];
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const int i = int(threadIdx.x) + e * NT;
    move[e] = false;
    if (i >= r.n) continue;
    const int p = source_of(r, parent, members, i);
    move[e] = p != i;
    len[e] = p < 0 ? 0 : kv_len(c, r.first + p);
  }
  __syncthreads();
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    if (!move[e]) continue;
    const int s = r.first + int(threadIdx.x) + e * NT;
    c.len[s] = len[e];
    c.fresh[s] = 0;
  }
}

}  // namespace

int64_t kv_reorder_parts(const tav2_kv& c) { return 2 * int64_t(c.layers) * c.kv_heads + TABLES; }

hipError_t launch_kv_reorder(const tav2_kv& c, const tav2_kv_groups& g, const int32_t* parent, int members,
                             hipStream_t st) {
  static_assert(TAV2_BEAMS_MAX % NT == 0 && TAV2_BEAMS_MAX <= NT * HOLD, "a place of every member at once");
  ProfScope prof("kv_reorder", st);
  // Pieces of a group, by the host's estimate of its members' tokens.  One group of 8, 64 features: 4 (layer, head) pairs with 4
  // tokens (4096) 5.5 us for 9.5 with two launches, 16 pairs with 3 tokens (14336) 14.2 for 11.4: one workgroup's scattered
  // pieces then take longer than a launch.
  const int64_t pieces = int64_t(g.max_members) * c.layers * c.kv_heads * (std::min<int>(g.max_own, KVP - 1) + 4) * c.head_dim / 4;
  if (pieces <= 6144) {
    kv_reorder_small_kernel<<<unsigned(g.num_groups), ONE, 0, st>>>(c, g, parent, members);
    return hipGetLastError();
  }
  const int64_t groups = kv_reorder_parts(c) * g.num_groups;
  const unsigned z = unsigned(std::max<int64_t>(1, std::min<int64_t>(8, 1024 / groups)));
  kv_reorder_kernel<<<dim3(unsigned(kv_reorder_parts(c)), unsigned(g.num_groups), z), NT, 0, st>>>(c, g, parent,
                                                                                                members);
  kv_reorder_lengths<<<unsigned(g.num_groups), NT, 0, st>>>(c, g, parent, members);
  return hipGetLastError();
}

}  // namespace tav2
