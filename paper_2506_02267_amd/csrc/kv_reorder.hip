// Reordering of the cache's sequences after beams were selected: members of a group continue one another.
//
// Every member's new state is another's old one, in any order (cycles among them), in place.  The moves of one
// place in a tail or one column of the tables depend only on that place in the group's other
// members, so a workgroup takes the same places of all members of a group: it loads what they are to become into
// registers, waits, and stores.  Nothing is copied aside and a byte is read and written once.
// The counts change by atomics on integers (any order).  The lengths, which the first launch reads, are
// written by a second one.
#include "common.h"
#include "internal.h"
#include "kv_common.h"

namespace tav2 {

namespace {

constexpr int NT = 256;      // threads
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

// blockIdx.y: a group.  blockIdx.x: a (layer, head, side) of the tails, and then the tables' share.
__global__ __launch_bounds__(NT) void kv_reorder_kernel(tav2_kv c, tav2_kv_groups g,
                                                        const int32_t* __restrict__ parent, int members) {
  __shared__ int who[TAV2_BEAMS_MAX], from[TAV2_BEAMS_MAX], held[TAV2_BEAMS_MAX], had[TAV2_BEAMS_MAX];
  __shared__ int moved, most;
  Group r;
  if (!group_of(c, g, blockIdx.y, r)) return;
  const int tid = threadIdx.x, D = c.head_dim, H = c.kv_heads;
  const int part = blockIdx.x, tails = 2 * c.layers * H;
  const bool table = part >= tails;
  const int side = part % 2;
  if (tid == 0) moved = most = 0;
  __syncthreads();
  for (int i = tid; i < r.n; i += NT) {
    const int p = source_of(r, parent, members, i);
    if (p == i) continue;
    const int len = p < 0 ? 0 : kv_len(c, r.first + p), old = kv_len(c, r.first + i);
    int n;
    if (table) {
      n = max(len, old) / KVP;
    } else {
      n = len % KVP;
    }
    if (n == 0) continue;
    const int k = atomicAdd(&moved, 1);   // (the order does not matter)
    who[k] = i;
    from[k] = p;
    held[k] = len;
    had[k] = old;
    atomicMax(&most, n);
  }
  __syncthreads();
  const int M = moved;
  if (M == 0) return;
  const int per = NT * HOLD / M;   // places of a member that are taken at once
  if (table) {
    const int step = per * TABLES;
    for (int b0 = (part - tails) * per; b0 < most; b0 += step) {
      int now[HOLD], was[HOLD];
#pragma unroll
      for (int e = 0; e < HOLD; ++e) {
        const int x = tid + e * NT, k = x / per, b = b0 + x % per;
        now[e] = was[e] = -1;
        if (k >= M) continue;
        if (b < held[k] / KVP) now[e] = c.table[int64_t(r.first + from[k]) * c.max_blocks + b];
        if (b < had[k] / KVP) was[e] = c.table[int64_t(r.first + who[k]) * c.max_blocks + b];
      }
      __syncthreads();
#pragma unroll
      for (int e = 0; e < HOLD; ++e) {
        if (now[e] == was[e]) continue;
        const int x = tid + e * NT;
        c.table[int64_t(r.first + who[x / per]) * c.max_blocks + b0 + x % per] = now[e];
        if (now[e] >= 0 && now[e] < c.pages) atomicAdd(c.refs + now[e], 1);
        if (was[e] >= 0 && was[e] < c.pages) atomicSub(c.refs + was[e], 1);
      }
    }
    return;
  }
  const int layer = part / 2 / H, h = part / 2 % H;
  uint16_t* const base = (side == 0 ? c.k_tail : c.v_tail) + kv_tail(c, layer, r.first, h);
  const int64_t seq = int64_t(H) * KVP * D;   // elements from a sequence's tail to the next one's
  // Places are 16-byte pieces, the same ones for all members: keys lie by token, values by feature (wide pieces
  // of each).  A piece's first element, and how many of its eight member k takes over.
  const int wide = (most + 7) / 8, pieces = side == 0 ? most * (D / 8) : D * wide;
  auto piece = [&](int k, int x, int* n) {
    const int t = held[k] % KVP;
    if (side == 0) {
      *n = x < t * (D / 8) ? 8 : 0;
      return x * 8;
    }
    const int f = x / wide, part = x % wide;
    *n = f < D ? min(8, t - 8 * part) : 0;
    return f * KVP + 8 * part;
  };
  for (int b0 = 0; b0 < pieces; b0 += per) {
    uint4 v[HOLD];
#pragma unroll
    for (int e = 0; e < HOLD; ++e) {
      const int x = tid + e * NT, k = x / per;
      int n = 0;
      const int at = k < M ? piece(k, b0 + x % per, &n) : 0;
      if (n > 0) v[e] = *reinterpret_cast<const uint4*>(base + from[k] * seq + at);
    }
    __syncthreads();
#pragma unroll
    for (int e = 0; e < HOLD; ++e) {
      const int x = tid + e * NT, k = x / per;
      int n = 0;
      const int at = k < M ? piece(k, b0 + x % per, &n) : 0;
      uint16_t* to = base + (k < M ? who[k] : 0) * seq + at;
      if (n == 8) {
        *reinterpret_cast<uint4*>(to) = v[e];
      } else if (n > 0) {   // the last tokens of a feature: what lies behind them stays
        uint2 w = make_uint2(v[e].x, v[e].y);
        if (n & 4) {
          *reinterpret_cast<uint2*>(to) = w;
          to += 4;
          w = make_uint2(v[e].z, v[e].w);
        }
        if (n & 2) {
          *reinterpret_cast<uint32_t*>(to) = w.x;
          to += 2;
          w.x = w.y;
        }
        if (n & 1) *to = uint16_t(w.x);
      }
    }
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
  kv_reorder_kernel<<<dim3(unsigned(kv_reorder_parts(c)), unsigned(g.num_groups)), NT, 0, st>>>(
      c, g, parent, members);
  kv_reorder_lengths<<<unsigned(g.num_groups), NT, 0, st>>>(c, g, parent, members);
  return hipGetLastError();
}

}  // namespace tav2
