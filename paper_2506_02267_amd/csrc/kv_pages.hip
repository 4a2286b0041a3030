// The page operators of the 8-bit cache: extend, fork, free, trim, compact.
//
// The pool's state is refs[page] alone: how many sequences hold the page, 0 where it is
// free.  Free pages are found by a scan in ascending order, so what a call does depends on the
// state and its arguments only: no list whose order would follow the order of atomics.  Page numbers and
// lengths are clamped before they index anything, so a corrupted table cannot make a kernel leave its
// buffers.
#include <atomic>

#include "common.h"
#include "internal.h"
#include "kv_common.h"

namespace tav2 {

namespace {

constexpr int EXT_NT = 1024;                 // threads of the one-workgroup scans
constexpr int EXT_NW = EXT_NT / WAVE;
constexpr int SCAN = 4;                      // pages per thread and step of a scan

// Inclusive prefix sum over the workgroup's threads; *total = the sum.  sums: EXT_NW words.
__device__ __forceinline__ int block_scan(int v, int* sums, int* total) {
  const int lane = threadIdx.x % WAVE, wid = threadIdx.x / WAVE;
#pragma unroll
  for (int o = 1; o < WAVE; o <<= 1) {
    const int u = __shfl_up(v, o, WAVE);
    if (lane >= o) v += u;
  }
  __syncthreads();   // the last use of sums is over
  if (lane == WAVE - 1) sums[wid] = v;
  __syncthreads();
  int below = 0, all = 0;
#pragma unroll
  for (int w = 0; w < EXT_NW; ++w) {
    const int x = sums[w];
    below += w < wid ? x : 0;
    all += x;
  }
  *total = all;
  return v + below;
}

// The flags of SCAN * EXT_NT consecutive pages, flag j of thread t being page j EXT_NT + t:
// rank[j] = set flags before it; returns how many are set.  cnt: SCAN * EXT_NW words.
__device__ __forceinline__ int block_rank(const bool (&flag)[SCAN], int (&rank)[SCAN], int* cnt) {
  const int lane = threadIdx.x % WAVE, wid = threadIdx.x / WAVE;
  uint64_t bal[SCAN];
  __syncthreads();   // the last use of cnt is over
#pragma unroll
  for (int j = 0; j < SCAN; ++j) {
    bal[j] = __ballot(flag[j]);
    if (lane == 0) cnt[j * EXT_NW + wid] = __popcll(bal[j]);
  }
  __syncthreads();
  static_assert(SCAN * EXT_NW == WAVE, "one count per lane");
  const int mine = cnt[lane];   // every wave scans the 64 counts
  int v = mine;
#pragma unroll
  for (int o = 1; o < WAVE; o <<= 1) {
    const int u = __shfl_up(v, o, WAVE);
    if (lane >= o) v += u;
  }
#pragma unroll
  for (int j = 0; j < SCAN; ++j)
    rank[j] = __shfl(v - mine, j * EXT_NW + wid, WAVE) +
              __popcll(bal[j] & ((uint64_t(1) << lane) - 1));
  return __shfl(v, WAVE - 1, WAVE);
}

// One workgroup.  upto[s] (LDS) = pages that sequences 0..s ask for; the free pages, in ascending
// order, go to the rank-th place of that list as they are found, and what went to a sequence
// that then proved too large is put back.
__global__ __launch_bounds__(EXT_NT) void kv_extend_kernel(tav2_kv c, const int32_t* __restrict__ count) {
  extern __shared__ int upto[];   // [num_seqs]
  __shared__ int sums[EXT_NW], cnt[SCAN * EXT_NW];
  const int S = c.num_seqs, tid = threadIdx.x;
  int want = 0;   // pages asked for
  for (int s0 = 0; s0 < S; s0 += EXT_NT) {
    const int s = s0 + tid;
    int need = 0;
    if (s < S) {
      const int64_t old = kv_len(c, s), n = count[s];
      if (n > 0 && (old + n) / KVP <= c.max_blocks) need = int((old + n) / KVP - old / KVP);
    }
    int total;   // at most 1024 sequences of 2^20 blocks; the running sum saturates
    const int v = block_scan(need, sums, &total);
    const int64_t u = int64_t(want) + v;
    if (s < S) upto[s] = u > 0x7fffffff ? 0x7fffffff : int(u);
    const int64_t w = int64_t(want) + total;
    want = w > 0x7fffffff ? 0x7fffffff : int(w);
  }
  __syncthreads();
  int found = 0;
  for (int64_t p0 = 0; p0 < c.pages && found < want; p0 += SCAN * EXT_NT) {
    bool flag[SCAN];
    int rank[SCAN];
#pragma unroll
    for (int j = 0; j < SCAN; ++j) {
      const int64_t p = p0 + j * EXT_NT + tid;
      flag[j] = p < c.pages && c.refs[p] == 0;
    }
    const int n = block_rank(flag, rank, cnt);
#pragma unroll
    for (int j = 0; j < SCAN; ++j) {
      const int r = found + rank[j];
      if (!flag[j] || r >= want) continue;
      int lo = 0, hi = S - 1;   // the first sequence with upto > r
      while (lo < hi) {
        const int mid = (lo + hi) / 2;
        if (upto[mid] > r) hi = mid; else lo = mid + 1;
      }
      const int before = lo ? upto[lo - 1] : 0;
      const int64_t p = p0 + j * EXT_NT + tid;
      const int b = kv_len(c, lo) / KVP + (r - before);
      if (b < c.max_blocks) {
        c.table[int64_t(lo) * c.max_blocks + b] = int(p);
        c.refs[p] = 1;
      }
    }
    found += n;
  }
  if (found > want) found = want;
  __syncthreads();
  if (found < want) {   // the pages of the sequence that got only some of them
    int lo = 0, hi = S - 1;
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (upto[mid] > found) hi = mid; else lo = mid + 1;
    }
    const int before = lo ? upto[lo - 1] : 0;
    int32_t* e = c.table + int64_t(lo) * c.max_blocks + kv_len(c, lo) / KVP;
    for (int r = tid; r < found - before; r += EXT_NT) {
      c.refs[e[r]] = 0;
      e[r] = -1;
    }
    __syncthreads();   // the lengths are read no more
  }
  for (int s = tid; s < S; s += EXT_NT) {
    const int old = kv_len(c, s), n = count[s];
    const bool fits = n > 0 && (int64_t(old) + n) / KVP <= c.max_blocks;
    const bool granted = fits && upto[s] <= found;
    c.fresh[s] = granted ? n : 0;
    if (granted) c.len[s] = old + n;
  }
}

// Pages of one sequence per workgroup: those whose blocks lie in [lo, hi) are given up.
__device__ __forceinline__ void release(const tav2_kv& c, int s, int lo, int hi) {
  for (int b = lo + int(threadIdx.x); b < hi; b += int(blockDim.x)) {
    int32_t* e = c.table + int64_t(s) * c.max_blocks + b;
    const int p = *e;
    if (p >= 0 && p < c.pages) atomicSub(c.refs + p, 1);   // an integer count: any order
    if (p != -1) *e = -1;
  }
}

__global__ __launch_bounds__(256) void kv_free_kernel(tav2_kv c, const uint8_t* __restrict__ drop) {
  const int s = blockIdx.x;
  if (!drop[s]) return;
  release(c, s, 0, kv_len(c, s) / KVP);
  __syncthreads();   // every thread has read the length
  if (threadIdx.x == 0) {
    c.len[s] = 0;
    c.fresh[s] = 0;
  }
}

__global__ __launch_bounds__(256) void kv_trim_kernel(tav2_kv c, int window, int sinks) {
  const int s = blockIdx.x;
  const int len = kv_len(c, s);
  const int last = len - window + 1;   // the first position that stays visible
  release(c, s, sinks / KVP + (sinks % KVP != 0), last > 0 ? last / KVP : 0);
}

// Whether this call makes sequence s a copy, and of which one.
__device__ __forceinline__ int fork_source(const tav2_kv& c, const int32_t* parent, int s) {
  const int p = parent[s];
  if (p < 0 || p >= c.num_seqs || parent[p] >= 0) return -1;
  return c.len[s] == 0 ? p : -1;
}

// The tails: blockIdx.x a sequence, blockIdx.y a (layer, head).  Only the tokens that the parent
// holds are copied.
__global__ __launch_bounds__(256) void kv_fork_tails(tav2_kv c, const int32_t* __restrict__ parent) {
  const int s = blockIdx.x;
  const int p = fork_source(c, parent, s);
  if (p < 0) return;
  const int n = kv_len(c, p) % KVP;
  if (n == 0) return;
  const int D = c.head_dim, H = c.kv_heads;
  const int layer = blockIdx.y / H, h = blockIdx.y % H;
  const int64_t from = kv_tail(c, layer, p, h), to = kv_tail(c, layer, s, h);
  const uint4* ks = reinterpret_cast<const uint4*>(c.k_tail + from);
  uint4* kd = reinterpret_cast<uint4*>(c.k_tail + to);
  for (int e = threadIdx.x; e < n * D / 8; e += 256) kd[e] = ks[e];
  // by feature: rows of 64 tokens, whole groups of 8 and the rest one by one
  const uint16_t* vs = c.v_tail + from;
  uint16_t* vd = c.v_tail + to;
  for (int e = threadIdx.x; e < D * 8; e += 256) {
    const int at = (e >> 3) * KVP + (e & 7) * 8, held = n - (e & 7) * 8;
    if (held >= 8) {
      *reinterpret_cast<uint4*>(vd + at) = *reinterpret_cast<const uint4*>(vs + at);
    } else {
      for (int i = 0; i < held; ++i) vd[at + i] = vs[at + i];
    }
  }
}

// The tables, after the tails (whose condition is that the child is still empty).
__global__ __launch_bounds__(256) void kv_fork_tables(tav2_kv c, const int32_t* __restrict__ parent) {
  const int s = blockIdx.x;
  const int p = fork_source(c, parent, s);
  if (p < 0) return;
  const int len = kv_len(c, p);
  for (int b = threadIdx.x; b < len / KVP; b += 256) {
    const int id = c.table[int64_t(p) * c.max_blocks + b];
    c.table[int64_t(s) * c.max_blocks + b] = id;
    if (id >= 0 && id < c.pages) atomicAdd(c.refs + id, 1);
  }
  __syncthreads();   // every thread has seen the child empty
  if (threadIdx.x == 0) {
    c.len[s] = len;
    c.fresh[s] = 0;
  }
}

// One workgroup: counts the used pages, lists the holes below that count and the used pages from
// it on (both ascending), and moves the refs.  ws: [moves, hole[pages / 2], from[pages / 2], to[pages]].
__global__ __launch_bounds__(EXT_NT) void kv_plan_kernel(tav2_kv c, int32_t* __restrict__ used,
                                                        KvPlan plan) {
  __shared__ int sums[EXT_NW], cnt[SCAN * EXT_NW];
  const int tid = threadIdx.x;
  int mine = 0;
#pragma unroll 8
  for (int64_t p = tid; p < c.pages; p += EXT_NT) mine += c.refs[p] > 0;
  int U;
  block_scan(mine, sums, &U);
  int holes = 0, moves = 0;
  for (int64_t p0 = 0; p0 < c.pages; p0 += SCAN * EXT_NT) {
    bool held[SCAN], flag[SCAN];
    int rank[SCAN];
#pragma unroll
    for (int j = 0; j < SCAN; ++j) {
      const int64_t p = p0 + j * EXT_NT + tid;
      held[j] = c.refs[p < c.pages ? p : 0] > 0 && p < c.pages;
    }
    if (p0 < U) {
#pragma unroll
      for (int j = 0; j < SCAN; ++j) flag[j] = p0 + j * EXT_NT + tid < U && !held[j];
      const int n = block_rank(flag, rank, cnt);
#pragma unroll
      for (int j = 0; j < SCAN; ++j)
        if (flag[j]) plan.hole[holes + rank[j]] = int(p0 + j * EXT_NT + tid);
      holes += n;
    }
    if (p0 + SCAN * EXT_NT > U) {
#pragma unroll
      for (int j = 0; j < SCAN; ++j) flag[j] = p0 + j * EXT_NT + tid >= U && held[j];
      const int n = block_rank(flag, rank, cnt);
#pragma unroll
      for (int j = 0; j < SCAN; ++j)
        if (flag[j]) plan.from[moves + rank[j]] = int(p0 + j * EXT_NT + tid);
      moves += n;
    }
  }
  __threadfence_block();
  __syncthreads();   // the lists are whole (as many holes as moves, by counting)
  for (int i = tid; i < moves; i += EXT_NT) {
    const int p = plan.from[i], q = plan.hole[i];
    plan.to[p] = q;
    c.refs[q] = c.refs[p];
    c.refs[p] = 0;
  }
  if (tid == 0) {
    *plan.moves = moves;
    plan.moves[1] = U;
    *used = U;
  }
}

// Workgroups copy (page, layer, head) units in turn; the tables' entries are renumbered by all.
__global__ __launch_bounds__(256) void kv_compact_kernel(tav2_kv c, KvPlan plan) {
  const int moves = plan.moves[0], U = plan.moves[1];
  if (moves == 0) return;
  const int H = c.kv_heads, D = c.head_dim;
  const int64_t units = int64_t(moves) * c.layers * H;
  const int n = KVP * D / 16;   // 16-byte pieces of one side: 128 .. 512
  for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
    const int h = int(u % H);
    const int layer = int(u / H / moves), i = int(u / H % moves);
    const int64_t a = kv_unit(c, layer, plan.from[i], h), b = kv_unit(c, layer, plan.hole[i], h);
    const uint4* ks = reinterpret_cast<const uint4*>(c.k + a * KVP * D);
    const uint4* vs = reinterpret_cast<const uint4*>(c.v + a * KVP * D);
    uint4* kd = reinterpret_cast<uint4*>(c.k + b * KVP * D);
    uint4* vd = reinterpret_cast<uint4*>(c.v + b * KVP * D);
    for (int e = threadIdx.x; e < 2 * n; e += 256)
      if (e < n) kd[e] = ks[e]; else vd[e - n] = vs[e - n];
    if (threadIdx.x == 0) c.k_scale[b] = c.k_scale[a];
    if (threadIdx.x == 1) c.v_scale[b] = c.v_scale[a];
  }
  const int64_t entries = int64_t(c.num_seqs) * c.max_blocks;
  for (int64_t e = int64_t(blockIdx.x) * 256 + threadIdx.x; e < entries; e += int64_t(gridDim.x) * 256) {
    const int p = c.table[e];
    if (p >= U && p < c.pages) c.table[e] = plan.to[p];
  }
}

}  // namespace

hipError_t launch_kv_extend(const tav2_kv& c, const int32_t* count, hipStream_t st) {
  static_assert(TAV2_KV_SEQS_MAX * 4 <= 128 * 1024, "the prefix sums fit LDS");
  if (c.num_seqs > 8192) {   // more LDS than a kernel has without asking
    static std::atomic<bool> done[64] = {};
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= 64 || !done[dev].load(std::memory_order_acquire)) {
      e = hipFuncSetAttribute(reinterpret_cast<const void*>(kv_extend_kernel),
                              hipFuncAttributeMaxDynamicSharedMemorySize, TAV2_KV_SEQS_MAX * 4);
      if (e != hipSuccess) return e;
      if (dev >= 0 && dev < 64) done[dev].store(true, std::memory_order_release);
    }
  }
  ProfScope prof("kv_extend", st);
  kv_extend_kernel<<<1, EXT_NT, size_t(c.num_seqs) * 4, st>>>(c, count);
  return hipGetLastError();
}

hipError_t launch_kv_fork(const tav2_kv& c, const int32_t* parent, hipStream_t st) {
  ProfScope prof("kv_fork", st);
  kv_fork_tails<<<dim3(unsigned(c.num_seqs), unsigned(c.layers * c.kv_heads)), 256, 0, st>>>(c, parent);
  kv_fork_tables<<<unsigned(c.num_seqs), 256, 0, st>>>(c, parent);
  return hipGetLastError();
}

hipError_t launch_kv_free(const tav2_kv& c, const uint8_t* drop, hipStream_t st) {
  ProfScope prof("kv_free", st);
  kv_free_kernel<<<unsigned(c.num_seqs), 256, 0, st>>>(c, drop);
  return hipGetLastError();
}

hipError_t launch_kv_trim(const tav2_kv& c, int window, int sinks, hipStream_t st) {
  ProfScope prof("kv_trim", st);
  kv_trim_kernel<<<unsigned(c.num_seqs), 256, 0, st>>>(c, window, sinks);
  return hipGetLastError();
}

size_t kv_plan_bytes(const tav2_kv& c) {
  return align_up(8 + (size_t(c.pages) / 2 + 1) * 8 + size_t(c.pages) * 4, 256);
}

hipError_t launch_kv_compact(const tav2_kv& c, int32_t* used, void* ws, hipStream_t st) {
  KvPlan plan;
  plan.moves = static_cast<int32_t*>(ws);
  plan.hole = plan.moves + 2;
  plan.from = plan.hole + c.pages / 2 + 1;
  plan.to = plan.from + c.pages / 2 + 1;
  {
    ProfScope prof("kv_plan", st);
    kv_plan_kernel<<<1, EXT_NT, 0, st>>>(c, used, plan);
  }
  ProfScope prof("kv_compact", st);
  kv_compact_kernel<<<2048, 256, 0, st>>>(c, plan);
  return hipGetLastError();
}

}  // namespace tav2
