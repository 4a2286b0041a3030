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
#include "kv_attend_core.h"

namespace tav2 {

namespace {

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
  __device__ __forceinline__ bool parts() const { return splits > 1; }
};

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

// The positions that query row `row` of the job sees: below hi, at least lo.
__device__ __forceinline__ void row_seen(const AttendArgs& a, const Job& j, int row, int* hi, int* lo) {
  const int64_t pos = a.causal ? j.first_pos + row / j.G : j.first_pos;
  const int64_t end = pos + 1 < j.len ? pos + 1 : j.len;
  *hi = int(end > 0 ? end : 0);
  const int64_t low = pos - a.q.window + 1;
  *lo = a.q.window > 0 && low > 0 ? int(low) : 0;
}
// And those that all of a tile's rows see.
__device__ __forceinline__ void tile_seen(const AttendArgs& a, const Job& j, int64_t* hi, int64_t* lo) {
  *hi = j.lo_pos + 1 < j.len ? j.lo_pos + 1 : j.len;
  *lo = a.q.window > 0 ? j.hi_pos - a.q.window + 1 : 0;
}
__device__ __forceinline__ int tile_sinks(const AttendArgs& a, const Job&) { return a.q.sinks; }

template <int D, int QT>
__global__ __launch_bounds__(256, 2) void kv_attend_kernel(AttendArgs a) {
  Job j;
  if (my_job(a, 32 * QT, j)) attend_rows<D, QT>(a, j);
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

// At most 16 query rows (attend16).  Half the vector work of a 32-row tile: new actions of 64 users (4 rows) 35.4 us for 40.2 with
// that, 8 copies each of 16 histories 79 for 109.  Where rows are few enough, neighbouring sequences share
// a tile over the pages that they have in common (shared_set): the copies take 92 us without.
template <int D>
__global__ __launch_bounds__(256, D <= 64 ? 3 : 2) void kv_attend16_kernel(AttendArgs a) {
  constexpr int ND = D / 16;         // tiles of O^T
  __shared__ u32x4 stage[4][8 * D];  // a wave's page on its way, then its state (D / 16 x 64)
  __shared__ float mm[4][2][16];
  const tav2_kv& c = a.c;
  Job j;
  if (!my_job(a, 16, j)) return;
  const int lane = threadIdx.x % WAVE, m = lane % 16, g = lane / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int full = j.len / KVP;
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
  auto open_blocks = [&](auto open_block) {
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
  };
  auto finish = [&](float M, float l, auto tile) {
    if (!valid) return;
    const int64_t part = int64_t(j.split) * a.q.total * a.q.heads + at;
    const bool some = l > 0.f || l != l;
    const float inv = some ? 1.f / l : 0.f;
    for (int d = wave; d < ND; d += 4) {
      const f32x4 x = tile(d);
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
  };
  attend16<D>(a, j, feed, page, stage, mm, qi, row % j.G, hi, lo, open_blocks, finish);
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
