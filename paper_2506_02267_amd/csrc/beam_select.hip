// Selection of the best continuations of a request's beams over the vocabulary.
//
// A continuation is worth c = (score - Z) + z, Z the row's log-sum-exp; it is computed in 64 bits, since the values
// of different beams have to be put in order: with an error of 1e-7 two of a request's best would change places
// now and then.
//
// The first launch reads the logits once.  A wave takes a segment of a row, VPT 16-byte loads a lane, holds it in
// registers, and leaves its largest logit, its sum of exponentials, and each lane's largest logit (a group's: the
// lane's VPT x 8 or x 4 tokens).  The second launch has a workgroup a request.  The K-th largest of its segments'
// maxima, and then of the groups' in the segments that reach it, is a bound that K continuations reach; only
// the groups that reach it are read again, about K of them, and what reaches it there, little more than K, is put in
// order.  Where more than fit the list reach it (equal logits by the thousand), the bound is drawn closer over all of the
// request's continuations.
#include <float.h>

#include <type_traits>

#include "common.h"
#include "internal.h"

namespace tav2 {

namespace {

struct BeamArgs {
  tav2_beams b;
  int keep;
  bool in_place;
  int32_t* parent;
  int32_t* token;
  float* score;
  uint8_t* done;     // nullable
  // of each segment of each row: the sum of exp(z - top), the largest logit `top` (NONE: none), and the largest that may be
  // selected; of each of its lanes the largest that may be selected
  int vpt, segs;     // loads of 16 bytes a lane; a row's segments
  double* seg_sum;
  float* seg_top;
  float* seg_best;
  float* best;       // [rows, segs, 64]
};

constexpr float NONE = -INFINITY;   // a logit that is not there

// 16 bytes of a row, which may begin anywhere.
typedef uint32_t piece2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t piece4 __attribute__((ext_vector_type(4), aligned(4)));

template <bool BF>
struct Logits {
  static constexpr int EL = BF ? 8 : 4;   // in 16 bytes
  using piece = std::conditional_t<BF, piece2, piece4>;
  using T = std::conditional_t<BF, bf16_t, float>;
  static __device__ __forceinline__ float one(const T* p) {
    if constexpr (BF) return bf2f(*p);
    else return *p;
  }
};

template <bool BF>
__device__ __forceinline__ float logit(const BeamArgs& a, int64_t row, int v) {
  const float z = Logits<BF>::one(static_cast<const typename Logits<BF>::T*>(a.b.logits) + row * a.b.ld + v);
  return __builtin_isfinite(z) ? z : NONE;
}

// 2^t for t <= 0 or so: 2^n times a polynomial of f = t - n, |f| <= 1/2, that is off by at most 8e-13 of 2^f (fitted
// to the relative error's maximum).  Far below 0: 0.
__device__ __forceinline__ double exp2_neg(double t) {
  const double n = __builtin_rint(t), f = t - n;
  double p = 1.3175854784954272e-06;
  p = __builtin_fma(p, f, 1.530973767019622e-05);
  p = __builtin_fma(p, f, 1.5403851768737496e-04);
  p = __builtin_fma(p, f, 1.333345206150456e-03);
  p = __builtin_fma(p, f, 9.61812854282085e-03);
  p = __builtin_fma(p, f, 5.550410939341938e-02);
  p = __builtin_fma(p, f, 0.24022650698880715);
  p = __builtin_fma(p, f, 0.6931471805465146);
  p = __builtin_fma(p, f, 0.9999999999997632);
  return __builtin_ldexp(p, int(n));
}

constexpr double LOG2E_64 = 1.4426950408889634074;

// A segment of a row: each lane's largest logit that may be selected, and, alike in all lanes, the segment's
// largest logit and sum.
struct Segment {
  float best, top;
  double sum;
};
template <bool BF, int VPT>
__device__ __forceinline__ Segment scan(const BeamArgs& a, int64_t row, int seg) {
  using L = Logits<BF>;
  constexpr int EL = L::EL, SEG = WAVE * VPT * EL;
  const int lane = threadIdx.x % WAVE, V = a.b.vocab;
  const typename L::T* const p = static_cast<const typename L::T*>(a.b.logits) + row * a.b.ld;
  const int v0 = seg * SEG + lane * EL;   // of load i: + i 64 EL
  float z[VPT][EL];
  if (seg * SEG + SEG <= V) {
    typename L::piece w[VPT];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
      w[i] = *reinterpret_cast<const typename L::piece*>(p + v0 + i * WAVE * EL);
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int e = 0; e < EL; ++e)
        z[i][e] = __uint_as_float(!BF ? w[i][e] : e % 2 ? w[i][e / 2] & 0xFFFF0000u : w[i][e / 2] << 16);
  } else {
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int e = 0; e < EL; ++e) {
        const int v = v0 + i * WAVE * EL + e;
        z[i][e] = v < V ? L::one(p + v) : NONE;
      }
  }
  Segment r;
  float top = NONE;
#pragma unroll
  for (int i = 0; i < VPT; ++i)
#pragma unroll
    for (int e = 0; e < EL; ++e) {
      z[i][e] = __builtin_isfinite(z[i][e]) ? z[i][e] : NONE;
      top = vmax(top, z[i][e]);
    }
  r.best = top;
  if (a.b.allowed) {
    const uint8_t* const ok = a.b.allowed + row * a.b.allowed_ld;
    r.best = NONE;
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int v = v0 + i * WAVE * EL;
      const uint32_t bits = v < V ? ok[v / 8] >> (v % 8) : 0;   // (EL divides 8)
#pragma unroll
      for (int e = 0; e < EL; ++e) r.best = bits >> e & 1 ? vmax(r.best, z[i][e]) : r.best;
    }
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) top = vmax(top, __shfl_xor(top, o, WAVE));
  r.top = top;
  double s = 0.0;
  if (top > NONE) {
    const double m = top;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int e = 0; e < EL; ++e) s += exp2_neg(__builtin_fmax(double(z[i][e]) - m, -1e4) * LOG2E_64);
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o, WAVE);
  r.sum = s;
  return r;
}

// Four segments a workgroup.
template <bool BF, int VPT>
__global__ __launch_bounds__(256) void beam_scan_kernel(BeamArgs a) {
  const int per = (a.segs + 3) / 4;
  const int64_t row = blockIdx.x / per;
  if ((a.b.done && a.b.done[row]) || (a.b.score && !__builtin_isfinite(a.b.score[row]))) return;
  const int seg = int(blockIdx.x % per) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  if (seg >= a.segs) return;
  const Segment r = scan<BF, VPT>(a, row, seg);
  const int64_t at = row * a.segs + seg;
  a.best[at * WAVE + threadIdx.x % WAVE] = r.best;
  float b = r.best;
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) b = vmax(b, __shfl_xor(b, o, WAVE));
  if (threadIdx.x % WAVE == 0) {
    a.seg_sum[at] = r.sum;
    a.seg_top[at] = r.top;
    a.seg_best[at] = b;
  }
}

// Order-preserving key of a value: larger value <=> larger key; 0: no continuation.
__device__ __forceinline__ uint64_t value_key(double x) {
  const uint64_t u = __builtin_bit_cast(uint64_t, x + 0.0);
  return u >> 63 ? ~u : u | uint64_t(1) << 63;
}
__device__ __forceinline__ double key_value(uint64_t k) {
  return __builtin_bit_cast(double, k >> 63 ? k & ~(uint64_t(1) << 63) : ~k);
}
// And of a value rounded to 32 bits, which keeps the order but for ties.
__device__ __forceinline__ uint32_t near_key(double x) { return score_key(float(x)); }

constexpr int PICK = 1024;    // threads
constexpr int NW = PICK / WAVE;
constexpr int BINS = 2048;
constexpr int CAP = 2048;     // continuations that are put in order at last
constexpr int LIST = 4096;    // segments, and then groups, that may hold some of the best

struct PickShared {
  double base[TAV2_BEAMS_MAX];   // score - Z; a finished beam's score; NaN: no beam
  uint32_t bins[BINS];
  union {
    struct {
      uint64_t keys[CAP];
      uint32_t flats[CAP];
    };
    uint32_t segs[LIST];         // read before there are keys
  };
  union {
    struct {
      int parent[TAV2_K_MAX], token[TAV2_K_MAX], first_of[TAV2_BEAMS_MAX];
      double value[TAV2_K_MAX];
    };
    uint32_t groups[LIST];       // read before anything is put in order
  };
  uint32_t wsum[NW], wmin[NW], wmax[NW];
  uint32_t n, bin, above;
};

// The bin that the `need`-th from the top is in (BINS: there are fewer), and how many lie in the bins above it.
__device__ __forceinline__ void find_bin(PickShared& sh, uint32_t need) {
  const int tid = threadIdx.x, lane = tid % WAVE, wid = tid / WAVE;
  const uint32_t c0 = sh.bins[BINS - 1 - 2 * tid], c1 = sh.bins[BINS - 2 - 2 * tid];
  uint32_t v = c0 + c1;
#pragma unroll
  for (int o = 1; o < WAVE; o <<= 1) {
    const uint32_t u = __shfl_up(v, o, WAVE);
    if (lane >= o) v += u;
  }
  if (lane == WAVE - 1) sh.wsum[wid] = v;
  if (tid == 0) sh.bin = BINS;
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < NW; ++w) before += w < wid ? sh.wsum[w] : 0;
  const uint32_t upto = before + v, from = upto - c0 - c1;
  if (from < need && upto >= need) {
    const bool first = from + c0 >= need;
    sh.bin = BINS - 1 - 2 * tid - (first ? 0 : 1);
    sh.above = first ? from : from + c0;
  }
  __syncthreads();
}

// A key that at least K of the keys that visit(f) calls f with reach, and at most about `most`, unless more are equal;
// 1 where there are fewer than K.  Keys of 0 are none.
template <class Visit>
__device__ __forceinline__ uint32_t bound_of(PickShared& sh, Visit visit, uint32_t K, uint32_t most) {
  const int tid = threadIdx.x;
  uint32_t lo = ~0u, hi = 0;
  visit([&](uint32_t k) {
    if (k) lo = min(lo, k);
    hi = max(hi, k);
  });
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) {
    lo = min(lo, uint32_t(__shfl_xor(int(lo), o, WAVE)));
    hi = max(hi, uint32_t(__shfl_xor(int(hi), o, WAVE)));
  }
  if (tid % WAVE == 0) {
    sh.wmin[tid / WAVE] = lo;
    sh.wmax[tid / WAVE] = hi;
  }
  __syncthreads();
  for (int w = 0; w < NW; ++w) {
    lo = min(lo, sh.wmin[w]);
    hi = max(hi, sh.wmax[w]);
  }
  if (hi == 0) return 1;
  uint32_t above = 0;
  while (true) {
    int shift = 0;
    while ((hi - lo) >> shift >= BINS) ++shift;
    for (int i = tid; i < BINS; i += PICK) sh.bins[i] = 0;
    __syncthreads();
    visit([&](uint32_t k) {
      if (k >= lo && k <= hi && k) atomicAdd(&sh.bins[(k - lo) >> shift], 1u);
    });
    __syncthreads();
    find_bin(sh, K - above);
    if (sh.bin == BINS) return 1;
    const uint32_t in = sh.bins[sh.bin], l = lo + (sh.bin << shift), h = l + ((1u << shift) - 1);
    above += sh.above;
    lo = l;
    hi = min(hi, h);
    __syncthreads();
    if (above + in <= most || shift == 0) return lo;
  }
}

// A workgroup a request.
template <bool BF>
__global__ __launch_bounds__(PICK) void beam_pick_kernel(BeamArgs a) {
  constexpr int EL = Logits<BF>::EL;
  __shared__ PickShared sh;
  const int B = a.b.beams, V = a.b.vocab, K = a.keep, S = a.segs;
  const int tid = threadIdx.x, lane = tid % WAVE, wid = __builtin_amdgcn_readfirstlane(tid / WAVE);
  const int64_t row0 = int64_t(blockIdx.x) * B;
  const int eos0 = a.b.eos < 0 ? 0 : a.b.eos;
  const uint8_t* const done = a.b.done ? a.b.done + row0 : nullptr;
  // the beams' bases: a wave a beam
  for (int b = wid; b < B; b += NW) {
    const float s = a.b.score ? a.b.score[row0 + b] : 0.f;
    double x = __builtin_nan("");
    if (__builtin_isfinite(s)) {
      if (done && done[b]) {
        x = s;
      } else {
        const float* const tops = a.seg_top + (row0 + b) * S;
        const double* const sums = a.seg_sum + (row0 + b) * S;
        float m = NONE;
        for (int i = lane; i < S; i += WAVE) m = vmax(m, tops[i]);
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) m = vmax(m, __shfl_xor(m, o, WAVE));
        double z = 0.0;
        for (int i = lane; i < S; i += WAVE)
          z += sums[i] * exp2_neg(__builtin_fmax(double(tops[i]) - double(m), -1e4) * LOG2E_64);
#pragma unroll
        for (int o = 32; o >= 1; o >>= 1) z += __shfl_xor(z, o, WAVE);
        if (m > NONE) x = double(s) - (double(m) + log(z));
      }
    }
    if (lane == 0) sh.base[b] = x;
  }
  __syncthreads();

  // what segment s of beam b, and lane l's group of it, hold at best; a finished beam's one continuation counts as its first
  // segment's first group
  auto seg_key = [&](int b, int s) -> uint32_t {
    const double x = sh.base[b];
    if (x != x) return 0;
    if (done && done[b]) return s == 0 ? near_key(x) : 0;
    const float z = a.seg_best[(row0 + b) * S + s];
    return z > NONE ? near_key(x + double(z)) : 0;
  };
  auto group_key = [&](int b, int s, int l) -> uint32_t {
    const double x = sh.base[b];
    if (x != x) return 0;
    if (done && done[b]) return s == 0 && l == 0 ? near_key(x) : 0;
    const float z = a.best[((row0 + b) * S + s) * WAVE + l];
    return z > NONE ? near_key(x + double(z)) : 0;
  };
  // the key of beam b continued by v
  auto key_of = [&](int b, int v) -> uint64_t {
    const double x = sh.base[b];
    if (x != x) return 0;
    if (done && done[b]) return v == eos0 ? value_key(x) : 0;
    const float z = logit<BF>(a, row0 + b, v);
    if (!(z > NONE)) return 0;
    if (a.b.allowed && !(a.b.allowed[(row0 + b) * a.b.allowed_ld + v / 8] >> (v % 8) & 1)) return 0;
    return value_key(x + double(z));
  };
  auto list = [&](uint64_t k, uint32_t flat) {
    const uint32_t at = atomicAdd(&sh.n, 1u);
    if (at < CAP) {
      sh.keys[at] = k;
      sh.flats[at] = flat;
    }
  };

  const uint32_t total = uint32_t(B) * uint32_t(V), segs = uint32_t(B) * uint32_t(S);   // below 2^31
  bool fits = true;
  uint32_t bound = 1;
  if (segs >= 2 * uint32_t(K))
    bound = bound_of(sh, [&](auto f) {
      for (uint32_t i = tid; i < segs; i += PICK) f(seg_key(i / S, i % S));
    }, K, K + K / 4);
  if (tid == 0) sh.n = 0;
  __syncthreads();
  for (uint32_t i = tid; i < segs; i += PICK) {
    if (seg_key(i / S, i % S) < bound) continue;
    const uint32_t at = atomicAdd(&sh.n, 1u);
    if (at < LIST) sh.segs[at] = i;
  }
  __syncthreads();
  const uint32_t n_segs = sh.n;
  fits = n_segs <= LIST;
  if (fits) {
    auto groups = [&](auto f) {
#pragma unroll 4
      for (uint32_t i = wid; i < n_segs; i += NW) {
        const uint32_t s = sh.segs[i];
        f(group_key(s / S, s % S, lane));
      }
    };
    bound = max(bound, bound_of(sh, groups, K, K + K / 8));
    __syncthreads();
    if (tid == 0) sh.n = 0;
    __syncthreads();
    for (uint32_t i = wid; i < n_segs; i += NW) {
      const uint32_t s = sh.segs[i];
      if (group_key(s / S, s % S, lane) < bound) continue;
      const uint32_t at = atomicAdd(&sh.n, 1u);
      if (at < LIST) sh.groups[at] = s * WAVE + lane;
    }
    __syncthreads();
    const uint32_t n_groups = sh.n;
    fits = n_groups <= LIST;
    __syncthreads();
    if (tid == 0) sh.n = 0;
    __syncthreads();
    if (fits) {
      // a group's tokens: those of one load are neighbours
      const int i = lane / EL, e = lane % EL;
#pragma unroll 2
      for (uint32_t k = wid; k < n_groups; k += NW) {
        const uint32_t g = sh.groups[k], s = g / WAVE;
        const int b = int(s / S), seg = int(s % S);
        if (done && done[b]) {
          if (lane == 0) list(value_key(sh.base[b]), uint32_t(b) * V + eos0);
          continue;
        }
        const int v = (seg * a.vpt + i) * (WAVE * EL) + int(g % WAVE) * EL + e;
        if (i >= a.vpt || v >= V) continue;
        const uint64_t x = key_of(b, v);
        if (x && near_key(key_value(x)) >= bound) list(x, uint32_t(b) * V + v);
      }
    }
    __syncthreads();
    fits = fits && sh.n <= CAP;
    __syncthreads();
  }
  if (!fits) {
    // The interval [lo, hi] of keys, and then of one key's flat numbers, that the K-th lies in, drawn closer until what is
    // not below it fits; `above`: how many are above it.
    uint64_t lo = 1, hi = ~uint64_t(0);
    uint32_t flo = 0, fhi = total - 1, above = 0;
    bool by_flat = false;
    while (true) {
      const uint64_t width = by_flat ? fhi - flo : hi - lo;
      int shift = 0;
      while (width >> shift >= BINS) ++shift;
      for (int i = tid; i < BINS; i += PICK) sh.bins[i] = 0;
      __syncthreads();
      for (uint32_t i = tid; i < total; i += PICK) {
        const uint64_t k = key_of(i / V, i % V);
        if (k < lo || k > hi) continue;
        if (by_flat) {
          if (i >= flo && i <= fhi) atomicAdd(&sh.bins[BINS - 1 - ((i - flo) >> shift)], 1u);   // lower ones are better
        } else {
          atomicAdd(&sh.bins[(k - lo) >> shift], 1u);
        }
      }
      __syncthreads();
      find_bin(sh, K - above);
      if (sh.bin == BINS) break;   // fewer than K: all of them
      const uint32_t in = sh.bins[sh.bin];
      if (by_flat) {
        const uint64_t l = flo + (uint64_t(BINS - 1 - sh.bin) << shift), h = l + (uint64_t(1) << shift) - 1;
        flo = uint32_t(l);
        fhi = h < fhi ? uint32_t(h) : fhi;
      } else {
        const uint64_t l = lo + (uint64_t(sh.bin) << shift), h = l + ((uint64_t(1) << shift) - 1);
        lo = l;
        hi = h < hi ? h : hi;
      }
      above += sh.above;
      __syncthreads();
      if (above + in <= CAP) break;
      if (!by_flat && lo == hi) by_flat = true;   // (a bin of one flat number holds one)
    }
    if (tid == 0) sh.n = 0;
    __syncthreads();
    for (uint32_t i = tid; i < total; i += PICK) {
      const uint64_t k = key_of(i / V, i % V);
      if (k < lo || (by_flat && k == lo && i > fhi)) continue;
      list(k, i);
    }
    __syncthreads();
  }

  // in order: each one's place is the number of better ones
  const uint32_t n = min(sh.n, uint32_t(CAP));
  for (int k = tid; k < K; k += PICK) sh.parent[k] = -1;
  for (int b = tid; b < TAV2_BEAMS_MAX; b += PICK) sh.first_of[b] = TAV2_K_MAX;
  __syncthreads();
  for (uint32_t i = tid; i < n; i += PICK) {
    const uint64_t k = sh.keys[i];
    const uint32_t f = sh.flats[i];
    uint32_t rank = 0;
    for (uint32_t j = 0; j < n; ++j) rank += sh.keys[j] > k || (sh.keys[j] == k && sh.flats[j] < f);
    if (rank < uint32_t(K)) {
      sh.parent[rank] = int(f / V);
      sh.token[rank] = int(f % V);
      sh.value[rank] = key_value(k);
    }
  }
  __syncthreads();
  // (K <= PICK: a thread a place)
  const int p = tid < K ? sh.parent[tid] : -1;
  int slot = tid;
  if (a.in_place) {
    if (p >= 0) atomicMin(&sh.first_of[p], tid);
    __syncthreads();
    // the places of beams that are not continued, in order, for those that do not head a beam's
    const bool heads = p >= 0 && sh.first_of[p] == tid;
    const bool later = tid < K && !heads, free = tid < K && sh.first_of[tid] == TAV2_K_MAX;
    const uint64_t lb = __ballot(later), fb = __ballot(free), below = (uint64_t(1) << lane) - 1;
    if (lane == 0) sh.wsum[wid] = uint32_t(__popcll(lb)) | uint32_t(__popcll(fb)) << 16;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < wid; ++w) before += sh.wsum[w];
    const uint32_t nth = (before & 0xFFFF) + __popcll(lb & below), place = (before >> 16) + __popcll(fb & below);
    if (free) sh.bins[place] = tid;
    __syncthreads();
    if (later) slot = int(sh.bins[nth]);
    if (heads) slot = p;
  }
  if (tid >= K) return;
  const int64_t at = int64_t(blockIdx.x) * K + slot;
  a.parent[at] = p;
  const bool was = p >= 0 && done && done[p];
  a.token[at] = p < 0 ? -1 : was ? a.b.eos : sh.token[tid];
  a.score[at] = p < 0 ? -INFINITY : fmaxf(float(sh.value[tid]), -FLT_MAX);
  if (a.done) a.done[at] = p >= 0 && (was || (a.b.eos >= 0 && sh.token[tid] == a.b.eos));
}

// Loads a lane: as many as leave workgroups enough to fill the CUs, and no row mostly empty segments.
int vectors(const tav2_beams& b) {
  const int el = b.dtype == TAV2_BF16 ? 8 : 4;
  const int64_t rows = int64_t(b.num_requests) * b.beams;
  int vpt = 8;
  while (vpt > 1 && (rows * cdiv(b.vocab, WAVE * el * vpt) < 4096 || b.vocab <= WAVE * el * vpt / 2)) vpt /= 2;
  return vpt;
}
int64_t segments(const tav2_beams& b) {
  return cdiv(b.vocab, WAVE * (b.dtype == TAV2_BF16 ? 8 : 4) * vectors(b));
}

}  // namespace

int64_t beam_select_groups(const tav2_beams& b, int keep) {
  return int64_t(b.num_requests) * b.beams * cdiv(segments(b), 4);
}

size_t beam_select_bytes(const tav2_beams& b, int keep) {
  return align_up(size_t(b.num_requests) * b.beams * segments(b) * (8 + 4 + 4 + 4 * WAVE), 256);
}

template <bool BF>
static void launch_scan(const BeamArgs& a, unsigned n, hipStream_t st) {
  if (a.vpt == 8) beam_scan_kernel<BF, 8><<<n, 256, 0, st>>>(a);
  else if (a.vpt == 4) beam_scan_kernel<BF, 4><<<n, 256, 0, st>>>(a);
  else if (a.vpt == 2) beam_scan_kernel<BF, 2><<<n, 256, 0, st>>>(a);
  else beam_scan_kernel<BF, 1><<<n, 256, 0, st>>>(a);
}

hipError_t launch_beam_select(const tav2_beams& b, int keep, bool in_place, int32_t* parent,
                              int32_t* token, float* score, uint8_t* done, void* ws, hipStream_t st) {
  BeamArgs a{};
  a.b = b;
  a.keep = keep;
  a.in_place = in_place;
  a.parent = parent;
  a.token = token;
  a.score = score;
  a.done = done;
  a.vpt = vectors(b);
  a.segs = int(segments(b));
  const size_t n = size_t(b.num_requests) * b.beams * a.segs;
  a.seg_sum = static_cast<double*>(ws);
  a.best = reinterpret_cast<float*>(a.seg_sum + n);
  a.seg_top = a.best + n * WAVE;
  a.seg_best = a.seg_top + n;
  {
    ProfScope prof("beam_scan", st);
    const unsigned groups = unsigned(beam_select_groups(b, keep));
    if (b.dtype == TAV2_BF16) launch_scan<true>(a, groups, st);
    else launch_scan<false>(a, groups, st);
  }
  ProfScope prof("beam_pick", st);
  if (b.dtype == TAV2_BF16) beam_pick_kernel<true><<<unsigned(b.num_requests), PICK, 0, st>>>(a);
  else beam_pick_kernel<false><<<unsigned(b.num_requests), PICK, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace tav2
