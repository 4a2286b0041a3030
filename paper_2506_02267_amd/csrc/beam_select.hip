// Selection of the best continuations of a request's beams over the vocabulary.
//
// A continuation is worth c = (score - log S) + (z - top), S the row's sum of exp(z - top), top its largest logit; it is
// computed in 64 bits, since the values of different beams have to be put in order: with an error of 1e-7 two of a
// request's best would change places now and then.  top and log S stay apart: their sum would drop log S where logits are
// large (a row filled with the type's lowest value: every token would be worth the score itself).
//
// The first launch reads the logits once.  A wave takes a segment of a row, VPT 16-byte loads a lane, holds it in
// registers, and leaves its largest logit, its sum of exponentials, and each lane's largest logit (a group's: the
// lane's VPT x 8 or x 4 tokens).  The second launch has a workgroup a request.  The K-th largest of its segments'
// maxima, and then of the groups' in the segments that reach it, is a bound that K continuations reach; only
// the groups that reach it are read again, about K of them, and what reaches it there, little more than K, is put in
// order.  Where more than fit the list reach it (equal logits by the thousand), the bound is drawn closer over all of the
// request's continuations, by one workgroup in up to ten passes: about 10 ns a logit (32 x 131072: 40 ms).
#include <float.h>

#include <algorithm>
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

// Exponentials in 64 bits: 2^(n / 64) from a table in LDS, times 1 + g (C1 + g (C2 + g C3)) for the rest g / 64, |g| <= 1/2:
// off by at most 6.2e-12 of it (2^-37; fitted to the relative error's maximum, exact at 0).  n comes from the low bits of a
// sum with 1.5 2^52; its multiples of 64 go into the exponent by an addition, as what converts or scales 64-bit numbers
// takes several times as long.  14.7 instructions a logit; with a polynomial alone, 16.7, the largest case took 77.7 us for 74.
constexpr double ROUND = 6755399441055744.0;
constexpr double LOG2E_64 = 64 * 1.4426950408889634074;
constexpr double C1 = 0.01083042469637773, C2 = 5.86491682817601e-05, C3 = 2.1173090131387150e-07;
__device__ const double EXP2_64[64] = {
    1.0, 1.0108892860517005, 1.0218971486541166, 1.0330248790212284,
    1.0442737824274138, 1.0556451783605572, 1.0671404006768237, 1.0787607977571199,
    1.0905077326652577, 1.102382583307841, 1.1143867425958924, 1.1265216186082418,
    1.1387886347566916, 1.1511892299529827, 1.1637248587775775, 1.1763969916502812,
    1.189207115002721, 1.202156731452703, 1.215247359980469, 1.22848053610687,
    1.241857812073484, 1.255380757024691, 1.2690509571917332, 1.2828700160787783,
    1.2968395546510096, 1.3109612115247644, 1.3252366431597413, 1.339667524053303,
    1.3542555469368927, 1.3690024229745905, 1.383909881963832, 1.3989796725383112,
    1.4142135623730951, 1.42961333839197, 1.4451808069770467, 1.460917794180647,
    1.4768261459394993, 1.4929077282912648, 1.5091644275934228, 1.5255981507445384,
    1.5422108254079407, 1.559004400237837, 1.5759808451078865, 1.593142151342267,
    1.6104903319492543, 1.6280274218573478, 1.645755478153965, 1.6636765803267364,
    1.681792830507429, 1.7001063537185235, 1.718619298122478, 1.7373338352737062,
    1.7562521603732995, 1.7753764925265212, 1.7947090750031072, 1.8142521755003989,
    1.8340080864093424, 1.8539791250833855, 1.8741676341103, 1.8945759815869656,
    1.9152065613971474, 1.9360617934922943, 1.9571441241754002, 1.978456026387951,
};

// The table in LDS, an entry's exponent less what its own n adds (n << 14).
__device__ __forceinline__ void load_table(uint2* table) {
  if (threadIdx.x < 64) {
    const uint64_t u = __builtin_bit_cast(uint64_t, EXP2_64[threadIdx.x]);
    table[threadIdx.x] = make_uint2(uint32_t(u), uint32_t(u >> 32) - (threadIdx.x << 14));
  }
  __syncthreads();
}
// s + 2^((n + g) / 64), n the low 32 bits of k.
__device__ __forceinline__ double add_exp2(double s, double g, double k, const uint2* table) {
  typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
  const uint32_t n = __builtin_bit_cast(u32x2, k).x;
  const uint2 t = table[n & 63];
  const u32x2 u = {t.x, t.y + (n << 14)};
  const double q = __builtin_fma(__builtin_fma(C3, g, C2), g, C1);
  return __builtin_fma(__builtin_bit_cast(double, u), __builtin_fma(q, g, 1.0), s);
}

// exp(x - m) for x <= m, where x is not there 0 or next to it.
__device__ __forceinline__ double weight(float x, double m, const uint2* table) {
  const double d = __builtin_fmax(double(x) - m, -700.0), k = __builtin_fma(d, LOG2E_64, ROUND);
  return add_exp2(0.0, __builtin_fma(d, LOG2E_64, -(k - ROUND)), k, table);
}

// v joined over a wave's lanes by op, alike in all of them, on the vector unit alone: neighbours in fours, eights and
// sixteens, then the halves (a third of the time that six passes through LDS take).
template <int CTRL>
__device__ __forceinline__ uint32_t lane_move(uint32_t v) {
  return uint32_t(__builtin_amdgcn_update_dpp(int(v), int(v), CTRL, 0xF, 0xF, false));
}
template <class T, class Op>
__device__ __forceinline__ T wave_all(T v, Op op) {
  constexpr int N = sizeof(T) / 4;
  struct Words { uint32_t w[N]; };
  auto moved = [](T x, auto f) {
    Words a = __builtin_bit_cast(Words, x);
#pragma unroll
    for (int i = 0; i < N; ++i) a.w[i] = f(a.w[i]);
    return __builtin_bit_cast(T, a);
  };
  v = op(v, moved(v, [](uint32_t w) { return lane_move<0xB1>(w); }));    // 1 0 3 2
  v = op(v, moved(v, [](uint32_t w) { return lane_move<0x4E>(w); }));    // 2 3 0 1
  v = op(v, moved(v, [](uint32_t w) { return lane_move<0x141>(w); }));   // 7 - i of eight
  v = op(v, moved(v, [](uint32_t w) { return lane_move<0x140>(w); }));   // 15 - i of sixteen
  T a = v, b = v;
  auto swap = [&](auto f) {
    Words x = __builtin_bit_cast(Words, v), y = x;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const auto r = f(x.w[i]);
      x.w[i] = r[0];
      y.w[i] = r[1];
    }
    a = __builtin_bit_cast(T, x);
    b = __builtin_bit_cast(T, y);
  };
  swap([](uint32_t w) { return __builtin_amdgcn_permlane16_swap(w, w, false, false); });
  v = op(a, b);
  swap([](uint32_t w) { return __builtin_amdgcn_permlane32_swap(w, w, false, false); });
  return op(a, b);
}
__device__ __forceinline__ float wave_max(float v) { return wave_all(v, [](float a, float b) { return vmax(a, b); }); }
__device__ __forceinline__ double wave_sum(double v) { return wave_all(v, [](double a, double b) { return a + b; }); }

// A segment of a row: each lane's largest logit that may be selected, and, alike in all lanes, the segment's
// largest logit and sum.
struct Segment {
  float best, top;
  double sum;
};
template <bool BF, int VPT>
__device__ __forceinline__ Segment scan(const BeamArgs& a, int64_t row, int seg, const uint2* table) {
  using L = Logits<BF>;
  constexpr int EL = L::EL, SEG = WAVE * VPT * EL;
  const int lane = threadIdx.x % WAVE, V = a.b.vocab;
  const typename L::T* const p = static_cast<const typename L::T*>(a.b.logits) + row * a.b.ld;
  const int v0 = seg * SEG + lane * EL;   // of load i: + i 64 EL
  float z[VPT][EL];
  typename L::piece w[VPT];
  if (seg * SEG + SEG <= V) {
#pragma unroll
    for (int i = 0; i < VPT; ++i)
      w[i] = *reinterpret_cast<const typename L::piece*>(p + v0 + i * WAVE * EL);
  } else if (V >= EL) {
    // the row ends in this segment: its last 16 bytes in place of those that pass it, moved to where they would stand
#pragma unroll
    for (int i = 0; i < VPT; ++i)
      w[i] = *reinterpret_cast<const typename L::piece*>(p + min(v0 + i * WAVE * EL, V - EL));
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
      const int past = v0 + i * WAVE * EL - (V - EL);   // tokens
      const auto bits = __builtin_bit_cast(unsigned __int128, w[i]);
      w[i] = __builtin_bit_cast(typename L::piece, past > 0 ? bits >> (past < EL ? past * (128 / EL) : 127) : bits);
    }
  } else {
#pragma unroll
    for (int i = 0; i < VPT; ++i) w[i] = (typename L::piece){0, 0, 0, 0};
    if (v0 < V)
      for (int v = 0; v < V; ++v) {   // (the first lane has them all)
        const uint32_t u = __float_as_uint(L::one(p + v));
        w[0][BF ? v / 2 : v] |= !BF || v % 2 ? u : u >> 16;
      }
  }
#pragma unroll
  for (int i = 0; i < VPT; ++i) {
#pragma unroll
    for (int e = 0; e < EL; ++e)
      z[i][e] = __uint_as_float(!BF ? w[i][e] : e % 2 ? w[i][e / 2] & 0xFFFF0000u : w[i][e / 2] << 16);
  }
  // the largest and the least, NaN where one is; what is no finite number is not there
  float top = z[0][0], low = z[0][0];
#pragma unroll
  for (int i = 0; i < VPT; ++i)
#pragma unroll
    for (int e = 0; e < EL; ++e) {
      top = vmax(top, z[i][e]);
      low = __builtin_elementwise_minimum(low, z[i][e]);
    }
  const bool odd = !(top < INFINITY && low > -INFINITY);
  if (seg * SEG + SEG > V || __any(odd)) {
    top = NONE;
    low = -INFINITY;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int e = 0; e < EL; ++e) {
        z[i][e] = v0 + i * WAVE * EL + e < V && __builtin_isfinite(z[i][e]) ? z[i][e] : NONE;
        top = vmax(top, z[i][e]);
      }
  }
  Segment r;
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
  top = wave_max(top);
  r.top = top;
  double s = 0.0;
  const double m = top;
  if (__all(low >= top - 700.f && __builtin_fabsf(top) < 16384.f)) {
    // the usual sizes: exp(z) against 2^(N / 64) next to exp(m), two instructions less for each
    const double N = __builtin_rint(m * LOG2E_64), R = ROUND - N;
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int e = 0; e < EL; ++e) {
        const double x = z[i][e], k = __builtin_fma(x, LOG2E_64, R);
        s = add_exp2(s, __builtin_fma(x, LOG2E_64, -(k - R)), k, table);
      }
    s *= add_exp2(0.0, __builtin_fma(m, -LOG2E_64, N), ROUND, table);
  } else if (top > NONE) {
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
      for (int e = 0; e < EL; ++e) s += weight(z[i][e], m, table);
  }
  r.sum = wave_sum(s);
  return r;
}

// Waves take segments in turn.
template <bool BF, int VPT>
__global__ __launch_bounds__(256) void beam_scan_kernel(BeamArgs a) {
  __shared__ uint2 table[64];
  load_table(table);
  const int lane = threadIdx.x % WAVE, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int64_t all = int64_t(a.b.num_requests) * a.b.beams * a.segs;
  for (int64_t at = int64_t(blockIdx.x) * 4 + wave; at < all; at += int64_t(gridDim.x) * 4) {
    const int64_t row = at / a.segs;
    if ((a.b.done && a.b.done[row]) || (a.b.score && !__builtin_isfinite(a.b.score[row]))) continue;
    const Segment r = scan<BF, VPT>(a, row, int(at % a.segs), table);
    a.best[at * WAVE + lane] = r.best;
    const float b = wave_max(r.best);
    if (lane == 0) {
      a.seg_sum[at] = r.sum;
      a.seg_top[at] = r.top;
      a.seg_best[at] = b;
    }
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
constexpr int BIN_BITS = 11, BINS = 1 << BIN_BITS;
constexpr int CAP = 2048;     // continuations that are put in order at last
constexpr int LIST = 4096;    // segments, and then groups, that may hold some of the best

static_assert(BINS == 2 * PICK && TAV2_K_MAX <= PICK && TAV2_BEAMS_MAX <= PICK && TAV2_K_MAX <= CAP,
              "two bins, a place, a beam for each thread; room for all that is asked for");

struct PickShared {
  double base[TAV2_BEAMS_MAX];   // score - log S; a finished beam's score; NaN: no beam
  float top[TAV2_BEAMS_MAX];     // the largest logit (of a finished beam: anything)
  bool ended[TAV2_BEAMS_MAX];    // finished
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
  uint2 table[64];
};

// The bin that the `need`-th from the top is in (BINS: there are fewer), and how many lie in the bins above it.
__device__ __forceinline__ void find_bin(PickShared& sh, uint32_t need) {
  const int tid = threadIdx.x, lane = tid % WAVE, wid = tid / WAVE;
  const uint32_t c0 = sh.bins[BINS - 1 - 2 * tid], c1 = sh.bins[BINS - 2 - 2 * tid];
  // the sum over the lanes up to this one: within sixteen by shifts of 1, 2, 4 and 8 (0x110 + n), then from lane 15 of each
  // sixteen to the next (0x142), and from lane 31 to the upper half (0x143)
  uint32_t v = c0 + c1;
  v += __builtin_amdgcn_update_dpp(0, int(v), 0x111, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, int(v), 0x112, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, int(v), 0x114, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, int(v), 0x118, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, int(v), 0x142, 0xA, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, int(v), 0x143, 0xC, 0xF, false);
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
  lo = wave_all(lo, [](uint32_t a, uint32_t b) { return min(a, b); });
  hi = wave_all(hi, [](uint32_t a, uint32_t b) { return max(a, b); });
  if (tid % WAVE == 0) {
    sh.wmin[tid / WAVE] = lo;
    sh.wmax[tid / WAVE] = hi;
  }
  for (int i = tid; i < BINS; i += PICK) sh.bins[i] = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < NW; ++w) {
    lo = min(lo, sh.wmin[w]);
    hi = max(hi, sh.wmax[w]);
  }
  if (hi == 0) return 1;
  uint32_t above = 0;
  while (true) {
    const int shift = max(0, 32 - __builtin_clz(hi - lo | 1) - BIN_BITS);
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
    for (int i = tid; i < BINS; i += PICK) sh.bins[i] = 0;
    __syncthreads();
  }
}

// A beam's base, from its score, its row's largest logit and its sum of exponentials.
__device__ __forceinline__ double base_of(float s, bool ended, float top, double sum) {
  if (!__builtin_isfinite(s)) return __builtin_nan("");
  if (ended) return s;
  return top > NONE ? double(s) - log(sum) : __builtin_nan("");
}
// What the token of logit z is worth.
__device__ __forceinline__ double worth(double base, float top, float z) { return base + (double(z) - double(top)); }

// What a segment or a group of beam b holds at best, of which z is the largest logit; a finished beam's one
// continuation counts as its first one's.
__device__ __forceinline__ uint32_t best_key(double base, float top, bool done, bool first, float z) {
  if (done) return first && base == base ? near_key(base) : 0;
  return base == base && z > NONE ? near_key(worth(base, top, z)) : 0;
}

// The selection of a request, whose bases and largest logits are in sh.  visit(f) calls f(key, group) for the groups that hold all of the
// best; a group is (beam * segments + segment) * 64 + lane.
template <bool BF, class Visit>
__device__ __forceinline__ void pick(const BeamArgs& a, PickShared& sh, int64_t row0, uint32_t bound, bool fits, Visit visit) {
  constexpr int EL = Logits<BF>::EL;
  const int B = a.b.beams, V = a.b.vocab, K = a.keep, S = a.segs;
  const int tid = threadIdx.x, lane = tid % WAVE, wid = __builtin_amdgcn_readfirstlane(tid / WAVE);
  const int eos0 = a.b.eos < 0 ? 0 : a.b.eos;
  const uint32_t total = uint32_t(B) * uint32_t(V);   // below 2^31
  // the key of beam b continued by v
  auto key_of = [&](int b, int v) -> uint64_t {
    const double x = sh.base[b];
    if (x != x) return 0;
    if (sh.ended[b]) return v == eos0 ? value_key(x) : 0;
    const float z = logit<BF>(a, row0 + b, v);
    if (!(z > NONE)) return 0;
    if (a.b.allowed && !(a.b.allowed[(row0 + b) * a.b.allowed_ld + v / 8] >> (v % 8) & 1)) return 0;
    return value_key(worth(x, sh.top[b], z));
  };
  auto list = [&](uint64_t k, uint32_t flat) {
    const uint32_t at = atomicAdd(&sh.n, 1u);
    if (at < CAP) {
      sh.keys[at] = k;
      sh.flats[at] = flat;
    }
  };
  uint32_t n_groups = 0;
  auto list_groups = [&]() {
    if (tid == 0) sh.n = 0;
    __syncthreads();
    visit([&](uint32_t k, uint32_t g) {
      if (k < bound) return;
      const uint32_t at = atomicAdd(&sh.n, 1u);
      if (at < LIST) sh.groups[at] = g;
    });
    __syncthreads();
    n_groups = sh.n;
    __syncthreads();
  };
  // (the groups' own bound where the segments' leaves too many, or there is none)
  if (fits && bound > 1) list_groups();
  if (fits && (bound == 1 || n_groups > 2 * uint32_t(K) + 64)) {
    bound = max(bound, bound_of(sh, [&](auto f) { visit([&](uint32_t k, uint32_t) { f(k); }); }, K, K + K / 8));
    list_groups();
  }
  if (fits) {
    fits = n_groups <= LIST;
    if (tid == 0) sh.n = 0;
    __syncthreads();
    if (fits) {
      // a lane a token, four at once, so that their loads are on the way together
      const int size = a.vpt * EL;   // of a group: 4 .. 64, a power of two; tokens of one load are neighbours
      const int each = WAVE / size, mine = lane / size, i = lane % size / EL, e = lane % EL;
      for (uint32_t k0 = wid * each + mine; k0 - mine < n_groups; k0 += 4 * NW * each) {
        int beam[4], v[4];
        float z[4];
        uint32_t ok[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint32_t k = k0 + u * NW * each;
          const uint32_t g = sh.groups[min(k, n_groups - 1)], s = g / WAVE;
          beam[u] = int(s / S);
          v[u] = (int(s % S) * a.vpt + i) * (WAVE * EL) + int(g % WAVE) * EL + e;
          if (k >= n_groups || v[u] >= V) v[u] = -1;
          const int at = max(v[u], 0);
          z[u] = logit<BF>(a, row0 + beam[u], at);
          ok[u] = a.b.allowed ? a.b.allowed[(row0 + beam[u]) * a.b.allowed_ld + at / 8] >> (at % 8) & 1 : 1;
        }
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const double c = worth(sh.base[beam[u]], sh.top[beam[u]], z[u]);
          if (sh.ended[beam[u]]) {
            if (lane % size == 0 && k0 + u * NW * each < n_groups)
              list(value_key(sh.base[beam[u]]), uint32_t(beam[u]) * V + eos0);
          } else if (v[u] >= 0 && ok[u] && z[u] > NONE && near_key(c) >= bound) {
            list(value_key(c), uint32_t(beam[u]) * V + v[u]);
          }
        }
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
  // sixteen threads each, which look at every sixteenth
  for (uint32_t i0 = 0; i0 < n; i0 += PICK / 16) {
    const uint32_t i = min(i0 + tid / 16, n - 1), f = sh.flats[i];
    const uint64_t k = sh.keys[i];
    uint32_t rank = 0;
#pragma unroll 4
    for (uint32_t j = tid % 16; j < n; j += 16) {
      const uint64_t kj = sh.keys[j];
      rank += kj > k || (kj == k && sh.flats[j] < f);
    }
    rank += lane_move<0xB1>(rank);
    rank += lane_move<0x4E>(rank);
    rank += lane_move<0x141>(rank);
    rank += lane_move<0x140>(rank);
    if (tid % 16 == 0 && i0 + tid / 16 < n && rank < uint32_t(K)) {
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
  const bool was = p >= 0 && sh.ended[p];
  a.token[at] = p < 0 ? -1 : was ? a.b.eos : sh.token[tid];
  a.score[at] = p < 0 ? -INFINITY : fmaxf(float(sh.value[tid]), -FLT_MAX);
  if (a.done) a.done[at] = p >= 0 && (was || (a.b.eos >= 0 && sh.token[tid] == a.b.eos));
}

// A workgroup a request, whose segments the first launch took.
template <bool BF>
__global__ __launch_bounds__(PICK) void beam_pick_kernel(BeamArgs a) {
  __shared__ PickShared sh;
  const int B = a.b.beams, K = a.keep, S = a.segs;
  const int tid = threadIdx.x, lane = tid % WAVE, wid = __builtin_amdgcn_readfirstlane(tid / WAVE);
  const int64_t row0 = int64_t(blockIdx.x) * B;
  // (all that does not depend on anything is on the way first; what a finished beam's rows hold is not used)
  const bool ended = tid < B && a.b.done && a.b.done[row0 + tid];
  const float score = tid < B && a.b.score ? a.b.score[row0 + tid] : 0.f;
  const float* const seg_best = a.seg_best + row0 * S;
  const float* const best = a.best + row0 * S * WAVE;
  load_table(sh.table);
  // (the segments' best logits are on the way while the bases are found)
  const uint32_t segs = uint32_t(B) * uint32_t(S);
  const bool held = segs <= 4 * PICK;
  float seg_z[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) seg_z[e] = held && tid + e * PICK < segs ? seg_best[tid + e * PICK] : NONE;
  // the beams' largest logits and sums, a wave two beams at once; then their bases, a thread a beam
  for (int b0 = wid; b0 < B; b0 += 2 * NW) {
    float top[2], m[2];
    double sum[2], z[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int b = min(b0 + u * NW, B - 1);
      top[u] = lane < S ? a.seg_top[(row0 + b) * S + lane] : NONE;
      sum[u] = lane < S ? a.seg_sum[(row0 + b) * S + lane] : 0.0;
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int b = min(b0 + u * NW, B - 1);
      const float* const tops = a.seg_top + (row0 + b) * S;
      const double* const sums = a.seg_sum + (row0 + b) * S;
      m[u] = top[u];
      for (int i = lane + WAVE; i < S; i += WAVE) m[u] = vmax(m[u], tops[i]);
      m[u] = wave_max(m[u]);
      z[u] = sum[u] * weight(top[u], m[u], sh.table);
      for (int i = lane + WAVE; i < S; i += WAVE) z[u] += sums[i] * weight(tops[i], m[u], sh.table);
      z[u] = wave_sum(z[u]);
      if (lane == 0 && b0 + u * NW < B) {
        sh.base[b] = z[u];
        sh.top[b] = m[u];
      }
    }
  }
  __syncthreads();
  if (tid < B) {
    sh.base[tid] = base_of(score, ended, sh.top[tid], sh.base[tid]);
    sh.ended[tid] = ended;
  }
  __syncthreads();

  auto seg_key = [&](uint32_t i, float z) -> uint32_t {
    const int b = int(i / S);
    return best_key(sh.base[b], sh.top[b], sh.ended[b], i % S == 0, z);
  };
  uint32_t bound = 1, seg_keys[4];
#pragma unroll
  for (int e = 0; e < 4; ++e)
    seg_keys[e] = held && tid + e * PICK < segs ? seg_key(tid + e * PICK, seg_z[e]) : 0;
  if (segs >= 2 * uint32_t(K)) {
    bound = bound_of(sh, [&](auto f) {
      if (held) {
#pragma unroll
        for (int e = 0; e < 4; ++e) f(seg_keys[e]);
      } else {
        for (uint32_t i = tid; i < segs; i += PICK) f(seg_key(i, seg_best[i]));
      }
    }, K, K + K / 4);
  }
  if (tid == 0) sh.n = 0;
  __syncthreads();
  auto list_segment = [&](uint32_t i, uint32_t key) {
    if (key < bound) return;
    const uint32_t at = atomicAdd(&sh.n, 1u);
    if (at < LIST) sh.segs[at] = i;
  };
  if (held) {
#pragma unroll
    for (int e = 0; e < 4; ++e) list_segment(tid + e * PICK, seg_keys[e]);
  } else {
    for (uint32_t i = tid; i < segs; i += PICK) list_segment(i, seg_key(i, seg_best[i]));
  }
  __syncthreads();
  const uint32_t n_segs = sh.n;
  __syncthreads();
  auto group_key = [&](uint32_t i) -> uint32_t {
    const int b = int(i / S);
    return best_key(sh.base[b], sh.top[b], sh.ended[b], i % S == 0 && lane == 0, best[int64_t(i) * WAVE + lane]);
  };
  constexpr int HELD = 8;   // segments of a wave whose groups' keys it holds
  if (n_segs <= HELD * NW) {
    uint32_t at[HELD], keys[HELD];
#pragma unroll
    for (int e = 0; e < HELD; ++e) {
      const uint32_t k = wid + e * NW;
      at[e] = k < n_segs ? sh.segs[k] : 0;
      keys[e] = k < n_segs ? group_key(at[e]) : 0;
    }
    pick<BF>(a, sh, row0, bound, true, [&](auto f) {
#pragma unroll
      for (int e = 0; e < HELD; ++e) f(keys[e], at[e] * WAVE + lane);
    });
  } else {
    pick<BF>(a, sh, row0, bound, n_segs <= LIST, [&](auto f) {
#pragma unroll 4
      for (uint32_t k = wid; k < n_segs; k += NW) {
        const uint32_t i = sh.segs[k];
        f(group_key(i), i * WAVE + lane);
      }
    });
  }
}

// Rows of one segment, few enough for one workgroup a request: both in one launch, with nothing between them in memory.
template <bool BF, int VPT, int ROWS>
__global__ __launch_bounds__(PICK) void beam_small_kernel(BeamArgs a) {
  __shared__ PickShared sh;
  const int B = a.b.beams;
  const int lane = threadIdx.x % WAVE, wid = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  const int64_t row0 = int64_t(blockIdx.x) * B;
  const uint8_t* const done = a.b.done ? a.b.done + row0 : nullptr;
  load_table(sh.table);
  uint32_t keys[ROWS];
#pragma unroll
  for (int e = 0; e < ROWS; ++e) {
    const int b = wid + e * NW;
    keys[e] = 0;
    if (b >= B) continue;
    const bool ended = done && done[b];
    const float score = a.b.score ? a.b.score[row0 + b] : 0.f;
    Segment r{NONE, NONE, 0.0};
    if (!ended && __builtin_isfinite(score)) r = scan<BF, VPT>(a, row0 + b, 0, sh.table);
    const double x = base_of(score, ended, r.top, r.sum);
    if (lane == 0) {
      sh.base[b] = x;
      sh.top[b] = r.top;
      sh.ended[b] = ended;
    }
    keys[e] = best_key(x, r.top, ended, lane == 0, r.best);
  }
  __syncthreads();
  pick<BF>(a, sh, row0, 1, true, [&](auto f) {
#pragma unroll
    for (int e = 0; e < ROWS; ++e) f(keys[e], uint32_t(wid + e * NW) * WAVE + lane);
  });
}

// Workgroups of the first launch, at most: as many as run at once.
constexpr int64_t SCANS = 2048;

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
// Of beam_small_kernel: loads a lane, 0: not with these sizes.  One launch and two, us, bf16, requests of 16, 32 and 64 beams.
// 1024 tokens: 1 request 12.5 / 15.9, 15.4 / 17.8, 20.5 / 19.6; 256 requests 14.1 / 18.8, 15.8 / 21.2, 24.1 / 29.8.
// 4096 tokens: 1 request 15.2 / 17.4, 25.3 / 18.1, 43.8 / 20.0; 16 requests 15.7 / 17.9, 25.9 / 18.3, 44.7 / 21.4;
// 64 requests 16.9 / 18.6, 26.7 / 20.4, 45.9 / 29.0; 256 requests 17.3 / 24.4, 30.8 / 32.9, 52.6 / 53.3.  The rule is by what
// many requests take: few requests of more than 16 beams of thousands of tokens would be faster in two.
int small_vectors(const tav2_beams& b) {
  const int el = b.dtype == TAV2_BF16 ? 8 : 4;
  if (b.beams > 4 * NW || b.vocab > WAVE * el * 8) return 0;
  int vpt = 8;
  while (vpt > 1 && b.vocab <= WAVE * el * vpt / 2) vpt /= 2;
  return vpt;
}

template <bool BF>
void launch_scan(const BeamArgs& a, unsigned n, hipStream_t st) {
  if (a.vpt == 8) beam_scan_kernel<BF, 8><<<n, 256, 0, st>>>(a);
  else if (a.vpt == 4) beam_scan_kernel<BF, 4><<<n, 256, 0, st>>>(a);
  else if (a.vpt == 2) beam_scan_kernel<BF, 2><<<n, 256, 0, st>>>(a);
  else beam_scan_kernel<BF, 1><<<n, 256, 0, st>>>(a);
}
template <bool BF, int VPT>
void launch_small(const BeamArgs& a, hipStream_t st) {
  const unsigned n = unsigned(a.b.num_requests);
  if (a.b.beams <= NW) beam_small_kernel<BF, VPT, 1><<<n, PICK, 0, st>>>(a);
  else if (a.b.beams <= 2 * NW) beam_small_kernel<BF, VPT, 2><<<n, PICK, 0, st>>>(a);
  else beam_small_kernel<BF, VPT, 4><<<n, PICK, 0, st>>>(a);
}
template <bool BF>
void launch_small(const BeamArgs& a, hipStream_t st) {
  if (a.vpt == 8) launch_small<BF, 8>(a, st);
  else if (a.vpt == 4) launch_small<BF, 4>(a, st);
  else if (a.vpt == 2) launch_small<BF, 2>(a, st);
  else launch_small<BF, 1>(a, st);
}

}  // namespace

int64_t beam_select_groups(const tav2_beams& b, int keep) {
  if (small_vectors(b)) return int64_t(b.num_requests) * (PICK / 256);
  return std::max<int64_t>(SCANS, int64_t(b.num_requests) * (PICK / 256));
}

size_t beam_select_bytes(const tav2_beams& b, int keep) {
  if (small_vectors(b)) return 0;
  return align_up(size_t(b.num_requests) * b.beams * segments(b) * (8 + 4 + 4 + 4 * WAVE), 256);
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
  if ((a.vpt = small_vectors(b))) {
    a.segs = 1;
    ProfScope prof("beam_pick", st);
    if (b.dtype == TAV2_BF16) launch_small<true>(a, st);
    else launch_small<false>(a, st);
    return hipGetLastError();
  }
  a.vpt = vectors(b);
  a.segs = int(segments(b));
  const size_t n = size_t(b.num_requests) * b.beams * a.segs;
  a.seg_sum = static_cast<double*>(ws);
  a.best = reinterpret_cast<float*>(a.seg_sum + n);
  a.seg_top = a.best + n * WAVE;
  a.seg_best = a.seg_top + n;
  {
    ProfScope prof("beam_scan", st);
    const unsigned groups = unsigned(std::min<int64_t>(SCANS, cdiv(int64_t(n), 4)));
    if (b.dtype == TAV2_BF16) launch_scan<true>(a, groups, st);
    else launch_scan<false>(a, groups, st);
  }
  ProfScope prof("beam_pick", st);
  if (b.dtype == TAV2_BF16) beam_pick_kernel<true><<<unsigned(b.num_requests), PICK, 0, st>>>(a);
  else beam_pick_kernel<false><<<unsigned(b.num_requests), PICK, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace tav2
