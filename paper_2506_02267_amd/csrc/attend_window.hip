// Causal attention of packed sequences with a window and sink tokens.
//
// A workgroup takes 128 consecutive (position, head) rows of one kv head of a sequence; its four waves
// (or eight, below) share each 64-key tile through LDS: keys as rows, values by feature (two keys a 32-bit
// word, turned while they are written).  The next tile's loads are in flight while the present one is
// multiplied, one barrier a tile.  Tiles that no row of the workgroup sees are not
// visited, and a wave skips those that none of its own sees, so the work is that of the window.
// Bound by the vector units: an exponential, a scaling, a maximum, a sum and a rounding for each
// score, beside 4 D matrix operations; the two add up, as the three waves a SIMD (four with the kernel of
// eight waves) seldom meet in different ones.  16384 tokens with a window of 1024, 4 heads of 64: 34 us (13 at
// a large product's rate); 32 sequences of 203 - 4000 tokens, 4 heads on 2: 143 us (73).
#include <algorithm>

#include "attend_core.h"
#include "internal.h"

namespace tav2 {

namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int TK = 64;   // keys of a tile (bf16)
constexpr int ROWS = 128;   // rows of a workgroup, 32 a wave
// Workgroups up to which a second four waves take the other half of each tile's keys: few ones leave
// SIMDs idle.  Both sides, us: 512 workgroups, 16384 tokens whole 227 and 291, with a window of 1024 35.0
// and 38.4, 4 x 4096 62.8 and 78.5; 1024, 8 x 4096 108.7 and 104; some 2000 (32 histories of 203 - 4000 tokens)
// 155 and 147; 4096, 64 x 2048 with a window of 512 151 and 136.
constexpr int64_t SPLIT_GROUPS = 768;
constexpr int BUNDLE = 4;   // tiles of a sequence that are neighbours on an XCD (rows_of)

struct WindowArgs {
  tav2_window a;
  float scale;
  int tiles;   // row tiles per (sequence, kv head)
};

// Rows of this workgroup, (position, head) pairs: from row0 on of a sequence's `rows`; `len` tokens from row `off`.
struct Rows {
  int64_t off;
  int len, rows, row0, h, G;
};

__device__ __forceinline__ bool rows_of(const WindowArgs& w, int per, Rows& r) {
  const tav2_window& a = w.a;
  // The rows with the most keys first.  Workgroups go to the 8 XCDs in turn: BUNDLE neighbouring tiles of
  // a sequence go to the same one together, where they read the same keys at about the same time, the
  // next of them to another (with a sequence's tiles all on one, some XCDs ended long after the others: 32
  // sequences of 203 - 4000 tokens 287 us for 168).  Bundles of 1, 2, 4, 8 and 16, us: 8 sequences in fp32 21.2,
  // 20.0, 19.4, 19.8, 20.1; 8 x 4096 tokens in bf16 103.8, 99.9, 100.5, 105.8, 110.
  const int units = a.num_requests * a.kv_heads;
  const int slot = int(blockIdx.x) / 8;
  const int bundle = slot / BUNDLE * 8 + int(blockIdx.x) % 8;
  const int turn = bundle / units * BUNDLE + slot % BUNDLE;
  const int unit = (bundle + bundle / units) % units;
  const int tile = w.tiles - 1 - turn;
  if (tile < 0) return false;
  const int s = unit / a.kv_heads;
  r.h = unit % a.kv_heads;
  r.G = a.heads / a.kv_heads;
  r.off = a.offset[s];
  r.len = a.len[s] < a.max_len ? a.len[s] : a.max_len;
  r.rows = r.len * r.G;
  r.row0 = tile * per;
  return r.row0 < r.rows;
}

// The tiles that positions lo .. hi see: [0, sink) and [first, last).
struct Tiles {
  int sink, first, last;
  __device__ __forceinline__ int count() const { return sink + last - first; }
  __device__ __forceinline__ int at(int i) const { return i < sink ? i : first + i - sink; }
};
__device__ __forceinline__ Tiles tiles_seen(int lo, int hi, int window, int sinks, int tk) {
  Tiles t;
  t.last = hi / tk + 1;
  t.first = window > 0 && lo >= window ? (lo - window + 1) / tk : 0;
  t.sink = window > 0 ? min(int((int64_t(sinks) + tk - 1) / tk), t.first) : 0;
  return t;
}

// What a wave's rows see of the tile at k0: 0 nothing, 1 some, 2 all of it.
__device__ __forceinline__ int tile_seen(int k0, int tk, int lo, int hi, int window, int sinks) {
  if (k0 > hi) return 0;
  if (window > 0 && int64_t(k0) + tk + window <= int64_t(lo) + 1 && k0 >= sinks) return 0;
  const bool low = window == 0 || int64_t(k0) + window > hi || int64_t(k0) + tk <= sinks;
  return low && k0 + tk - 1 <= lo ? 2 : 1;
}

// The row of a half tile's operand that key k is (key_row's inverse).
__device__ __forceinline__ int operand_row(int k) { return 8 * ((k >> 2) & 3) + 4 * (k >> 4 & 1) + (k & 3); }

template <int D, bool SPLIT>
__global__ __launch_bounds__(SPLIT ? 512 : 256, SPLIT && D <= 64 ? 4 : 2) void attend_window_bf16(WindowArgs w) {
  constexpr int CH = D / 8;                       // 16-byte pieces of a row
  constexpr int NK = TK * CH / 256;               // pieces of K per thread
  constexpr int NV = (TK / 2 * CH + 255) / 256;   // pairs of pieces of V per thread
  // Rows of 16 bytes more than their numbers take, so that the 8 neighbouring rows that lanes read together
  // begin 4 banks apart; keys in the order of the operand's rows; a feature's 16-byte pieces of
  // keys xor'ed by feature / 8, so that the writes of 8 features by 8 lanes do not meet either.
  // Addresses are fixed and constants.
  constexpr int KS = D * 2 + 16, VS = TK * 2 + 16;
  __shared__ __align__(16) uint8_t lds[2 * (TK * KS + D * VS)];
  auto lk = [&](int buf) { return lds + buf * (TK * KS); };
  auto lv = [&](int buf) { return lds + 2 * TK * KS + buf * (D * VS); };
  Rows r;
  if (!rows_of(w, ROWS, r)) return;
  const tav2_window& a = w.a;
  const int tid = threadIdx.x, lane = tid % WAVE, m = lane % 32, half = lane / 32;
  // (scalar, for scalar branches; with SPLIT the second four waves take the same rows, and each four
  // one half of a tile's keys)
  const int wave = __builtin_amdgcn_readfirstlane(tid / WAVE) % 4;
  const int part = SPLIT ? __builtin_amdgcn_readfirstlane(tid / 256) : 0;
  const int wrow0 = r.row0 + wave * 32;
  const bf16_t* kb = static_cast<const bf16_t*>(a.k) + r.off * a.k_ld + r.h * D;
  const bf16_t* vb = static_cast<const bf16_t*>(a.v) + r.off * a.v_ld + r.h * D;

  bf16x8 qf[1][D / 16];
  AttSeen<1> seen;
  seen.sinks = a.sinks;
  {
    const int row = min(wrow0 + m, r.rows - 1);
    const int pos = row / r.G;
    const bf16_t* p = static_cast<const bf16_t*>(a.q) + (r.off + pos) * a.q_ld +
                      (r.h * r.G + row % r.G) * D + half * (D / 2);
#pragma unroll
    for (int t = 0; t < D / 16; ++t) qf[0][t] = as_bf16x8(*reinterpret_cast<const uint4*>(p + 8 * t));
    seen.hi[0] = pos + 1;
    seen.lo[0] = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
  }
  const int last_row = min(r.row0 + ROWS, r.rows) - 1;
  const Tiles tiles = tiles_seen(r.row0 / r.G, last_row / r.G, a.window, a.sinks, TK);
  const bool idle = wrow0 >= r.rows;
  const int wlo = wrow0 / r.G, whi = min(wrow0 + 31, r.rows - 1) / r.G;

  // A thread's pieces of a tile, as byte offsets from the tile's first row: fixed but for a sequence's
  // last tile, where rows past the end become its last one (their weights are 0).  With SPLIT the first
  // four waves bring the values, the others the keys.
  constexpr int NP = SPLIT ? 2 * NV : NK + 2 * NV;
  constexpr int VP = SPLIT ? 0 : NK;   // the first of the values' pieces
  const int t256 = tid % 256;
  u32x4 piece[NP];
  uint32_t from[NP];
  auto offsets = [&](int last) {
#pragma unroll
    for (int i = 0; i < (SPLIT ? NP : NK); ++i) {
      if (SPLIT && part == 0) break;
      const int e = (t256 + 256 * i) % (TK * CH);
      from[i] = (uint32_t(min(e / CH, last)) * uint32_t(a.k_ld) + e % CH * 8) * 2;
    }
#pragma unroll
    for (int i = 0; i < 2 * NV; ++i) {
      if (SPLIT && part == 1) break;
      const int e = (t256 + 256 * (i / 2)) % (TK / 2 * CH);   // (32 features: the second half again)
      from[VP + i] = (uint32_t(min(e / CH * 2 + i % 2, last)) * uint32_t(a.v_ld) + e % CH * 8) * 2;
    }
  };
  offsets(TK - 1);
  auto load = [&](int k0) {
    if (k0 + TK > r.len) offsets(r.len - 1 - k0);   // (the last tile visited)
    const char* kt = reinterpret_cast<const char*>(kb + int64_t(k0) * a.k_ld);
    const char* vt = reinterpret_cast<const char*>(vb + int64_t(k0) * a.v_ld);
    if (SPLIT && part == 0) kt = vt;
#pragma unroll
    for (int i = 0; i < NP; ++i)
      piece[i] = *reinterpret_cast<const u32x4*>((SPLIT || i < NK ? kt : vt) + from[i]);
  };
  // and its places in LDS
  uint32_t sk[SPLIT ? NP : NK], sv[NV];
#pragma unroll
  for (int i = 0; i < (SPLIT ? NP : NK); ++i) {
    const int e = (t256 + 256 * i) % (TK * CH), k = e / CH;
    sk[i] = (k / 32 * 32 + operand_row(k % 32)) * KS + e % CH * 16;
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int e = (t256 + 256 * i) % (TK / 2 * CH);
    sv[i] = e % CH * 8 * VS + (((e / CH) / 4) ^ (e % CH % 8)) * 16 + (e / CH) % 4 * 4;
  }
  auto store = [&](int buf) {
    if (!SPLIT || part == 1) {
#pragma unroll
      for (int i = 0; i < (SPLIT ? NP : NK); ++i) *reinterpret_cast<u32x4*>(lk(buf) + sk[i]) = piece[i];
    }
    if (!SPLIT || part == 0) {
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int f = 0; f < 8; ++f)
          *reinterpret_cast<uint32_t*>(lv(buf) + sv[i] + f * VS) =
              __builtin_amdgcn_perm(piece[VP + 2 * i + 1][f / 2], piece[VP + 2 * i][f / 2],
                                    f % 2 ? 0x07060302u : 0x05040100u);
    }
  };
  // where this lane reads its operands: key row, features; feature row, keys
  // (with SPLIT, of the wave's half)
  const uint32_t ak = (32 * part + m) * KS + half * D;
  uint32_t av[2][2];   // [keys' half, xor features' parity of 32][keys 8 t ..]
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int t = 0; t < 2; ++t) av[x][t] = m * VS + ((4 * (x ^ part) + 2 * half + t) ^ (m / 8)) * 16;

  AttState<D, 1> st;
  st.clear();
  const float c[1] = {w.scale * LOG2E};
  const int n = tiles.count();
  load(tiles.at(0) * TK);
  store(0);
  __syncthreads();
  int i = 0;
  do {   // (a row sees itself: there is a tile)
    const int k0 = tiles.at(i) * TK, buf = i & 1;
    if (i + 1 < n) load(tiles.at(i + 1) * TK);
    const int see = idle ? 0 : tile_seen(k0, TK, wlo, whi, a.window, a.sinks);
    if (see) {
      const uint8_t* const kl = lk(buf) + ak;
      const uint8_t* const vl = lv(buf);
      // With 128 features both halves of the tile at once: one look at the reference for 64 keys, and longer
      // runs of products (8 x 4096 tokens of 4 heads 176 us for 187); with fewer the halves in turn, in fewer
      // registers (64 x 2048 tokens with a window of 512 128 us for 131; 32 features 133 for 139).
      constexpr int NB = !SPLIT && D == 128 ? 2 : 1;
#pragma unroll
      for (int u0 = 0; u0 < (SPLIT ? 1 : 2); u0 += NB) {
        auto keys = [&](int b, bf16x8(&kf)[D / 16]) {
          const int u = u0 + b;
#pragma unroll
          for (int t = 0; t < D / 16; ++t)
            kf[t] = as_bf16x8(*reinterpret_cast<const uint4*>(kl + 32 * u * KS + 16 * t));
        };
        auto values = [&](int b, bf16x8(&vf)[D / 32][2]) {
          const int u = u0 + b;
#pragma unroll
          for (int d = 0; d < D / 32; ++d)
#pragma unroll
            for (int t = 0; t < 2; ++t)
              vf[d][t] = as_bf16x8(*reinterpret_cast<const uint4*>(vl + 32 * d * VS + av[u ^ (d & 1)][t]));
        };
        att_step<bf16x8, NB, D, 1>(st, keys, values, qf, c, AttNoScale(), see == 1, seen,
                                   k0 + 32 * (u0 + part) + 16 * half);
      }
    }
    if (i + 1 < n) store(buf ^ 1);
    __syncthreads();
  } while (++i < n);
  if constexpr (SPLIT) {   // the second halves' states, through the tiles' LDS, into the first's
    static_assert(4 * (D / 32) * 16 * WAVE * 4 <= int(sizeof(lds)), "they fit");
    __shared__ float ml[4][2][WAVE];
    float* const their = reinterpret_cast<float*>(lds) + wave * (D / 32) * 16 * WAVE + lane;
    if (part == 1) {
      ml[wave][0][lane] = st.m[0];
      ml[wave][1][lane] = st.l[0];
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
#pragma unroll
        for (int e = 0; e < 16; ++e) their[(d * 16 + e) * WAVE] = st.o[d][0][e];
    }
    __syncthreads();
    if (part == 1) return;
    const float m2 = ml[wave][0][lane], M = m2 > st.m[0] ? m2 : st.m[0];
    const float f1 = __builtin_amdgcn_exp2f(st.m[0] - M), f2 = __builtin_amdgcn_exp2f(m2 - M);
    st.m[0] = M;
    st.l[0] = st.l[0] * f1 + ml[wave][1][lane] * f2;
#pragma unroll
    for (int d = 0; d < D / 32; ++d)
#pragma unroll
      for (int e = 0; e < 16; ++e) st.o[d][0][e] = st.o[d][0][e] * f1 + their[(d * 16 + e) * WAVE] * f2;
  }
  const int row = wrow0 + m;
  const float l = xsum32(st.l[0]);
  if (row >= r.rows) return;
  const int64_t at = (r.off + row / r.G) * a.heads + r.h * r.G + row % r.G;
  const float inv = 1.f / l;   // a row sees itself: l > 0
  bf16_t* out = static_cast<bf16_t*>(a.out) + at * D + 4 * half;
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<uint2*>(out + 32 * d + 8 * j) =
          make_uint2(pack2(st.o[d][0][4 * j] * inv, st.o[d][0][4 * j + 1] * inv),
                     pack2(st.o[d][0][4 * j + 2] * inv, st.o[d][0][4 * j + 3] * inv));
  if (a.lse && half == 0) a.lse[at] = (st.m[0] + __builtin_amdgcn_logf(l)) * LN2;
}

// fp32, on 32x32x2 fp32 products (the weights are operands as they are): a workgroup takes 32 rows,
// and its four waves take the 32-key tiles in turn, each through its own part of LDS, so that no wave
// waits for another until their states meet at the end.  8 sequences of 57 - 1000 tokens, a window of 200, 8 heads
// of 32: 19 us, the few tiles of a row one after the other (35 with 128 rows a workgroup); 4 x 2000 tokens of
// 64 features: 98 us for 160.  With 128 features a workgroup's LDS and registers fill a CU: 4 x 1000 - 2000 tokens, 4 heads
// on 2, 140 us.
constexpr int TF = 32;
constexpr int ROWS_F32 = 32;

template <int D>
__global__ __launch_bounds__(256, D <= 64 ? 2 : 1) void attend_window_f32(WindowArgs w) {
  constexpr int LS = D + 4;                 // an LDS row (floats)
  constexpr int CH = D / 4, NC = TF * CH / WAVE;
  __shared__ __align__(16) float lds[4][2 * TF * LS];
  __shared__ float ml[4][2][WAVE];
  Rows r;
  if (!rows_of(w, ROWS_F32, r)) return;
  const tav2_window& a = w.a;
  const int tid = threadIdx.x, lane = tid % WAVE, m = lane % 32, half = lane / 32;
  const int wave = __builtin_amdgcn_readfirstlane(tid / WAVE);   // (scalar branches)
  float* const lk = lds[wave];              // keys in the order of the operand's rows
  float* const lv = lk + TF * LS;           // values as they lie
  const float* kb = static_cast<const float*>(a.k) + r.off * a.k_ld + r.h * D;
  const float* vb = static_cast<const float*>(a.v) + r.off * a.v_ld + r.h * D;
  const int row = min(r.row0 + m, r.rows - 1), pos = row / r.G;
  f32x4 qf[D / 8];
  AttSeen<1> seen;
  seen.sinks = a.sinks;
  {
    const float* p = static_cast<const float*>(a.q) + (r.off + pos) * a.q_ld +
                     (r.h * r.G + row % r.G) * D + half * (D / 2);
#pragma unroll
    for (int t = 0; t < D / 8; ++t) qf[t] = *reinterpret_cast<const f32x4*>(p + 4 * t);
    seen.hi[0] = pos + 1;
    seen.lo[0] = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
  }
  const int lo = r.row0 / r.G, hi = (min(r.row0 + ROWS_F32, r.rows) - 1) / r.G;
  const Tiles tiles = tiles_seen(lo, hi, a.window, a.sinks, TF);
  f32x4 gk[NC], gv[NC];
  auto load = [&](int k0) {
#pragma unroll
    for (int i = 0; i < NC; ++i) {
      const int e = lane + WAVE * i, key = min(k0 + e / CH, r.len - 1), ch = e % CH * 4;
      gk[i] = *reinterpret_cast<const f32x4*>(kb + int64_t(key) * a.k_ld + ch);
      gv[i] = *reinterpret_cast<const f32x4*>(vb + int64_t(key) * a.v_ld + ch);
    }
  };
  AttState<D, 1> st;
  st.clear();
  const float c = w.scale * LOG2E;
  const int n = tiles.count();
  if (wave < n) load(tiles.at(wave) * TF);
  for (int i = wave; i < n; i += 4) {
    const int k0 = tiles.at(i) * TF;
    // (a wave's LDS operations are done in order; the barriers keep the compiler to it)
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int j = 0; j < NC; ++j) {
      const int e = lane + WAVE * j, key = e / CH, ch = e % CH * 4;
      *reinterpret_cast<f32x4*>(lk + operand_row(key) * LS + ch) = gk[j];
      *reinterpret_cast<f32x4*>(lv + key * LS + ch) = gv[j];
    }
    __builtin_amdgcn_wave_barrier();
    if (i + 4 < n) load(tiles.at(i + 4) * TF);
    f32x16 sc[1], &s = sc[0];
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
    const float* kr = lk + m * LS + half * (D / 2);
#pragma unroll
    for (int t = 0; t < D / 8; ++t) {
      const f32x4 k4 = *reinterpret_cast<const f32x4*>(kr + 4 * t);
#pragma unroll
      for (int e = 0; e < 4; ++e) s = __builtin_amdgcn_mfma_f32_32x32x2f32(k4[e], qf[t][e], s, 0, 0, 0);
    }
    att_softmax(st, 0, sc, c, AttNoScale(), tile_seen(k0, TF, lo, hi, a.window, a.sinks) != 2, seen,
                         k0 + 16 * half);
    const float* vr = lv + 16 * half * LS + m;
#pragma unroll
    for (int t = 0; t < 16; ++t)
#pragma unroll
      for (int d = 0; d < D / 32; ++d)
        st.o[d][0] = __builtin_amdgcn_mfma_f32_32x32x2f32(vr[t * LS + 32 * d], s[t], st.o[d][0], 0, 0, 0);
  }
  // the waves' states meet in LDS; wave w joins registers 4w .. 4w + 3 of each tile, in the order of the
  // waves: features 8w + 4 half .. of it
  __builtin_amdgcn_wave_barrier();
  static_assert(D / 32 * 16 * WAVE <= 2 * TF * LS, "a state fits");
  ml[wave][0][lane] = st.m[0];
  ml[wave][1][lane] = xsum32(st.l[0]);
#pragma unroll
  for (int d = 0; d < D / 32; ++d)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      reinterpret_cast<f32x4*>(lds[wave])[(d * 4 + j) * WAVE + lane] =
          (f32x4){st.o[d][0][4 * j], st.o[d][0][4 * j + 1], st.o[d][0][4 * j + 2], st.o[d][0][4 * j + 3]};
  __syncthreads();
  if (r.row0 + m >= r.rows) return;
  float M = -FLT_MAX, l = 0.f, f[4];
#pragma unroll
  for (int x = 0; x < 4; ++x) M = vmax(M, ml[x][0][lane]);
#pragma unroll
  for (int x = 0; x < 4; ++x) {
    f[x] = __builtin_amdgcn_exp2f(ml[x][0][lane] - M);
    l += ml[x][1][lane] * f[x];
  }
  const int64_t at = (r.off + pos) * a.heads + r.h * r.G + row % r.G;
  const float inv = 1.f / l;   // a row sees itself: l > 0
  float* out = static_cast<float*>(a.out) + at * D + 8 * wave + 4 * half;
#pragma unroll
  for (int d = 0; d < D / 32; ++d) {
    f32x4 o = (f32x4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int x = 0; x < 4; ++x) o += reinterpret_cast<const f32x4*>(lds[x])[(d * 4 + wave) * WAVE + lane] * f[x];
    *reinterpret_cast<f32x4*>(out + 32 * d) = o * inv;
  }
  if (a.lse && wave == 0 && half == 0) a.lse[at] = (M + __builtin_amdgcn_logf(l)) * LN2;
}

int rows_per_group(const tav2_window& a) { return a.dtype == TAV2_F32 ? ROWS_F32 : ROWS; }

}  // namespace

int64_t attend_window_groups(const tav2_window& a) {
  const int64_t tiles = cdiv(int64_t(a.max_len) * (a.heads / a.kv_heads), rows_per_group(a));
  return cdiv(int64_t(a.num_requests) * a.kv_heads * cdiv(tiles, BUNDLE), 8) * 8 * BUNDLE;
}

hipError_t launch_attend_window(const tav2_window& a, hipStream_t st) {
  WindowArgs w;
  w.a = a;
  w.scale = a.scale > 0.f ? a.scale : 1.f / sqrtf(float(a.head_dim));
  w.tiles = int(cdiv(int64_t(a.max_len) * (a.heads / a.kv_heads), rows_per_group(a)));
  const unsigned grid = unsigned(attend_window_groups(a));
  ProfScope prof("attend_window", st);
  if (a.dtype == TAV2_F32) {
    if (a.head_dim == 32) attend_window_f32<32><<<grid, 256, 0, st>>>(w);
    else if (a.head_dim == 64) attend_window_f32<64><<<grid, 256, 0, st>>>(w);
    else attend_window_f32<128><<<grid, 256, 0, st>>>(w);
  } else {
    const bool split = int64_t(a.num_requests) * a.kv_heads * w.tiles <= SPLIT_GROUPS;
    if (a.head_dim == 32 && split) attend_window_bf16<32, true><<<grid, 512, 0, st>>>(w);
    else if (a.head_dim == 32) attend_window_bf16<32, false><<<grid, 256, 0, st>>>(w);
    else if (a.head_dim == 64 && split) attend_window_bf16<64, true><<<grid, 512, 0, st>>>(w);
    else if (a.head_dim == 64) attend_window_bf16<64, false><<<grid, 256, 0, st>>>(w);
    else if (split) attend_window_bf16<128, true><<<grid, 512, 0, st>>>(w);
    else attend_window_bf16<128, false><<<grid, 256, 0, st>>>(w);
  }
  return hipGetLastError();
}

}  // namespace tav2
