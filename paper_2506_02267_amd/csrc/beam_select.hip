// Selection of the best continuations of a request's beams over the vocabulary.
//
// A continuation is worth c = (score - Z) + z, Z the row's log-sum-exp; it is computed in 64 bits, since the values
// of different beams have to be put in order: with an error of 1e-7 two of a request's best would change places
// now and then.
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
  float* row_max;    // [rows]: -inf where a row has no finite logit
  double* row_sum;   // [rows]: of exp(z - max)
};

template <bool BF>
__device__ __forceinline__ float logit(const BeamArgs& a, int64_t row, int v) {
  const int64_t at = row * a.b.ld + v;
  float z;
  if constexpr (BF) z = bf2f(static_cast<const bf16_t*>(a.b.logits)[at]);
  else z = static_cast<const float*>(a.b.logits)[at];
  return __builtin_isfinite(z) ? z : -INFINITY;
}

// 2^t for t <= 0 (any, -inf too), relative error below 2^-36: 2^n times the polynomial of 2^f, |f| <= 1/2, whose
// terms are (f ln 2)^i / i!; the first one left out is below 7e-12.
__device__ __forceinline__ double exp2_neg(double t) {
  t = __builtin_fmax(t, -1100.0);
  const double n = __builtin_rint(t), f = t - n;
  double p = 1.0178086009239696e-07;
  p = __builtin_fma(p, f, 1.3215486790144305e-06);
  p = __builtin_fma(p, f, 1.5252733804059838e-05);
  p = __builtin_fma(p, f, 0.00015403530393381606);
  p = __builtin_fma(p, f, 0.0013333558146428441);
  p = __builtin_fma(p, f, 0.009618129107628477);
  p = __builtin_fma(p, f, 0.055504108664821576);
  p = __builtin_fma(p, f, 0.2402265069591007);
  p = __builtin_fma(p, f, 0.6931471805599453);
  p = __builtin_fma(p, f, 1.0);
  return __builtin_ldexp(p, int(n));
}

constexpr double LOG2E_64 = 1.4426950408889634074;

// A row's largest logit and its sum: a workgroup a row.
template <bool BF>
__global__ __launch_bounds__(256) void beam_scan_kernel(BeamArgs a) {
  __shared__ float top[4];
  __shared__ double part[4];
  const int64_t row = blockIdx.x;
  const int tid = threadIdx.x;
  float m = -INFINITY;
  for (int v = tid; v < a.b.vocab; v += 256) m = fmaxf(m, logit<BF>(a, row, v));
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, WAVE));
  if (tid % WAVE == 0) top[tid / WAVE] = m;
  __syncthreads();
  m = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
  double s = 0.0;
  if (m > -INFINITY)
    for (int v = tid; v < a.b.vocab; v += 256)
      s += exp2_neg((double(logit<BF>(a, row, v)) - double(m)) * LOG2E_64);
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) s += __shfl_xor(s, o, WAVE);
  if (tid % WAVE == 0) part[tid / WAVE] = s;
  __syncthreads();
  if (tid == 0) {
    a.row_max[row] = m;
    a.row_sum[row] = part[0] + part[1] + part[2] + part[3];
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

constexpr int PICK = 1024;    // threads
constexpr int BINS = 2048;
constexpr int CAP = 2048;     // continuations that are put in order at last

// A workgroup a request.
template <bool BF>
__global__ __launch_bounds__(PICK) void beam_pick_kernel(BeamArgs a) {
  constexpr int NW = PICK / WAVE;
  __shared__ double base[TAV2_BEAMS_MAX];     // score - Z; a finished beam's score; NaN: no beam
  __shared__ uint32_t bins[BINS];
  __shared__ uint32_t wsum[NW];
  __shared__ uint64_t keys[CAP];
  __shared__ uint32_t flats[CAP];
  __shared__ uint32_t n_list, s_bin, s_above;
  __shared__ int r_parent[TAV2_K_MAX], r_token[TAV2_K_MAX], first_of[TAV2_BEAMS_MAX];
  __shared__ double r_value[TAV2_K_MAX];
  const int B = a.b.beams, V = a.b.vocab, K = a.keep, tid = threadIdx.x;
  const int64_t row0 = int64_t(blockIdx.x) * B;
  const int eos0 = a.b.eos < 0 ? 0 : a.b.eos;
  for (int b = tid; b < B; b += PICK) {
    const float s = a.b.score ? a.b.score[row0 + b] : 0.f;
    const bool done = a.b.done && a.b.done[row0 + b];
    double x = __builtin_nan("");
    if (__builtin_isfinite(s)) {
      if (done) x = s;
      else if (a.row_max[row0 + b] > -INFINITY)
        x = double(s) - (double(a.row_max[row0 + b]) + log(a.row_sum[row0 + b]));
    }
    base[b] = x;
  }
  __syncthreads();
  // the key of beam b continued by v
  auto key_of = [&](int b, int v) -> uint64_t {
    const double x = base[b];
    if (x != x) return 0;
    if (a.b.done && a.b.done[row0 + b]) return v == eos0 ? value_key(x) : 0;
    const float z = logit<BF>(a, row0 + b, v);
    if (!(z > -INFINITY)) return 0;
    if (a.b.allowed && !(a.b.allowed[(row0 + b) * a.b.allowed_ld + v / 8] >> (v % 8) & 1)) return 0;
    return value_key(x + double(z));
  };
  const uint32_t total = uint32_t(B) * uint32_t(V);   // below 2^31

  // [lo, hi]: keys (then, of one key, flat numbers) among which the K-th lies; `above` continuations are better
  uint64_t lo = 1, hi = ~uint64_t(0);
  uint32_t flo = 0, fhi = total - 1;
  uint32_t above = 0;
  bool by_flat = false;
  while (true) {
    const uint64_t width = by_flat ? fhi - flo : hi - lo;
    int shift = 0;
    while (width >> shift >= BINS) ++shift;
    for (int i = tid; i < BINS; i += PICK) bins[i] = 0;
    __syncthreads();
    for (uint32_t i = tid; i < total; i += PICK) {
      const uint64_t k = key_of(i / V, i % V);
      if (k < lo || k > hi) continue;
      if (by_flat) {
        if (i >= flo && i <= fhi) atomicAdd(&bins[BINS - 1 - ((i - flo) >> shift)], 1u);   // lower ones are better
      } else {
        atomicAdd(&bins[(k - lo) >> shift], 1u);
      }
    }
    __syncthreads();
    // counts of the bins from each one up; the bin that the K-th is in
    const int lane = tid % WAVE, wid = tid / WAVE;
    uint32_t c0 = bins[BINS - 1 - 2 * tid], c1 = bins[BINS - 2 - 2 * tid], v = c0 + c1;
#pragma unroll
    for (int o = 1; o < WAVE; o <<= 1) {
      const uint32_t u = __shfl_up(v, o, WAVE);
      if (lane >= o) v += u;
    }
    if (lane == WAVE - 1) wsum[wid] = v;
    if (tid == 0) s_bin = BINS;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < NW; ++w) before += w < wid ? wsum[w] : 0;
    const uint32_t need = K - above;
    const uint32_t upto = before + v, from = upto - c0 - c1;
    if (from < need && upto >= need) {
      const bool first = from + c0 >= need;
      s_bin = BINS - 1 - 2 * tid - (first ? 0 : 1);
      s_above = first ? from : from + c0;
    }
    __syncthreads();
    if (s_bin == BINS) break;   // fewer than K: all of them
    const uint32_t in = bins[s_bin];
    if (by_flat) {
      const uint32_t from_low = BINS - 1 - s_bin;
      const uint64_t l = flo + (uint64_t(from_low) << shift), h = l + (uint64_t(1) << shift) - 1;
      flo = uint32_t(l);
      fhi = h < fhi ? uint32_t(h) : fhi;
    } else {
      const uint64_t l = lo + (uint64_t(s_bin) << shift), h = l + ((uint64_t(1) << shift) - 1);
      lo = l;
      hi = h < hi ? h : hi;
    }
    above += s_above;
    __syncthreads();
    if (above + in <= CAP) break;
    if (!by_flat && lo == hi) by_flat = true;
    // (a bin of one flat number holds one)
  }
  // those at or above the bin: all of them fit the list
  if (tid == 0) n_list = 0;
  __syncthreads();
  for (uint32_t i = tid; i < total; i += PICK) {
    const uint64_t k = key_of(i / V, i % V);
    if (k < lo || (by_flat && k == lo && i > fhi)) continue;
    const uint32_t at = atomicAdd(&n_list, 1u);
    if (at < CAP) {
      keys[at] = k;
      flats[at] = i;
    }
  }
  __syncthreads();
  const uint32_t n = n_list < CAP ? n_list : CAP;
  for (int k = tid; k < K; k += PICK) r_parent[k] = -1;
  for (int b = tid; b < TAV2_BEAMS_MAX; b += PICK) first_of[b] = TAV2_K_MAX;
  __syncthreads();
  for (uint32_t i = tid; i < n; i += PICK) {
    const uint64_t k = keys[i];
    const uint32_t f = flats[i];
    uint32_t rank = 0;
    for (uint32_t j = 0; j < n; ++j) rank += keys[j] > k || (keys[j] == k && flats[j] < f);
    if (rank < uint32_t(K)) {
      r_parent[rank] = int(f / V);
      r_token[rank] = int(f % V);
      r_value[rank] = key_value(k);
    }
  }
  __syncthreads();
  // (K <= PICK: a thread a place)
  const int p = tid < K ? r_parent[tid] : -1;
  int slot = tid;
  if (a.in_place) {
    if (p >= 0) atomicMin(&first_of[p], tid);
    __syncthreads();
    const bool heads = p >= 0 && first_of[p] == tid;
    // the places of beams that are not continued, in order, for those that do not head a beam's
    const bool later = tid < K && !heads, free = tid < K && first_of[tid] == TAV2_K_MAX;
    const int lane = tid % WAVE, wid = tid / WAVE;
    const uint64_t lb = __ballot(later), fb = __ballot(free), below = (uint64_t(1) << lane) - 1;
    if (lane == 0) wsum[wid] = uint32_t(__popcll(lb)) | uint32_t(__popcll(fb)) << 16;
    __syncthreads();
    uint32_t before = 0;
    for (int w = 0; w < wid; ++w) before += wsum[w];
    const uint32_t nth = (before & 0xFFFF) + __popcll(lb & below), place = (before >> 16) + __popcll(fb & below);
    if (free) bins[place] = tid;
    __syncthreads();
    if (later) slot = int(bins[nth]);
    if (heads) slot = p;
  }
  if (tid >= K) return;
  const int64_t at = int64_t(blockIdx.x) * K + slot;
  a.parent[at] = p;
  const bool was = p >= 0 && a.b.done && a.b.done[row0 + p];
  a.token[at] = p < 0 ? -1 : was ? a.b.eos : r_token[tid];
  float s = -INFINITY;
  if (p >= 0) s = fmaxf(float(r_value[tid]), -3.402823466e38f);
  a.score[at] = s;
  if (a.done) a.done[at] = p >= 0 && (was || (a.b.eos >= 0 && r_token[tid] == a.b.eos));
}

}  // namespace

int64_t beam_select_groups(const tav2_beams& b, int keep) { return int64_t(b.num_requests) * b.beams; }

size_t beam_select_bytes(const tav2_beams& b, int keep) {
  return align_up(size_t(b.num_requests) * b.beams * 12 + 8, 256);
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
  const size_t rows = size_t(b.num_requests) * b.beams;
  a.row_sum = static_cast<double*>(ws);
  a.row_max = reinterpret_cast<float*>(a.row_sum + rows);
  {
    ProfScope prof("beam_scan", st);
    if (b.dtype == TAV2_BF16) beam_scan_kernel<true><<<unsigned(rows), 256, 0, st>>>(a);
    else beam_scan_kernel<false><<<unsigned(rows), 256, 0, st>>>(a);
  }
  ProfScope prof("beam_pick", st);
  const unsigned n = unsigned(b.num_requests);
  if (b.dtype == TAV2_BF16) beam_pick_kernel<true><<<n, PICK, 0, st>>>(a);
  else beam_pick_kernel<false><<<n, PICK, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace tav2
