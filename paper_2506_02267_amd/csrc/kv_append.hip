// New tokens into the 8-bit cache: full blocks to their pages, the rest to the tail.
//
// A workgroup takes one block of one sequence and head, keys or values: 64 tokens x D features, read
// once (bf16), its largest magnitude found, codes and scale written once.  Bound by HBM: 2 bytes
// read and 1 written per value.
#include "common.h"
#include "internal.h"
#include "kv_common.h"

namespace tav2 {

namespace {

constexpr float KV_TINY = 7.8886090522101181e-31f;   // 2^-100: blocks below it are zeros

struct AppendArgs {
  tav2_kv c;
  int layer;
  const bf16_t* x[2];   // keys, values
  int64_t ld[2];
  const int64_t* offset;
  int max_count;
  int blocks;           // grid's blocks per sequence
};

// 127 x / top rounded half to even, exactly.  x and top are bf16 values scaled so that top lies in
// [2, 4): 127 x has 15 significant bits.  n is the nearest whole number to an approximate
// quotient, so at most one off where the true one is near a half; the remainder
// e = 127 x - n top is exact (whole multiples of x's last place, below 2^24 of them), and says
// which side it is on.
__device__ __forceinline__ int kv_code(float x, float top, float inv) {
  const float a = 127.f * x;
  float n = __builtin_rintf(a * inv);
  const float e = __builtin_fmaf(-n, top, a);
  const float twice = 2.f * __builtin_fabsf(e);
  const bool odd = int(n) & 1;
  if (twice > top || (twice == top && odd)) n += e > 0.f ? 1.f : -1.f;
  return int(n);
}

template <int D>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a) {
  constexpr int F = D / 4;                 // features per thread: a quarter of a token's
  constexpr int LDT = KVP + 4;             // LDS row of codes by feature (bytes)
  __shared__ float wmax[4];
  __shared__ __align__(16) int8_t codes[D * LDT];
  const tav2_kv& c = a.c;
  const int H = c.kv_heads;
  int64_t u = blockIdx.x;
  const int side = int(u % 2);
  u /= 2;
  const int h = int(u % H);
  u /= H;
  const int j = int(u % a.blocks), s = int(u / a.blocks);
  const int now = kv_len(c, s);
  int n_new = c.fresh[s];
  n_new = n_new < 0 ? 0 : n_new > now ? now : n_new;
  const int old = now - n_new;
  const int end = old + (n_new < a.max_count ? n_new : a.max_count);   // (max_count bounds fresh)
  const int b = old / KVP + j;
  if (n_new == 0 || b > end / KVP || (j > 0 && b == end / KVP)) return;

  const int tid = threadIdx.x, t = tid / 4, f0 = (tid % 4) * F;
  const bf16_t* src = a.x[side];
  const int64_t ld = a.ld[side], row0 = a.offset[s];
  bf16_t* tail = (side ? c.v_tail : c.k_tail) + kv_tail(c, a.layer, s, h);
  const int pos = b * KVP + t;
  __align__(16) bf16_t x[F];
  auto load = [&](const bf16_t* p) {
#pragma unroll
    for (int i = 0; i < F; i += 8) __builtin_memcpy(x + i, __builtin_assume_aligned(p + i, 16), 16);
  };
  auto load_new = [&](int p) { load(src + (row0 + p - old) * ld + h * D + f0); };
  if (b < end / KVP) {   // a full block: to its page
    if (pos >= old) {
      load_new(pos);
    } else if (side == 0) {
      load(tail + t * D + f0);
    } else {
#pragma unroll
      for (int i = 0; i < F; ++i) x[i] = tail[(f0 + i) * KVP + t];
    }
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < F; ++i) top = fmaxf(top, __builtin_fabsf(bf2f(x[i])));
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, WAVE));
    if (tid % WAVE == 0) wmax[tid / WAVE] = top;
    __syncthreads();
    top = fmaxf(fmaxf(wmax[0], wmax[1]), fmaxf(wmax[2], wmax[3]));
    const bool zero = !(top >= KV_TINY);
    const int page = c.table[int64_t(s) * c.max_blocks + b];
    if (page >= 0 && page < c.pages) {   // (uniform)
      const int64_t unit = kv_unit(c, a.layer, page, h);
      if (tid == 0) (side ? c.v_scale : c.k_scale)[unit] = zero ? 1.f : top / 127.f;
      // by a power of two into [2, 4): exact (what leaves the normal range has code 0)
      const uint32_t ex = __float_as_uint(top) >> 23;
      const float f = __uint_as_float((255u - ex) << 23);
      const float topn = top * f, inv = 1.f / topn;
      int q[F];
#pragma unroll
      for (int i = 0; i < F; ++i) q[i] = zero ? 0 : kv_code(bf2f(x[i]) * f, topn, inv);
      if (side == 0) {
        uint32_t w[F / 4];
#pragma unroll
        for (int i = 0; i < F / 4; ++i)
          w[i] = (q[4 * i] & 0xFF) | (q[4 * i + 1] & 0xFF) << 8 | (q[4 * i + 2] & 0xFF) << 16 |
                 uint32_t(q[4 * i + 3]) << 24;
        uint32_t* d = reinterpret_cast<uint32_t*>(c.k + unit * KVP * D + t * D + f0);
#pragma unroll
        for (int i = 0; i < F / 4; ++i) d[i] = w[i];
      } else {   // by feature, through LDS
#pragma unroll
        for (int i = 0; i < F; ++i) codes[(f0 + i) * LDT + t] = int8_t(q[i]);
        __syncthreads();
        for (int e = tid; e < D * KVP / 4; e += 256)
          reinterpret_cast<uint32_t*>(c.v + unit * KVP * D)[e] =
              *reinterpret_cast<const uint32_t*>(codes + (e / 16) * LDT + (e % 16) * 4);
      }
    }
    __syncthreads();   // the old tail has been read
  }
  // the new open block: written by the workgroup of the first block, the only one that read
  // the old one
  if (j == 0) {
    const int p = end / KVP * KVP + t;
    if (p < end && p >= old) {
      load_new(p);
      if (side == 0) {
        bf16_t* d = tail + t * D + f0;
#pragma unroll
        for (int i = 0; i < F; i += 8) __builtin_memcpy(__builtin_assume_aligned(d + i, 16), x + i, 16);
      } else {
#pragma unroll
        for (int i = 0; i < F; ++i) tail[(f0 + i) * KVP + t] = x[i];
      }
    }
  }
}

}  // namespace

int64_t kv_append_groups(const tav2_kv& c, int max_count) {
  return int64_t(c.num_seqs) * cdiv(max_count, KVP) * c.kv_heads * 2;
}

hipError_t launch_kv_append(const tav2_kv& c, int layer, const void* k, int64_t k_ld, const void* v,
                            int64_t v_ld, const int64_t* offset, int max_count, hipStream_t st) {
  AppendArgs a{};
  a.c = c;
  a.layer = layer;
  a.x[0] = static_cast<const bf16_t*>(k);
  a.x[1] = static_cast<const bf16_t*>(v);
  a.ld[0] = k_ld;
  a.ld[1] = v_ld;
  a.offset = offset;
  a.max_count = max_count;
  // blocks that max_count tokens can fill, or the first of them
  a.blocks = int(cdiv(max_count, KVP));
  const unsigned grid = unsigned(kv_append_groups(c, max_count));
  ProfScope prof("kv_append", st);
  switch (c.head_dim) {
    case 32: kv_append_kernel<32><<<grid, 256, 0, st>>>(a); break;
    case 64: kv_append_kernel<64><<<grid, 256, 0, st>>>(a); break;
    default: kv_append_kernel<128><<<grid, 256, 0, st>>>(a); break;
  }
  return hipGetLastError();
}

}  // namespace tav2
