// New tokens into the 8-bit cache: full blocks to their pages, the rest to the tail.
//
// A wave takes one block of one sequence and head, keys or values: 64 tokens x D features, read once
// (bf16, 16 bytes a lane and load), codes and scale written once.  A lane holds 8 features of 4, 8 or
// 16 consecutive tokens, so that both orders of codes (by token for keys, by feature for
// values) are whole words of its own: no LDS, no barrier, the largest magnitude from lane exchanges.
// Bound by HBM: 2 bytes read and 1 written per value.
#include "common.h"
#include "internal.h"
#include "kv_common.h"
#include "token_source.h"

namespace tav2 {

namespace {

constexpr float KV_TINY = 0x1p-100f;   // blocks whose magnitudes are all below it are zeros

struct AppendArgs {
  tav2_kv c;
  int layer;
  const bf16_t* x[2];   // keys, values
  int64_t ld[2];
  const int64_t* offset;
  int max_count;
  int blocks;           // units' blocks per sequence
};

__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 8; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, WAVE));
  return xmax32(xmax16(v));
}

// The word of codes of 4 values.  A code is 127 x / top rounded half to even, exactly: scaled by the
// power of two that takes top into [2, 4), 127 x (f127 = 127 times that power) has 15 significant
// bits and is exact; q, the quotient by an approximate reciprocal, is off by at most 2^-22 of
// itself, while a quotient that is no half is at least 2^-17 of itself away from the next one; and
// where it is a half, the exact remainder (first fma) corrects q to it.  Adding 1.5 2^23 rounds
// to a whole number, whose lowest byte is the code.
__device__ __forceinline__ uint32_t codes4(const float (&x)[4], float f127, float top, float inv) {
  uint32_t b[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a = x[i] * f127;
    const float q = a * inv;
    const float r = __builtin_fmaf(-q, top, a);
    b[i] = __float_as_uint(__builtin_fmaf(r, inv, q) + 12582912.f);
  }
  const uint32_t lo = __builtin_amdgcn_perm(b[1], b[0], 0x0c0c0400u);
  const uint32_t hi = __builtin_amdgcn_perm(b[3], b[2], 0x0c0c0400u);
  return lo | hi << 16;
}

__device__ __forceinline__ float half_of(uint32_t w, int i) {   // bf16 i of a word
  return __uint_as_float(i ? w & 0xFFFF0000u : w << 16);
}

template <int D>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a) {
  constexpr int CH = D / 8;        // lanes to a token's row
  constexpr int NT = KVP * CH / WAVE;   // consecutive tokens per lane: 4, 8, 16
  const tav2_kv& c = a.c;
  const int H = c.kv_heads;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / WAVE);
  int64_t u = int64_t(blockIdx.x) * 4 + wave;
  const int h = int(u % H);
  u /= H;
  const int side = int(u % 2);
  u /= 2;
  const int j = int(u % a.blocks), s = int(u / a.blocks);
  if (s >= c.num_seqs) return;
  const int now = kv_len(c, s);
  int n_new = ld_meta(c.fresh + s);
  n_new = n_new < 0 ? 0 : n_new > now ? now : n_new;
  const int old = now - n_new;
  const int end = old + (n_new < a.max_count ? n_new : a.max_count);   // (max_count bounds fresh)
  const int b = old / KVP + j;
  if (n_new == 0 || b > end / KVP || (j > 0 && b == end / KVP)) return;

  const int lane = threadIdx.x % WAVE, c8 = lane % CH * 8, t0 = lane / CH * NT;
  const int64_t ld = a.ld[side];
  // the row of position p, this lane's features
  const bf16_t* rows = a.x[side] + (ld_meta(a.offset + s) - old) * ld + h * D + c8;
  bf16_t* tail = (side ? c.v_tail : c.k_tail) + kv_tail(c, a.layer, s, h);
  if (b < end / KVP) {   // a full block: to its page
    const int page = ld_meta(c.table + int64_t(s) * c.max_blocks + b);
    uint4 w[NT];
    if (b * KVP >= old) {
#pragma unroll
      for (int i = 0; i < NT; ++i)
        w[i] = *reinterpret_cast<const uint4*>(rows + int64_t(b * KVP + t0 + i) * ld);
    } else {   // begun before: its first tokens lie in the tail
#pragma unroll
      for (int i = 0; i < NT; ++i) {
        const int t = t0 + i;
        if (b * KVP + t >= old) {
          w[i] = *reinterpret_cast<const uint4*>(rows + int64_t(b * KVP + t) * ld);
        } else if (side == 0) {
          w[i] = *reinterpret_cast<const uint4*>(tail + t * D + c8);
        } else {
          uint32_t x[4];
#pragma unroll
          for (int f = 0; f < 4; ++f)
            x[f] = tail[(c8 + 2 * f) * KVP + t] | uint32_t(tail[(c8 + 2 * f + 1) * KVP + t]) << 16;
          w[i] = make_uint4(x[0], x[1], x[2], x[3]);
        }
      }
    }
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < NT; ++i) {
      const uint32_t x[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
      for (int f = 0; f < 4; ++f)
        top = fmaxf(top, fmaxf(__builtin_fabsf(half_of(x[f], 0)), __builtin_fabsf(half_of(x[f], 1))));
    }
    top = wave_max(top);
    const bool zero = !(top >= KV_TINY);
    if (page >= 0 && page < c.pages) {
      const int64_t unit = kv_unit(c, a.layer, page, h);
      if (lane == 0) (side ? c.v_scale : c.k_scale)[unit] = zero ? 1.f : top / 127.f;
      // into [2, 4) by a power of two (what leaves the normal range has code 0); zeros: all codes 0
      const float f = zero ? 0.f : __uint_as_float((255u - (__float_as_uint(top) >> 23)) << 23);
      const float topn = zero ? 1.f : top * f, inv = 1.f / topn, f127 = 127.f * f;
      if (side == 0) {
        int8_t* d = c.k + unit * KVP * D + t0 * D + c8;
#pragma unroll
        for (int i = 0; i < NT; ++i) {
          const float lo[4] = {half_of(w[i].x, 0), half_of(w[i].x, 1), half_of(w[i].y, 0), half_of(w[i].y, 1)};
          const float hi[4] = {half_of(w[i].z, 0), half_of(w[i].z, 1), half_of(w[i].w, 0), half_of(w[i].w, 1)};
          *reinterpret_cast<uint2*>(d + i * D) =
              make_uint2(codes4(lo, f127, topn, inv), codes4(hi, f127, topn, inv));
        }
      } else {
        int8_t* d = c.v + unit * KVP * D + c8 * KVP + t0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          uint32_t q[NT / 4];
#pragma unroll
          for (int i = 0; i < NT; i += 4) {
            float x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const uint32_t y[4] = {w[i + k].x, w[i + k].y, w[i + k].z, w[i + k].w};
              x[k] = half_of(y[e / 2], e % 2);
            }
            q[i / 4] = codes4(x, f127, topn, inv);
          }
          __builtin_memcpy(__builtin_assume_aligned(d + e * KVP, NT), q, NT);
        }
      }
    }
  }
  // the new open block: written by the wave of the first block, the only one that reads the old
  // one (its loads have returned: the largest magnitude came from them)
  if (j == 0) {
    const int p0 = end / KVP * KVP + t0;
#pragma unroll 1
    for (int i = 0; i < NT; ++i) {
      if (p0 + i >= end || p0 + i < old) continue;
      const uint4 w = *reinterpret_cast<const uint4*>(rows + int64_t(p0 + i) * ld);
      if (side == 0) {
        *reinterpret_cast<uint4*>(tail + (t0 + i) * D + c8) = w;
      } else {
        const uint32_t x[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int f = 0; f < 8; ++f)
          tail[(c8 + f) * KVP + t0 + i] = bf16_t(f % 2 ? x[f / 2] >> 16 : x[f / 2]);
      }
    }
  }
}

}  // namespace

int64_t kv_append_groups(const tav2_kv& c, int max_count) {
  return cdiv(int64_t(c.num_seqs) * cdiv(max_count, KVP) * c.kv_heads * 2, 4);
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
