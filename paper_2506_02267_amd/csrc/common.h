// Device helpers shared by the gfx950 kernels of the NN-select + encode path.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t bf16_t;   // raw bf16 storage

namespace tav2 {

constexpr int WAVE = 64;

// Partner values across lane halves without LDS: the gfx950 permlane swaps of a
// register with itself leave {v[l], v[l ^ 32]} (or {v[l], v[l ^ 16]}) in the pair.
// Maximum without NaN quieting (gfx950 v_maximum3_f32): fmaxf's IEEE semantics
// make the compiler canonicalize every operand that is not the result of an
// arithmetic instruction (MFMA results, lane swaps), one extra instruction each.
// The operands here are finite or -inf.
__device__ __forceinline__ float vmax(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float xmax32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                  false);
  return vmax(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float xmax16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                  false);
  return vmax(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float xsum32(float v) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                  false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}
__device__ __forceinline__ float xsum16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false,
                                                  false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// v moved around within sixteen lanes by N, on the vector unit.
template <int N>
__device__ __forceinline__ float ror16(float v) {
  return __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), 0x120 + N, 0xF, 0xF, true));
}
// v joined by op with those of the lanes of the same sixteen that lie a multiple of `step` (1, 2, 4, 8 or 16) away.
template <class Op>
__device__ __forceinline__ float steps16(float v, int step, Op op) {
  if (step <= 8) v = op(v, ror16<8>(v));
  if (step <= 4) v = op(v, ror16<4>(v));
  if (step <= 2) v = op(v, ror16<2>(v));
  if (step <= 1) v = op(v, ror16<1>(v));
  return v;
}

__device__ __forceinline__ float bf2f(bf16_t b) { return __uint_as_float(uint32_t(b) << 16); }

// float -> bf16, round to nearest even (inputs are finite).
__device__ __forceinline__ bf16_t f2bf(float f) {
  uint32_t u = __float_as_uint(f);
  u += 0x7FFFu + ((u >> 16) & 1u);
  return bf16_t(u >> 16);
}

// 32x32x16 bf16 MFMA, fp32 accumulate.  Operand layout (lane l, h = l / 32):
//   A[32 x 16]: row l % 32, k = 8h .. 8h+7;  B[16 x 32]: column l % 32, k = 8h .. 8h+7;
//   D[32 x 32]: column l % 32, register r = 4j + i holds row 8j + 4h + i.
__device__ __forceinline__ f32x16 mfma32(const bf16x8& a, const bf16x8& b, const f32x16& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ bf16x8 as_bf16x8(const uint4& v) {
  return __builtin_bit_cast(bf16x8, v);
}
__device__ __forceinline__ bf16x8 as_bf16x8(const uint2& lo, const uint2& hi) {
  uint4 v = make_uint4(lo.x, lo.y, hi.x, hi.y);
  return __builtin_bit_cast(bf16x8, v);
}
// Two floats -> packed bf16 pair (a in the low half), round to nearest even: the
// gfx950 conversion instruction, one per pair.  (A vector conversion: two scalar
// conversions are not always merged, e.g. when the pair feeds packed 16-bit
// arithmetic, and then cost two conversions and a permute.)
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){a, b}, bf16x2_t));
}

// Order-preserving 32-bit key of an fp32 score: larger score <=> larger key,
// -0.0 maps to the key of +0.0.  Key 0 lies below every finite score and -inf.
__device__ __forceinline__ uint32_t score_key(float s) {
  uint32_t u = __float_as_uint(s);
  if (u == 0x80000000u) u = 0u;
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float key_score(uint32_t k) {
  uint32_t u = (k & 0x80000000u) ? (k & 0x7FFFFFFFu) : ~k;
  return __uint_as_float(u);
}

__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, WAVE);
  return v;
}
__device__ __forceinline__ int wave_sum_i(int v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, WAVE);
  return v;
}

__host__ __device__ __forceinline__ int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }
__host__ __device__ __forceinline__ size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

}  // namespace tav2
