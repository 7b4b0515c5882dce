// INT2 codes of the packed records as fp16 matrix-core operands.
#pragma once

#include "common.h"

namespace int2kv {

typedef _Float16 cd_h2_t __attribute__((ext_vector_type(2)));
typedef _Float16 cd_h8_t __attribute__((ext_vector_type(8)));
typedef __bf16 cd_b8_t __attribute__((ext_vector_type(8)));
typedef float cd_f16_t __attribute__((ext_vector_type(16)));
typedef uint32_t cd_u2_t __attribute__((ext_vector_type(2)));
typedef uint32_t cd_u4_t __attribute__((ext_vector_type(4)));

// A constant in a vector register: with its mask in a scalar one, AND and OR are one instruction (which takes one scalar)
__device__ __forceinline__ uint32_t in_vgpr(uint32_t x) {
  asm("" : "+v"(x));
  return x;
}
__device__ __forceinline__ uint32_t in_sgpr(uint32_t x) {
  asm("" : "+s"(x));
  return x;
}

// The codes at bits X, X + 1 of a word's two 16-bit halves as two fp16 numbers. In an fp16 number of exponent 10 - X
// mantissa bit X weighs 1, so the code bits joined with 2^(10 - X) make 2^(10 - X) + code, and the subtraction is exact.
template <int X>
__device__ __forceinline__ cd_h2_t land_codes(uint32_t w) {
  static_assert(X >= 0 && X <= 8, "the codes have to lie in the ten mantissa bits");
  constexpr uint32_t mask = (3u << X) * 0x10001u, magic = ((25u - X) << 10) * 0x10001u;
  const cd_h2_t base = {(_Float16)(float)(1 << (10 - X)), (_Float16)(float)(1 << (10 - X))};
  return __builtin_bit_cast(cd_h2_t, (w & in_sgpr(mask)) | in_vgpr(magic)) - base;
}

// The codes of position p (0..7) of a word's two halves: channels 16 p + m of halves m = 2 w, 2 w + 1. `hi` is w >> 10.
template <int P>
__device__ __forceinline__ cd_h2_t land_position(uint32_t w, uint32_t hi) {
  if constexpr (P < 5)
    return land_codes<2 * P>(w);
  else
    return land_codes<2 * P - 10>(hi);
}

// An fp16 number in both halves
__device__ __forceinline__ cd_h2_t both_lo(uint32_t sz) { return __builtin_bit_cast(cd_h2_t, __builtin_amdgcn_perm(sz, sz, 0x01000100u)); }
__device__ __forceinline__ cd_h2_t both_hi(uint32_t sz) { return __builtin_bit_cast(cd_h2_t, __builtin_amdgcn_perm(sz, sz, 0x03020302u)); }

// The two operands that one word of a token's row makes: operand o holds positions 4 o .. 4 o + 3, element 2 i + e
// channel 16 (4 o + i) + 2 w + e. s, z: the token's scale and zero of each group in both halves of a pair; each value is
// code * s + z with one rounding to fp16.
template <int NG>
__device__ __forceinline__ void word_operands(uint32_t w, const cd_h2_t (&s)[NG], const cd_h2_t (&z)[NG], cd_h8_t (&out)[2]) {
  const uint32_t hi = w >> 10;
  cd_h2_t v[8];
#define INT2KV_POS(P) v[P] = __builtin_elementwise_fma(land_position<P>(w, hi), s[P * NG / 8], z[P * NG / 8]);
  INT2KV_POS(0) INT2KV_POS(1) INT2KV_POS(2) INT2KV_POS(3) INT2KV_POS(4) INT2KV_POS(5) INT2KV_POS(6) INT2KV_POS(7)
#undef INT2KV_POS
#pragma unroll
  for (int o = 0; o < 2; ++o)
#pragma unroll
    for (int i = 0; i < 4; ++i) out[o][2 * i] = v[4 * o + i].x, out[o][2 * i + 1] = v[4 * o + i].y;
}

// Channel of element j of operand kk (0..7) in lane half hh: lane half hh of a token holds words 4 hh .. 4 hh + 3 of its
// row, operand kk takes positions 4 (kk % 2) .. of word 4 hh + kk / 2.
__host__ __device__ __forceinline__ int code_channel(int kk, int hh, int j) {
  return 16 * (4 * (kk & 1) + (j >> 1)) + 2 * (4 * hh + (kk >> 1)) + (j & 1);
}

// Eight numbers rounded to fp16; bf16 numbers as fp16 ones (exact within fp16's normal range)
__device__ __forceinline__ cd_h8_t pack_half8(const float* x) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  cd_h8_t y;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const cd_h2_t p = __builtin_convertvector((f2{x[2 * i], x[2 * i + 1]}), cd_h2_t);
    y[2 * i] = p.x, y[2 * i + 1] = p.y;
  }
  return y;
}
__device__ __forceinline__ cd_h8_t half_of(const cd_b8_t& x) {
  float y[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = (float)x[i];
  return pack_half8(y);
}

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f2{a, b}), b2));
}

}  // namespace int2kv
