// What the kernels of the chunk attention share: the units of a context, the order of tokens in the products, scores to
// probabilities.
#pragma once

#include "codes.h"
#include "common.h"
#include "kernels.h"

namespace int2kv {

constexpr int kUnit = 64;                     // tokens of a unit: two 32-token halves, four pages
constexpr int kUnitPages = kUnit / kBlock;
constexpr float kLogit2 = 1.4426950408889634f * 0.08838834764831845f;  // log2(e) / sqrt(128)
constexpr float kLazy = 8.0f;   // the running maximum moves when a score exceeds it by 2^8
constexpr float kBias = 7.0f;   // probabilities are held times 2^7: the largest is below 2^15, and fp16's normal range
                                // reaches 2^-21 below the maximum
constexpr float kNone = -1.0e30f;  // running maximum of a row that has seen nothing
constexpr float kMove = kBias + kLazy;

// Row m of S^T's 32-token half is token 16 (m / 16) + row_token(m % 16): registers 8 p .. 8 p + 7 of a lane half hh are
// then tokens 8 hh .. 8 hh + 7 of page p, which lie side by side in the records.
__device__ __forceinline__ int row_token(int m) { return (m & 3) | ((m & 4) << 1) | ((m & 8) >> 1); }
// The token (of its half) of register i, without the lane half's 8
__device__ __forceinline__ constexpr int reg_token(int i) { return 16 * (i >> 3) + (i & 7); }

struct Seq {
  int start, n, ctx;
};
__device__ __forceinline__ Seq seq_of(const ChunkArgs& a, int b) {
  Seq s;
  s.start = min(max(a.starts[b], 0), a.total_q);
  const int end = min(max(a.starts[b + 1], 0), a.total_q);
  s.n = min(max(end - s.start, 0), a.max_q);
  const long long room = (long long)a.max_blocks * kBlock;
  s.ctx = min(max(a.lens[b], 0), (int)(room < a.max_ctx ? room : a.max_ctx));
  return s;
}
// Units of a tile whose last new token is i: INT2 units, then units of the chunk's own tokens
__device__ __forceinline__ int int2_units(const ChunkArgs& a, const Seq& s, int i) {
  const int lim = a.k_new ? s.ctx : min(s.ctx, max(0, s.ctx - s.n + i + 1));
  return (lim + kUnit - 1) / kUnit;
}
__device__ __forceinline__ int own_units(const ChunkArgs& a, int i) { return a.k_new ? i / kUnit + 1 : 0; }

__device__ __forceinline__ cd_f16_t splat16(float x) {
  cd_f16_t v;
#pragma unroll
  for (int r = 0; r < 16; ++r) v[r] = x;
  return v;
}
// max / sum over a lane and its partner (lane ^ 32)
__device__ __forceinline__ float pair_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float pair_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// fp16 operands: INT2 units. The rotated queries carry log2(e) / sqrt(128), so scores are base-2 logarithms as they are.
struct HalfOps {
  typedef cd_h8_t vec;
  static __device__ __forceinline__ cd_f16_t mfma(const cd_h8_t& a, const vec& b, const cd_f16_t& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ float start(float base) { return base; }
  static __device__ __forceinline__ float score(float s, float) { return s; }
  static __device__ __forceinline__ uint32_t pack(float a, float b, float& sum) {
    typedef float f2 __attribute__((ext_vector_type(2)));
    const cd_h2_t p = __builtin_convertvector((f2{a, b}), cd_h2_t);
    sum = __builtin_amdgcn_fdot2(p, cd_h2_t{(_Float16)1.0f, (_Float16)1.0f}, sum, false);
    return __builtin_bit_cast(uint32_t, p);
  }
  // the halves of a pair that are not finite
  static __device__ __forceinline__ uint32_t odd(uint32_t x) {
    return ((x & 0x7C00u) == 0x7C00u ? 0xFFFFu : 0u) | ((x & 0x7C000000u) == 0x7C000000u ? 0xFFFF0000u : 0u);
  }
};
// bf16 operands: the chunk's own units, whose scores are scaled in fp32
struct BfOps {
  typedef cd_b8_t vec;
  static __device__ __forceinline__ cd_f16_t mfma(const cd_h8_t& a, const vec& b, const cd_f16_t& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(cd_b8_t, a), b, c, 0, 0, 0);
  }
  static __device__ __forceinline__ float start(float) { return 0.0f; }
  static __device__ __forceinline__ float score(float s, float base) { return __builtin_fmaf(s, kLogit2, base); }
  static __device__ __forceinline__ uint32_t pack(float a, float b, float& sum) {
    sum += a + b;
    return pack_bf16(a, b);
  }
  static __device__ __forceinline__ uint32_t odd(uint32_t x) {
    return ((x & 0x7F80u) == 0x7F80u ? 0xFFFFu : 0u) | ((x & 0x7F800000u) == 0x7F800000u ? 0xFFFF0000u : 0u);
  }
};

// Moves m where a score of the step exceeds it by 2^kLazy (the lane's own scores and its partner's)
template <class Ops, int TILES>
__device__ __forceinline__ void settle(cd_f16_t& X, float& base, float& m, float& sum, float& thr, cd_f16_t (&O)[TILES]) {
  float a = fmaxf(X[0], X[1]);
#pragma unroll
  for (int i = 2; i < 16; i += 2) a = fmaxf(fmaxf(a, X[i]), X[i + 1]);
  const float top = Ops::score(pair_max(a), base);
  const bool move = top > thr;
  if (__any(move)) {
    const float d = move ? top - kBias : 0.0f;
    const float f = !move ? 1.0f : thr < 0.0f ? 0.0f : __builtin_amdgcn_exp2f(-d);
    m += d;
    base -= d;
    sum *= f;
    thr = move ? kMove : thr;
#pragma unroll
    for (int i = 0; i < TILES; ++i) O[i] *= f;
    X -= splat16(Ops::start(d));
  }
}
// Probabilities of a step as operands: page pg of the half takes registers 8 pg .. 8 pg + 7
template <class Ops>
__device__ __forceinline__ void soften(const cd_f16_t& X, float base, float& sum, cd_u4_t (&P)[2]) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    P[i >> 2][i & 3] =
        Ops::pack(__builtin_amdgcn_exp2f(Ops::score(X[2 * i], base)), __builtin_amdgcn_exp2f(Ops::score(X[2 * i + 1], base)), sum);
}
// An operand with all but element j of the lanes that hold token t of a page cleared
__device__ __forceinline__ cd_u4_t only_token(cd_u4_t x, int t) {
  const bool has = ((threadIdx.x >> 5) & 1) == (uint32_t)((t >> 3) & 1);
  const int j = t & 7;
#pragma unroll
  for (int y = 0; y < 4; ++y) x[y] = has && y == (j >> 1) ? x[y] & (j & 1 ? 0xFFFF0000u : 0xFFFFu) : 0u;
  return x;
}

}  // namespace int2kv
