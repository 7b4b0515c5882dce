// Rows read back from the INT2 cache (int2kv_read_rows).
//
//   rotated rows   k^ = code * s + z,            v^ = code * s + z
//   model's basis  k~ = k^ R_K^T (+ mu),         v~ = v^ R_V^T
//
// The product is formed transposed, D^T = R x^T (32 x 32 x 16 matrix products, R's rows as the A operand, a token per lane
// as the B operand): lane (token, half hh) holds words 4 hh .. 4 hh + 3 of its token's codes, which are its channels of all
// eight operands, so nothing moves between lanes; D leaves 64 output channels in a lane, eight consecutive ones per store
// (tile 2 a + e holds channels 64 a + 2 m + e in its rows m). R is converted once per work-group into LDS, in operand
// order; a work-group then walks over tokens, a wave 32 at a time with the next tile's records on their way.
//
// bf16 rows: x^ and R in one fp16 term each, an error of about 3e-4 of the row's root mean square against the output's
// rounding of 2^-9 of each value. fp32 rows: two fp16 terms each, three products (the fourth is below 2^-22).
#include "codes.h"
#include "common.h"
#include "kernels.h"

namespace int2kv {

namespace {

constexpr int kReadThreads = 256;
constexpr int kReadTile = 32;                 // tokens of a wave's step
constexpr int kFrag = 64;                     // lanes of an operand, 16 bytes each

// One token's half row as loaded: its four words and its groups' (s, z)
template <int NG>
struct RawRow {
  uint32_t w[4], s[NG], z[NG];  // s, z: fp16 bits
  bool ok;
};

template <int NG>
__device__ __forceinline__ RawRow<NG> load_row(const CacheView& cv, int slot, bool in, int h, int kv, int hh) {
  using Lay = Rec<NG>;
  RawRow<NG> r;
  r.ok = in && slot >= 0 && slot < cv.num_blocks * kBlock;
  const int at = r.ok ? slot : 0, t = at & 15;
  const uint8_t* rec = cv.pool + ((size_t)(at >> 4) * cv.num_kv_heads + h) * Lay::kBytes;
  if (kv == 0) {
    const cd_u4_t w = *reinterpret_cast<const cd_u4_t*>(rec + kOffKCodes + 32 * t + 16 * hh);
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = w[i];
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const uint32_t m = *reinterpret_cast<const uint32_t*>(rec + Lay::kOffKMeta + 4 * NG * t + 4 * g);
      r.s[g] = m & 0xFFFFu;
      r.z[g] = m >> 16;
    }
  } else {
    const uint16_t* c = reinterpret_cast<const uint16_t*>(rec + kOffVCodes) + 128 * hh + t;  // half m of token t: 16 m + t
#pragma unroll
    for (int i = 0; i < 4; ++i) r.w[i] = (uint32_t)c[32 * i] | ((uint32_t)c[32 * i + 16] << 16);
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      r.s[g] = *reinterpret_cast<const uint16_t*>(rec + Lay::kOffVScale + 32 * g + 2 * t);
      r.z[g] = *reinterpret_cast<const uint16_t*>(rec + Lay::kOffVZero + 32 * g + 2 * t);
    }
  }
  return r;
}

// Word W's two operands in fp32 steps, as two fp16 terms
template <int NG>
__device__ __forceinline__ void word_terms(uint32_t w, const float (&s)[NG], const float (&z)[NG], cd_h8_t (&hi)[2],
                                           cd_h8_t (&lo)[2]) {
  const uint32_t up = w >> 10;
#define INT2KV_POS(P)                                                         \
  {                                                                           \
    const cd_h2_t c = land_position<P>(w, up);                                \
    const float a = __builtin_fmaf((float)c.x, s[P * NG / 8], z[P * NG / 8]); \
    const float b = __builtin_fmaf((float)c.y, s[P * NG / 8], z[P * NG / 8]); \
    const _Float16 ah = (_Float16)a, bh = (_Float16)b;                        \
    hi[P / 4][2 * (P % 4)] = ah, hi[P / 4][2 * (P % 4) + 1] = bh;             \
    lo[P / 4][2 * (P % 4)] = (_Float16)(a - (float)ah);                       \
    lo[P / 4][2 * (P % 4) + 1] = (_Float16)(b - (float)bh);                   \
  }
  INT2KV_POS(0) INT2KV_POS(1) INT2KV_POS(2) INT2KV_POS(3) INT2KV_POS(4) INT2KV_POS(5) INT2KV_POS(6) INT2KV_POS(7)
#undef INT2KV_POS
}

}  // namespace

// Work-group (block x of gridDim.x, KV head y, keys z = 0 / values z = 1)
template <int NG, bool F32>
__global__ __launch_bounds__(kReadThreads, 2) void read_rows_kernel(CacheView cv, const int32_t* __restrict__ slots, int n,
                                                                    const float* __restrict__ R_k,
                                                                    const float* __restrict__ R_v,
                                                                    const float* __restrict__ mu, void* __restrict__ k_out,
                                                                    void* __restrict__ v_out, int z0) {
  constexpr int kTerms = F32 ? 2 : 1;
  __shared__ __align__(16) uint32_t frag[kTerms][4][8][kFrag][4];  // [term][tile][operand][lane][8 fp16]
  __shared__ float off[kHeadDim];
  const int tid = threadIdx.x, l = tid & 63, wave = tid >> 6, m = l & 31, hh = l >> 5;
  const int h = blockIdx.y, kv = blockIdx.z + z0, H = cv.num_kv_heads;
  void* out = kv ? v_out : k_out;
  // ---- R into LDS. A thread takes two neighbouring channels of one row; lane chunk m of operand kk lies at m ^ kk, so
  // that a row's 64 pairs, which differ in operand and place but not in m, spread over the banks
  const float* R = (kv ? R_v : R_k) + (size_t)h * kHeadDim * kHeadDim;
  for (int i = tid; i < kHeadDim * kHeadDim / 2; i += kReadThreads) {
    const int row = i >> 6, c2 = i & 63, p = c2 >> 3, w = c2 & 7, kk = 2 * (w & 3) + (p >> 2);
    const float2 r = *reinterpret_cast<const float2*>(R + row * kHeadDim + 2 * c2);
    const int tile = 2 * (row >> 6) + (row & 1), at = (w >> 2) * 32 + (((row & 63) >> 1) ^ kk);
    const cd_h2_t hi = {(_Float16)r.x, (_Float16)r.y};
    frag[0][tile][kk][at][p & 3] = __builtin_bit_cast(uint32_t, hi);
    if constexpr (F32) {
      const cd_h2_t lo = {(_Float16)(r.x - (float)hi.x), (_Float16)(r.y - (float)hi.y)};
      frag[kTerms - 1][tile][kk][at][p & 3] = __builtin_bit_cast(uint32_t, lo);
    }
  }
  if (tid < kHeadDim) off[tid] = kv == 0 && mu ? mu[(size_t)h * kHeadDim + tid] : 0.0f;
  __syncthreads();

  const int tiles = (n + kReadTile - 1) / kReadTile, hop = gridDim.x * (kReadThreads / 64);
  int tile = blockIdx.x * (kReadThreads / 64) + wave;
  auto slot_of = [&](int t) { return slots[min(t * kReadTile + m, n - 1)]; };
  auto inside = [&](int t) { return t * kReadTile + m < n; };
  if (tile >= tiles) return;
  RawRow<NG> raw = load_row<NG>(cv, slot_of(tile), inside(tile), h, kv, hh);
  int slot_next = tile + hop < tiles ? slot_of(tile + hop) : -1;
  for (; tile < tiles; tile += hop) {
    const RawRow<NG> cur = raw;
    if (tile + hop < tiles) {
      raw = load_row<NG>(cv, slot_next, inside(tile + hop), h, kv, hh);
      if (tile + 2 * hop < tiles) slot_next = slot_of(tile + 2 * hop);
    }
    cd_f16_t acc[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[i][r] = 0.0f;
    auto A = [&](int term, int i, int kk) { return *reinterpret_cast<const cd_h8_t*>(&frag[term][i][kk][hh * 32 + (m ^ kk)][0]); };
    if constexpr (F32) {
      float s[NG], z[NG];
#pragma unroll
      for (int g = 0; g < NG; ++g) s[g] = f16_bits_to_f32(cur.s[g]), z[g] = f16_bits_to_f32(cur.z[g]);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        cd_h8_t hi[2], lo[2];
        word_terms<NG>(cur.w[w], s, z, hi, lo);
#pragma unroll
        for (int o = 0; o < 2; ++o)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const cd_h8_t a = A(0, i, 2 * w + o);
            acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(A(kTerms - 1, i, 2 * w + o), hi[o], acc[i], 0, 0, 0);
            acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, lo[o], acc[i], 0, 0, 0);
            acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a, hi[o], acc[i], 0, 0, 0);
          }
      }
    } else {
      cd_h2_t s[NG], z[NG];
#pragma unroll
      for (int g = 0; g < NG; ++g) s[g] = both_lo(cur.s[g]), z[g] = both_lo(cur.z[g]);
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        cd_h8_t x[2];
        word_operands<NG>(cur.w[w], s, z, x);
#pragma unroll
        for (int o = 0; o < 2; ++o)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            acc[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(A(0, i, 2 * w + o), x[o], acc[i], 0, 0, 0);
      }
    }
    if (cur.ok) {
      // register 4 u + v of tile 2 a + e: channel 64 a + 16 u + 8 hh + 2 v + e
      const size_t at = ((size_t)(tile * kReadTile + m) * H + h) * kHeadDim + 8 * hh;
#pragma unroll
      for (int a = 0; a < 2; ++a)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const int c = 64 * a + 16 * u;
          float y[8];
#pragma unroll
          for (int v = 0; v < 8; ++v) y[v] = acc[2 * a + (v & 1)][4 * u + (v >> 1)] + off[c + 8 * hh + v];
          if constexpr (F32) {
            float4* o = reinterpret_cast<float4*>(static_cast<float*>(out) + at + c);
            o[0] = make_float4(y[0], y[1], y[2], y[3]);
            o[1] = make_float4(y[4], y[5], y[6], y[7]);
          } else {
            *reinterpret_cast<uint4*>(static_cast<uint16_t*>(out) + at + c) =
                make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
          }
        }
    }
  }
}

// Rows as stored: thread (token, KV head, word w) has channels 16 p + 2 w and + 1. Exact before the output's rounding.
template <int NG, bool F32>
__global__ __launch_bounds__(256) void read_rotated_kernel(CacheView cv, const int32_t* __restrict__ slots, int n,
                                                           void* __restrict__ k_out, void* __restrict__ v_out, int z0) {
  using Lay = Rec<NG>;
  const int H = cv.num_kv_heads, kv = blockIdx.y + z0;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x, row = i >> 3;
  if (row >= (long long)n * H) return;
  const int w = (int)(i & 7), h = (int)(row % H), slot = slots[row / H];
  if (slot < 0 || slot >= cv.num_blocks * kBlock) return;
  const int t = slot & 15;
  const uint8_t* rec = cv.pool + ((size_t)(slot >> 4) * H + h) * Lay::kBytes;
  uint32_t word;
  float s[NG], z[NG];
  if (kv == 0) {
    word = *reinterpret_cast<const uint32_t*>(rec + kOffKCodes + 32 * t + 4 * w);
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const uint32_t m = *reinterpret_cast<const uint32_t*>(rec + Lay::kOffKMeta + 4 * NG * t + 4 * g);
      s[g] = f16_bits_to_f32(m & 0xFFFFu);
      z[g] = f16_bits_to_f32(m >> 16);
    }
  } else {
    const uint16_t* c = reinterpret_cast<const uint16_t*>(rec + kOffVCodes) + 32 * w + t;
    word = (uint32_t)c[0] | ((uint32_t)c[16] << 16);
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      s[g] = f16_bits_to_f32(*reinterpret_cast<const uint16_t*>(rec + Lay::kOffVScale + 32 * g + 2 * t));
      z[g] = f16_bits_to_f32(*reinterpret_cast<const uint16_t*>(rec + Lay::kOffVZero + 32 * g + 2 * t));
    }
  }
  void* out = kv ? v_out : k_out;
#pragma unroll
  for (int p = 0; p < 8; ++p) {
    const float a = __builtin_fmaf((float)((word >> (2 * p)) & 3u), s[p * NG / 8], z[p * NG / 8]);
    const float b = __builtin_fmaf((float)((word >> (16 + 2 * p)) & 3u), s[p * NG / 8], z[p * NG / 8]);
    const size_t at = (size_t)row * kHeadDim + 16 * p + 2 * w;
    if constexpr (F32)
      *reinterpret_cast<float2*>(static_cast<float*>(out) + at) = make_float2(a, b);
    else
      *reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(out) + at) = pack_bf16(a, b);
  }
}

namespace {

template <int NG, bool F32>
hipError_t launch_read(CacheView c, const int32_t* slots, int n, const float* R_k, const float* R_v, const float* mu,
                       void* k_out, void* v_out, hipStream_t s) {
  const int H = c.num_kv_heads;
  // keys, values or both in one launch where they take the same kernel
  auto rotated = [&](int z0, int nz) {
    const long long blocks = ((long long)n * H * 8 + 255) / 256;
    hipLaunchKernelGGL((read_rotated_kernel<NG, F32>), dim3((unsigned)blocks, nz), dim3(256), 0, s, c, slots, n, k_out, v_out, z0);
  };
  auto turned = [&](int z0, int nz) {
    const int tiles = (n + kReadTile - 1) / kReadTile, waves = kReadThreads / 64;
    int nb = (2 * num_cus() + nz * H - 1) / (nz * H);  // two work-groups a compute unit share R's conversion
    nb = nb < 1 ? 1 : nb;
    const int most = (tiles + waves - 1) / waves;
    hipLaunchKernelGGL((read_rows_kernel<NG, F32>), dim3(nb < most ? nb : most, H, nz), dim3(kReadThreads), 0, s, c, slots, n,
                       R_k, R_v, mu, k_out, v_out, z0);
  };
  if (k_out && v_out && !R_k == !R_v) {
    R_k ? turned(0, 2) : rotated(0, 2);
  } else {
    if (k_out) R_k ? turned(0, 1) : rotated(0, 1);
    if (v_out) R_v ? turned(1, 1) : rotated(1, 1);
  }
  return hipGetLastError();
}

}  // namespace

hipError_t launch_read_rows(CacheView c, const int32_t* slots, int n, const float* R_k, const float* R_v, const float* mu,
                            bool f32, void* k_out, void* v_out, hipStream_t s) {
  if (c.groups == 4)
    return f32 ? launch_read<4, true>(c, slots, n, R_k, R_v, mu, k_out, v_out, s)
               : launch_read<4, false>(c, slots, n, R_k, R_v, mu, k_out, v_out, s);
  return f32 ? launch_read<1, true>(c, slots, n, R_k, R_v, mu, k_out, v_out, s)
             : launch_read<1, false>(c, slots, n, R_k, R_v, mu, k_out, v_out, s);
}

}  // namespace int2kv
