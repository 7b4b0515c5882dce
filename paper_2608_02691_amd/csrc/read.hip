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
// Bound by the rows written (256 or 512 bytes a row; the records are 96, in whole pages where neighbours are wanted too).
// Rows leave through LDS as whole 256-byte pieces by stores that bypass the caches: 32,768 scattered tokens of 8 heads, keys
// and values, take 32 us (160 MB, 5.0 TB/s); 32-byte pieces straight from the accumulators took 71.
//
// bf16 rows: x^ and R in one fp16 term each, an error of about 3e-4 of the row's root mean square against the output's
// rounding of 2^-9 of each value. fp32 rows: two fp16 terms each, three products (the fourth is below 2^-22).
#include "codes.h"
#include "common.h"
#include "kernels.h"

namespace int2kv {

namespace {

constexpr int kReadThreads = 512;
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
  __shared__ __align__(16) uint4 rows[kReadThreads / 64][kReadTile * 16];  // results on their way out
  __shared__ __align__(16) float off[kHeadDim];
  const int tid = threadIdx.x, l = tid & 63, wave = tid >> 6, m = l & 31, hh = l >> 5;
  const int h = blockIdx.y, kv = blockIdx.z + z0, H = cv.num_kv_heads;
  void* out = kv ? v_out : k_out;
  // ---- R into LDS. A thread takes four neighbouring channels of one row; lane chunk m of operand kk lies at m ^ kk, so that
  // a row's pieces, which differ in operand and place but not in m, spread over the banks
  const float* R = (kv ? R_v : R_k) + (size_t)h * kHeadDim * kHeadDim;
  constexpr int kLoads = kHeadDim * kHeadDim / 4 / kReadThreads;
  float4 r4[kLoads];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) r4[i] = reinterpret_cast<const float4*>(R)[tid + kReadThreads * i];
#pragma unroll
  for (int i = 0; i < kLoads; ++i) {
    const int e = tid + kReadThreads * i, row = e >> 5, c4 = e & 31, p = c4 >> 2;
    const int tile = 2 * (row >> 6) + (row & 1);
#pragma unroll
    for (int x = 0; x < 2; ++x) {  // channels 16 p + 2 w, + 1
      const int w = 2 * (c4 & 3) + x, kk = 2 * (w & 3) + (p >> 2), at = (w >> 2) * 32 + (((row & 63) >> 1) ^ kk);
      const float u = x ? r4[i].z : r4[i].x, v = x ? r4[i].w : r4[i].y;
      const cd_h2_t hi = {(_Float16)u, (_Float16)v};
      frag[0][tile][kk][at][p & 3] = __builtin_bit_cast(uint32_t, hi);
      if constexpr (F32) {
        const cd_h2_t lo = {(_Float16)(u - (float)hi.x), (_Float16)(v - (float)hi.y)};
        frag[kTerms - 1][tile][kk][at][p & 3] = __builtin_bit_cast(uint32_t, lo);
      }
    }
  }
  const bool centered = kv == 0 && mu;
  if (centered && tid < kHeadDim) off[tid] = mu[(size_t)h * kHeadDim + tid];
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
    // The next tile's loads are waited for here: behind the stores, which count in the same order, the wait would be for them
#pragma unroll
    for (int i = 0; i < 4; ++i) asm volatile("" : "+v"(raw.w[i]));
#pragma unroll
    for (int g = 0; g < NG; ++g) asm volatile("" : "+v"(raw.s[g]), "+v"(raw.z[g]));
    asm volatile("" : "+v"(slot_next));
    // (the stores bypass the caches: through them they take a quarter longer)
    // register 4 u + v of tile 2 a + e: channel 64 a + 16 u + 8 hh + 2 v + e. Through the wave's own piece of LDS, 256 bytes a
    // token at a time (chunk x of token m at x ^ m), so that a store writes four whole pieces of rows
    const unsigned long long live = __ballot(cur.ok);
    uint4* box = rows[wave];
#pragma unroll
    for (int part = 0; part < (F32 ? 2 : 1); ++part) {
#pragma unroll
      for (int a = F32 ? part : 0; a < (F32 ? part + 1 : 2); ++a)
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          float y[8];
#pragma unroll
          for (int v = 0; v < 8; ++v) y[v] = acc[2 * a + (v & 1)][4 * u + (v >> 1)];
          if (centered) {
            const float4* mu4 = reinterpret_cast<const float4*>(off + 64 * a + 16 * u + 8 * hh);
            const float4 m0 = mu4[0], m1 = mu4[1];
            y[0] += m0.x, y[1] += m0.y, y[2] += m0.z, y[3] += m0.w, y[4] += m1.x, y[5] += m1.y, y[6] += m1.z, y[7] += m1.w;
          }
          if constexpr (F32) {
            const int x = 4 * u + 2 * hh;
            box[16 * m + (x ^ (m & 15))] = make_uint4(__float_as_uint(y[0]), __float_as_uint(y[1]), __float_as_uint(y[2]), __float_as_uint(y[3]));
            box[16 * m + ((x + 1) ^ (m & 15))] = make_uint4(__float_as_uint(y[4]), __float_as_uint(y[5]), __float_as_uint(y[6]), __float_as_uint(y[7]));
          } else {
            box[16 * m + ((8 * a + 2 * u + hh) ^ (m & 15))] =
                make_uint4(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7]));
          }
        }
      __builtin_amdgcn_wave_barrier();
      uint8_t* o = static_cast<uint8_t*>(out) + ((size_t)tile * kReadTile * H + h) * (kHeadDim * (F32 ? 4 : 2)) + 256 * part + 16 * (l & 15);
#pragma unroll
      for (int r = 0; r < kReadTile; r += 4) {
        const int t = r + (l >> 4);
        const uint4 y = box[16 * t + ((l & 15) ^ (t & 15))];
        if ((live >> t) & 1) __builtin_nontemporal_store(cd_u4_t{y.x, y.y, y.z, y.w}, reinterpret_cast<cd_u4_t*>(o + (size_t)t * H * (kHeadDim * (F32 ? 4 : 2))));
      }
      __builtin_amdgcn_wave_barrier();
    }
  }
}

// Rows as stored: thread (token, KV head, position p, half x) has the eight channels 16 p + 8 x .., which are bits 2 p of
// halves 8 x .. 8 x + 7. Exact before the output's rounding.
template <int NG, bool F32>
__global__ __launch_bounds__(256) void read_rotated_kernel(CacheView cv, const int32_t* __restrict__ slots, int n,
                                                           void* __restrict__ k_out, void* __restrict__ v_out, int z0) {
  using Lay = Rec<NG>;
  const int H = cv.num_kv_heads, kv = blockIdx.y + z0;
  const long long i = (long long)blockIdx.x * 256 + threadIdx.x, row = i >> 4;
  if (row >= (long long)n * H) return;
  const int x = (int)(i & 1), p = (int)(i >> 1) & 7, g = p * NG / 8, h = (int)(row % H), slot = slots[row / H];
  if (slot < 0 || slot >= cv.num_blocks * kBlock) return;
  const int t = slot & 15;
  const uint8_t* rec = cv.pool + ((size_t)(slot >> 4) * H + h) * Lay::kBytes;
  uint32_t w[4];
  float s, z;
  if (kv == 0) {
    const cd_u4_t c = *reinterpret_cast<const cd_u4_t*>(rec + kOffKCodes + 32 * t + 16 * x);
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = c[j];
    const uint32_t m = *reinterpret_cast<const uint32_t*>(rec + Lay::kOffKMeta + 4 * NG * t + 4 * g);
    s = f16_bits_to_f32(m & 0xFFFFu);
    z = f16_bits_to_f32(m >> 16);
  } else {
    // a lane of the row loads one half; the halves 8 x .. come from the lanes that have them
    const int l = threadIdx.x & 63;
    const int half = *reinterpret_cast<const uint16_t*>(rec + kOffVCodes + 32 * (l & 15) + 2 * t);
    const int pair = half | (__builtin_amdgcn_update_dpp(0, half, 0xB1, 0xF, 0xF, false) << 16);  // (even lanes)
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = (uint32_t)__builtin_amdgcn_ds_bpermute(4 * ((l & 48) + 8 * x + 2 * j), pair);
    s = f16_bits_to_f32(*reinterpret_cast<const uint16_t*>(rec + Lay::kOffVScale + 32 * g + 2 * t));
    z = f16_bits_to_f32(*reinterpret_cast<const uint16_t*>(rec + Lay::kOffVZero + 32 * g + 2 * t));
  }
  float y[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) y[j] = __builtin_fmaf((float)((w[j >> 1] >> (16 * (j & 1) + 2 * p)) & 3u), s, z);
  void* out = kv ? v_out : k_out;
  const size_t at = (size_t)row * kHeadDim + 16 * p + 8 * x;
  if constexpr (F32) {
    typedef float f4 __attribute__((ext_vector_type(4)));
    f4* o = reinterpret_cast<f4*>(static_cast<float*>(out) + at);
    __builtin_nontemporal_store(f4{y[0], y[1], y[2], y[3]}, o);
    __builtin_nontemporal_store(f4{y[4], y[5], y[6], y[7]}, o + 1);
  } else {
    __builtin_nontemporal_store(cd_u4_t{pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]), pack_bf16(y[4], y[5]), pack_bf16(y[6], y[7])},
                                reinterpret_cast<cd_u4_t*>(static_cast<uint16_t*>(out) + at));
  }
}

namespace {

template <int NG, bool F32>
hipError_t launch_read(CacheView c, const int32_t* slots, int n, const float* R_k, const float* R_v, const float* mu,
                       void* k_out, void* v_out, hipStream_t s) {
  const int H = c.num_kv_heads;
  // keys, values or both in one launch where they take the same kernel
  auto rotated = [&](int z0, int nz) {
    const long long blocks = ((long long)n * H * 16 + 255) / 256;
    hipLaunchKernelGGL((read_rotated_kernel<NG, F32>), dim3((unsigned)blocks, nz), dim3(256), 0, s, c, slots, n, k_out, v_out, z0);
  };
  auto turned = [&](int z0, int nz) {
    const int tiles = (n + kReadTile - 1) / kReadTile, waves = kReadThreads / 64;
    int nb = (num_cus() + nz * H - 1) / (nz * H);  // a work-group a compute unit
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
