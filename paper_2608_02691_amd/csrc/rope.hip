// Rotary positions with several axes of a chunk's queries and keys (int2kv_rope_axes).
//
//   y_i = x_i cos - x_{i+64} sin,  y_{i+64} = x_{i+64} cos + x_i sin,  i < 64,
// (cos, sin) of pair i at the token's position on the pair's axis: row positions[axis(i)][token] of the caller's
// table. Each value is the fp64 result (exact products of bf16 and fp32) rounded once to bf16, as in the cache write's
// RoPE, whose arithmetic (rope_pairs) this uses.
//
// Bound by the rows it moves, 512 bytes a (token, head). A token's table rows and positions are read once per thread and
// used for all the heads the thread takes: thread (token, piece j) holds the eight pairs 8 j .. 8 j + 7 of its token and
// walks over heads, four threads of the token abreast, so a wave's loads are whole 128-byte half rows. The stores bypass the
// caches: 24,576 tokens of 32 + 8 heads take 97 us (516 MB, 5.3 TB/s), 101 with ordinary stores.
#include "append_core.h"
#include "common.h"
#include "kernels.h"

namespace int2kv {

namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeTokens = 8;  // tokens of a block: 32 threads each
constexpr int kRopeAhead = 4;   // heads a thread loads before it turns the first

// RUNS: the eight pairs of every piece lie on one axis, so their cosines are two 16-byte loads
template <bool RUNS>
__global__ __launch_bounds__(kRopeThreads) void rope_axes_kernel(RopeAxesArgs a) {
  const int tid = threadIdx.x, j = tid & 7, sub = (tid >> 3) & 3;
  const int tok = blockIdx.x * kRopeTokens + (tid >> 5), t = min(tok, a.n - 1);
  bool ok = tok < a.n;
  for (int x = 0; x < a.num_axes; ++x) {
    const int p = a.positions[(size_t)x * a.n + t];
    ok = ok && p >= 0 && p < a.max_pos;
  }
  // the piece's eight axes, four bits each
  uint32_t ax = a.axis[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) ax = j == i ? a.axis[i] : ax;
  float cs[16];
  auto row = [&](int axis) {
    const int p = a.positions[(size_t)axis * a.n + t];
    return a.cos_sin + (size_t)(ok ? p : 0) * kHeadDim + 8 * j;
  };
  if constexpr (RUNS) {
    const float4* c = reinterpret_cast<const float4*>(row(ax & 15));
    const float4 c0 = c[0], c1 = c[1], s0 = c[16], s1 = c[17];
    cs[0] = c0.x, cs[1] = c0.y, cs[2] = c0.z, cs[3] = c0.w, cs[4] = c1.x, cs[5] = c1.y, cs[6] = c1.z, cs[7] = c1.w;
    cs[8] = s0.x, cs[9] = s0.y, cs[10] = s0.z, cs[11] = s0.w, cs[12] = s1.x, cs[13] = s1.y, cs[14] = s1.z, cs[15] = s1.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float* c = row((ax >> (4 * i)) & 15) + i;
      cs[i] = c[0];
      cs[8 + i] = c[64];
    }
  }
  const int last = min(a.hq + a.hk, ((int)blockIdx.y + 1) * a.heads_per_block);
  for (int h0 = blockIdx.y * a.heads_per_block + sub; h0 < last; h0 += 4 * kRopeAhead) {
    ap_u4_t x0[kRopeAhead], x1[kRopeAhead];
    uint16_t* dst[kRopeAhead];
#pragma unroll
    for (int u = 0; u < kRopeAhead; ++u) {
      const int h = h0 + 4 * u;
      dst[u] = nullptr;
      if (ok && h < last) {
        const bool is_q = h < a.hq;
        const size_t c = (size_t)(is_q ? h : h - a.hq) * kHeadDim + 8 * j;
        const uint16_t* src = (is_q ? a.q + t * a.q_stride : a.k + t * a.k_stride) + c;
        dst[u] = (is_q ? a.q_out + t * a.q_out_stride : a.k_out + t * a.k_out_stride) + c;
        x0[u] = *reinterpret_cast<const ap_u4_t*>(src);
        x1[u] = *reinterpret_cast<const ap_u4_t*>(src + 64);
      }
    }
#pragma unroll
    for (int u = 0; u < kRopeAhead; ++u) {
      if (dst[u]) {
        rope_pairs(x0[u], x1[u], cs);
        __builtin_nontemporal_store(x0[u], reinterpret_cast<ap_u4_t*>(dst[u]));
        __builtin_nontemporal_store(x1[u], reinterpret_cast<ap_u4_t*>(dst[u] + 64));
      }
    }
  }
}

}  // namespace

hipError_t launch_rope_axes(RopeAxesArgs a, const uint8_t* pair_axis, hipStream_t s) {
  bool runs = true;
  for (int j = 0; j < 8; ++j) {
    a.axis[j] = 0;
    for (int i = 0; i < 8; ++i) {
      a.axis[j] |= (uint32_t)pair_axis[8 * j + i] << (4 * i);
      runs = runs && pair_axis[8 * j + i] == pair_axis[8 * j];
    }
  }
  // a token's heads are split over blocks only while the tokens alone leave compute units idle
  const int blocks = (a.n + kRopeTokens - 1) / kRopeTokens, quads = (a.hq + a.hk + 3) / 4;
  int split = (4 * num_cus() + blocks - 1) / blocks;
  split = split < 1 ? 1 : split > quads ? quads : split;
  a.heads_per_block = 4 * ((quads + split - 1) / split);
  const dim3 grid(blocks, (quads * 4 + a.heads_per_block - 1) / a.heads_per_block);
  if (runs)
    hipLaunchKernelGGL(rope_axes_kernel<true>, grid, dim3(kRopeThreads), 0, s, a);
  else
    hipLaunchKernelGGL(rope_axes_kernel<false>, grid, dim3(kRopeThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace int2kv
