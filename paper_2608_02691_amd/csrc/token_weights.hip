// Attention weight that every cached token receives (int2kv_token_weights).
//
// Rows are (new token i of sequence b, query head j of the KV head's group), row i * G_q + j of the sequence, in tiles of 32;
// a row sees the cached s < limit_i. With x_rs = log2(e) / sqrt(128) (q_r R_K) k^_s^T:
//     w_out[s] = decay w_in[s] + sum_r 2^(x_rs - L_r),   L_r = log2(sum_s 2^x_rs).
// Four launches: the rows' operands; each row's maximum and sum over ranges of 256 tokens; L_r; the sums over the rows.
//
// The results are fp32 sums, so scores are formed to fp32's precision: k^ = code s_g + z_g by groups, and
//     x = sum_g s_g D_g + sum_g z_g Q_g,   D_g = sum_{c in g} q'_c code_c,   Q_g = sum_{c in g} q'_c,
// where a code is exact in fp16, q' and Q_g are two fp16 terms each (22 bits) and z_g is fp16 as stored, all products are
// exact in fp32, and s_g enters in fp32.
#include "chunk_core.h"

namespace int2kv {

namespace {

constexpr int kRows = 32;                                     // rows of a tile
constexpr int kOpBytes = 2 * 8 * 64 * 16 + 64 * 16;           // a tile's operands: high terms, low terms, Q_g
constexpr int kWaves = 8;
static_assert(kRangeTokens == 32 * kWaves, "a wave takes 32 tokens of a range");

struct Span {
  int start, n, ctx, past;  // as Seq
  int tile0;                // first of the sequence's row tiles
  __device__ __forceinline__ int limit(int i) const { return max(min(ctx, past + i + 1), 0); }
};
// The tiles of sequence b start at start * gq / 32 + b: never before the end of the one before.
__device__ __forceinline__ Span span_of(const TokenWeightsArgs& a, int b) {
  Span s;
  s.start = min(max(a.starts[b], 0), a.total_q);
  const int end = min(max(a.starts[b + 1], 0), a.total_q);
  const int count = max(end - s.start, 0), len = max(a.lens[b], 0);
  s.n = min(count, a.max_q);
  const long long room = (long long)a.max_blocks * kBlock;
  s.ctx = min(len, (int)(room < a.max_ctx ? room : a.max_ctx));
  s.past = len - count;
  s.tile0 = (int)((long long)s.start * a.gq / kRows) + b;
  return s;
}

__device__ __forceinline__ cd_u4_t pack_terms(const float* x) {  // eight bf16 numbers, each the upper half of its word
  cd_u4_t y;
#pragma unroll
  for (int i = 0; i < 4; ++i) y[i] = __builtin_amdgcn_perm(__float_as_uint(x[2 * i + 1]), __float_as_uint(x[2 * i]), 0x07060302u);
  return y;
}
__device__ __forceinline__ float upper(float x) { return __uint_as_float(__float_as_uint(x) & 0xFFFF0000u); }

// Where channel c lies in the operands: product 2 g + x of group g takes positions 2 g, 2 g + 1 of words 2 x, 2 x + 1 of the
// lane half's four
struct Spot {
  int product, half, element;
};
__device__ __forceinline__ Spot spot_of(int c) {
  const int g = c >> 5, p = (c >> 4) & 1, word = (c & 15) >> 1;
  return Spot{2 * g + ((word & 3) >> 1), word >> 2, ((word & 1) << 2) | (p << 1) | (c & 1)};
}

// A lane's token: its codes as operands, its scales and the operand of its zeros
template <int NG>
struct Token {
  cd_h8_t code[8];
  float scale[NG];
  cd_h8_t zero;
  bool real;
  __device__ __forceinline__ void load(const TokenWeightsArgs& a, int b, int h, int token, int ctx, int hh) {
    int id = -1;
    if (token < ctx) id = a.table[(size_t)b * a.max_blocks + token / kBlock];
    real = id >= 0 && id < a.cv.num_blocks;
    const uint8_t* rec = a.cv.pool + ((size_t)(uint32_t)(real ? id : 0) * a.cv.num_kv_heads + h) * Rec<NG>::kBytes;
    const int t = token & 15;
    const cd_u4_t w = *reinterpret_cast<const cd_u4_t*>(rec + kOffKCodes + 32 * t + 16 * hh);
    const uint32_t* m = reinterpret_cast<const uint32_t*>(rec + Rec<NG>::kOffKMeta + 4 * NG * t);
    zero = cd_h8_t{};
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      const uint32_t sz = m[g];
      scale[g] = f16_bits_to_f32(sz & 0xFFFFu);
      const _Float16 z = __builtin_bit_cast(cd_h2_t, sz).y;
      zero[g] = hh == 0 ? z : (_Float16)0.0f;
      zero[4 + g] = zero[g];
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const uint32_t u = w[2 * x], v = w[2 * x + 1];
      const uint32_t uh = u >> 10, vh = v >> 10;
      auto put = [&](cd_h8_t& c, cd_h2_t p, cd_h2_t q, cd_h2_t r, cd_h2_t y) { c = cd_h8_t{p.x, p.y, q.x, q.y, r.x, r.y, y.x, y.y}; };
      put(code[0 + x], land_position<0>(u, uh), land_position<1>(u, uh), land_position<0>(v, vh), land_position<1>(v, vh));
      put(code[2 + x], land_position<2>(u, uh), land_position<3>(u, uh), land_position<2>(v, vh), land_position<3>(v, vh));
      put(code[4 + x], land_position<4>(u, uh), land_position<5>(u, uh), land_position<4>(v, vh), land_position<5>(v, vh));
      put(code[6 + x], land_position<6>(u, uh), land_position<7>(u, uh), land_position<6>(v, vh), land_position<7>(v, vh));
    }
  }
};

// A row tile's operands in LDS
struct Ops {
  cd_h8_t hi[8][64], lo[8][64], group[64];
};
static_assert(sizeof(Ops) == kOpBytes, "as the workspace holds them");

__device__ __forceinline__ cd_f16_t product(const cd_h8_t& x, const cd_h8_t& y, const cd_f16_t& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(x, y, c, 0, 0, 0);
}

// Brings a tile's operands to LDS by all threads of the block
__device__ __forceinline__ void bring(const uint8_t* from, Ops& to) {
  const uint4* s = reinterpret_cast<const uint4*>(from);
  uint4* d = reinterpret_cast<uint4*>(&to);
  for (int i = threadIdx.x; i < kOpBytes / 16; i += 64 * kWaves) d[i] = s[i];
}

}  // namespace

// ---- The rows' operands. Block: row tiles of one KV head, one after the other; wave w forms channels 32 w .. of q R_K on the
// matrix cores, R_K in three bf16 terms that sum to it exactly. A tile's rows are scaled by one power of two that brings
// the largest element to 2^7 .. 2^8: what the low terms lose, 2^-24, is 2^-31 of it, and a group's sum fits fp16.
__global__ __launch_bounds__(256) void weight_rows_kernel(TokenWeightsArgs a, int tiles_per_block) {
  __shared__ float top[4], sums[4][kRows];
  const int H = a.cv.num_kv_heads, blocks = (a.seq_tiles + tiles_per_block - 1) / tiles_per_block;
  const int at = blockIdx.x % blocks, h = blockIdx.x / blocks % H, b = blockIdx.x / blocks / H;
  const Span s = span_of(a, b);
  const int tiles = (s.n * a.gq + kRows - 1) / kRows;
  const int w = threadIdx.x >> 6, l = threadIdx.x & 63, n = l & 31, hh = l >> 5;
  if (at * tiles_per_block >= tiles) return;
  cd_u4_t R[8][3];  // of column 32 w + n, rows 16 kk + 8 hh ..
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) {
    float x[8], y[8], z[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float r = a.R_k[((size_t)h * kHeadDim + 16 * kk + 8 * hh + j) * kHeadDim + 32 * w + n];
      x[j] = upper(r), y[j] = upper(r - x[j]), z[j] = r - x[j] - y[j];
    }
    R[kk][0] = pack_terms(x), R[kk][1] = pack_terms(y), R[kk][2] = pack_terms(z);
  }
  for (int t = at * tiles_per_block; t < min(tiles, (at + 1) * tiles_per_block); ++t) {
    const int row = kRows * t + n, tok = row / a.gq;
    const bool live = row < s.n * a.gq;
    const uint16_t* q = a.q + (s.start + (live ? tok : 0)) * a.q_stride + (size_t)(h * a.gq + (live ? row - tok * a.gq : 0)) * kHeadDim + 8 * hh;
    cd_f16_t d = splat16(0.0f);
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      cd_u4_t x = *reinterpret_cast<const cd_u4_t*>(q + 16 * kk);
      if (!live) x = cd_u4_t{0, 0, 0, 0};
#pragma unroll
      for (int i = 0; i < 3; ++i)
        d = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(cd_b8_t, R[kk][i]), __builtin_bit_cast(cd_b8_t, x), d, 0, 0, 0);
    }
    // register r: channel 32 w + 8 (r / 4) + 4 hh + r % 4 of row n
    float big = 0.0f, sum = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      d[r] *= kLogit2;
      big = fmaxf(big, fabsf(d[r]));
    }
#pragma unroll
    for (int step = 32; step > 0; step >>= 1) big = fmaxf(big, __shfl_xor(big, step));
    __syncthreads();  // (the tile before is done with them)
    if (l == 0) top[w] = big;
    __syncthreads();
    big = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    const uint32_t e = min(max(__float_as_uint(big) >> 23, 8u), 254u);
    const float up = __uint_as_float((261u - e) << 23), down = __uint_as_float((e - 7u) << 23);
    const size_t tile = ((size_t)(s.tile0 + t) * H + h);
    Ops& out = *reinterpret_cast<Ops*>(a.ops + tile * kOpBytes);
#pragma unroll
    for (int r = 0; r < 16; r += 2) {
      const float x = d[r] * up, y = d[r + 1] * up;
      sum += x + y;
      const Spot p = spot_of(32 * w + 8 * (r >> 2) + 4 * hh + (r & 3));
      const cd_h2_t hi = {(_Float16)x, (_Float16)y}, lo = {(_Float16)(x - (float)hi.x), (_Float16)(y - (float)hi.y)};
      *reinterpret_cast<cd_h2_t*>(reinterpret_cast<_Float16*>(&out.hi[p.product][32 * p.half + n]) + p.element) = hi;
      *reinterpret_cast<cd_h2_t*>(reinterpret_cast<_Float16*>(&out.lo[p.product][32 * p.half + n]) + p.element) = lo;
    }
    sum = pair_sum(sum);
    if (hh == 0) sums[w][n] = sum;
    __syncthreads();
    if (w == 0) {
      cd_h8_t g{};
      if (hh == 0) {
        float x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = sums[i][n];
        if (a.cv.groups == 1) x[0] = (x[0] + x[1]) + (x[2] + x[3]), x[1] = x[2] = x[3] = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) g[i] = (_Float16)x[i], g[4 + i] = (_Float16)(x[i] - (float)g[i]);
      }
      out.group[l] = g;
      if (l == 0) a.down[tile] = down;
    }
  }
}

// ---- Maximum and sum of the rows over a range. Block: 256 tokens of one KV head over a slice of the row tiles, wave w
// with 32 of them. Products are codes x rows, so that a lane holds a row and the sums are its own.
template <int NG>
__global__ __launch_bounds__(64 * kWaves, 2) void weight_stats_kernel(TokenWeightsArgs a) {
  __shared__ Ops ops;
  __shared__ float scales[kWaves][32][NG];
  __shared__ float2 both[kWaves][kRows];
  const int H = a.cv.num_kv_heads;
  const int range = blockIdx.x % a.ranges, slice = blockIdx.x / a.ranges % a.slices, bh = blockIdx.x / a.ranges / a.slices, b = bh / H, h = bh % H;
  const Span s = span_of(a, b);
  const int rows = s.n * a.gq, tiles = (rows + kRows - 1) / kRows, per = (tiles + a.slices - 1) / a.slices;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, n = l & 31, hh = l >> 5, first = kRangeTokens * range, t0 = first + 32 * w;
  if (first >= s.ctx) return;
  Token<NG> tok;
  tok.load(a, b, h, t0 + n, s.ctx, hh);
  if (hh == 0) {
#pragma unroll
    for (int g = 0; g < NG; ++g) scales[w][n][g] = tok.scale[g];
  }
  const uint32_t real = (uint32_t)__ballot(tok.real);  // (the lane halves hold the same tokens)
  __syncthreads();
  float sc[NG][16];
#pragma unroll
  for (int r = 0; r < 16; ++r)
#pragma unroll
    for (int g = 0; g < NG; ++g) sc[g][r] = scales[w][8 * (r >> 2) + 4 * hh + (r & 3)][g];
  for (int t = slice * per; t < min(tiles, (slice + 1) * per); ++t) {
    if (s.limit(min(kRows * t + kRows - 1, rows - 1) / a.gq) <= first) continue;  // none of its rows sees the range
    const size_t tile = (size_t)(s.tile0 + t) * H + h;
    __syncthreads();
    bring(a.ops + tile * kOpBytes, ops);
    const float down = a.down[tile];
    __syncthreads();
    cd_f16_t S = product(tok.zero, ops.group[l], splat16(0.0f));
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      cd_f16_t D = splat16(0.0f);
#pragma unroll
      for (int x = 8 / NG * g; x < 8 / NG * (g + 1); ++x) {
        D = product(tok.code[x], ops.hi[x][l], D);
        D = product(tok.code[x], ops.lo[x][l], D);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) S[r] = __builtin_fmaf(sc[g][r], D[r], S[r]);
    }
    const int lim = s.limit(min(kRows * t + n, rows - 1) / a.gq) - t0;
    float m = -INFINITY;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int x = 8 * (r >> 2) + 4 * hh + (r & 3);
      S[r] = x < lim && ((real >> x) & 1) ? S[r] * down : -INFINITY;
      m = fmaxf(m, S[r]);
    }
    m = pair_max(m);
    const float base = m == -INFINITY ? 0.0f : m;
    float sum = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) sum += __builtin_amdgcn_exp2f(S[r] - base);
    sum = pair_sum(sum);
    if (hh == 0) both[w][n] = make_float2(m, sum);
    __syncthreads();
    if (threadIdx.x < kRows) {
      float top = -INFINITY, all = 0.0f;
#pragma unroll
      for (int x = 0; x < kWaves; ++x) top = fmaxf(top, both[x][threadIdx.x].x);
#pragma unroll
      for (int x = 0; x < kWaves; ++x) {
        const float2 v = both[x][threadIdx.x];
        all += v.y == 0.0f ? 0.0f : v.y * __builtin_amdgcn_exp2f(v.x - top);
      }
      a.stats[(((size_t)range * a.tiles + s.tile0 + t) * H + h) * kRows + threadIdx.x] = make_float2(top, all);
    }
  }
}

// ---- L_r of every row; infinite for rows that see nothing and behind the last one, so that their weights are zero
__global__ __launch_bounds__(256) void weight_lse_kernel(TokenWeightsArgs a) {
  const int H = a.cv.num_kv_heads, n = threadIdx.x & 31;
  const long long item = (long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (item >= (long long)a.B * H * a.seq_tiles) return;
  const int t = (int)(item % a.seq_tiles), h = (int)(item / a.seq_tiles % H), b = (int)(item / a.seq_tiles / H);
  const Span s = span_of(a, b);
  const int rows = s.n * a.gq, row = kRows * t + n;
  if (kRows * t >= rows) return;
  const int ranges = row < rows ? (s.limit(row / a.gq) + kRangeTokens - 1) / kRangeTokens : 0;
  float m = -INFINITY, sum = 0.0f;
  for (int r = 0; r < ranges; ++r) {
    const float2 v = a.stats[(((size_t)r * a.tiles + s.tile0 + t) * H + h) * kRows + n];
    const float top = fmaxf(m, v.x), base = top == -INFINITY ? 0.0f : top;
    sum = sum * __builtin_amdgcn_exp2f(m - base) + v.y * __builtin_amdgcn_exp2f(v.x - base);
    m = top;
  }
  a.lse[((size_t)(s.tile0 + t) * H + h) * kRows + n] = sum == 0.0f ? INFINITY : m + __builtin_amdgcn_logf(sum);
}

// ---- The sums over the rows. Products are rows x codes, so that a lane holds a token.
template <int NG>
__global__ __launch_bounds__(64 * kWaves, 2) void weight_sums_kernel(TokenWeightsArgs a) {
  __shared__ Ops ops;
  __shared__ float lse[kRows];
  const int H = a.cv.num_kv_heads;
  const int range = blockIdx.x % a.ranges, slice = blockIdx.x / a.ranges % a.slices, bh = blockIdx.x / a.ranges / a.slices, b = bh / H, h = bh % H;
  const Span s = span_of(a, b);
  const int rows = s.n * a.gq, tiles = (rows + kRows - 1) / kRows, per = (tiles + a.slices - 1) / a.slices;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, n = l & 31, hh = l >> 5, first = kRangeTokens * range, t0 = first + 32 * w;
  if (first >= s.ctx) return;
  Token<NG> tok;
  tok.load(a, b, h, t0 + n, s.ctx, hh);
  float sum = 0.0f;
  for (int t = slice * per; t < min(tiles, (slice + 1) * per); ++t) {
    if (s.limit(min(kRows * t + kRows - 1, rows - 1) / a.gq) <= first) continue;
    const size_t tile = (size_t)(s.tile0 + t) * H + h;
    __syncthreads();
    bring(a.ops + tile * kOpBytes, ops);
    if (threadIdx.x < kRows) lse[threadIdx.x] = a.lse[tile * kRows + threadIdx.x];
    const float down = a.down[tile];
    __syncthreads();
    cd_f16_t S = product(ops.group[l], tok.zero, splat16(0.0f));
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      cd_f16_t D = splat16(0.0f);
#pragma unroll
      for (int x = 8 / NG * g; x < 8 / NG * (g + 1); ++x) {
        D = product(ops.hi[x][l], tok.code[x], D);
        D = product(ops.lo[x][l], tok.code[x], D);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) S[r] = __builtin_fmaf(tok.scale[g], D[r], S[r]);
    }
    float add = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int x = 8 * (r >> 2) + 4 * hh + (r & 3);
      const bool sees = kRows * t + x < rows && t0 + n < s.limit((kRows * t + x) / a.gq);
      add += sees ? __builtin_amdgcn_exp2f(__builtin_fmaf(S[r], down, -lse[x])) : 0.0f;
    }
    sum += add;
  }
  sum = pair_sum(sum);
  if (!tok.real) sum = 0.0f;
  if (hh || t0 + n >= s.ctx) return;
  if (a.slices > 1) {
    a.part[((size_t)slice * a.B * H + bh) * ((size_t)a.ranges * kRangeTokens) + t0 + n] = sum;
  } else {
    const size_t at = (size_t)bh * a.w_stride + t0 + n;
    a.w_out[at] = a.w_in ? __builtin_fmaf(a.decay, a.w_in[at], sum) : sum;
  }
}

__global__ __launch_bounds__(256) void weight_join_kernel(TokenWeightsArgs a) {
  const int H = a.cv.num_kv_heads, range = blockIdx.x % a.ranges, bh = blockIdx.x / a.ranges, t = kRangeTokens * range + threadIdx.x;
  const Span s = span_of(a, bh / H);
  if (t >= s.ctx) return;
  float sum = 0.0f;
  for (int x = 0; x < a.slices; ++x) sum += a.part[((size_t)x * a.B * H + bh) * ((size_t)a.ranges * kRangeTokens) + t];
  const size_t at = (size_t)bh * a.w_stride + t;
  a.w_out[at] = a.w_in ? __builtin_fmaf(a.decay, a.w_in[at], sum) : sum;
}

TokenWeightsPlan make_token_weights_plan(int B, int Hq, int H, int total_q, int max_q, int max_ctx) {
  TokenWeightsPlan p{};
  const int gq = Hq / H;
  p.seq_tiles = (int)(((long long)max_q * gq + kRows - 1) / kRows);
  p.ranges = (int)(((long long)max_ctx + kRangeTokens - 1) / kRangeTokens);
  if (p.ranges < 1) p.ranges = 1;
  p.tiles = (int)((long long)total_q * gq / kRows + B + 1);
  // slices of the row tiles while the ranges leave places on the chip free
  const long long blocks = (long long)B * H * p.ranges, places = 2LL * num_cus();
  long long slices = places / (blocks < 1 ? 1 : blocks);
  if (slices > (p.seq_tiles + 3) / 4) slices = (p.seq_tiles + 3) / 4;
  p.slices = slices < 1 ? 1 : (int)slices;
  auto up = [](size_t x) { return (x + 255) & ~size_t(255); };
  size_t off = 0;
  p.off_ops = off, off = up(off + (size_t)p.tiles * H * kOpBytes);
  p.off_down = off, off = up(off + (size_t)p.tiles * H * sizeof(float));
  p.off_stats = off, off = up(off + (size_t)p.ranges * p.tiles * H * kRows * sizeof(float2));
  p.off_lse = off, off = up(off + (size_t)p.tiles * H * kRows * sizeof(float));
  p.off_part = off, off = up(off + (size_t)places * kRangeTokens * sizeof(float));  // (a smaller call may take more slices)
  p.total = off;
  return p;
}

namespace {

template <int NG>
hipError_t launch_ng(const TokenWeightsArgs& a, hipStream_t s) {
  const long long H = a.cv.num_kv_heads;
  hipError_t e = hipSuccess;
  if (a.seq_tiles > 0) {
    const long long items = a.B * H * a.seq_tiles;
    const int per = (int)(items / 1024 < 1 ? 1 : items / 1024 > 8 ? 8 : items / 1024);
    hipLaunchKernelGGL(weight_rows_kernel, dim3((unsigned)(a.B * H * ((a.seq_tiles + per - 1) / per))), dim3(256), 0, s, a, per);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(weight_stats_kernel<NG>, dim3((unsigned)(a.B * H * a.slices * a.ranges)), dim3(64 * kWaves), 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(weight_lse_kernel, dim3((unsigned)((items + 7) / 8)), dim3(256), 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  hipLaunchKernelGGL(weight_sums_kernel<NG>, dim3((unsigned)(a.B * H * a.slices * a.ranges)), dim3(64 * kWaves), 0, s, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  if (a.slices > 1) {
    hipLaunchKernelGGL(weight_join_kernel, dim3((unsigned)(a.B * H * a.ranges)), dim3(kRangeTokens), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

hipError_t launch_token_weights(TokenWeightsArgs a, const TokenWeightsPlan& p, uint8_t* ws, hipStream_t s) {
  a.seq_tiles = p.seq_tiles, a.ranges = p.ranges, a.slices = p.slices, a.tiles = p.tiles;
  a.ops = ws + p.off_ops;
  a.down = reinterpret_cast<float*>(ws + p.off_down);
  a.stats = reinterpret_cast<float2*>(ws + p.off_stats);
  a.lse = reinterpret_cast<float*>(ws + p.off_lse);
  a.part = reinterpret_cast<float*>(ws + p.off_part);
  return a.cv.groups == 4 ? launch_ng<4>(a, s) : launch_ng<1>(a, s);
}

}  // namespace int2kv
