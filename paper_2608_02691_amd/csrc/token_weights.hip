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

// ---- Few rows a sequence (decode steps): up to kFewRows rows of one KV head. The scores are formed once and kept; the second
// pass goes over them and not over the keys.
namespace {

constexpr int kFewRows = 8;
constexpr int kPieceTokens = 512, kPiecePages = kPieceTokens / kBlock / 4;  // of a block; pages of each of its four waves
constexpr int kJoinTokens = 1024;

// The rows' operands for products of 16 rows x 16 tokens: row 4 j + g of tile t holds group g's channels of query row
// 4 t + j and zeros elsewhere, so that D's registers are the four groups' sums of one query row and token. A lane's
// eight channels (lane = 16 quad + 4 j + g): positions 2 g, 2 g + 1 of words 2 quad, 2 quad + 1.
struct FewOps {
  cd_h8_t term[2][2][64];  // [tile][high, low]
  float sum[2][4][4];      // Q_g of [tile][row]
  float down, pad[3];
};

__device__ __forceinline__ cd_f4_t product16(const cd_h8_t& x, const cd_h8_t& y, const cd_f4_t& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, c, 0, 0, 0);
}

}  // namespace

// Block: one (sequence, KV head). Thread: channel c of every other row.
__global__ __launch_bounds__(256) void weight_few_rows_kernel(TokenWeightsArgs a) {
  __shared__ float q[kFewRows][kHeadDim], top[4];
  const int H = a.cv.num_kv_heads, h = blockIdx.x % H, b = blockIdx.x / H, c = threadIdx.x & 127, odd = threadIdx.x >> 7;
  const Span s = span_of(a, b);
  const int rows = min(s.n * a.gq, kFewRows);
  if (rows == 0 || s.ctx == 0) return;
  for (int i = threadIdx.x; i < kFewRows * kHeadDim; i += 256) {
    const int r = i >> 7, tok = r / a.gq;
    q[r][i & 127] = r < rows ? bf16_bits_to_f32(a.q[(s.start + tok) * a.q_stride + (size_t)(h * a.gq + r - tok * a.gq) * kHeadDim + (i & 127)]) : 0.0f;
  }
  __syncthreads();
  float d[kFewRows / 2] = {};
  const float* R = a.R_k + (size_t)h * kHeadDim * kHeadDim + c;
#pragma unroll 32
  for (int k = 0; k < kHeadDim; ++k) {
    const float x = R[(size_t)k * kHeadDim];
#pragma unroll
    for (int i = 0; i < kFewRows / 2; ++i) d[i] = __builtin_fmaf(q[2 * i + odd][k], x, d[i]);
  }
  float big = 0.0f;
#pragma unroll
  for (int i = 0; i < kFewRows / 2; ++i) {
    d[i] *= kLogit2;
    big = fmaxf(big, fabsf(d[i]));
  }
#pragma unroll
  for (int step = 32; step > 0; step >>= 1) big = fmaxf(big, __shfl_xor(big, step));
  if ((threadIdx.x & 63) == 0) top[threadIdx.x >> 6] = big;
  __syncthreads();
  big = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
  const uint32_t e = min(max(__float_as_uint(big) >> 23, 8u), 254u);
  const float up = __uint_as_float((261u - e) << 23);
  FewOps& out = reinterpret_cast<FewOps*>(a.few)[(size_t)b * H + h];
  const int g = c >> 5, p = (c >> 4) & 1, word = (c & 15) >> 1, element = ((word & 1) << 2) | (p << 1) | (c & 1);
#pragma unroll
  for (int i = 0; i < kFewRows / 2; ++i) {
    const int r = 2 * i + odd, lane = 16 * (word >> 1) + 4 * (r & 3) + g;
    const float x = d[i] * up;
    const _Float16 hi = (_Float16)x;
    reinterpret_cast<_Float16*>(&out.term[r >> 2][0][lane])[element] = hi;
    reinterpret_cast<_Float16*>(&out.term[r >> 2][1][lane])[element] = (_Float16)(x - (float)hi);
    float sum = x;  // over the group: 32 lanes
#pragma unroll
    for (int step = 16; step > 0; step >>= 1) sum += __shfl_xor(sum, step);
    if ((c & 31) == 0) out.sum[r >> 2][r & 3][g] = sum;
  }
  if (threadIdx.x == 0) out.down = __uint_as_float((e - 7u) << 23);
}

// Block: 512 tokens of one KV head, a wave eight pages of them; all loads of a wave are on their way at once. Lane: one token
// of a page and one row of each tile. TILES: of four rows.
template <int NG, int TILES>
__global__ __launch_bounds__(256) void weight_few_scores_kernel(TokenWeightsArgs a) {
  using Lay = Rec<NG>;
  __shared__ float2 both[4][kFewRows];
  const int H = a.cv.num_kv_heads, h = blockIdx.x % H, piece = blockIdx.x / H % a.pieces, b = blockIdx.x / H / a.pieces;
  const Span s = span_of(a, b);
  if (kPieceTokens * piece >= s.ctx || s.n == 0) return;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, t = l & 15, quad = l >> 4;
  const int page0 = kPieceTokens / kBlock * piece + kPiecePages * w, pages = (s.ctx + kBlock - 1) / kBlock;
  int id = -1;
  if (l < kPiecePages && page0 + l < pages) id = a.table[(size_t)b * a.max_blocks + page0 + l];
  const uint32_t real = (uint32_t)__ballot(id >= 0 && id < a.cv.num_blocks);
  cd_u2_t code[kPiecePages];
  uint32_t meta[kPiecePages][NG];
#pragma unroll
  for (int i = 0; i < kPiecePages; ++i) {
    const int x = __builtin_amdgcn_readlane(id, i);
    const uint8_t* rec = a.cv.pool + ((size_t)(uint32_t)((real >> i) & 1 ? x : 0) * H + h) * Lay::kBytes;
    code[i] = *reinterpret_cast<const cd_u2_t*>(rec + kOffKCodes + 32 * t + 8 * quad);
#pragma unroll
    for (int g = 0; g < NG; ++g) meta[i][g] = reinterpret_cast<const uint32_t*>(rec + Lay::kOffKMeta + 4 * NG * t)[g];
  }
  const FewOps& ops = reinterpret_cast<const FewOps*>(a.few)[(size_t)b * H + h];
  const float down = ops.down;
  cd_h8_t A[TILES][2][4];  // [tile][high, low][group]
  float Q[TILES][4];
  int lim[TILES];
  const cd_h8_t none{};
#pragma unroll
  for (int k = 0; k < TILES; ++k) {
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const cd_h8_t y = ops.term[k][x][l];
#pragma unroll
      for (int g = 0; g < 4; ++g) A[k][x][g] = (l & 3) == g ? y : none;
    }
    const float4 v = *reinterpret_cast<const float4*>(ops.sum[k][quad]);
    Q[k][0] = v.x * down, Q[k][1] = v.y * down, Q[k][2] = v.z * down, Q[k][3] = v.w * down;
    const int row = 4 * k + quad;
    lim[k] = row < s.n * a.gq ? s.limit(row / a.gq) : 0;
  }
  float m[TILES], sum[TILES];
#pragma unroll
  for (int k = 0; k < TILES; ++k) m[k] = kNone, sum[k] = 0.0f;
  float* scores = a.scores + ((size_t)b * H + h) * a.page_cap * (kBlock * a.row_cap);
#pragma unroll
  for (int i = 0; i < kPiecePages; ++i) {
    if (page0 + i >= pages) break;
    cd_h8_t c[4];
    const uint32_t u = code[i].x, v = code[i].y, uh = u >> 10, vh = v >> 10;
    auto put = [&](cd_h8_t& y, cd_h2_t p, cd_h2_t q, cd_h2_t r, cd_h2_t z) { y = cd_h8_t{p.x, p.y, q.x, q.y, r.x, r.y, z.x, z.y}; };
    put(c[0], land_position<0>(u, uh), land_position<1>(u, uh), land_position<0>(v, vh), land_position<1>(v, vh));
    put(c[1], land_position<2>(u, uh), land_position<3>(u, uh), land_position<2>(v, vh), land_position<3>(v, vh));
    put(c[2], land_position<4>(u, uh), land_position<5>(u, uh), land_position<4>(v, vh), land_position<5>(v, vh));
    put(c[3], land_position<6>(u, uh), land_position<7>(u, uh), land_position<6>(v, vh), land_position<7>(v, vh));
    const int token = kBlock * (page0 + i) + t;
#pragma unroll
    for (int k = 0; k < TILES; ++k) {
      cd_f4_t D = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        D = product16(A[k][0][g], c[g], D);
        D = product16(A[k][1][g], c[g], D);
      }
      float x = 0.0f;
      if constexpr (NG == 4) {
        float z = 0.0f;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          x = __builtin_fmaf(f16_bits_to_f32(meta[i][g] & 0xFFFFu), D[g], x);
          z = __builtin_fmaf(f16_bits_to_f32(meta[i][g] >> 16), Q[k][g], z);
        }
        x = __builtin_fmaf(x, down, z);
      } else {
        x = __builtin_fmaf(f16_bits_to_f32(meta[i][0] & 0xFFFFu) * down, (D[0] + D[1]) + (D[2] + D[3]),
                           f16_bits_to_f32(meta[i][0] >> 16) * ((Q[k][0] + Q[k][1]) + (Q[k][2] + Q[k][3])));
      }
      x = (real >> i) & 1 && token < lim[k] ? x : -INFINITY;
      // the reference moves when a score exceeds it by 2^40, which fp32's sums have room for
      if (__any(x > m[k] + 40.0f)) {
        const float top = fmaxf(m[k], x);
        sum[k] *= __builtin_amdgcn_exp2f(m[k] - top);
        m[k] = top;
      }
      sum[k] += __builtin_amdgcn_exp2f(x - m[k]);
      if (4 * k + quad < a.row_cap) scores[((size_t)(page0 + i) * a.row_cap + 4 * k + quad) * kBlock + t] = x;
    }
  }
#pragma unroll
  for (int k = 0; k < TILES; ++k) {
    const float top = row_max16(m[k]);
    const float all = row_sum16(sum[k] * __builtin_amdgcn_exp2f(m[k] - top));
    if (t == 0) both[w][4 * k + quad] = make_float2(top, all);
  }
  __syncthreads();
  if (threadIdx.x < 4 * TILES) {
    float top = kNone, all = 0.0f;
#pragma unroll
    for (int x = 0; x < 4; ++x) top = fmaxf(top, both[x][threadIdx.x].x);
#pragma unroll
    for (int x = 0; x < 4; ++x) all += both[x][threadIdx.x].y * __builtin_amdgcn_exp2f(both[x][threadIdx.x].x - top);
    a.stats[(((size_t)b * H + h) * a.pieces + piece) * kFewRows + threadIdx.x] = make_float2(top, all);
  }
}

// Block: 1,024 tokens of one KV head, a thread four of them. Each wave joins the pieces of its rows first.
__global__ __launch_bounds__(256) void weight_few_join_kernel(TokenWeightsArgs a) {
  __shared__ float lse[kFewRows];
  const int H = a.cv.num_kv_heads, joins = (a.page_cap * kBlock + kJoinTokens - 1) / kJoinTokens;
  const int h = blockIdx.x % H, join = blockIdx.x / H % joins, b = blockIdx.x / H / joins, w = threadIdx.x >> 6, l = threadIdx.x & 63;
  const Span s = span_of(a, b);
  if (kJoinTokens * join >= s.ctx) return;
  const int rows = min(s.n * a.gq, a.row_cap), pieces = (s.ctx + kPieceTokens - 1) / kPieceTokens;
  const float2* stats = a.stats + ((size_t)b * H + h) * a.pieces * kFewRows;
  for (int r = w; r < rows; r += 4) {
    float top = kNone, all = 0.0f;
    for (int x = l; x < pieces; x += 64) {
      const float2 v = stats[(size_t)x * kFewRows + r];
      const float next = fmaxf(top, v.x);
      all = all * __builtin_amdgcn_exp2f(top - next) + v.y * __builtin_amdgcn_exp2f(v.x - next);
      top = next;
    }
    float most = top;
#pragma unroll
    for (int step = 32; step > 0; step >>= 1) most = fmaxf(most, __shfl_xor(most, step));
    all *= __builtin_amdgcn_exp2f(top - most);
#pragma unroll
    for (int step = 32; step > 0; step >>= 1) all += __shfl_xor(all, step);
    if (l == 0) lse[r] = all == 0.0f ? INFINITY : most + __builtin_amdgcn_logf(all);
  }
  __syncthreads();
  const int t = kJoinTokens * join + 4 * threadIdx.x;
  if (t >= s.ctx) return;
  const float* scores = a.scores + (((size_t)b * H + h) * a.page_cap + t / kBlock) * (kBlock * a.row_cap) + (t & 15);
  float sum[4] = {};
  for (int r = 0; r < rows; ++r) {
    const float4 x = *reinterpret_cast<const float4*>(scores + r * kBlock);
    sum[0] += __builtin_amdgcn_exp2f(x.x - lse[r]), sum[1] += __builtin_amdgcn_exp2f(x.y - lse[r]);
    sum[2] += __builtin_amdgcn_exp2f(x.z - lse[r]), sum[3] += __builtin_amdgcn_exp2f(x.w - lse[r]);
  }
  const size_t at = ((size_t)b * H + h) * a.w_stride + t;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (t + i < s.ctx) a.w_out[at + i] = a.w_in ? __builtin_fmaf(a.decay, a.w_in[at + i], sum[i]) : sum[i];
}

TokenWeightsPlan make_token_weights_plan(int B, int Hq, int H, int total_q, int max_q, int max_ctx) {
  TokenWeightsPlan p{};
  const int gq = Hq / H;
  const long long seq_rows = (long long)max_q * gq;
  p.few = seq_rows > 0 && seq_rows <= kFewRows;
  p.seq_tiles = (int)((seq_rows + kRows - 1) / kRows);
  p.ranges = (int)(((long long)max_ctx + kRangeTokens - 1) / kRangeTokens);
  if (p.ranges < 1) p.ranges = 1;
  p.pieces = (int)(((long long)max_ctx + kPieceTokens - 1) / kPieceTokens);
  p.page_cap = (int)(((long long)max_ctx + kBlock - 1) / kBlock);
  p.row_cap = (int)(seq_rows < kFewRows ? seq_rows : kFewRows);
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
  // few rows: a call within these bounds may have them, whether or not this one does
  off = 0;
  p.off_few = off, off = up(off + (size_t)B * H * sizeof(FewOps));
  p.off_few_stats = off, off = up(off + (size_t)B * H * p.pieces * kFewRows * sizeof(float2));
  p.off_scores = off, off = up(off + (size_t)B * H * p.page_cap * kBlock * p.row_cap * sizeof(float));
  p.total = p.total > off ? p.total : off;
  return p;
}

namespace {

template <int NG>
hipError_t launch_few(const TokenWeightsArgs& a, hipStream_t s) {
  const long long H = a.cv.num_kv_heads;
  hipLaunchKernelGGL(weight_few_rows_kernel, dim3((unsigned)(a.B * H)), dim3(256), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)(a.B * H * a.pieces));
  if (a.row_cap <= 4)
    hipLaunchKernelGGL((weight_few_scores_kernel<NG, 1>), grid, dim3(256), 0, s, a);
  else
    hipLaunchKernelGGL((weight_few_scores_kernel<NG, 2>), grid, dim3(256), 0, s, a);
  if ((e = hipGetLastError()) != hipSuccess) return e;
  const long long joins = ((long long)a.page_cap * kBlock + kJoinTokens - 1) / kJoinTokens;
  hipLaunchKernelGGL(weight_few_join_kernel, dim3((unsigned)(a.B * H * joins)), dim3(256), 0, s, a);
  return hipGetLastError();
}

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
  if (p.few) {
    a.few = ws + p.off_few;
    a.stats = reinterpret_cast<float2*>(ws + p.off_few_stats);
    a.scores = reinterpret_cast<float*>(ws + p.off_scores);
    a.pieces = p.pieces, a.page_cap = p.page_cap, a.row_cap = p.row_cap;
    return a.cv.groups == 4 ? launch_few<4>(a, s) : launch_few<1>(a, s);
  }
  return a.cv.groups == 4 ? launch_ng<4>(a, s) : launch_ng<1>(a, s);
}

}  // namespace int2kv
