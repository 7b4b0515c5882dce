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
#include <type_traits>

#include "append_core.h"
#include "chunk_core.h"

namespace int2kv {

namespace {

constexpr int kRows = 32;                                     // rows of a tile
constexpr int kChunkTiles = 32;                               // row tiles of a block at most
constexpr size_t kSlabBytes = size_t(1) << 30;                // of the workspace, beyond which row tiles are taken in slabs
constexpr float kSure = 60.0f;  // ref lies above a row's largest score by less than this; sums reach 2^-66 of the largest term
constexpr float kFar = 100.0f;  // scores above ref by more than this are summed relative to their own maximum
static_assert(kRangeTokens == 4 * 64, "the waves' tokens");

struct Span {
  int start, n, ctx, past;  // as Seq (but the table does not cut ctx)
  int tile0;                // place of the sequence's first row tile (in slabs: as if there were one)
  __device__ __forceinline__ int limit(int i) const { return max(min(ctx, past + i + 1), 0); }
};
// The tiles of sequence b start at start * gq / 32 + b: never before the end of the one before. In slabs every sequence has the
// same number of places, for its tiles from the slab's first one on.
__device__ __forceinline__ Span span_of(const TokenWeightsArgs& a, int b) {
  Span s;
  s.start = min(max(a.starts[b], 0), a.total_q);
  const int end = min(max(a.starts[b + 1], 0), a.total_q);
  const int count = max(end - s.start, 0), len = max(a.lens[b], 0);
  s.n = min(count, a.max_q);
  s.ctx = min(len, a.max_ctx);  // tokens behind the table's end lie in no block: their sums decay with the others
  s.past = len - count;
  s.tile0 = a.slab_tiles > 0 ? b * a.slab_tiles - a.chunk0 * a.chunk_tiles : (int)((long long)s.start * a.gq / kRows) + b;
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
  float scale[NG], low[NG];
  cd_h8_t zero;
  bool real;
  __device__ __forceinline__ void load(const TokenWeightsArgs& a, int b, int h, int token, int ctx, int hh) {
    int id = -1;
    if (token < ctx && token / kBlock < a.max_blocks) id = a.table[(size_t)b * a.max_blocks + token / kBlock];
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
      low[g] = f16_bits_to_f32(sz >> 16);
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

// A row tile's operands, and beside them what else its readers need
struct RowTile {
  cd_h8_t hi[8][64], lo[8][64];
  cd_h8_t group[32];       // Q_g: high terms, low terms (the other lane half's is zero)
  float ref[kRows];        // near the row's largest score over the first tokens: its sums are formed relative to it
  float lse[kRows];        // L_r; infinite for rows that see nothing and behind the last one, so that their weights are zero
  float down;              // what brings the scores back to size
  uint32_t unsure;         // not zero: some row's ref names no score of its own, or may lie far above it
  float pad[62];
};
constexpr int kTileBytes = sizeof(RowTile), kPieces = kTileBytes / 1024;
static_assert(kTileBytes == 17 * 1024, "pieces of 64 lanes x 16 bytes");

__device__ __forceinline__ cd_f16_t product(const cd_h8_t& x, const cd_h8_t& y, const cd_f16_t& c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(x, y, c, 0, 0, 0);
}

// A block's share: a range of tokens of one KV head and a chunk of the row tiles that see it
struct Share {
  int b, h, bh, range, chunk, first, t0, t1;  // first token; tiles
};
__device__ __forceinline__ Share share_of(const TokenWeightsArgs& a, int bh, int range, int chunk, const Span& s) {
  Share x;
  x.bh = bh, x.range = range, x.chunk = chunk;
  x.b = bh / a.cv.num_kv_heads, x.h = bh - x.b * a.cv.num_kv_heads;
  x.first = kRangeTokens * range;
  x.t0 = x.t1 = 0;
  if (x.first < s.ctx) {
    const int rows = s.n * a.gq, tiles = (rows + kRows - 1) / kRows;
    // the first row that sees the first token
    x.t0 = max(a.chunk_tiles * chunk, max(x.first - s.past, 0) * a.gq / kRows);
    x.t1 = min(tiles, a.chunk_tiles * (chunk + 1));
  }
  return x;
}

}  // namespace

// ---- The rows' operands. Block: row tiles of one KV head, one after the other; wave w forms channels 32 w .. of q R_K on the
// matrix cores, R_K in three bf16 terms that sum to it exactly. A tile's rows are scaled by one power of two that brings
// the largest element to 2^7 .. 2^8: what the low terms lose, 2^-24, is 2^-31 of it, and a group's sum fits fp16. The
// last wave forms the rows' scores over the sequence's first 32 tokens, in one fp16 term: their maximum is where the first pass starts.
// Its roundings, 2^-11 of a query and of a key, may come to many powers of two where scores are large: up to 2^-10 sum |q'_c k_c|, at
// most 2^-10 128 max |q'| max |k|. Above a row's scores by 126 and more it would leave nothing of the row's sums, so tiles in which the
// bound passes kSure are summed relative to their own maxima.
// Bound by the operands it writes, 17 KB a tile: 14,200 tokens of 32 + 8 heads 95 us, 3.7 TB/s. Blocks of several tiles bring R_K
// once: with one tile each, whole prompts of 4 x 4,000 tokens take 1,448 us, with up to eight 1,380.
template <int NG>
__global__ __launch_bounds__(256) void weight_rows_kernel(TokenWeightsArgs a, int tiles_per_block) {
  __shared__ float top[4], sums[4][kRows];
  __shared__ cd_h8_t keys[8][64];  // the first tokens' rows, rounded to fp16: the last wave's
  __shared__ cd_u4_t in[2][8][64];
  __shared__ __align__(16) RowTile out;
  const int H = a.cv.num_kv_heads, blocks = (a.seq_tiles + tiles_per_block - 1) / tiles_per_block;
  const int h = blockIdx.x % H, at = blockIdx.x / H % blocks, b = blockIdx.x / H / blocks;
  const Span s = span_of(a, b);
  const int slab0 = a.chunk0 * a.chunk_tiles, tiles = min((s.n * a.gq + kRows - 1) / kRows, slab0 + a.seq_tiles), t0 = slab0 + at * tiles_per_block;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, n = l & 31, hh = l >> 5;
  if (t0 >= tiles || s.ctx == 0) return;
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
  uint32_t real = 0;
  float key_top = 0x1p-14f;  // the largest element of the lane's part of the keys (below 2^-14 fp16's steps no longer shrink)
  if (w == 3) {
    Token<NG> first;
    first.load(a, b, h, n, s.ctx, hh);
    real = (uint32_t)__ballot(first.real);
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      cd_h8_t k;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float y = __builtin_fmaf((float)first.code[x][j], first.scale[x * NG / 8], first.low[x * NG / 8]);
        key_top = first.real ? fmaxf(key_top, fabsf(y)) : key_top;
        k[j] = (_Float16)y;
      }
      keys[x][l] = k;
    }
  }
  const int t1 = min(tiles, t0 + tiles_per_block), rows = s.n * a.gq;
  // a tile's rows on their way to LDS as the products take them, a quarter by each wave; the last one's again behind the last
  auto fetch = [&](int t) {
    const int row = min(kRows * t + n, rows - 1), tok = quotient(row, a.gq);
    const uint16_t* q = a.q + (s.start + tok) * a.q_stride + (size_t)(h * a.gq + row - tok * a.gq) * kHeadDim + 8 * hh;
#pragma unroll
    for (int i = 0; i < 2; ++i) ap_dma16(q + 16 * (2 * w + i), (uint32_t)(uintptr_t)&in[t & 1][2 * w + i][0]);
  };
  fetch(t0);
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  for (int t = t0; t < t1; ++t) {
    if (t + 1 < t1) fetch(t + 1);
    const bool live = kRows * t + n < rows;
    cd_f16_t d = splat16(0.0f);
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      const cd_u4_t x = live ? in[t & 1][kk][l] : cd_u4_t{0, 0, 0, 0};
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
    if (l == 0) top[w] = big;
    __syncthreads();  // (and the tile before has left)
    big = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    const uint32_t e = min(max(__float_as_uint(big) >> 23, 8u), 254u);
    const float up = __uint_as_float((261u - e) << 23), down = __uint_as_float((e - 7u) << 23);
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
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the next tile's rows (and the last one's stores)
    __syncthreads();
    uint4* to = reinterpret_cast<uint4*>(a.ops + ((size_t)(s.tile0 + t) * H + h) * kTileBytes);
    RowTile& tile = *reinterpret_cast<RowTile*>(to);
    const uint4* from = reinterpret_cast<const uint4*>(&out);
    if (w == 3) {
      cd_f16_t S = splat16(0.0f);
#pragma unroll
      for (int x = 0; x < 8; ++x) S = product(keys[x][l], out.hi[x][l], S);
      const int lim = live ? s.limit(quotient(kRows * t + n, a.gq)) : 0;
      float m = -INFINITY;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int x = 8 * (r >> 2) + 4 * hh + (r & 3);
        m = fmaxf(m, x < lim && ((real >> x) & 1) ? S[r] : -INFINITY);
      }
      m = pair_max(m) * down;
      const bool good = fabsf(m) < 1.0e30f;
      if (hh == 0) tile.ref[n] = good ? m : 0.0f;
      const bool unsure = __any((lim > 0 && !good) || 0.125f * big * key_top > kSure);
      if (l == 0) tile.unsure = unsure;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) to[threadIdx.x + 256 * i] = from[threadIdx.x + 256 * i];
    if (threadIdx.x < kRows) {
      float x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = sums[i][n];
      if (a.cv.groups == 1) x[0] = (x[0] + x[1]) + (x[2] + x[3]), x[1] = x[2] = x[3] = 0.0f;
      cd_h8_t g;
#pragma unroll
      for (int i = 0; i < 4; ++i) g[i] = (_Float16)x[i], g[4 + i] = (_Float16)(x[i] - (float)g[i]);
      to[1024 + n] = __builtin_bit_cast(uint4, g);
      if (n == 0) tile.down = down;
    }
  }
}

// ---- The two passes over the keys. Block: 256 tokens of one KV head and a chunk of the row tiles that see them; a wave has
// 64 tokens. Products are rows x codes, so that a lane holds a token and its scales. PASS 1 sums each row's 2^(x - ref)
// over the range, PASS 2 each token's 2^(x - L) over the rows. Whole prompts of 3,000 to 4,096 tokens (210 GFLOP of scores, in two
// terms): 560 and 450 us, 0.75 and 0.93 PFLOP/s; matrix pipe 33 and 44 %, vector ALU 52 and 57 % of cycles, at 1.9 GHz.
namespace {

constexpr int kSlots = 4;

// Sums over the 32 lanes of a half for all sixteen registers: halves of what is left change places, so that a lane ends with the
// sum of one register, lane_register()
__device__ __forceinline__ float fold(cd_f16_t v, const bool max_of) {
  auto f = [&](float x, float y) { return max_of ? fmaxf(x, y) : x + y; };
  const int l = threadIdx.x;
  float a[8], b[4], c[2];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[i]), __float_as_uint(v[i + 8]), false, false);
    a[i] = f(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) b[i] = f(l & 8 ? a[i + 4] : a[i], dppf<0x128>(l & 8 ? a[i] : a[i + 4]));        // row_ror:8
#pragma unroll
  for (int i = 0; i < 2; ++i) c[i] = f(l & 4 ? b[i + 2] : b[i], dppf<0x141>(l & 4 ? b[i] : b[i + 2]));        // row_half_mirror
  const float d = f(l & 2 ? c[1] : c[0], dppf<0x4E>(l & 2 ? c[0] : c[1]));                                     // quad_perm 2 3 0 1
  return f(d, dppf<0xB1>(d));                                                                                 // quad_perm 1 0 3 2
}
// Of the instructions around: a product, then V of the vector ALU, N times
template <int N, int V>
__device__ __forceinline__ void in_turn() {
  if constexpr (N > 0) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x402, V, 0);
    in_turn<N - 1, V>();
  }
}
// The row (of its tile) of a lane's fold
__device__ __forceinline__ int fold_row(int l) {
  const int r = ((l >> 4) & 1) << 3 | ((l >> 3) & 1) << 2 | ((l >> 2) & 1) << 1 | ((l >> 1) & 1);
  return 8 * (r >> 2) + 4 * (l >> 5) + (r & 3);
}

}  // namespace

template <int NG, int PASS>
__global__ __launch_bounds__(256, 2) void weight_scan_kernel(TokenWeightsArgs a) {
  __shared__ __align__(16) RowTile lds[kSlots];
  __shared__ float2 both[2][4][kRows], stats[PASS == 1 ? kChunkTiles : 1][kRows];
  __shared__ float top_of[4][kRows];
  __shared__ float2 unused[PASS == 1 ? 64 : 1];
  // Heads come first, so that the blocks of a head share an XCD's L2, then ranges: the engines of an XCD take
  // blocks in turn, which by sequences of different lengths leaves some with more to do. Last chunks go first: those that most ranges see
  const int H = a.cv.num_kv_heads, BH = a.B * H, other = blockIdx.x / H, bh = other / a.ranges % a.B * H + blockIdx.x % H;
  const Span s = span_of(a, bh / H);
  const Share me = share_of(a, bh, other % a.ranges, a.chunk0 + a.chunks - 1 - other / a.ranges / a.B, s);
  if (me.t0 >= me.t1 && (PASS == 1 || a.part || me.first >= s.ctx)) return;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, n = l & 31, hh = l >> 5, token0 = me.first + 64 * w;
  // ---- Row tiles on their way to LDS, tile t in slot t % kSlots. Half way through a tile (at its start) the next one has landed for every wave
  // and the one before is done with, so that no wave waits between tiles.
  const uint8_t* tiles = a.ops + ((ptrdiff_t)s.tile0 * H + me.h) * kTileBytes + 16 * l;  // of tile 0, which a slab may not hold
  const size_t stride = (size_t)H * kTileBytes;
  const uint32_t lds0 = (uint32_t)(uintptr_t)&lds[0];
  auto slot = [&](int t) -> const RowTile& { return lds[t & (kSlots - 1)]; };
  auto issue = [&](int t) {  // 17 pieces by four waves: the first has one more
    if (t >= me.t1) return;
    for (int c = w; c < kPieces; c += 4) ap_dma16(tiles + t * stride + 1024 * c, lds0 + (uint32_t)((t & (kSlots - 1)) * kTileBytes + 1024 * c));
  };
  // until tile t has landed, with what came after it, up to `after` tiles, on its way
  auto landed = [&](int t, auto after) {
    constexpr int A = decltype(after)::value;
    if (t + A >= me.t1)
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    else if (w == 0)
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(A * (kPieces / 4 + 1)) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"(A * (kPieces / 4)) : "memory");
    __syncthreads();
  };
#pragma unroll
  for (int t = 0; t < kSlots - 1; ++t) issue(me.t0 + t);

  Token<NG> tok[2];
  float sum[2] = {0.0f, 0.0f};
  int from[2];  // rows that see the lane's tokens, less its half's 4
#pragma unroll
  for (int u = 0; u < 2; ++u) {
    tok[u].load(a, me.b, me.h, token0 + 32 * u + n, s.ctx, hh);
    from[u] = tok[u].real ? max(token0 + 32 * u + n - s.past, 0) * a.gq - 4 * hh : INT32_MAX;
  }
  const bool whole = __all(tok[0].real && tok[1].real), any = __any(tok[0].real || tok[1].real);
  // tiles from which all of the wave's tokens are seen by every row, some by some
  const int all_from = PASS == 1 && !whole ? me.t1 : (max(min(token0 + 63, s.ctx - 1) - s.past, 0) * a.gq + kRows - 1) / kRows;
  const int some_from = any ? max(token0 - s.past, 0) * a.gq / kRows : me.t1;

  // Eight steps a tile (a quarter of the products of one token tile each): while the matrix cores form a step's products the
  // vector ALU adds the last one's to the scores, in the first two also sums the tile before. X: that tile's
  // scores less ref (L), then this one's.
  cd_f16_t X[2] = {splat16(-INFINITY), splat16(-INFINITY)};
  bool pending = false;
  auto scores = [&](const RowTile& ops, auto&& beside, auto&& middle) {
    if constexpr (PASS == 2) middle();  // (in the middle it would cost the second pass registers it does not have)
    const cd_h8_t group = ops.group[n];  // (the other lane half's tokens have zeros there)
    cd_h8_t op[2][2][2];  // [quarter][high, low]
    auto read = [&](int q) {
#pragma unroll
      for (int x = 0; x < 2; ++x) op[q & 1][0][x] = ops.hi[2 * q + x][l], op[q & 1][1][x] = ops.lo[2 * q + x][l];
    };
    read(0);
    cd_f16_t D[2];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if (PASS == 1 && q == 2 && u == 0) middle();
        if (u == 1 && q < 3) read(q + 1);
        const cd_h8_t(&y)[2][2] = op[q & 1];
        D[u] = product(y[0][0], tok[u].code[2 * q], NG == 4 || q == 0 ? splat16(0.0f) : D[u]);
        D[u] = product(y[1][0], tok[u].code[2 * q], D[u]);
        D[u] = product(y[0][1], tok[u].code[2 * q + 1], D[u]);
        D[u] = product(y[1][1], tok[u].code[2 * q + 1], D[u]);
        beside(2 * q + u);
        if (q == 0) X[u] = product(group, tok[u].zero, splat16(0.0f));
        if (NG == 4 && q + u > 0) {
          const int v = u ^ 1, g = u == 1 ? q : q - 1;
#pragma unroll
          for (int r = 0; r < 16; ++r) X[v][r] = __builtin_fmaf(tok[v].scale[NG == 4 ? g : 0], D[v][r], X[v][r]);
        }
        // products and vector instructions in turn: a wave issues in order, and each product waits for the one before
        if (q == 0) {
          if (u == 0) __builtin_amdgcn_sched_group_barrier(0x402, 8, 0);
          in_turn<5, 8>();
        } else
          in_turn<4, 4>();
        __builtin_amdgcn_sched_barrier(0);
      }
    const float* base = PASS == 1 ? ops.ref : ops.lse;
    const float down = ops.down;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float4 v = *reinterpret_cast<const float4*>(&base[8 * x + 4 * hh]);
      const float less[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int y = 0; y < 4; ++y)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int r = 4 * x + y;
          if (u == 1 || NG == 1) X[u][r] = __builtin_fmaf(tok[u].scale[NG - 1], D[u][r], X[u][r]);
          X[u][r] = __builtin_fmaf(X[u][r], down, -less[y]);
        }
    }
  };
  // A tile's sums from its X: step 0 and 1 the token tiles', step 2, in PASS 1, over the wave's tokens
  cd_f16_t v;
  auto sums = [&](int i, int t) {
    if (i > 2) return;
    if (i == 2) {
      if (PASS == 2) return;
      // (by the address, not by a branch, into which the compiler would move the exponentials, behind the products)
      float2* to = pending ? &both[t & 1][w][fold_row(l)] : &unused[l];
      *to = make_float2(0.0f, fold(v, false));  // lanes of a pair the same
      return;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float x = __builtin_amdgcn_exp2f(X[i][r]);
      if constexpr (PASS == 2)
        sum[i] += x;
      else
        v[r] = i == 0 ? x : v[r] + x;
    }
  };
  auto all_sums = [&](int t) {
    for (int i = 0; i < 3; ++i) sums(i, t);
    X[0] = X[1] = splat16(-INFINITY);
    pending = false;
  };
  // PASS 1: relative to the rows' maxima, which lie far from ref
  auto peak_sums = [&](int t) {
#pragma unroll
    for (int r = 0; r < 16; ++r) v[r] = fmaxf(X[0][r], X[1][r]);
    float top = fold(v, true);
    top = top == -INFINITY ? 0.0f : top;
    top_of[w][fold_row(l)] = top;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float m = top_of[w][8 * (r >> 2) + 4 * hh + (r & 3)];
      v[r] = __builtin_amdgcn_exp2f(X[0][r] - m) + __builtin_amdgcn_exp2f(X[1][r] - m);
    }
    const float all = fold(v, false);
    if ((l & 1) == 0) both[t & 1][w][fold_row(l)] = make_float2(top, all);
    X[0] = X[1] = splat16(-INFINITY);
    pending = false;
  };
  auto far_off = [&]() {
    float m = X[0][0];
#pragma unroll
    for (int r = 1; r < 32; ++r) m = fmaxf(m, X[r >> 4][r & 15]);
    return __any(m > kFar);
  };
  // PASS 1: the waves' sums of a tile, relative to its ref
  auto join = [&](int t) {
    const float2(&x)[4][kRows] = both[t & 1];
    float top = -INFINITY, all = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) top = fmaxf(top, x[i][n].y == 0.0f ? -INFINITY : x[i][n].x);
    const float base = top == -INFINITY ? 0.0f : top;
#pragma unroll
    for (int i = 0; i < 4; ++i) all = x[i][n].y == 0.0f ? all : __builtin_fmaf(x[i][n].y, __builtin_amdgcn_exp2f(x[i][n].x - base), all);
    stats[t - me.t0][n] = make_float2(base, all);
  };
  if (me.t0 < me.t1) landed(me.t0, std::integral_constant<int, 2>());
  for (int t = me.t0; t < me.t1; ++t) {
    const RowTile& ops = slot(t);
    auto middle = [&] {
      landed(t + 1, std::integral_constant<int, 1>());
      issue(t + 3);
      if (PASS == 1 && t > me.t0 && w == (t & 3)) join(t - 1);  // every wave's sums of it are in LDS
    };
    if (t >= all_from) {
      scores(ops, [&](int i) { sums(i, t - 1); }, middle);
      pending = true;
    } else {
      if (pending) all_sums(t - 1);
      if (t >= some_from) {
        scores(ops, [](int) {}, middle);
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int least = from[u] - kRows * t;  // of the lane's rows, less its half's 4
#pragma unroll
          for (int r = 0; r < 16; ++r) X[u][r] = 8 * (r >> 2) + (r & 3) >= least ? X[u][r] : -INFINITY;
        }
        pending = true;
      } else {
        if (PASS == 1 && l < kRows) both[t & 1][w][l] = make_float2(0.0f, 0.0f);
        middle();
      }
    }
    if (PASS == 1 && pending && (ops.unsure || far_off())) peak_sums(t);
  }
  if (pending) all_sums(me.t1 - 1);
  if constexpr (PASS == 1) {
    __syncthreads();
    if (w == 0) join(me.t1 - 1);
    __syncthreads();
    for (int i = threadIdx.x; i < (me.t1 - me.t0) * kRows; i += 256) {
      const size_t tile = (size_t)(s.tile0 + me.t0 + i / kRows) * H + me.h;
      const float2 v = stats[i / kRows][i % kRows];
      a.stats[((size_t)me.range * a.tiles * H + tile) * kRows + i % kRows] = make_float2(v.x + reinterpret_cast<const RowTile*>(a.ops + tile * kTileBytes)->ref[i % kRows], v.y);
    }
  } else {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int t = token0 + 32 * u + n;
      float x = pair_sum(sum[u]);
      if (!tok[u].real) x = 0.0f;
      if (hh || t >= s.ctx) continue;
      if (a.part) {
        a.part[((size_t)(me.chunk - a.chunk0) * BH + bh) * ((size_t)a.ranges * kRangeTokens) + t] = x;
      } else {
        const size_t at = (size_t)bh * a.w_stride + t;
        a.w_out[at] = a.w_in ? __builtin_fmaf(a.decay, a.w_in[at], x) : x;
      }
    }
  }
}

// ---- L_r of every row. Block: a row tile; eight threads a row, each with every eighth range. Bound by latency: 17 us for 15,840 tiles.
__global__ __launch_bounds__(256) void weight_lse_kernel(TokenWeightsArgs a) {
  __shared__ float2 part[8][kRows];
  const int H = a.cv.num_kv_heads, n = threadIdx.x & 31, k = threadIdx.x >> 5;
  const int h = blockIdx.x % H, t = a.chunk0 * a.chunk_tiles + blockIdx.x / H % a.seq_tiles, b = blockIdx.x / H / a.seq_tiles;
  const Span s = span_of(a, b);
  const int rows = s.n * a.gq, row = kRows * t + n;
  if (kRows * t >= rows || s.ctx == 0) return;
  const int ranges = row < rows ? (s.limit(row / a.gq) + kRangeTokens - 1) / kRangeTokens : 0;
  float m = -INFINITY, sum = 0.0f;
#pragma unroll 4
  for (int r = k; r < ranges; r += 8) {
    const float2 v = a.stats[(((size_t)r * a.tiles + s.tile0 + t) * H + h) * kRows + n];
    if (v.y == 0.0f) continue;  // nothing seen there: its reference must not count
    const float top = fmaxf(m, v.x), base = top == -INFINITY ? 0.0f : top;
    sum = sum * __builtin_amdgcn_exp2f(m - base) + v.y * __builtin_amdgcn_exp2f(v.x - base);
    m = top;
  }
  part[k][n] = make_float2(m, sum);
  __syncthreads();
  if (k) return;
#pragma unroll
  for (int x = 1; x < 8; ++x) m = fmaxf(m, part[x][n].x);
  const float base = m == -INFINITY ? 0.0f : m;
  sum = 0.0f;
#pragma unroll
  for (int x = 0; x < 8; ++x) sum = __builtin_fmaf(part[x][n].y, __builtin_amdgcn_exp2f(part[x][n].x - base), sum);
  reinterpret_cast<RowTile*>(a.ops + ((size_t)(s.tile0 + t) * H + h) * kTileBytes)->lse[n] = sum == 0.0f ? INFINITY : m + __builtin_amdgcn_logf(sum);
}

// ---- The chunks' sums, behind those of the slabs before, and the running ones: 8 us for up to 16 chunks of 4 x 4,096 tokens and 8 heads
__global__ __launch_bounds__(256) void weight_join_kernel(TokenWeightsArgs a) {
  const int BH = a.B * a.cv.num_kv_heads, bh = blockIdx.x % BH, range = blockIdx.x / BH, t = kRangeTokens * range + threadIdx.x;
  const Span s = span_of(a, bh / a.cv.num_kv_heads);
  if (t >= s.ctx) return;
  const size_t places = (size_t)a.ranges * kRangeTokens;
  float sum = a.chunk0 > 0 ? a.run[bh * places + t] : 0.0f;
  for (int x = 0; x < a.chunks; ++x) {
    const Share share = share_of(a, bh, range, a.chunk0 + x, s);
    if (share.t0 < share.t1) sum += a.part[((size_t)x * BH + bh) * places + t];
  }
  if (!a.last) {
    a.run[bh * places + t] = sum;
    return;
  }
  const size_t at = (size_t)bh * a.w_stride + t;
  a.w_out[at] = a.w_in ? __builtin_fmaf(a.decay, a.w_in[at], sum) : sum;
}

// ---- Few rows a sequence (decode steps): up to kFewRows rows of one KV head. The scores are formed once and kept; the second
// pass goes over them and not over the keys: 64 sequences of 512 to 32,768 tokens with five rows 188 us, by the kernels above about
// three times as much (64 x 2 tokens of 8,000: 120 and 362 us; 2 of 1,000: 12 and 19). More rows than that have only those, at a tile
// of 32: 64 x 1 token of 8,000 and 4 KV heads, 8 rows 71 us, 12 or 16 rows 175.
namespace {

constexpr int kFewRows = 8;
constexpr int kPieceTokens = 512;  // of a block
constexpr int kJoinTokens = 1024;

// The rows' operands for products of 16 rows x 16 tokens, with zeros where a row has no part in a group, so that one chain of
// products forms several groups' sums. Up to four rows: operand row 4 j + g is group g of row j, and D's registers are the four groups of
// one row. Up to eight: operand row 2 j + g % 2, two D, for g / 2. A lane's eight channels (lane = 16 quad + operand
// row): positions 2 g, 2 g + 1 of words 2 quad, 2 quad + 1.
// Codes are normal numbers: taken as they lie, as subnormal ones code 2^(2 p - 24), they would spare an instruction for two
// channels, but the matrix cores align a product by its operands' exponents, and the leading zeros of a subnormal one cost the
// sum as many of its last bits (weights off by 8e-6 of themselves in place of 5e-7).
struct FewOps {
  cd_h8_t term[2][2][64];  // [group / 2 (up to eight rows)][high, low]
  float sum[kFewRows][4];  // of a row's channels of each group
  float down, pad[3];
};

__device__ __forceinline__ cd_f4_t product16(const cd_h8_t& x, const cd_h8_t& y, const cd_f4_t& c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, c, 0, 0, 0);
}
// Positions P, P + 1 of two words
template <int P>
__device__ __forceinline__ cd_h8_t codes_of(uint32_t u, uint32_t uh, uint32_t v, uint32_t vh) {
  const cd_h2_t a = land_position<P>(u, uh), b = land_position<P + 1>(u, uh), c = land_position<P>(v, vh), d = land_position<P + 1>(v, vh);
  return cd_h8_t{a.x, a.y, b.x, b.y, c.x, c.y, d.x, d.y};
}

}  // namespace

namespace {

struct FewLds {
  float q[kFewRows][kHeadDim], part[8][kFewRows][kHeadDim], top[16];
};

// The operands of one (sequence, KV head) by T threads: thread (channel c, part k of the sum's terms), all its loads on their
// way at once (R, given by rotation_part); then (channel, row). All threads of the block call it.
template <int T>
struct RotationPart {
  float x[kHeadDim / (T / kHeadDim)];
};
template <int T>
__device__ __forceinline__ void rotation_part(const TokenWeightsArgs& a, int h, RotationPart<T>& p) {
  constexpr int kTerms = kHeadDim / (T / kHeadDim);
  const float* R = a.R_k + ((size_t)h * kHeadDim + kTerms * (threadIdx.x >> 7)) * kHeadDim + (threadIdx.x & 127);
#pragma unroll
  for (int i = 0; i < kTerms; ++i) p.x[i] = R[(size_t)i * kHeadDim];
}
template <int T>
__device__ __forceinline__ void few_operands(const TokenWeightsArgs& a, const Span& s, int h, const RotationPart<T>& p, FewLds& lds, FewOps& out) {
  constexpr int kParts = T / kHeadDim, kTerms = kHeadDim / kParts, kEach = kFewRows / kParts;  // rows of a thread in the second half
  const int c = threadIdx.x & 127, k = threadIdx.x >> 7, rows = min(s.n * a.gq, kFewRows);
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int r = k + kParts * i, tok = r / a.gq;
    lds.q[r][c] = r < rows ? bf16_bits_to_f32(a.q[(s.start + tok) * a.q_stride + (size_t)(h * a.gq + r - tok * a.gq) * kHeadDim + c]) : 0.0f;
  }
  __syncthreads();
  for (int r = 0; r < rows; ++r) {
    float d = 0.0f;
#pragma unroll
    for (int i = 0; i < kTerms; ++i) d = __builtin_fmaf(lds.q[r][kTerms * k + i], p.x[i], d);
    lds.part[k][r][c] = d;
  }
  __syncthreads();
  float d[kEach], big = 0.0f;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int r = k + kParts * i;
    d[i] = 0.0f;
    if (r < rows) {
#pragma unroll
      for (int x = 0; x < kParts; ++x) d[i] += lds.part[x][r][c];
    }
    d[i] *= kLogit2;
    big = fmaxf(big, fabsf(d[i]));
  }
#pragma unroll
  for (int step = 32; step > 0; step >>= 1) big = fmaxf(big, __shfl_xor(big, step));
  if ((threadIdx.x & 63) == 0) lds.top[threadIdx.x >> 6] = big;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < T / 64; ++i) big = fmaxf(big, lds.top[i]);
  // the largest element to 2^13 .. 2^14
  const uint32_t e = min(max(__float_as_uint(big) >> 23, 14u), 240u);
  const int g = c >> 5, pos = c >> 4, word = (c & 15) >> 1, element = ((word & 1) << 2) | ((pos & 1) << 1) | (c & 1);
  const bool narrow = a.row_cap <= 4;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int r = k + kParts * i;
    const float y = d[i] * __uint_as_float((267u - e) << 23);
    const _Float16 hi = (_Float16)y, lo = (_Float16)(y - (float)hi);
    if (!narrow || r < 4) {
      const int at = narrow ? 0 : g >> 1, lane = 16 * (word >> 1) + (narrow ? 4 * r + g : 2 * r + (g & 1));
      reinterpret_cast<_Float16*>(&out.term[at][0][lane])[element] = hi;
      reinterpret_cast<_Float16*>(&out.term[at][1][lane])[element] = lo;
    }
    float sum = y;  // over the group: 32 lanes
#pragma unroll
    for (int step = 16; step > 0; step >>= 1) sum += __shfl_xor(sum, step);
    if ((c & 31) == 0) out.sum[r][g] = sum;
  }
  if (threadIdx.x == 0) out.down = __uint_as_float((e - 13u) << 23);
}

}  // namespace

// Block: one (sequence, KV head). Bound by the latency of its loads: 10 us for 512 of them.
__global__ __launch_bounds__(1024) void weight_few_rows_kernel(TokenWeightsArgs a) {
  __shared__ FewLds lds;
  const int H = a.cv.num_kv_heads, h = blockIdx.x % H, b = blockIdx.x / H;
  RotationPart<1024> R;
  rotation_part(a, h, R);
  const Span s = span_of(a, b);
  if (s.n == 0 || s.ctx == 0) return;
  few_operands<1024>(a, s, h, R, lds, reinterpret_cast<FewOps*>(a.few)[(size_t)b * H + h]);
}

// Block: W waves with PAGES pages of one KV head each; all loads of a wave are on their way at once. Lane: one token of a page
// and ROWS rows, 1 (up to four of a KV head) or 2. ALONE: forms its operands itself, while the keys are on their way. WHOLE: the
// block has the whole context, so that scores and statistics stay in registers and LDS, and forms the sums too. Bound by the vector
// ALU (82 % of cycles) and the rows it moves: 64 sequences of 512 to 32,768 tokens, 40 + 8 heads, 130 to 140 us, 3.8 TB/s of
// keys read and scores written.
template <int NG, int ROWS, int W, int PAGES, bool ALONE, bool WHOLE>
__global__ __launch_bounds__(64 * W, 4) void weight_few_scores_kernel(TokenWeightsArgs a) {
  using Lay = Rec<NG>;
  static_assert(WHOLE ? ALONE && W <= 16 && PAGES % 4 == 0 : W * PAGES * kBlock == kPieceTokens, "a lane of sixteen a wave; pieces");
  __shared__ float2 both[W][kFewRows];
  __shared__ typename std::conditional<ALONE, FewLds, int>::type work;
  __shared__ typename std::conditional<ALONE, FewOps, int>::type own;
  const int H = a.cv.num_kv_heads, h = blockIdx.x % H, piece = WHOLE ? 0 : blockIdx.x / H % a.pieces, b = WHOLE ? blockIdx.x / H : blockIdx.x / H / a.pieces;
  RotationPart<64 * W> R;
  if constexpr (ALONE) rotation_part(a, h, R);
  const Span s = span_of(a, b);
  if (kPieceTokens * piece >= s.ctx || (!WHOLE && s.n == 0)) return;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), l = threadIdx.x & 63, t = l & 15, quad = l >> 4;
  const int page0 = W * PAGES * piece + PAGES * w, pages = (s.ctx + kBlock - 1) / kBlock;
  int id = -1;
  if (l < PAGES && page0 + l < min(pages, a.max_blocks)) id = a.table[(size_t)b * a.max_blocks + page0 + l];
  const uint32_t real = (uint32_t)__ballot(id >= 0 && id < a.cv.num_blocks);
  cd_u2_t code[PAGES];
  uint32_t meta[PAGES][NG];
#pragma unroll
  for (int i = 0; i < PAGES; ++i) {
    const int x = __builtin_amdgcn_readlane(id, i);
    const uint8_t* rec = a.cv.pool + ((size_t)(uint32_t)((real >> i) & 1 ? x : 0) * H + h) * Lay::kBytes;
    // (each key is read once: past the caches, so that the scores stay in them)
    code[i] = __builtin_nontemporal_load(reinterpret_cast<const cd_u2_t*>(rec + kOffKCodes + 32 * t + 8 * quad));
    if constexpr (NG == 4) {
      const cd_u4_t y = __builtin_nontemporal_load(reinterpret_cast<const cd_u4_t*>(rec + Lay::kOffKMeta + 16 * t));
#pragma unroll
      for (int g = 0; g < 4; ++g) meta[i][g] = y[g];
    } else {
      meta[i][0] = __builtin_nontemporal_load(reinterpret_cast<const uint32_t*>(rec + Lay::kOffKMeta + 4 * t));
    }
  }
  // WHOLE: a lane's tokens in the sums are those of pages 4 j + quad
  const size_t at = ((size_t)b * H + h) * a.w_stride;
  const int token0 = kBlock * (page0 + quad) + t;
  float before[WHOLE ? PAGES / 4 : 1], kept[PAGES][ROWS];
  if constexpr (WHOLE) {
#pragma unroll
    for (int j = 0; j < PAGES / 4; ++j) before[j] = a.w_in && token0 + 64 * j < s.ctx ? a.w_in[at + token0 + 64 * j] : 0.0f;
  }
  const FewOps* from = reinterpret_cast<const FewOps*>(a.few) + ((size_t)b * H + h);
  if constexpr (ALONE) {
    few_operands<64 * W>(a, s, h, R, work, own);
    __syncthreads();
    from = &own;
  }
  const FewOps& ops = *from;
  const float down = ops.down;
  cd_h8_t A[2][4];  // [high, low][group]
  float Q[ROWS][4];
  int lim[ROWS];
  const cd_h8_t none{};
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      if constexpr (ROWS == 1)
        A[x][g] = (l & 3) == g ? ops.term[0][x][l] : none;
      else
        A[x][g] = (l & 1) == (g & 1) ? ops.term[g >> 1][x][l] : none;
    }
#pragma unroll
  for (int k = 0; k < ROWS; ++k) {
    const int row = ROWS * quad + k;
    const float4 v = *reinterpret_cast<const float4*>(ops.sum[row]);
    Q[k][0] = v.x * down, Q[k][1] = v.y * down, Q[k][2] = v.z * down, Q[k][3] = v.w * down;
    if constexpr (NG == 1) Q[k][0] = (Q[k][0] + Q[k][1]) + (Q[k][2] + Q[k][3]);
    lim[k] = row < s.n * a.gq ? s.limit(row / a.gq) : 0;
  }
  float* scores = WHOLE ? nullptr : a.scores + (((size_t)b * H + h) * a.page_cap + page0) * (kBlock * a.row_cap) + ROWS * quad * kBlock + t;
#pragma unroll
  for (int i = 0; i < PAGES; ++i) {
    const uint32_t u = code[i].x, v = code[i].y, uh = u >> 10, vh = v >> 10;
    const cd_h8_t c[4] = {codes_of<0>(u, uh, v, vh), codes_of<2>(u, uh, v, vh), codes_of<4>(u, uh, v, vh), codes_of<6>(u, uh, v, vh)};
    const int token = kBlock * (page0 + i) + t;
    cd_f4_t D[ROWS];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      cd_f4_t& d = D[ROWS == 1 ? 0 : g >> 1];
      if (g == 0 || (ROWS == 2 && g == 2)) d = cd_f4_t{0.0f, 0.0f, 0.0f, 0.0f};
      d = product16(A[0][g], c[g], d);
      d = product16(A[1][g], c[g], d);
    }
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      float d[4];  // the row's groups
#pragma unroll
      for (int g = 0; g < 4; ++g) d[g] = ROWS == 1 ? D[0][g] : D[g >> 1][2 * k + (g & 1)];
      float x = 0.0f, z = 0.0f;
      if constexpr (NG == 4) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          x = __builtin_fmaf(f16_bits_to_f32(meta[i][g] & 0xFFFFu), d[g], x);
          z = __builtin_fmaf(f16_bits_to_f32(meta[i][g] >> 16), Q[k][g], z);
        }
      } else {
        x = f16_bits_to_f32(meta[i][0] & 0xFFFFu) * ((d[0] + d[1]) + (d[2] + d[3]));
        z = f16_bits_to_f32(meta[i][0] >> 16) * Q[k][0];
      }
      x = __builtin_fmaf(x, down, z);
      x = (real >> i) & 1 && token < lim[k] ? x : -INFINITY;
      kept[i][k] = x;
    }
  }
  if constexpr (!WHOLE) {  // (here, so that the products of several pages may overlap)
#pragma unroll
    for (int k = 0; k < ROWS; ++k)
      if (ROWS * quad + k < a.row_cap) {
#pragma unroll
        for (int i = 0; i < PAGES; ++i)
          if (page0 + i < pages) scores[i * (kBlock * a.row_cap) + k * kBlock] = kept[i][k];
      }
  }
#pragma unroll
  for (int k = 0; k < ROWS; ++k) {
    float top = kNone, all = 0.0f;
#pragma unroll
    for (int i = 0; i < PAGES; ++i) top = fmaxf(top, kept[i][k]);
    top = row_max16(top);
#pragma unroll
    for (int i = 0; i < PAGES; ++i) all += __builtin_amdgcn_exp2f(kept[i][k] - top);
    all = row_sum16(all);
    if (t == 0) both[w][ROWS * quad + k] = make_float2(top, all);
  }
  __syncthreads();
  if constexpr (WHOLE) {
    float lse[ROWS];
#pragma unroll
    for (int k = 0; k < ROWS; ++k) {
      const float2 v = t < W ? both[min(t, W - 1)][ROWS * quad + k] : make_float2(kNone, 0.0f);
      const float top = row_max16(v.x), all = row_sum16(v.y * __builtin_amdgcn_exp2f(v.x - top));
      lse[k] = all == 0.0f ? INFINITY : top + __builtin_amdgcn_logf(all);
    }
#pragma unroll
    for (int j = 0; j < PAGES / 4; ++j) {
      float mine = 0.0f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        float x = __builtin_amdgcn_exp2f(kept[4 * j + i][0] - lse[0]);
        if constexpr (ROWS == 2) x += __builtin_amdgcn_exp2f(kept[4 * j + i][1] - lse[1]);
        x += __shfl_xor(x, 16);
        x += __shfl_xor(x, 32);
        mine = quad == i ? x : mine;
      }
      if (token0 + 64 * j < s.ctx) a.w_out[at + token0 + 64 * j] = a.w_in ? __builtin_fmaf(a.decay, before[j], mine) : mine;
    }
  } else if (threadIdx.x < 4 * ROWS) {
    float top = kNone, all = 0.0f;
#pragma unroll
    for (int x = 0; x < W; ++x) top = fmaxf(top, both[x][threadIdx.x].x);
#pragma unroll
    for (int x = 0; x < W; ++x) all += both[x][threadIdx.x].y * __builtin_amdgcn_exp2f(both[x][threadIdx.x].x - top);
    a.stats[(((size_t)b * H + h) * a.pieces + piece) * kFewRows + threadIdx.x] = make_float2(top, all);
  }
}

// Block: 1,024 tokens of one KV head, a thread four of them. Each wave joins the pieces of its rows first. Bound by the scores it
// reads: the same batch 47 us, 4.9 TB/s.
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
  // Chunks of the row tiles: shorter ones, as long as there are fewer than four blocks a compute unit, where they take less time: rounds
  // of two blocks a compute unit, half of a prompt's own square empty, each of its tiles and 1.8 tiles' time before the first. 64 tokens
  // (32 + 8 heads) of 8,000: chunks of 4 tiles 41.5 us, of 8 46; of four times 4,000, a whole round: 68 and 60.5; 256 of 4,000: of 4, 8,
  // 32 tiles 78, 83, 114
  const long long ranges = (long long)B * H * p.ranges, places = 4LL * num_cus();
  auto chunks = [&](int tiles) { return ((long long)p.seq_tiles + tiles - 1) / tiles; };
  const double seen = max_ctx > 0 ? 1.0 - 0.5 * (max_q < max_ctx ? max_q : max_ctx) / max_ctx : 1.0;
  auto cost = [&](int tiles) {
    const long long rounds = ((long long)(seen * (double)(ranges * chunks(tiles))) + 2 * num_cus() - 1) / (2 * num_cus());
    return (double)(rounds < 1 ? 1 : rounds) * ((tiles < p.seq_tiles ? tiles : p.seq_tiles) + 1.8);
  };
  p.chunk_tiles = kChunkTiles;
  for (int tiles = kChunkTiles; tiles > 4 && ranges * chunks(tiles) < places;) {
    tiles /= 2;
    if (cost(tiles) < cost(p.chunk_tiles)) p.chunk_tiles = tiles;
  }
  p.chunks = p.slab_chunks = (int)chunks(p.chunk_tiles);
  auto up = [](size_t x) { return (x + 255) & ~size_t(255); };
  size_t off = 0;
  auto lay = [&](size_t tiles, size_t parts, size_t runs) {
    off = 0;
    p.off_ops = off, off = up(off + tiles * H * kTileBytes);
    p.off_stats = off, off = up(off + (size_t)p.ranges * tiles * H * kRows * sizeof(float2));
    p.off_part = off, off = up(off + parts * kRangeTokens * sizeof(float));
    p.off_run = off, off = up(off + runs * kRangeTokens * sizeof(float));
    return off;
  };
  // (a smaller call may take shorter chunks: fewer than twice as many as there are places, and one a range)
  const long long most = ranges * chunks(kChunkTiles), shorter = 2 * places + ranges;
  const size_t whole = lay(p.tiles, (size_t)(most > shorter ? most : shorter), 0);
  // A row's statistics take 8 bytes a range, so that those of whole prompts would grow with the square of their length (32 + 8 heads:
  // 32,768 tokens 1.8 GB, 131,072 21.6). Beyond kSlabBytes, or what one chunk of every sequence takes where that is more, the chunks are
  // taken a slab at a time, as many as have room; sums are added up in the same order. One prompt of 32,768 tokens 18.7 ms either way, of
  // 65,536 74.4 ms and 72.8 with all statistics at once, of 131,072 294 and 287.
  const size_t least = lay((size_t)B * kChunkTiles, ranges, ranges), room = least > kSlabBytes ? least : kSlabBytes;
  if (whole <= room) {
    p.total = lay(p.tiles, (size_t)(most > shorter ? most : shorter), 0);
  } else {
    auto slab = [&](long long n) { return lay((size_t)B * n * p.chunk_tiles, (size_t)(ranges * n), ranges); };
    long long n = 1, beyond = (long long)p.chunks + 1;  // n chunks have room
    while (beyond - n > 1) {
      const long long mid = (n + beyond) / 2;
      if (slab(mid) <= room) n = mid;
      else beyond = mid;
    }
    slab(n);
    p.slab_chunks = (int)n, p.slab_tiles = (int)n * p.chunk_tiles, p.tiles = B * p.slab_tiles;
    p.total = room;
  }
  // few rows: a call within these bounds may have them, whether or not this one does
  off = 0;
  p.off_few = off, off = up(off + (size_t)B * H * sizeof(FewOps));
  p.off_few_stats = off, off = up(off + (size_t)B * H * p.pieces * kFewRows * sizeof(float2));
  p.off_scores = off, off = up(off + (size_t)B * H * p.page_cap * kBlock * p.row_cap * sizeof(float));
  p.total = p.total > off ? p.total : off;
  return p;
}

namespace {

// W, PAGES, ALONE, WHOLE: as weight_few_scores_kernel
template <int NG, int W, int PAGES, bool ALONE, bool WHOLE>
hipError_t launch_scores(const TokenWeightsArgs& a, hipStream_t s) {
  const long long BH = (long long)a.B * a.cv.num_kv_heads;
  if (!ALONE) {
    hipLaunchKernelGGL(weight_few_rows_kernel, dim3((unsigned)BH), dim3(1024), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  const dim3 grid((unsigned)(BH * (WHOLE ? 1 : a.pieces)));
  if (a.row_cap <= 4)
    hipLaunchKernelGGL((weight_few_scores_kernel<NG, 1, W, PAGES, ALONE, WHOLE>), grid, dim3(64 * W), 0, s, a);
  else
    hipLaunchKernelGGL((weight_few_scores_kernel<NG, 2, W, PAGES, ALONE, WHOLE>), grid, dim3(64 * W), 0, s, a);
  return hipGetLastError();
}
template <int NG>
hipError_t launch_few(const TokenWeightsArgs& a, hipStream_t s) {
  const long long H = a.cv.num_kv_heads;
  // Contexts that a block holds take one launch and keep no scores in memory (32 + 8 heads): 500 tokens of 256 sequences 35 us, in
  // pieces 48; 1,000 of one 11 and 13, of 64 20 and 29 (40 + 8 heads); 2,000 of 128 61 and 68
  if (a.max_ctx <= 8 * 4 * kBlock) return launch_scores<NG, 8, 4, true, true>(a, s);
  if (a.max_ctx <= 16 * 4 * kBlock) return launch_scores<NG, 16, 4, true, true>(a, s);
  if (a.max_ctx <= 16 * 8 * kBlock) return launch_scores<NG, 16, 8, true, true>(a, s);
  // While every compute unit has at most one block, each rotates its own queries, a launch less: 16,000 tokens of one sequence (32 + 8
  // heads) 16.5 us, with the launch 18.2; 32,000, twice the blocks, 26.1 and 20.5
  const hipError_t e = a.B * H * a.pieces <= num_cus() ? launch_scores<NG, 8, 4, true, false>(a, s) : launch_scores<NG, 4, 8, false, false>(a, s);
  if (e != hipSuccess) return e;
  const long long joins = ((long long)a.page_cap * kBlock + kJoinTokens - 1) / kJoinTokens;
  hipLaunchKernelGGL(weight_few_join_kernel, dim3((unsigned)(a.B * H * joins)), dim3(256), 0, s, a);
  return hipGetLastError();
}

// The chunks chunk0 .. chunk0 + chunks - 1
template <int NG>
hipError_t launch_slab(const TokenWeightsArgs& a, hipStream_t s) {
  const long long BH = (long long)a.B * a.cv.num_kv_heads;
  hipError_t e = hipSuccess;
  if (a.seq_tiles > 0) {
    const long long items = BH * a.seq_tiles;
    const int per = (int)(items / 1024 < 1 ? 1 : items / 1024 > 8 ? 8 : items / 1024);
    const dim3 shares((unsigned)(BH * a.ranges * a.chunks));
    hipLaunchKernelGGL(weight_rows_kernel<NG>, dim3((unsigned)(BH * ((a.seq_tiles + per - 1) / per))), dim3(256), 0, s, a, per);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL((weight_scan_kernel<NG, 1>), shares, dim3(256), 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL(weight_lse_kernel, dim3((unsigned)items), dim3(256), 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
    hipLaunchKernelGGL((weight_scan_kernel<NG, 2>), shares, dim3(256), 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.part) {
    hipLaunchKernelGGL(weight_join_kernel, dim3((unsigned)(BH * a.ranges)), dim3(kRangeTokens), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

template <int NG>
hipError_t launch_many(TokenWeightsArgs a, const TokenWeightsPlan& p, hipStream_t s) {
  for (int c = 0;;) {
    a.chunk0 = c, a.chunks = min(p.slab_chunks, p.chunks - c), a.last = c + a.chunks == p.chunks;
    a.seq_tiles = min(a.chunks * p.chunk_tiles, p.seq_tiles - c * p.chunk_tiles);
    const hipError_t e = launch_slab<NG>(a, s);
    c += a.chunks;
    if (e != hipSuccess || a.last) return e;
  }
}

}  // namespace

hipError_t launch_token_weights(TokenWeightsArgs a, const TokenWeightsPlan& p, uint8_t* ws, hipStream_t s) {
  a.ranges = p.ranges, a.chunk_tiles = p.chunk_tiles, a.tiles = p.tiles, a.slab_tiles = p.slab_tiles;
  a.ops = ws + p.off_ops;
  a.stats = reinterpret_cast<float2*>(ws + p.off_stats);
  // one chunk of all rows writes the results itself
  a.part = p.chunks == 1 && p.slab_tiles == 0 ? nullptr : reinterpret_cast<float*>(ws + p.off_part);
  a.run = reinterpret_cast<float*>(ws + p.off_run);
  if (p.few) {
    a.few = ws + p.off_few;
    a.stats = reinterpret_cast<float2*>(ws + p.off_few_stats);
    a.scores = reinterpret_cast<float*>(ws + p.off_scores);
    a.pieces = p.pieces, a.page_cap = p.page_cap, a.row_cap = p.row_cap;
    return a.cv.groups == 4 ? launch_few<4>(a, s) : launch_few<1>(a, s);
  }
  return a.cv.groups == 4 ? launch_many<4>(a, p, s) : launch_many<1>(a, p, s);
}

}  // namespace int2kv
