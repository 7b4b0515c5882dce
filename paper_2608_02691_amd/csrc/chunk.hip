// Attention of a chunk of new tokens over the paged INT2 cache (int2kv_chunk_attention).
//
// Rows are (new token i of sequence b, query head j of the KV head's group), row i * G_q + j of the sequence. A row sees
// S = {cached s < limit} and, where the chunk's own keys and values are given in bf16, {new t <= i}:
//     a_s = c (q R_K) k^_s^T,   a_t = c (q k_t^T - q mu^T)   (both with centered keys; c = 1 / sqrt(128)),
//     o = (sum_s p_s v^_s) R_V^T + sum_t p_t v_t,   p = softmax over S.
// Three launches:
//   chunk_prep_kernel   rotates the queries (q' = q R_K as fp16 operands), lays R_V out as operands, and plans the work;
//   chunk_attn_kernel   a work-group takes a tile of rows of one KV head over a range of 64-token units of the context:
//                       the INT2 units first, their sum un-rotated, then the chunk's own bf16 units;
//   chunk_merge_kernel  joins the pieces of tiles whose context was split.
//
// Products are formed transposed (S^T = K Q^T, O^T = V^T P^T, 32 x 32 x 16): a lane holds one query row, so the softmax is
// lane-local but for one exchange of halves, the rescaling is one factor per lane, and the probabilities are the second
// product's B operand as they lie (its k order is the order of S^T's rows in a lane; V^T is laid out to match). INT2 codes
// become fp16 operands once per work-group and unit and are shared through LDS in operand order.
#include "codes.h"
#include "common.h"
#include "kernels.h"

namespace int2kv {

namespace {

constexpr int kUnit = 64;                     // tokens of a unit: two 32-token halves, four pages
constexpr int kUnitPages = kUnit / kBlock;
constexpr float kLogit2 = 1.4426950408889634f * 0.08838834764831845f;  // log2(e) / sqrt(128)
constexpr float kLazy = 8.0f;   // the running maximum moves when a score exceeds it by 2^8
constexpr float kBias = 7.0f;   // probabilities are held times 2^7: the largest is below 2^15, and fp16's normal range
                                // reaches 2^-21 below the maximum
constexpr float kNone = -1.0e30f;  // running maximum of a row that has seen nothing
constexpr int kPrepThreads = 256;

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

// Inclusive sum over the block; total to every thread. tmp: a word per wave and one more.
__device__ __forceinline__ int block_scan(int x, int* tmp, int& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(x, d);
    if (lane >= d) x += y;
  }
  __syncthreads();
  if (lane == 63) tmp[wave] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kPrepThreads / 64; ++w) {
    before += w < wave ? tmp[w] : 0;
    total += tmp[w];
  }
  return x + before;
}

// Plan of the attention launch, by one block: tiles of bm rows in sequence order, cut into pieces of at most L units so
// that all heads' pieces come to about `target`; the last tiles first, since under a causal mask they are the longest.
__device__ void plan_work(const ChunkArgs& a) {
  __shared__ int tmp[kPrepThreads / 64];
  __shared__ unsigned long long sum;
  const int tid = threadIdx.x;
  int carry = 0, total;
  for (int b0 = 0; b0 < a.B; b0 += kPrepThreads) {
    const int b = b0 + tid;
    const int rows = b < a.B ? seq_of(a, b).n * a.gq : 0, mine = (rows + a.bm - 1) / a.bm;
    const int upto = block_scan(mine, tmp, total);
    if (b < a.B) a.tile_start[b] = carry + upto - mine;
    carry = min(carry + total, 1 << 30);
  }
  // sequences that overlap can ask for more tiles than there is room for: the rest is left out
  const int T = min(carry, a.max_tiles);
  if (tid == 0) sum = 0;
  __syncthreads();
  unsigned long long mine = 0;
  for (int t = tid; t < T; t += kPrepThreads) {
    int lo = 0, hi = a.B - 1;  // the last sequence that starts at or before t (empty ones start where the next does)
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.tile_start[mid] <= t)
        lo = mid;
      else
        hi = mid - 1;
    }
    const Seq s = seq_of(a, lo);
    const int row0 = (t - a.tile_start[lo]) * a.bm, last = min(row0 + a.bm, s.n * a.gq) - 1;
    const int i = last / a.gq, units = int2_units(a, s, i) + own_units(a, i);
    ChunkTile& d = a.tiles[t];
    d.b = lo, d.row0 = row0, d.start = s.start, d.n = s.n, d.ctx = s.ctx, d.units = units;
    mine += units;
  }
  atomicAdd(&sum, mine);
  __syncthreads();
  const unsigned long long work = sum * a.cv.num_kv_heads;
  const int L = (int)max((unsigned long long)a.min_units, (work + a.target - 1) / a.target);
  int items = 0, slots = 0;
  for (int r0 = 0; r0 < T; r0 += kPrepThreads) {
    const int t = T - 1 - (r0 + tid);
    int units = 0, pieces = 0;
    if (t >= 0) {
      units = a.tiles[t].units;
      pieces = units > L ? (units + L - 1) / L : 1;
    }
    int want = pieces > 1 ? pieces : 0;
    int n_slots, n_items;
    const int slot_end = slots + block_scan(want, tmp, n_slots);
    if (want && slot_end > a.max_slots) pieces = 1, want = 0;  // cannot happen within the bounds the host sized for
    const int item_end = items + block_scan(pieces, tmp, n_items);
    if (t >= 0) {
      ChunkTile d = a.tiles[t];
      d.pieces = pieces, d.slot = want ? slot_end - want : -1;
      a.tiles[t] = d;
      for (int p = 0; p < pieces; ++p) {
        const int at = item_end - pieces + p;
        if (at >= a.max_items) break;
        ChunkItem it;
        it.tile = t;
        it.u0 = (int)((long long)units * p / pieces);
        it.u1 = (int)((long long)units * (p + 1) / pieces);
        it.slot = want ? d.slot + p : -1;
        a.items[at] = it;
      }
    }
    slots += n_slots;
    items += n_items;
  }
  if (tid == 0) {
    a.counts[0] = min(items, a.max_items);
    a.counts[1] = T;
  }
}

// R_V of a head as A operands of o = o' R_V^T: tile 2 a + e, row m is output channel 64 a + 2 m + e; operand (i, half)
// takes the channels 32 i + 16 half + {4 hh .. + 3, 8 + 4 hh .. + 3} a lane half holds of tile i of O^T.
__device__ void layout_rv(const ChunkArgs& a, int h, int part, int parts) {
  const float* R = a.R_v + (size_t)h * kHeadDim * kHeadDim;
  cd_h8_t* dst = reinterpret_cast<cd_h8_t*>(a.rv) + (size_t)h * 2048;
  for (int x = part * kPrepThreads + threadIdx.x; x < 2048; x += parts * kPrepThreads) {
    const int l = x & 63, m = l & 31, hh = l >> 5, op = (x >> 6) & 7, t = x >> 9;
    const float* src = R + (size_t)(64 * (t >> 1) + 2 * m + (t & 1)) * kHeadDim + 16 * op + 4 * hh;
    const float4 u = *reinterpret_cast<const float4*>(src), v = *reinterpret_cast<const float4*>(src + 8);
    dst[x] = cd_h8_t{(_Float16)u.x, (_Float16)u.y, (_Float16)u.z, (_Float16)u.w,
                     (_Float16)v.x, (_Float16)v.y, (_Float16)v.z, (_Float16)v.w};
  }
}

// Position (in a query row of the workspace) -> channel: chunk 2 kk + hh of eight is operand kk's piece of lane half hh
__device__ __forceinline__ int pos_channel(int pos) { return code_channel(pos >> 4, (pos >> 3) & 1, pos & 7); }

// Query rotation: q'^T = R_K^T q^T on the matrix cores, R_K in two bf16 terms (q is exact), a wave per 32 positions, row
// tiles of 32. q' is held in fp16 times a power of two that brings |q|, which bounds every |q'_c|, to [2^11, 2^12).
__device__ void rotate_queries(const ChunkArgs& a, int h, int part, int parts) {
  const int l = threadIdx.x & 63, wave = threadIdx.x >> 6, n = l & 31, hh = l >> 5;
  const float* R = a.R_k + (size_t)h * kHeadDim * kHeadDim;
  // A rows: row m = 8 u + 4 hh + v of the wave's tile is position 32 wave + 16 (u / 2) + 8 hh + 4 (u % 2) + v, so that a
  // lane's results are eight consecutive positions at a time
  const int mu_ = n >> 3, mh = (n >> 2) & 1, mv = n & 3;
  const int col = pos_channel(32 * wave + 16 * (mu_ >> 1) + 8 * mh + 4 * (mu_ & 1) + mv);
  cd_b8_t hi[8], lo[8];
#pragma unroll
  for (int kk = 0; kk < 8; ++kk)
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float r = R[(size_t)(16 * kk + 8 * hh + j) * kHeadDim + col];
      hi[kk][j] = (__bf16)r;
      lo[kk][j] = (__bf16)(r - (float)hi[kk][j]);
    }
  const int rows = a.total_q * a.gq, tiles = (rows + 31) / 32;
  for (int t = part; t < tiles; t += parts) {
    const int row = t * 32 + n, rc = min(row, rows - 1), tok = rc / a.gq;
    const uint16_t* q = a.q + tok * a.q_stride + (size_t)(h * a.gq + rc - tok * a.gq) * kHeadDim + 8 * hh;
    cd_b8_t x[8];
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) x[kk] = *reinterpret_cast<const cd_b8_t*>(q + 16 * kk);
    cd_f16_t d;
#pragma unroll
    for (int r = 0; r < 16; ++r) d[r] = 0.0f;
    float norm = 0.0f, off = 0.0f;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) {
      d = __builtin_amdgcn_mfma_f32_32x32x16_bf16(lo[kk], x[kk], d, 0, 0, 0);
      d = __builtin_amdgcn_mfma_f32_32x32x16_bf16(hi[kk], x[kk], d, 0, 0, 0);
#pragma unroll
      for (int j = 0; j < 8; ++j) norm = __builtin_fmaf((float)x[kk][j], (float)x[kk][j], norm);
    }
    if (a.mu && wave == 0) {
      const float* mu = a.mu + (size_t)h * kHeadDim + 8 * hh;
#pragma unroll
      for (int kk = 0; kk < 8; ++kk)
#pragma unroll
        for (int j = 0; j < 8; ++j) off = __builtin_fmaf((float)x[kk][j], mu[16 * kk + j], off);
    }
    norm += __shfl_xor(norm, 32);
    off += __shfl_xor(off, 32);
    // 2^e <= |q| < 2^(e + 1); zero, infinite and NaN rows are left as they are
    const int e = (int)((__float_as_uint(sqrtf(norm)) >> 23) & 255) - 127;
    const bool plain = !(norm > 0x1p-100f) || !(norm < 0x1p100f);
    const float up = plain ? 1.0f : __uint_as_float((uint32_t)(127 + 11 - e) << 23), down = plain ? 1.0f : __uint_as_float((uint32_t)(127 - 11 + e) << 23);
    if (row < rows) {
      uint16_t* o = a.qrot + ((size_t)h * rows + row) * kHeadDim + 32 * wave + 8 * hh;
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        cd_h8_t y;
#pragma unroll
        for (int r = 0; r < 8; ++r) y[r] = (_Float16)(d[8 * u + r] * up);
        *reinterpret_cast<cd_h8_t*>(o + 16 * u) = y;
      }
      if (wave == 0 && hh == 0) a.qscale[(size_t)h * rows + row] = make_float2(down * kLogit2, off * kLogit2);
    }
  }
}

}  // namespace

// Blocks: 0 plans; then H blocks of R_V; then a.rot_blocks per head of the query rotation.
__global__ __launch_bounds__(kPrepThreads) void chunk_prep_kernel(ChunkArgs a) {
  const int H = a.cv.num_kv_heads;
  int x = blockIdx.x;
  if (x == 0) return plan_work(a);
  if (--x < H) return layout_rv(a, x, 0, 1);
  x -= H;
  rotate_queries(a, x % H, x / H, a.rot_blocks);
}

namespace {

// What RW waves share: a unit's K and V^T operands, two units of them
struct ChunkLds {
  cd_h8_t k[2][16][64];  // [buffer][half tm, operand kk][lane]
  cd_h8_t v[2][16][64];  // [buffer][page, tile][lane]
  uint32_t bad[2][8];    // per building wave: a value of the unit is not finite (units that need masks)
};

}  // namespace

template <int NG, int RW>
__global__ __launch_bounds__(64 * RW, RW == 8 ? 2 : RW == 4 ? 2 : 1) void chunk_attn_kernel(ChunkArgs a) {
  using Lay = Rec<NG>;
  constexpr int KW = 8 / RW;                  // words of a token's half row that a wave makes operands of
  constexpr int PV = RW >= 4 ? 1 : 4 / RW;    // pages it makes V^T operands of
  constexpr int TV = RW == 8 ? 2 : 4;         // and tiles of each
  constexpr int GV = NG == 4 ? TV : 1;        // groups those tiles lie in
  __shared__ ChunkLds lds;
  const int H = a.cv.num_kv_heads;
  const int h = (int)(blockIdx.x % H), at = (int)(blockIdx.x / H);
  if (at >= a.counts[0]) return;
  const ChunkItem item = a.items[at];
  const ChunkTile tile = a.tiles[item.tile];
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = l & 31, hh = l >> 5;
  const int rows = tile.n * a.gq, row_w = tile.row0 + 32 * w;  // the wave's first row
  const int row = row_w + n, rc = min(row, rows - 1), tok = rc / a.gq, head = h * a.gq + rc - tok * a.gq;
  const int last_tok = min(tile.row0 + a.bm, rows) - 1;
  const int nI = int2_units(a, Seq{tile.start, tile.n, tile.ctx}, last_tok / a.gq);
  const int all_rows = a.total_q * a.gq;
  const size_t grow = (size_t)h * all_rows + (size_t)tile.start * a.gq + rc;
  const float2 qs = a.qscale[grow];

  cd_f16_t O[4];
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) O[i][r] = 0.0f;
  float m = kNone, sum = 0.0f;

  // ---- scores of a unit (S[tm][r]: token 32 tm + 8 (r / 4) + 4 hh + r % 4) to probabilities, moving m, sum and O
  auto soften = [&](cd_f16_t (&S)[2], float c, float off) {
    float mx = S[0][0];
#pragma unroll
    for (int tm = 0; tm < 2; ++tm)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, S[tm][r]);
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float top = __builtin_fmaf(mx, c, -off);
    const bool move = top > m + kLazy;
    if (__any(move)) {
      const float to = move ? top : m, f = __builtin_amdgcn_exp2f(m - to);
      m = to;
      sum *= f;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int r = 0; r < 16; ++r) O[i][r] *= f;
    }
    const float base = kBias - off - m;
#pragma unroll
    for (int tm = 0; tm < 2; ++tm)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        S[tm][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(S[tm][r], c, base));
        sum += S[tm][r];
      }
  };

  // ==== the INT2 units
  const int i1 = min(item.u1, nI);
  if (item.u0 < i1) {
    const int lim = a.k_new ? tile.ctx : tile.ctx - tile.n + tok + 1;  // tokens this row sees
    const int lim_min = a.k_new ? tile.ctx : tile.ctx - tile.n + min(row_w, rows - 1) / a.gq + 1;
    cd_h8_t Q[8];
#pragma unroll
    for (int kk = 0; kk < 8; ++kk)
      Q[kk] = *reinterpret_cast<const cd_h8_t*>(a.qrot + grow * kHeadDim + 16 * kk + 8 * hh);
    const int tmw = RW == 8 ? w >> 2 : RW == 4 ? w >> 1 : w;   // half whose K operands this wave makes
    const int word0 = RW == 8 ? w & 3 : RW == 4 ? 2 * (w & 1) : 0;
    const int page0 = RW == 8 ? w >> 1 : RW == 4 ? w : 2 * w;  // its (first) V page
    const int tile0 = RW == 8 ? 2 * (w & 1) : 0;
    struct Raw {
      uint32_t kw[KW], km[NG];
      cd_u2_t vc[PV][2], vs[PV][GV][2], vz[PV][GV][2];
      uint32_t ok;  // pages that exist
    } raw;
    const int32_t* table = a.table + (size_t)tile.b * a.max_blocks;
    const int pages = (tile.ctx + kBlock - 1) / kBlock;
    auto page_id = [&](int u) {  // lane l: the block of page l % 4 of unit u
      const int p = kUnitPages * u + (l & 3);
      return p < pages ? table[p] : -1;
    };
    auto fetch = [&](int pid) {
      const bool good = pid >= 0 && pid < a.cv.num_blocks;
      raw.ok = (uint32_t)__ballot(good) & 15u;
      const int id = good ? pid : 0;
      auto record = [&](int p) {
        return a.cv.pool + ((size_t)(uint32_t)__builtin_amdgcn_readlane(id, p) * H + h) * Lay::kBytes;
      };
      const uint8_t* ra = record(2 * tmw);
      const uint8_t* rb = record(2 * tmw + 1);
      const uint8_t* rk = n < 16 ? ra : rb;
      const int t = n & 15;
      const uint32_t* kw = reinterpret_cast<const uint32_t*>(rk + kOffKCodes + 32 * t + 16 * hh) + word0;
#pragma unroll
      for (int i = 0; i < KW; ++i) raw.kw[i] = kw[i];
      const uint32_t* km = reinterpret_cast<const uint32_t*>(rk + Lay::kOffKMeta + 4 * NG * t);
#pragma unroll
      for (int g = 0; g < NG; ++g) raw.km[g] = km[g];
#pragma unroll
      for (int p = 0; p < PV; ++p) {
        const uint8_t* rv = record(page0 + p);
        const uint8_t* vc = rv + kOffVCodes + 32 * (n & 15) + 8 * hh;
        const uint8_t* vm = rv + 8 * hh + (NG == 4 ? 32 * tile0 : 0);
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          raw.vc[p][x] = *reinterpret_cast<const cd_u2_t*>(vc + 16 * x);
#pragma unroll
          for (int g = 0; g < GV; ++g) {
            raw.vs[p][g][x] = *reinterpret_cast<const cd_u2_t*>(vm + Lay::kOffVScale + 32 * g + 16 * x);
            raw.vz[p][g][x] = *reinterpret_cast<const cd_u2_t*>(vm + Lay::kOffVZero + 32 * g + 16 * x);
          }
        }
      }
    };
    // whether some row of the tile may not see all of unit u (the same for every wave)
    const int lim_tile = a.k_new ? tile.ctx : tile.ctx - tile.n + tile.row0 / a.gq + 1;
    auto build = [&](int u, int buf) {
      cd_h2_t s[NG], z[NG];
#pragma unroll
      for (int g = 0; g < NG; ++g) s[g] = both_lo(raw.km[g]), z[g] = both_hi(raw.km[g]);
#pragma unroll
      for (int i = 0; i < KW; ++i) {
        cd_h8_t x[2];
        word_operands<NG>(raw.kw[i], s, z, x);
        lds.k[buf][8 * tmw + 2 * (word0 + i)][l] = x[0];
        lds.k[buf][8 * tmw + 2 * (word0 + i) + 1][l] = x[1];
      }
      const bool edge = raw.ok != 15u || kUnit * (u + 1) > tile.ctx, masked = edge || kUnit * (u + 1) > lim_tile;
      bool bad = false;
#pragma unroll
      for (int p = 0; p < PV; ++p) {
        // pairs of tokens (4 hh, + 1), (+ 2, + 3), (8 + 4 hh, + 1), (+ 2, + 3); tile i's channel 32 i + 16 ph + (n % 16)
        // lies at bits 2 (2 i + ph) of each half
        uint32_t word[4], keep[4] = {~0u, ~0u, ~0u, ~0u};
        const int shift = 2 * (n >> 4) + 4 * tile0;
#pragma unroll
        for (int x = 0; x < 4; ++x) word[x] = raw.vc[p][x >> 1][x & 1] >> shift;
        if (edge) {
          // tokens that do not exist: their values must not reach the product, where 0 * inf would be NaN
          int cnt = tile.ctx - (kUnit * u + kBlock * (page0 + p));
          cnt = (raw.ok >> (page0 + p)) & 1 ? cnt : 0;
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const int tb = 8 * (x >> 1) + 4 * hh + 2 * (x & 1);
            keep[x] = (tb < cnt ? 0xFFFFu : 0u) | (tb + 1 < cnt ? 0xFFFF0000u : 0u);
          }
        }
        auto one = [&](int i, int x, cd_h2_t code) {
          const int g = NG == 4 ? i : 0;
          // (copies: a bit cast of a vector's element takes element 0)
          const uint32_t sv = raw.vs[p][g][x >> 1][x & 1], zv = raw.vz[p][g][x >> 1][x & 1];
          const cd_h2_t y = __builtin_elementwise_fma(code, __builtin_bit_cast(cd_h2_t, sv), __builtin_bit_cast(cd_h2_t, zv));
          return __builtin_bit_cast(uint32_t, y) & keep[x];
        };
#pragma unroll
        for (int i = 0; i < TV; ++i) {
          cd_u4_t f;
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            const cd_h2_t code = i == 0   ? land_codes<0>(word[x])
                                 : i == 1 ? land_codes<4>(word[x])
                                 : i == 2 ? land_codes<8>(word[x])
                                          : land_codes<4>(word[x] >> 8);
            f[x] = one(i, x, code);
          }
          if (masked) {
#pragma unroll
            for (int x = 0; x < 4; ++x)
              bad = bad || (f[x] & 0x7C00u) == 0x7C00u || (f[x] & 0x7C000000u) == 0x7C000000u;
          }
          lds.v[buf][4 * (page0 + p) + tile0 + i][l] = __builtin_bit_cast(cd_h8_t, f);
        }
      }
      if (masked) {
        const bool any = __any(bad);
        if (l == 0) lds.bad[buf][w] = any;
      }
    };

    int u = item.u0;
    int pid = page_id(u);
    fetch(pid);
    pid = page_id(u + 1);
    build(u, 0);
    uint32_t ok = raw.ok;
    int buf = 0;
    for (; u < i1; ++u, buf ^= 1) {
      const bool more = u + 1 < i1;
      if (more) {
        fetch(pid);
        pid = page_id(u + 2);
      }
      __syncthreads();
      cd_f16_t S[2];
#pragma unroll
      for (int tm = 0; tm < 2; ++tm) {
#pragma unroll
        for (int r = 0; r < 16; ++r) S[tm][r] = 0.0f;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
          S[tm] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lds.k[buf][8 * tm + kk][l], Q[kk], S[tm], 0, 0, 0);
      }
      const bool masked = ok != 15u || kUnit * (u + 1) > lim_min;
      if (masked) {
#pragma unroll
        for (int tm = 0; tm < 2; ++tm)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int t = 32 * tm + 8 * (r >> 2) + 4 * hh + (r & 3);
            const bool see = ((ok >> (2 * tm + (r >> 3))) & 1) && kUnit * u + t < lim && kUnit * u + t < tile.ctx;
            S[tm][r] = see ? S[tm][r] : -INFINITY;
          }
      }
      soften(S, qs.x, 0.0f);
      cd_h8_t P[4];
#pragma unroll
      for (int pg = 0; pg < 4; ++pg)
#pragma unroll
        for (int j = 0; j < 8; ++j) P[pg][j] = (_Float16)S[pg >> 1][8 * (pg & 1) + j];
      uint32_t bad = 0;
      if (ok != 15u || kUnit * (u + 1) > lim_tile) {
#pragma unroll
        for (int x = 0; x < RW; ++x) bad |= lds.bad[buf][x];
      }
      if (__builtin_amdgcn_readfirstlane(bad)) {
        // a value that is not finite must not reach rows that do not see its token: one token at a time
        for (int t = 0; t < kUnit; ++t) {
          const int pg = t >> 4, j = ((t >> 3) & 1) * 4 + (t & 3), th = (t >> 2) & 1;
          const bool see = ((ok >> pg) & 1) && kUnit * u + t < lim && kUnit * u + t < tile.ctx;
          cd_h8_t p1 = P[0];
#pragma unroll
          for (int x = 1; x < 4; ++x) p1 = pg == x ? P[x] : p1;
#pragma unroll
          for (int x = 0; x < 8; ++x) p1[x] = x == j && hh == th ? p1[x] : (_Float16)0.0f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            cd_h8_t v1 = lds.v[buf][4 * pg + i][l];
#pragma unroll
            for (int x = 0; x < 8; ++x) v1[x] = x == j && hh == th ? v1[x] : (_Float16)0.0f;
            cd_f16_t d;
#pragma unroll
            for (int r = 0; r < 16; ++r) d[r] = 0.0f;
            d = __builtin_amdgcn_mfma_f32_32x32x16_f16(v1, p1, d, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 16; ++r) O[i][r] += see ? d[r] : 0.0f;
          }
        }
      } else {
#pragma unroll
        for (int pg = 0; pg < 4; ++pg)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            O[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(lds.v[buf][4 * pg + i][l], P[pg], O[i], 0, 0, 0);
      }
      if (more) build(u + 1, buf ^ 1);
      ok = raw.ok;
    }

    // ---- un-rotate: O^T <- R_V O^T, on the normalized sums (within fp16's range, being averages of the values)
    __syncthreads();
    cd_h8_t* rv = &lds.k[0][0][0];
    const cd_h8_t* src = reinterpret_cast<const cd_h8_t*>(a.rv) + (size_t)h * 2048;
    for (int x = threadIdx.x; x < 2048; x += 64 * RW) rv[x] = src[x];
    __syncthreads();
    const float all = sum + __shfl_xor(sum, 32), inv = all == 0.0f ? 0.0f : 1.0f / all;
    cd_h8_t B[8];
#pragma unroll
    for (int op = 0; op < 8; ++op)
#pragma unroll
      for (int j = 0; j < 8; ++j) B[op][j] = (_Float16)(O[op >> 1][8 * (op & 1) + j] * inv);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      cd_f16_t d;
#pragma unroll
      for (int r = 0; r < 16; ++r) d[r] = 0.0f;
#pragma unroll
      for (int op = 0; op < 8; ++op) d = __builtin_amdgcn_mfma_f32_32x32x16_f16(rv[512 * t + 64 * op + l], B[op], d, 0, 0, 0);
#pragma unroll
      for (int r = 0; r < 16; ++r) O[t][r] = d[r] * all;
    }
    __syncthreads();
  }

  // ==== the chunk's own tokens, bf16
  const int c0 = max(item.u0 - nI, 0), c1 = item.u1 - nI;
  if (c0 < c1) {
    constexpr int PP = TV / 2;  // tile pairs: one load of two neighbouring channels serves two tiles
    cd_b8_t Q[8];
    const uint16_t* qp = a.q + (tile.start + tok) * a.q_stride + (size_t)head * kHeadDim + 8 * hh;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) Q[kk] = *reinterpret_cast<const cd_b8_t*>(qp + 16 * kk);
    const int tmw = RW == 8 ? w >> 2 : RW == 4 ? w >> 1 : w;
    const int op0 = RW == 8 ? 2 * (w & 3) : RW == 4 ? 4 * (w & 1) : 0;
    const int page0 = RW == 8 ? w >> 1 : RW == 4 ? w : 2 * w;
    const int pair0 = RW == 8 ? w & 1 : 0;
    struct Raw {
      cd_u4_t k[2 * KW];
      uint32_t v[PV][PP][8];
    } raw;
    const uint16_t* kb = a.k_new + tile.start * a.k_stride + (size_t)h * kHeadDim + 8 * hh;
    const uint16_t* vb = a.v_new + tile.start * a.v_stride + (size_t)h * kHeadDim + 2 * n;
    auto fetch = [&](int u) {
      const int t = min(kUnit * u + 32 * tmw + n, tile.n - 1);
      const uint16_t* kr = kb + t * a.k_stride;
#pragma unroll
      for (int i = 0; i < 2 * KW; ++i) raw.k[i] = *reinterpret_cast<const cd_u4_t*>(kr + 16 * (op0 + i));
#pragma unroll
      for (int p = 0; p < PV; ++p)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int tv = min(kUnit * u + kBlock * (page0 + p) + 8 * (j >> 2) + 4 * hh + (j & 3), tile.n - 1);
          const uint16_t* vr = vb + tv * a.v_stride;
#pragma unroll
          for (int x = 0; x < PP; ++x) raw.v[p][x][j] = *reinterpret_cast<const uint32_t*>(vr + 64 * (pair0 + x));
        }
    };
    const int tok_tile = tile.row0 / a.gq, tok_w = min(row_w, rows - 1) / a.gq;  // first tokens of the tile and the wave
    auto build = [&](int u, int buf) {
#pragma unroll
      for (int i = 0; i < 2 * KW; ++i) lds.k[buf][8 * tmw + op0 + i][l] = __builtin_bit_cast(cd_h8_t, raw.k[i]);
      const bool masked = kUnit * u + kUnit - 1 > tok_tile;
      bool bad = false;
#pragma unroll
      for (int p = 0; p < PV; ++p) {
        if (masked) {
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            const int tv = kUnit * u + kBlock * (page0 + p) + 8 * (j >> 2) + 4 * hh + (j & 3);
#pragma unroll
            for (int x = 0; x < PP; ++x) {
              uint32_t& y = raw.v[p][x][j];
              y = tv < tile.n ? y : 0u;
              bad = bad || (y & 0x7F80u) == 0x7F80u || (y & 0x7F800000u) == 0x7F800000u;
            }
          }
        }
#pragma unroll
        for (int x = 0; x < PP; ++x) {
          cd_u4_t e, o;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            e[j] = __builtin_amdgcn_perm(raw.v[p][x][2 * j + 1], raw.v[p][x][2 * j], 0x05040100u);
            o[j] = __builtin_amdgcn_perm(raw.v[p][x][2 * j + 1], raw.v[p][x][2 * j], 0x07060302u);
          }
          lds.v[buf][4 * (page0 + p) + 2 * (pair0 + x)][l] = __builtin_bit_cast(cd_h8_t, e);
          lds.v[buf][4 * (page0 + p) + 2 * (pair0 + x) + 1][l] = __builtin_bit_cast(cd_h8_t, o);
        }
      }
      if (masked) {
        const bool any = __any(bad);
        if (l == 0) lds.bad[buf][w] = any;
      }
    };
    auto operand = [](const cd_h8_t& x) { return __builtin_bit_cast(cd_b8_t, x); };
    int u = c0, buf = 0;
    fetch(u);
    build(u, 0);
    for (; u < c1; ++u, buf ^= 1) {
      const bool more = u + 1 < c1;
      if (more) fetch(u + 1);
      __syncthreads();
      cd_f16_t S[2];
#pragma unroll
      for (int tm = 0; tm < 2; ++tm) {
#pragma unroll
        for (int r = 0; r < 16; ++r) S[tm][r] = 0.0f;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
          S[tm] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand(lds.k[buf][8 * tm + kk][l]), Q[kk], S[tm], 0, 0, 0);
      }
      if (kUnit * u + kUnit - 1 > tok_w) {
#pragma unroll
        for (int tm = 0; tm < 2; ++tm)
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const int t = kUnit * u + 32 * tm + 8 * (r >> 2) + 4 * hh + (r & 3);
            S[tm][r] = t <= tok ? S[tm][r] : -INFINITY;
          }
      }
      soften(S, kLogit2, qs.y);
      cd_b8_t P[4];
#pragma unroll
      for (int pg = 0; pg < 4; ++pg)
#pragma unroll
        for (int j = 0; j < 8; ++j) P[pg][j] = (__bf16)S[pg >> 1][8 * (pg & 1) + j];
      uint32_t bad = 0;
      if (kUnit * u + kUnit - 1 > tok_tile) {
#pragma unroll
        for (int x = 0; x < RW; ++x) bad |= lds.bad[buf][x];
      }
      if (__builtin_amdgcn_readfirstlane(bad)) {
        for (int t = 0; t < kUnit; ++t) {
          const int pg = t >> 4, j = ((t >> 3) & 1) * 4 + (t & 3), th = (t >> 2) & 1;
          const bool see = kUnit * u + t <= tok;
          cd_b8_t p1 = P[0];
#pragma unroll
          for (int x = 1; x < 4; ++x) p1 = pg == x ? P[x] : p1;
#pragma unroll
          for (int x = 0; x < 8; ++x) p1[x] = x == j && hh == th ? p1[x] : (__bf16)0.0f;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            cd_b8_t v1 = operand(lds.v[buf][4 * pg + i][l]);
#pragma unroll
            for (int x = 0; x < 8; ++x) v1[x] = x == j && hh == th ? v1[x] : (__bf16)0.0f;
            cd_f16_t d;
#pragma unroll
            for (int r = 0; r < 16; ++r) d[r] = 0.0f;
            d = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v1, p1, d, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 16; ++r) O[i][r] += see ? d[r] : 0.0f;
          }
        }
      } else {
#pragma unroll
        for (int pg = 0; pg < 4; ++pg)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            O[i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(operand(lds.v[buf][4 * pg + i][l]), P[pg], O[i], 0, 0, 0);
      }
      if (more) build(u + 1, buf ^ 1);
    }
  }

  // ---- results: register 4 u + v of tile 2 a + e is channel 64 a + 16 u + 8 hh + 2 v + e
  const float all = sum + __shfl_xor(sum, 32);
  if (row >= rows) return;
  if (item.slot < 0) {
    const float inv = all == 0.0f ? 0.0f : 1.0f / all;
    uint16_t* o = a.out + ((size_t)(tile.start + tok) * a.Hq + head) * kHeadDim + 8 * hh;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t y[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) y[v] = pack_bf16(O[2 * x][4 * q + v] * inv, O[2 * x + 1][4 * q + v] * inv);
        *reinterpret_cast<uint4*>(o + 64 * x + 16 * q) = make_uint4(y[0], y[1], y[2], y[3]);
      }
  } else {
    // partial: bm rows of 128 sums, then their (m, l)
    float* part = a.part + ((size_t)item.slot * H + h) * a.bm * kChunkPartStride;
    const int rt = row - tile.row0;
    float* o = part + (size_t)rt * kHeadDim + 8 * hh;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float4* d = reinterpret_cast<float4*>(o + 64 * x + 16 * q);
        d[0] = make_float4(O[2 * x][4 * q], O[2 * x + 1][4 * q], O[2 * x][4 * q + 1], O[2 * x + 1][4 * q + 1]);
        d[1] = make_float4(O[2 * x][4 * q + 2], O[2 * x + 1][4 * q + 2], O[2 * x][4 * q + 3], O[2 * x + 1][4 * q + 3]);
      }
    if (hh == 0) reinterpret_cast<float2*>(part + (size_t)a.bm * kHeadDim)[rt] = make_float2(m, all);
  }
}

// Block (tile, KV head, 16 rows): thread (row, eight channels) sums the tile's pieces in order.
__global__ __launch_bounds__(256) void chunk_merge_kernel(ChunkArgs a) {
  const int t = blockIdx.x, h = blockIdx.y, H = a.cv.num_kv_heads;
  if (t >= a.counts[1]) return;
  const ChunkTile tile = a.tiles[t];
  if (tile.slot < 0) return;
  const int rt = blockIdx.z * 16 + (threadIdx.x >> 4), c = 8 * (threadIdx.x & 15), row = tile.row0 + rt;
  if (row >= tile.n * a.gq) return;
  const size_t stride = (size_t)H * a.bm * kChunkPartStride;
  const float* part = a.part + ((size_t)tile.slot * H + h) * a.bm * kChunkPartStride;
  float top = kNone;
  for (int p = 0; p < tile.pieces; ++p) top = fmaxf(top, reinterpret_cast<const float2*>(part + p * stride + (size_t)a.bm * kHeadDim)[rt].x);
  float o[8] = {}, all = 0.0f;
  for (int p = 0; p < tile.pieces; ++p) {
    const float* x = part + p * stride;
    const float2 ml = reinterpret_cast<const float2*>(x + (size_t)a.bm * kHeadDim)[rt];
    const float4* d = reinterpret_cast<const float4*>(x + (size_t)rt * kHeadDim + c);
    const float4 u = d[0], v = d[1];
    const float f = __builtin_amdgcn_exp2f(ml.x - top);
    all = __builtin_fmaf(ml.y, f, all);
    o[0] = __builtin_fmaf(u.x, f, o[0]), o[1] = __builtin_fmaf(u.y, f, o[1]);
    o[2] = __builtin_fmaf(u.z, f, o[2]), o[3] = __builtin_fmaf(u.w, f, o[3]);
    o[4] = __builtin_fmaf(v.x, f, o[4]), o[5] = __builtin_fmaf(v.y, f, o[5]);
    o[6] = __builtin_fmaf(v.z, f, o[6]), o[7] = __builtin_fmaf(v.w, f, o[7]);
  }
  const float inv = all == 0.0f ? 0.0f : 1.0f / all;
  const int tok = row / a.gq;
  uint16_t* out = a.out + ((size_t)(tile.start + tok) * a.Hq + h * a.gq + row - tok * a.gq) * kHeadDim + c;
  *reinterpret_cast<uint4*>(out) = make_uint4(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv),
                                              pack_bf16(o[4] * inv, o[5] * inv), pack_bf16(o[6] * inv, o[7] * inv));
}

ChunkPlan make_chunk_plan(int B, int Hq, int H, int total_q, int max_q, int max_ctx) {
  ChunkPlan p{};
  const int gq = Hq / H;
  const long long seq_rows = (long long)max_q * gq, rows = (long long)total_q * gq;
  p.waves = seq_rows <= 64 ? 2 : seq_rows <= 128 ? 4 : 8;
  p.bm = 32 * p.waves;
  const long long per_seq = (seq_rows + p.bm - 1) / p.bm;
  long long tiles = B * per_seq, by_rows = rows / p.bm + B;
  tiles = tiles < by_rows ? tiles : by_rows;
  p.max_tiles = (int)(tiles < 1 ? 1 : tiles);
  // pieces of all heads: two rounds of the resident work-groups (an eight-wave group per unit, or as many smaller ones)
  const long long resident = (long long)num_cus() * (8 / p.waves);
  p.target = 2 * resident;
  p.min_units = 4;
  const long long extra = p.target / H + 1;
  const long long most = ((long long)max_ctx + 63) / 64 + ((long long)max_q + 63) / 64, cuts = (most + p.min_units - 1) / p.min_units;
  p.max_items = (int)(p.max_tiles + (extra < tiles * cuts ? extra : tiles * cuts));
  p.max_slots = (int)(2 * extra < tiles * cuts ? 2 * extra : tiles * cuts);
  const long long q_tiles = (rows + 31) / 32, want = (2LL * num_cus() + H - 1) / H;
  p.rot_blocks = (int)(q_tiles < want ? (q_tiles < 1 ? 1 : q_tiles) : want);
  auto up = [](size_t x) { return (x + 255) & ~size_t(255); };
  size_t off = 0;
  p.off_counts = off, off = up(off + 2 * sizeof(int32_t));
  p.off_start = off, off = up(off + (size_t)B * sizeof(int32_t));
  p.off_tiles = off, off = up(off + (size_t)p.max_tiles * sizeof(ChunkTile));
  p.off_items = off, off = up(off + (size_t)p.max_items * sizeof(ChunkItem));
  p.off_qrot = off, off = up(off + (size_t)H * rows * kHeadDim * sizeof(uint16_t));
  p.off_qscale = off, off = up(off + (size_t)H * rows * sizeof(float2));
  p.off_rv = off, off = up(off + (size_t)H * kHeadDim * kHeadDim * sizeof(uint16_t));
  p.off_part = off, off = up(off + (size_t)p.max_slots * H * p.bm * kChunkPartStride * sizeof(float));
  p.total = off;
  return p;
}

namespace {

template <int NG, int RW>
hipError_t launch_attn(const ChunkArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((chunk_attn_kernel<NG, RW>), dim3((unsigned)((long long)a.max_items * a.cv.num_kv_heads)), dim3(64 * RW),
                     0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_chunk_attention(ChunkArgs a, const ChunkPlan& p, uint8_t* ws, hipStream_t s) {
  a.bm = p.bm;
  a.max_tiles = p.max_tiles;
  a.max_items = p.max_items;
  a.max_slots = p.max_slots;
  a.target = p.target;
  a.min_units = p.min_units;
  a.rot_blocks = p.rot_blocks;
  a.counts = reinterpret_cast<int32_t*>(ws + p.off_counts);
  a.tile_start = reinterpret_cast<int32_t*>(ws + p.off_start);
  a.tiles = reinterpret_cast<ChunkTile*>(ws + p.off_tiles);
  a.items = reinterpret_cast<ChunkItem*>(ws + p.off_items);
  a.qrot = reinterpret_cast<uint16_t*>(ws + p.off_qrot);
  a.qscale = reinterpret_cast<float2*>(ws + p.off_qscale);
  a.rv = reinterpret_cast<uint16_t*>(ws + p.off_rv);
  a.part = reinterpret_cast<float*>(ws + p.off_part);
  const int H = a.cv.num_kv_heads;
  hipLaunchKernelGGL(chunk_prep_kernel, dim3(1 + H + H * p.rot_blocks), dim3(kPrepThreads), 0, s, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  if (a.cv.groups == 4)
    e = p.waves == 8 ? launch_attn<4, 8>(a, s) : p.waves == 4 ? launch_attn<4, 4>(a, s) : launch_attn<4, 2>(a, s);
  else
    e = p.waves == 8 ? launch_attn<1, 8>(a, s) : p.waves == 4 ? launch_attn<1, 4>(a, s) : launch_attn<1, 2>(a, s);
  if (e != hipSuccess) return e;
  if (p.max_slots > 1) {
    hipLaunchKernelGGL(chunk_merge_kernel, dim3(p.max_tiles, H, p.bm / 16), dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace int2kv
