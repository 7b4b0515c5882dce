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

// x / d for x >= 0, d > 0, without the long way of integer division: a float quotient is off by at most x / d * 2^-22, its
// remainder's by less than one
__device__ __forceinline__ int quotient(int x, int d) {
  const float inv = __builtin_amdgcn_rcpf((float)d);
  int q = (int)((float)x * inv);
  int r = x - q * d;
  const int more = (int)((float)r * inv);
  q += more;
  r -= more * d;
  q += r >= d ? 1 : 0;
  return q - (r < 0 ? 1 : 0);
}

struct Seq {
  int start, n, ctx;
  int past;  // cached tokens before the first new one where the cache holds both, by the whole sequence and its whole length
             // (n and ctx are cut to max_q, max_ctx and the table); negative where the length does not hold the sequence.
             // TREE: the tree's tokens before the first new one, by the same rule
};
struct Tree {  // rows of a sequence's tree in k_new and v_new
  int start, count;
};
__device__ __forceinline__ Tree tree_of(const ChunkArgs& a, int b) {
  const int start = min(max(a.tree_starts[b], 0), a.total_tree), end = min(max(a.tree_starts[b + 1], 0), a.total_tree);
  return Tree{start, max(end - start, 0)};
}
template <bool TREE>
__device__ __forceinline__ Seq seq_of(const ChunkArgs& a, int b) {
  Seq s;
  s.start = min(max(a.starts[b], 0), a.total_q);
  const int end = min(max(a.starts[b + 1], 0), a.total_q);
  const int count = max(end - s.start, 0), len = max(a.lens[b], 0);
  s.n = min(count, a.max_q);
  const long long room = (long long)a.max_blocks * kBlock;
  s.ctx = min(len, (int)(room < a.max_ctx ? room : a.max_ctx));
  s.past = (TREE ? tree_of(a, b).count : len) - count;
  return s;
}
// Cached tokens that new token i sees (not above zero: none)
__device__ __forceinline__ int limit_of(const ChunkArgs& a, const Seq& s, int i) { return a.own ? s.ctx : min(s.ctx, s.past + i + 1); }
// Units of a tile whose last new token is i: INT2 units, then units of the chunk's own tokens
__device__ __forceinline__ int int2_units(const ChunkArgs& a, const Seq& s, int i) {
  const int lim = a.own ? s.ctx : max(0, min(s.ctx, s.past + i + 1));
  return (lim + kUnit - 1) / kUnit;
}
template <bool TREE>
__device__ __forceinline__ int own_units(const ChunkArgs& a, const Seq& s, int i) {
  if constexpr (TREE) {
    const int t = min(s.past + i, a.max_tree - 1);
    return t < 0 ? 0 : t / kUnit + 1;
  }
  return a.own ? i / kUnit + 1 : 0;
}

// ---- The plan. A sequence's rows are tiles of bm; a tile is cut into equal pieces of at most about L units, by its own units
// where the tiles leave places on the chip free (up to 64 of them), else all tiles of a sequence like its longest; a
// work-group takes one piece of one KV head. L comes from an estimate of the time in units of work: while all pieces have a
// place on the chip at once, the longest; beyond that the average load and half a piece; a piece costs piece_units beside its
// own units, a partial merge_units.
struct Load {  // of one sequence: row tiles, and units of the last one; or of one tile
  int tiles, units;
};
template <bool TREE>
__device__ __forceinline__ Load load_of(const ChunkArgs& a, const Seq& s) {
  const int rows = s.n * a.gq;
  if (rows == 0) return Load{0, 0};
  return Load{quotient(rows + a.bm - 1, a.bm), int2_units(a, s, s.n - 1) + own_units<TREE>(a, s, s.n - 1)};
}
// Units of the tile of rows row0 ..
template <bool TREE>
__device__ __forceinline__ int tile_units(const ChunkArgs& a, const Seq& s, int row0) {
  const int i = quotient(max(min(row0 + a.bm, s.n * a.gq) - 1, 0), a.gq);
  return int2_units(a, s, i) + own_units<TREE>(a, s, i);
}
constexpr int kCuts = 16;
// Candidate k: units of a piece. The first leaves the tiles whole; the others lie above the size that would fill the places
// on the chip evenly, once or (from 10 on) up to three times. even: units of a place
__device__ __forceinline__ int cut_of(const ChunkArgs& a, int k, float even, int umax) {
  if (k == 0) return max(umax, 1);
  return max(a.min_piece, (int)fminf(even * (k < 10 ? 0.85f + 0.15f * (float)k : 0.32f + 0.12f * (float)(k - 10)), 1.0e9f) + 1);
}
// Pieces of a tile of so many units
__device__ __forceinline__ int pieces_of(int units, int L) { return max(1, quotient(units + L - 1, L)); }
// The time in units with pieces of at most c units, n of them a KV head, `parts` of them of tiles that are cut; places: a KV
// head's part of the chip
__device__ __forceinline__ float cost_of(const ChunkArgs& a, int c, int n, int parts, float even, float places, int umax) {
  const float one = (float)min(c, umax) + a.piece_units, fn = (float)n;
  const float load = even + fn * a.piece_units * __builtin_amdgcn_rcpf(places);
  // Two work-groups of a compute unit share it: one alone takes 0.6 of the time, the fullest pair lies between the average
  // and two of the longest. Where there are more pieces than places the longest may come last, by half.
  const float at_once = a.per_cu == 2 ? fmaxf(0.6f * one, 0.5f * (one + load)) : one;
  const float time = fn <= places ? at_once : fmaxf(load, one) + 0.5f * one;
  return time + (float)parts * (float)a.cv.num_kv_heads * a.merge_units;
}
// whether n pieces may be: they have room, and a place each while the tiles have one (more pieces than that never paid: the
// chip slows down as its places fill)
__device__ __forceinline__ bool fits(const ChunkArgs& a, int n, int T, float places) {
  return n <= a.max_slots && ((float)T > places || (float)n <= places);
}
__device__ __forceinline__ float places_of(const ChunkArgs& a) {
  return (float)a.resident * __builtin_amdgcn_rcpf((float)a.cv.num_kv_heads);
}
// Sum and maximum over the wave: rotations inside rows of 16 lanes, then swaps of rows and halves
template <class F>
__device__ __forceinline__ int wave_fold(int x, F f) {
  x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x128, 0xF, 0xF, false));
  x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x124, 0xF, 0xF, false));
  x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x122, 0xF, 0xF, false));
  x = f(x, __builtin_amdgcn_update_dpp(0, x, 0x121, 0xF, 0xF, false));
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = f((int)r[0], (int)r[1]);
  const auto h = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return f((int)h[0], (int)h[1]);
}
__device__ __forceinline__ int wave_sum(int x) {
  return wave_fold(x, [](int a, int b) { return a + b; });
}
__device__ __forceinline__ float wave_sum(float x) {  // the same order, so the same sum, in every wave
  return __int_as_float(wave_fold(__float_as_int(x), [](int a, int b) { return __float_as_int(__int_as_float(a) + __int_as_float(b)); }));
}
// Sum over the lanes l % 16
__device__ __forceinline__ int quarters_sum(int x) {
  const auto r = __builtin_amdgcn_permlane16_swap(x, x, false, false);
  x = (int)r[0] + (int)r[1];
  const auto h = __builtin_amdgcn_permlane32_swap(x, x, false, false);
  return (int)h[0] + (int)h[1];
}
// Inclusive sum over the wave: shifts inside rows of 16 lanes, then the rows' and the halves' last lanes onto those behind
__device__ __forceinline__ int wave_scan(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xF, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xA, 0xF, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xC, 0xF, false);
  return x;
}

// A work-group's piece
struct Place {
  Seq s;
  int b, row0;      // sequence, first row of the tile
  int u0, u1;       // units
  int slot;         // partial, -1: the result itself
  bool valid;
};
// The piece, longest first, of a KV head's work-group `at`. Where two work-groups share a compute unit and all have a place,
// the second ones (those from `half` on) come in the opposite order, the shortest beside the longest.
__device__ __forceinline__ int rank_of(const ChunkArgs& a, int at, int total) {
  const int half = quotient(a.resident >> 1, a.cv.num_kv_heads);
  return a.per_cu == 2 && at >= half && total * a.cv.num_kv_heads <= a.resident ? total - 1 - (at - half) : at;
}
// The piece of work-group `at`, found by every wave for itself: the sequences with the longest pieces come first, and of a
// sequence the last tiles, under a causal mask its longest. Writes the record of a cut tile for the merge (first piece, head 0).
template <bool TREE>
__device__ __forceinline__ Place locate(const ChunkArgs& a, int at, int h) {
  const int lane = threadIdx.x & 63;
  Place p;
  p.valid = false;
  Load load;
  int total, b, first, tile0, local, pieces, row = 0;
  // (expected, so that this path's code comes first: behind the other's it cost long chunks 0.6 %)
  if (__builtin_expect(a.B <= kChunkWaveSeqs, 1)) {
    Seq s{0, 0, 0, 0};
    if (lane < a.B) s = seq_of<TREE>(a, lane);
    load = load_of<TREE>(a, s);
    int tiles = wave_scan(load.tiles), lane_b = lane, lane_row = 0;
    const int T = __builtin_amdgcn_readlane(tiles, 63);
    const float places = places_of(a);
    const bool by_tile = T <= 64 && (float)T < places && __ballot(load.tiles > 1) != 0;
    if (by_tile) {  // a tile per lane: only those that are longer than others need be cut
      if (a.B > 1) {
        lane_b = 0;
#pragma unroll
        for (int step = 32; step > 0; step >>= 1) lane_b += __shfl(tiles, lane_b + step - 1) <= lane ? step : 0;
      } else {
        lane_b = 0;
      }
      const Seq q{0, __shfl(s.n, lane_b), __shfl(s.ctx, lane_b), __shfl(s.past, lane_b)};
      lane_row = (lane - __shfl(tiles - load.tiles, lane_b)) * a.bm;
      load = lane < T ? Load{1, tile_units<TREE>(a, q, lane_row)} : Load{0, 0};
      tiles = min(lane + 1, T);
    }
    const int umax = wave_fold(load.units, [](int x, int y) { return max(x, y); });
    const float W = wave_sum((float)load.tiles * (float)load.units), even = W * __builtin_amdgcn_rcpf(places);
    // A candidate per lane (of sixteen), a quarter of the sequences or tiles per sixteen lanes
    const int c = cut_of(a, lane & 15, even, umax), lanes = ((T <= 64 ? max(a.B, T) : a.B) + 3) & ~3;
    int n = 0, parts = 0;
    for (int i = lane >> 4; i < lanes; i += 4) {
      const int k = pieces_of(__shfl(load.units, i), c), x = __shfl(load.tiles, i) * k;
      n += x;
      parts += k > 1 ? x : 0;
    }
    n = quarters_sum(n), parts = quarters_sum(parts);
    const bool may = (lane & 15) == 0 || fits(a, n, T, places);
    const int cost = __float_as_int(may ? cost_of(a, c, n, parts, even, places, umax) : INFINITY);  // (positive: ordered as integers)
    const int best = wave_fold(cost, [](int x, int y) { return min(x, y); });
    const int L = __builtin_amdgcn_readlane(c, __ffsll(__ballot(cost == best)) - 1);
    const int mine_k = load.tiles > 0 ? pieces_of(load.units, L) : 0, mine = load.tiles * mine_k, upto = wave_scan(mine);
    total = __builtin_amdgcn_readlane(upto, 63);
    if (at == 0 && h == 0 && threadIdx.x == 0) a.head[1] = total > a.max_items || T > a.max_tiles ? 0 : T;
    total = min(total, a.max_items);
    if (at >= total) return p;
    const int r = rank_of(a, at, total), size = mine > 0 ? quotient(load.units + mine_k - 1, mine_k) : -1;
    // the length of piece r: the greatest that more than r pieces have
    int hi = wave_fold(size, [](int x, int y) { return max(x, y); }), lo = a.B == 1 && !by_tile ? hi : 0, above = 0;
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1, n = wave_sum(size >= mid ? mine : 0);
      if (n > r) lo = mid;
      else hi = mid - 1, above = n;
    }
    const int same = size == lo ? mine : 0, past = wave_scan(same);
    const int x = max(__ffsll(__ballot(past > r - above)) - 1, 0);
    local = r - above - __builtin_amdgcn_readlane(past - same, x);
    first = __builtin_amdgcn_readlane(upto - mine, x);
    tile0 = __builtin_amdgcn_readlane(tiles - load.tiles, x);
    pieces = __builtin_amdgcn_readlane(mine_k, x);
    load.tiles = __builtin_amdgcn_readlane(load.tiles, x);
    row = __builtin_amdgcn_readlane(lane_row, x);
    b = min(__builtin_amdgcn_readlane(lane_b, x), a.B - 1);
    p.s = Seq{__builtin_amdgcn_readlane(s.start, b), __builtin_amdgcn_readlane(s.n, b), __builtin_amdgcn_readlane(s.ctx, b),
              __builtin_amdgcn_readlane(s.past, b)};
  } else {
    total = a.head[0];
    if (at >= total) return p;
    const int r = rank_of(a, at, total);
    // the last sequence, in the order of their pieces' lengths, whose pieces start at or before r, 64 probes at a time
    int lo = 0, len = a.B;
    while (len > 1) {
      const int step = (len + 63) / 64, x = lo + lane * step;
      const int n = __popcll(__ballot(lane * step < len && a.item_start[min(x, a.B - 1)] <= r));
      lo += (n - 1) * step;
      len = min(step, len - (n - 1) * step);
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    b = a.order[lo];
    first = a.item_start[lo];
    local = r - first;
    tile0 = a.tile_start[b];
    p.s = seq_of<TREE>(a, b);
    load = load_of<TREE>(a, p.s);
    pieces = pieces_of(load.units, a.head[2]);
  }
  const int back = quotient(local, pieces), t = load.tiles - 1 - back, piece = local - back * pieces;
  p.b = b;
  p.row0 = row + t * a.bm;
  const int units = tile_units<TREE>(a, p.s, p.row0);
  const int each = quotient(units, pieces), more = units - each * pieces;  // the first `more` pieces have one more
  p.u0 = each * piece + min(piece, more);
  p.u1 = p.u0 + each + (piece < more ? 1 : 0);
  p.slot = pieces > 1 ? first + local : -1;
  p.valid = t >= 0 && p.slot < a.max_slots;
  if (piece == 0 && h == 0 && threadIdx.x == 0 && t >= 0 && tile0 + t < a.max_tiles)
    a.tiles[tile0 + t] = ChunkTile{p.row0, p.s.start, p.s.n, pieces, p.slot};
  // the same in every lane: into scalar registers
  auto one = [](int x) { return __builtin_amdgcn_readfirstlane(x); };
  p.s = Seq{one(p.s.start), one(p.s.n), one(p.s.ctx), one(p.s.past)};
  p.row0 = one(p.row0), p.u0 = one(p.u0), p.u1 = one(p.u1), p.slot = one(p.slot), p.b = one(p.b);
  return p;
}

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

// fp16 operands: INT2 units, whose codes, scales and zeros are fp16's own; probabilities are held times 2^kBias in it (with
// queries and rows together 0.0018 off from 64 bits in the row norm, the output's rounding alone 0.0017). The rotated queries carry log2(e) / sqrt(128), so scores are base-2 logarithms as they are.
struct HalfOps {
  typedef cd_h8_t vec;
  static __device__ __forceinline__ cd_f16_t mfma(const cd_h8_t& a, const vec& b, const cd_f16_t& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
  }
  static constexpr bool kBased = false;
  static __device__ __forceinline__ float score(float s, float base) { return s + base; }
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
// the same with products that start at base: one addition a score less, for 16 registers that hold it
struct BasedOps : HalfOps {
  static constexpr bool kBased = true;
  static __device__ __forceinline__ float score(float s, float) { return s; }
};
// bf16 operands: the chunk's own units, whose scores are scaled in fp32. The values are the caller's bf16 rows, whose range
// fp16 does not have, and a product takes one type: the probabilities are rounded to bf16 too, 2^-8 of each, with signs that
// average out over a row's tokens (a prompt of 2,011: 0.0021 off from 64 bits in the row norm, the output's rounding alone
// 0.0016).
struct BfOps {
  typedef cd_b8_t vec;
  static __device__ __forceinline__ cd_f16_t mfma(const cd_h8_t& a, const vec& b, const cd_f16_t& c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(cd_b8_t, a), b, c, 0, 0, 0);
  }
  static constexpr bool kBased = false;
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
template <class Ops, int N, int TILES>
__device__ __forceinline__ void settle(cd_f16_t (&X)[N], float& base, float& m, float& sum, float& thr, cd_f16_t (&O)[TILES],
                                       cd_f16_t* start = nullptr) {
  float a = fmaxf(X[0][0], X[0][1]);
#pragma unroll
  for (int i = 2; i < 16 * N; i += 2) a = fmaxf(fmaxf(a, X[i >> 4][i & 15]), X[i >> 4][(i & 15) + 1]);
  const float top = Ops::score(pair_max(a), base);
  const bool move = top > thr;
  if (__any(move)) {
    const float d = move ? top - kBias : 0.0f;
    const float f = !move ? 1.0f : thr < 0.0f ? 0.0f : __builtin_amdgcn_exp2f(-d);
    m += d;
    base -= d;
    if constexpr (Ops::kBased) {
      *start -= d;
#pragma unroll
      for (int i = 0; i < N; ++i) X[i] -= d;
    }
    sum *= f;
    thr = move ? kMove : thr;
#pragma unroll
    for (int i = 0; i < TILES; ++i) O[i] *= f;
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
// A row's INT2 sums are turned by R_V in fp16. They may be averages of long contexts, far below the values, so the row is
// brought to 2^12 .. 2^13 by a power of two (`down`, taken out again by `up`) that its largest element `top` names: what lies
// 2^-26 below that is still in fp16's normal range. (Unscaled, values of 1e-5 over 1,500 tokens came out 5 % off.)
struct RowScale {
  float down, up;
};
__device__ __forceinline__ RowScale row_scale(float top) {
  const uint32_t e = min(max(__float_as_uint(top) >> 23, 13u), 253u);  // (zeros: any)
  return RowScale{__uint_as_float((266u - e) << 23), __uint_as_float((e - 12u) << 23)};
}
// The largest element of a lane's registers and its partner's
__device__ __forceinline__ float row_top(const cd_f16_t (&O)[4]) {
  float top = 0.0f;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int r = 0; r < 16; r += 2) top = fmaxf(fmaxf(top, fabsf(O[i][r])), fabsf(O[i][r + 1]));
  return pair_max(top);
}
// q mu^T of a lane's query row, in the scores' unit
__device__ __forceinline__ float query_mean(const cd_b8_t (&Q)[8], const float* mu, int hh) {
  float off = 0.0f;
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) {
    const float4* x = reinterpret_cast<const float4*>(mu + 16 * kk + 8 * hh);
    const float4 u = x[0], v = x[1];
    const float y[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) off = __builtin_fmaf((float)Q[kk][j], y[j], off);
  }
  return pair_sum(off) * kLogit2;
}
// The query rotation q'^T = R_K^T q^T leaves positions 32 i .. 32 i + 31 of tile i in a lane's registers; position ->
// channel: eight positions 2 kk + hh make operand kk's piece of lane half hh. Row m = 8 u + 4 h + v of a tile's A operand is
// position 16 (u / 2) + 8 h + 4 (u % 2) + v, so that registers 8 x .. 8 x + 7 are operand 2 i + x as it is used.
__device__ __forceinline__ int pos_channel(int pos) { return code_channel(pos >> 4, (pos >> 3) & 1, pos & 7); }
__device__ __forceinline__ int row_position(int m) { return (m & 3) | ((m & 4) << 1) | ((m & 8) >> 1) | (m & 16); }

// ---- Trees: a token sees the tokens on its path, itself, its parent and so on to one whose parent is -1
constexpr float kAbsent = -1.0f;  // sum of a partial whose row has no path: sums of probabilities are never below zero, also where scores are infinite
typedef uint32_t path_t __attribute__((ext_vector_type(kTreeMost / 32)));  // bit t % 32 of word t / 32: token t lies on it
// The path of token t of a tree whose parents lie in LDS; nothing on it for a token that has none. A parent outside [-1, t)
// ends a walk that way, so each takes at most kTreeMost steps.
__device__ __forceinline__ path_t path_of(const int32_t* parents, int t, int count) {
  path_t p = 0;
  bool any = t >= 0 && t < count;
  int x = any ? t : -1;
  while (__any(x >= 0)) {
    const int next = parents[max(x, 0)];
#pragma unroll
    for (int i = 0; i < kTreeMost / 32; ++i) p[i] |= x >> 5 == i ? 1u << (x & 31) : 0u;
    const bool good = next >= -1 && next < x;
    any = any && (x < 0 || good);
    x = good ? next : -1;
  }
  const path_t none = 0;
  return any ? p : none;
}
__device__ __forceinline__ bool has_path(const path_t& p) {
  uint32_t x = 0;
#pragma unroll
  for (int i = 0; i < kTreeMost / 32; ++i) x |= p[i];
  return x != 0;
}
// Word i (the same in every lane)
__device__ __forceinline__ uint32_t path_word(const path_t& p, int i) {
  uint32_t x = p[0];
#pragma unroll
  for (int j = 1; j < kTreeMost / 32; ++j) {
    const uint32_t y = p[j];
    x = i == j ? y : x;
  }
  return x;
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
