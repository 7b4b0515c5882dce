// Attention of a chunk of new tokens over the paged INT2 cache (int2kv_chunk_attention).
//
// Rows are (new token i of sequence b, query head j of the KV head's group), row i * G_q + j of the sequence. A row sees
// S = {cached s < limit} and, where the chunk's own keys and values are given in bf16, {new t <= i}:
//     a_s = c (q R_K) k^_s^T,   a_t = c (q k_t^T - q mu^T)   (both with centered keys; c = 1 / sqrt(128)),
//     o = (sum_s p_s v^_s) R_V^T + sum_t p_t v_t,   p = softmax over S.
// A work-group takes a piece: a tile of rows of one KV head over a range of 64-token units of the context. It finds its
// piece by itself (chunk_core.h; a planning launch goes before it for large batches), rotates its queries, goes over the
// INT2 units, un-rotates their sum, and goes over the chunk's own bf16 units. chunk_merge_kernel joins the pieces of tiles
// that were cut.
//
// Products are formed transposed (S^T = K Q^T, O^T = V^T P^T, 32 x 32 x 16): a lane holds one query row, so the softmax is
// lane-local but for one exchange of halves, the rescaling is one factor per lane, and the probabilities are the second
// product's B operand as they lie (its k order is the order of S^T's rows in a lane; V^T is laid out to match). INT2 codes
// become fp16 operands once per work-group and unit and are shared through LDS in operand order.
//
// Bound by the clock, 2.0 of 2.4 GHz under this load, and by what two waves a SIMD hide of their waits (a third of their
// cycles): 4 x 2,048 tokens of 32 heads after 8,192 cached ones take 1.33 ms (943 TFLOP/s, where an 8,192^3 product reaches
// 1,270), with the matrix pipe busy 43 % of the cycles and the vector ALU 54 %. Eight waves share a unit's operands (256 rows a
// work-group); four waves do the same in 1.51 ms, their operands being made twice as often, and serve shorter sequences.
#include <type_traits>

#include "chunk_core.h"

namespace int2kv {

namespace {

constexpr int kPlanThreads = 256;

// Inclusive sum over the block; total to every thread
__device__ __forceinline__ int block_scan(int x, int* tmp, int& total) {
  const int wave = threadIdx.x >> 6;
  x = wave_scan(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 63) tmp[wave] = x;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    before += w < wave ? tmp[w] : 0;
    total += tmp[w];
  }
  return x + before;
}

}  // namespace

// The plan of a batch too large for every wave to hold, by one block: 72 us for 100 as for 256 sequences, which its LDS atomics
// take: the compiler sums their operands in loops over a wave's lanes
template <bool TREE>
__global__ __launch_bounds__(kPlanThreads) void chunk_plan_kernel(ChunkArgs a) {
  constexpr int kClasses = 64;
  __shared__ int tmp[kPlanThreads / 64], counts[kCuts], parts[kCuts], classes[kClasses], longest;
  __shared__ unsigned long long work;
  const int tid = threadIdx.x;
  if (tid < kCuts) counts[tid] = 0, parts[tid] = 0;
  if (tid < kClasses) classes[tid] = 0;
  if (tid == 0) longest = 0, work = 0;
  __syncthreads();
  int T = 0, total = 0;
  unsigned long long W = 0;
  for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
    const Load s = b0 + tid < a.B ? load_of<TREE>(a, seq_of<TREE>(a, b0 + tid)) : Load{0, 0};
    int n;
    block_scan(s.tiles, tmp, n);
    T = min(T + n, 1 << 28);
    atomicMax(&longest, s.units);
    W += (unsigned long long)s.tiles * s.units;
  }
  atomicAdd(&work, W);
  __syncthreads();
  const int umax = longest;
  const float places = places_of(a), even = (float)work * __builtin_amdgcn_rcpf(places);
  int mine[kCuts] = {}, cut[kCuts] = {};
  for (int b = tid; b < a.B; b += kPlanThreads) {
    const Load s = load_of<TREE>(a, seq_of<TREE>(a, b));
#pragma unroll
    for (int k = 0; k < kCuts; ++k) {
      const int n = pieces_of(s.units, cut_of(a, k, even, umax));
      mine[k] += s.tiles * n;
      cut[k] += n > 1 ? s.tiles * n : 0;
    }
  }
#pragma unroll
  for (int k = 0; k < kCuts; ++k) atomicAdd(&counts[k], mine[k]), atomicAdd(&parts[k], cut[k]);
  __syncthreads();
  float best = 0.0f;
  int L = 1;
  for (int k = 0; k < kCuts; ++k) {
    const int c = cut_of(a, k, even, umax);
    const float cost = cost_of(a, c, counts[k], parts[k], even, places, umax);
    if (k == 0 || (fits(a, counts[k], T, places) && cost < best)) best = cost, L = c;
  }
  // sequences by classes of their pieces' length; within a class in any order, which changes no result
  auto class_of = [&](const Load& s) {
    const int n = pieces_of(s.units, L);
    return s.tiles == 0 ? kClasses - 1 : (int)((float)(kClasses - 1) * (1.0f - (float)quotient(s.units + n - 1, n) / (float)max(umax, 1)));
  };
  T = 0;
  for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
    const int b = b0 + tid;
    const Load s = b < a.B ? load_of<TREE>(a, seq_of<TREE>(a, b)) : Load{0, 0};
    int n_tiles;
    const int t = T + block_scan(s.tiles, tmp, n_tiles) - s.tiles;
    if (b < a.B) {
      a.tile_start[b] = t;
      atomicAdd(&classes[class_of(s)], 1);
    }
    T = min(T + n_tiles, 1 << 28);
  }
  __syncthreads();
  if (tid < kClasses) {
    const int x = classes[tid];
    classes[tid] = wave_scan(x) - x;
  }
  __syncthreads();
  for (int b = tid; b < a.B; b += kPlanThreads) a.order[atomicAdd(&classes[class_of(load_of<TREE>(a, seq_of<TREE>(a, b)))], 1)] = b;
  __syncthreads();
  for (int b0 = 0; b0 < a.B; b0 += kPlanThreads) {
    const int x = b0 + tid;
    const Load s = x < a.B ? load_of<TREE>(a, seq_of<TREE>(a, a.order[x])) : Load{0, 0};
    const int items = s.tiles * pieces_of(s.units, L);
    int n_items;
    const int i = total + block_scan(items, tmp, n_items) - items;
    if (x < a.B) a.item_start[x] = i;
    total = min(total + n_items, 1 << 28);
  }
  if (tid == 0) {
    a.head[0] = min(total, a.max_items);
    a.head[1] = total > a.max_items || T > a.max_tiles ? 0 : T;
    a.head[2] = L;
  }
}

namespace {

// What the waves share: operands of K (two units) and V^T (three: a unit's values are read after the next unit's barrier)
struct ChunkLds {
  cd_h8_t k[2][16][64];  // [slot][32-token half, operand kk][lane]
  cd_h8_t v[3][16][64];  // [slot][page, tile][lane]
};

// Running state of a lane's row. Scores arrive with m taken off (the products start at base = kBias - m); thr is the score
// that moves m: any score for a row that has seen nothing.
struct RowState {
  cd_f16_t O[4];
  float m, sum, thr;
};

// The units u0 .. u1 of one kind. Src fetches a unit's rows into registers, makes operands of them (its share of the
// work-group's), and says which scores count. Steps are 32 tokens: while the matrix cores form the next step's scores the
// vector ALU turns this step's into probabilities, and while they add this step's values it takes the next step's maximum
// and makes the operands of the next unit.
template <class Ops, class Src>
__device__ __forceinline__ void attend(Src& src, RowState& st, ChunkLds& lds, const typename Ops::vec (&Q)[8], float off, int u0,
                                       int u1, bool live) {
  const int l = threadIdx.x & 63;
  cd_f16_t S[1], T[1];
  float base = kBias - st.m - off;
  cd_f16_t start = splat16(Ops::kBased ? base : 0.0f);
  // scores of half tm of the unit in slot kb
  auto scores = [&](cd_f16_t (&X)[1], int kb, int tm) {
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) X[0] = Ops::mfma(lds.k[kb][8 * tm + kk][l], Q[kk], kk == 0 ? start : X[0]);
  };
  // hides what a row does not see
  auto rest = [&](cd_f16_t (&X)[1], int u, int tm) {
    if (src.masked(u)) {
#pragma unroll
      for (int i = 0; i < 16; ++i) X[0][i] = src.sees(u, 32 * tm + reg_token(i)) ? X[0][i] : -INFINITY;
    }
    settle<Ops>(X, base, st.m, st.sum, st.thr, st.O, &start);
  };
  auto add = [&](const cd_u4_t (&P)[2], int vb, int tm) {
#pragma unroll
    for (int pg = 0; pg < 2; ++pg)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        st.O[i] = Ops::mfma(lds.v[vb][8 * tm + 4 * pg + i][l], __builtin_bit_cast(typename Ops::vec, P[pg]), st.O[i]);
  };

  // of the two waves of a SIMD (w and w + 4) one goes first, so that they come to lie half a step apart
  if (__builtin_amdgcn_readfirstlane(threadIdx.x >> 8)) __builtin_amdgcn_s_setprio(1);
  src.template build<false>(u0, lds, 0, 0);  // (fetched by the caller)
  if (u0 + 1 < u1) src.fetch(u0 + 1);
  __syncthreads();
  int kb = 0, vb = 0;
  if (live) {
    scores(S, 0, 0);
    rest(S, u0, 0);
    for (int u = u0; u < u1; ++u) {
      const bool more = u + 1 < u1;
      const int vn = vb == 2 ? 0 : vb + 1;
      cd_u4_t P[2];
      scores(T, kb, 1);
      soften<Ops>(S[0], base, st.sum, P);
      add(P, vb, 0);
      rest(T, u, 1);
      if (more) {
        src.template build<false>(u + 1, lds, kb ^ 1, vn);
        if (u + 2 < u1) src.fetch(u + 2);
      }
      __syncthreads();
      if (more) scores(S, kb ^ 1, 0);
      soften<Ops>(T[0], base, st.sum, P);
      add(P, vb, 1);
      if (more) rest(S, u + 1, 0);
      kb ^= 1;
      vb = vn;
    }
  } else {  // a wave without rows (the last tile's): its share of the operands, the same barriers
    for (int u = u0; u < u1; ++u) {
      const bool more = u + 1 < u1;
      const int vn = vb == 2 ? 0 : vb + 1;
      if (more) {
        src.template build<false>(u + 1, lds, kb ^ 1, vn);
        if (u + 2 < u1) src.fetch(u + 2);
      }
      __syncthreads();
      kb ^= 1;
      vb = vn;
    }
  }

  // Values that are not finite, in units that some row of the tile does not see all of, were left out above, where
  // 0 * inf would have reached rows that do not see them. They are added here, to the rows that do: a token at a time.
  __syncthreads();
  uint32_t* flags = reinterpret_cast<uint32_t*>(&lds.k[0][0][0]);
  const bool mine = __any(src.found != 0);
  if (l == 0) flags[threadIdx.x >> 6] = mine;
  __syncthreads();
  uint32_t found = 0;
  for (int w = 0; w < (int)(blockDim.x >> 6); ++w) found |= flags[w];
  if (__builtin_amdgcn_readfirstlane(found)) {
    for (int u = u0; u < u1; ++u) {
      src.refetch(u);
      if (!src.partial(u)) continue;
      __syncthreads();
      src.template build<true>(u, lds, 0, 0);
      __syncthreads();
      for (int tm = 0; live && tm < 2; ++tm) {
        scores(S, 0, tm);
#pragma unroll
        for (int i = 0; i < 16; ++i) S[0][i] = src.sees(u, 32 * tm + reg_token(i)) ? S[0][i] : -INFINITY;
        cd_u4_t P[2];
        float sum = 0.0f;  // already counted
        soften<Ops>(S[0], base, sum, P);
        for (int t = 0; t < 32; ++t) {
          const int pg = t >> 4;
          const bool see = src.sees_token(u, 32 * tm + t);
          const cd_u4_t p = only_token(pg ? P[1] : P[0], t);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const cd_u4_t v = only_token(__builtin_bit_cast(cd_u4_t, lds.v[0][8 * tm + 4 * pg + i][l]), t);
            const cd_f16_t d = Ops::mfma(__builtin_bit_cast(cd_h8_t, v), __builtin_bit_cast(typename Ops::vec, p), splat16(0.0f));
#pragma unroll
            for (int y = 0; y < 16; ++y) st.O[i][y] += see ? d[y] : 0.0f;
          }
        }
      }
    }
  }
}

// The INT2 units of a sequence. Of a unit's operands wave w of NW makes those of KW words of one half's keys, and TV tiles
// of one page's values.
template <int NG, int NW>
struct Int2Source {
  using Lay = Rec<NG>;
  static constexpr int KW = 8 / NW, TV = 16 / NW, GV = NG == 4 ? TV : 1;
  const ChunkArgs& a;
  const int32_t* table;
  int h, ctx, pages, lim, lim_min, lim_tile;  // tokens the lane's row sees; the least of the wave's and of the tile's
  int l, n, hh, half, word0, page, tile0;
  uint32_t kw[KW], km[NG];
  cd_u4_t vc, vs[GV], vz[GV];
  uint32_t ok, ok_prev;                 // pages of the fetched unit and of the one before
  int pid, fetched;
  uint32_t found = 0;                   // not zero: a value that is not finite was left out

  __device__ __forceinline__ Int2Source(const ChunkArgs& args, int head, int b, int tokens, int w, int limit, int least, int least_tile)
      : a(args), table(args.table + (size_t)b * args.max_blocks), h(head), ctx(tokens), pages((tokens + kBlock - 1) / kBlock),
        lim(limit), lim_min(least), lim_tile(least_tile), l(threadIdx.x & 63), n(l & 31), hh(l >> 5), half(w / (NW / 2)), word0(KW * (w % (NW / 2))),
        page(w / (NW / 4)), tile0(TV * (w % (NW / 4))), ok(0), ok_prev(0), pid(-1), fetched(-1) {}
  // lane l: the block of page l % 4 of unit u
  __device__ __forceinline__ int page_id(int u) const {
    const int p = kUnitPages * u + (l & 3);
    return p < pages ? table[p] : -1;
  }
  __device__ __forceinline__ void fetch(int u) {
    const int H = a.cv.num_kv_heads, now = fetched == u - 1 && fetched >= 0 ? pid : page_id(u);
    const bool good = now >= 0 && now < a.cv.num_blocks;
    ok_prev = ok;
    ok = (uint32_t)__ballot(good) & 15u;
    const int id = good ? now : 0;
    auto record = [&](int p) { return a.cv.pool + ((size_t)(uint32_t)__builtin_amdgcn_readlane(id, p) * H + h) * Lay::kBytes; };
    const uint8_t* ra = record(2 * half);
    const uint8_t* rb = record(2 * half + 1);
    const uint8_t* rk = n < 16 ? ra : rb;
    const int t = row_token(n & 15);
    const uint32_t* c = reinterpret_cast<const uint32_t*>(rk + kOffKCodes + 32 * t + 16 * hh) + word0;
#pragma unroll
    for (int i = 0; i < KW; ++i) kw[i] = c[i];
    const uint32_t* m = reinterpret_cast<const uint32_t*>(rk + Lay::kOffKMeta + 4 * NG * t);
#pragma unroll
    for (int g = 0; g < NG; ++g) km[g] = m[g];
    const uint8_t* rv = record(page) + 16 * hh;
    const uint8_t* rm = rv + (NG == 4 ? 32 * tile0 : 0);
    vc = *reinterpret_cast<const cd_u4_t*>(rv + kOffVCodes + 32 * (n & 15));
#pragma unroll
    for (int g = 0; g < GV; ++g) {
      vs[g] = *reinterpret_cast<const cd_u4_t*>(rm + Lay::kOffVScale + 32 * g);
      vz[g] = *reinterpret_cast<const cd_u4_t*>(rm + Lay::kOffVZero + 32 * g);
    }
    fetched = u;
    pid = page_id(u + 1);
  }
  __device__ __forceinline__ uint32_t pages_of(int u) const { return u == fetched ? ok : ok_prev; }
  // ODD: of the values only those that are not finite; else, in partial units, only those that are
  template <bool ODD>
  __device__ __forceinline__ void build(int u, ChunkLds& lds, int kb, int vb) {
    cd_h8_t(*k)[64] = lds.k[kb];
    cd_h8_t(*v)[64] = lds.v[vb];
    cd_h2_t s[NG], z[NG];
#pragma unroll
    for (int g = 0; g < NG; ++g) s[g] = both_lo(km[g]), z[g] = both_hi(km[g]);
#pragma unroll
    for (int i = 0; i < KW; ++i) {
      cd_h8_t x[2];
      word_operands<NG>(kw[i], s, z, x);
      k[8 * half + 2 * (word0 + i)][l] = x[0];
      k[8 * half + 2 * (word0 + i) + 1][l] = x[1];
    }
    // pairs of tokens 8 hh + 2 x, + 1; tile i's channel 32 i + 16 ph + (n % 16) lies at bits 2 (2 i + ph) of each half
    uint32_t word[4], keep[4] = {~0u, ~0u, ~0u, ~0u};
#pragma unroll
    for (int x = 0; x < 4; ++x) word[x] = vc[x] >> (2 * (n >> 4) + 4 * tile0);
    const bool part = ODD || partial(u);
    if (part) {
      // tokens that do not exist: their values must not reach the product, where 0 * inf would be NaN
      int cnt = ctx - (kUnit * u + kBlock * page);
      cnt = (ok >> page) & 1 ? cnt : 0;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int tb = 8 * hh + 2 * x;
        keep[x] = (tb < cnt ? 0xFFFFu : 0u) | (tb + 1 < cnt ? 0xFFFF0000u : 0u);
      }
    }
#pragma unroll
    for (int i = 0; i < TV; ++i) {
      cd_u4_t f;
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int g = NG == 4 ? i : 0;
        // (copies: a bit cast of a vector's element takes element 0)
        const uint32_t sv = vs[g][x], zv = vz[g][x];
        const cd_h2_t code = i == 0   ? land_codes<0>(word[x])
                             : i == 1 ? land_codes<4>(word[x])
                             : i == 2 ? land_codes<8>(word[x])
                                      : land_codes<4>(word[x] >> 8);
        const cd_h2_t y = __builtin_elementwise_fma(code, __builtin_bit_cast(cd_h2_t, sv), __builtin_bit_cast(cd_h2_t, zv));
        f[x] = __builtin_bit_cast(uint32_t, y) & keep[x];
      }
      if (part) {
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const uint32_t odd = HalfOps::odd(f[x]);
          found |= odd;
          f[x] &= ODD ? odd : ~odd;
        }
      }
      v[4 * page + tile0 + i][l] = __builtin_bit_cast(cd_h8_t, f);
    }
  }
  __device__ __forceinline__ void refetch(int u) {
    fetched = -1;
    fetch(u);
  }
  __device__ __forceinline__ bool partial(int u) const { return pages_of(u) != 15u || kUnit * (u + 1) > lim_tile; }
  __device__ __forceinline__ bool masked(int u) const { return pages_of(u) != 15u || kUnit * (u + 1) > lim_min; }
  // t: token of the unit without the lane half's 4
  __device__ __forceinline__ bool sees(int u, int t) const { return sees_token(u, t + 8 * hh); }
  __device__ __forceinline__ bool sees_token(int u, int t) const { return ((pages_of(u) >> (t >> 4)) & 1) && kUnit * u + t < lim; }
};

// The chunk's own units: bf16 rows. A wave's K operands are 16-byte pieces of its half's rows; its page's values come two
// channels a load and are paired over tokens, so that tile 2 e + o holds channels 64 e + 2 m + o.
// TREE: a token sees those on its path, and every unit counts as one that some row does not see all of.
template <int NW, bool TREE>
struct OwnSource {
  static constexpr int KO = 16 / NW, PV = 8 / NW;  // K operands, pairs of V^T tiles
  const ChunkArgs& a;
  int n_tok, tok, tok_min, tok_tile;  // the lane's row's token, the wave's and the tile's first
  int l, n, hh, half, op0, page, pair0;
  const uint16_t *kb, *vb;
  cd_u4_t k[KO];
  uint32_t v[PV][8];
  uint32_t found = 0;
  path_t path = 0;

  // start, count: the rows in k_new and v_new
  __device__ __forceinline__ OwnSource(const ChunkArgs& args, int h, int start, int count, int row0, int w, int row_tok, int least)
      : a(args), n_tok(count), tok(row_tok), tok_min(least), tok_tile(quotient(row0, args.gq)), l(threadIdx.x & 63), n(l & 31), hh(l >> 5), half(w / (NW / 2)),
        op0(KO * (w % (NW / 2))), page(w / (NW / 4)), pair0(PV * (w % (NW / 4))),
        kb(args.k_new + start * args.k_stride + (size_t)h * kHeadDim + 8 * hh + 16 * op0),
        vb(args.v_new + start * args.v_stride + (size_t)h * kHeadDim + 2 * n + 64 * pair0) {}
  __device__ __forceinline__ void fetch(int u) {
    const uint16_t* row = kb + min(kUnit * u + 32 * half + (n & 16) + row_token(n & 15), n_tok - 1) * a.k_stride;
#pragma unroll
    for (int i = 0; i < KO; ++i) k[i] = *reinterpret_cast<const cd_u4_t*>(row + 16 * i);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint16_t* p = vb + min(kUnit * u + kBlock * page + 8 * hh + j, n_tok - 1) * a.v_stride;
#pragma unroll
      for (int x = 0; x < PV; ++x) v[x][j] = *reinterpret_cast<const uint32_t*>(p + 64 * x);
    }
  }
  template <bool ODD>
  __device__ __forceinline__ void build(int u, ChunkLds& lds, int kbuf, int vbuf) {
    cd_h8_t(*ko)[64] = lds.k[kbuf];
    cd_h8_t(*vo)[64] = lds.v[vbuf];
#pragma unroll
    for (int i = 0; i < KO; ++i) ko[8 * half + op0 + i][l] = __builtin_bit_cast(cd_h8_t, k[i]);
    const bool part = ODD || partial(u);
#pragma unroll
    for (int x = 0; x < PV; ++x) {
      uint32_t y[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) y[j] = v[x][j];
      if (part) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          y[j] = kUnit * u + kBlock * page + 8 * hh + j < n_tok ? y[j] : 0u;
          const uint32_t odd = BfOps::odd(y[j]);
          found |= odd;
          y[j] &= ODD ? odd : ~odd;
        }
      }
      cd_u4_t e, o;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        e[j] = __builtin_amdgcn_perm(y[2 * j + 1], y[2 * j], 0x05040100u);
        o[j] = __builtin_amdgcn_perm(y[2 * j + 1], y[2 * j], 0x07060302u);
      }
      vo[4 * page + 2 * (pair0 + x)][l] = __builtin_bit_cast(cd_h8_t, e);
      vo[4 * page + 2 * (pair0 + x) + 1][l] = __builtin_bit_cast(cd_h8_t, o);
    }
  }
  __device__ __forceinline__ void refetch(int u) { fetch(u); }
  __device__ __forceinline__ bool partial(int u) const { return TREE || kUnit * u + kUnit - 1 > tok_tile; }
  __device__ __forceinline__ bool masked(int u) const { return TREE || kUnit * u + kUnit - 1 > tok_min; }
  __device__ __forceinline__ bool sees(int u, int t) const {  // (the lane half's 8 never crosses a word)
    if constexpr (TREE) return (path_word(path, 2 * u + (t >> 5)) >> ((t + 8 * hh) & 31)) & 1;
    return kUnit * u + t + 8 * hh <= tok;
  }
  __device__ __forceinline__ bool sees_token(int u, int t) const {
    if constexpr (TREE) return (path_word(path, 2 * u + (t >> 5)) >> (t & 31)) & 1;
    return kUnit * u + t <= tok;
  }
};

// R_K's elements that a thread brings into LDS: eight channels 8 oct .. of a column at a time
template <int NW>
struct KeyRotation {
  static constexpr int N = 2048 / (64 * NW);
  float r[N][8];
  __device__ __forceinline__ void load(const float* R) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = threadIdx.x + 64 * NW * i, oct = e >> 7, c = e & 127;
#pragma unroll
      for (int j = 0; j < 8; ++j) r[i][j] = R[(size_t)(8 * oct + j) * kHeadDim + c];
    }
  }
};
// q' = q R_K of the lane's row as fp16 operands with log2(e) / sqrt(128) folded in (what a small q' loses among fp16's
// subnormals, 2^-25 an element, is nothing in a score). q is exact in fp16, R_K's elements are rounded to it: 2^-12 of each,
// as the result's own rounding.
template <int NW>
__device__ __forceinline__ void rotate_query(const KeyRotation<NW>& R, ChunkLds& lds, const cd_b8_t (&x)[8], cd_h8_t (&Q)[8]) {
  cd_h8_t* rk = reinterpret_cast<cd_h8_t*>(&lds);  // [tile][operand][lane]
#pragma unroll
  for (int i = 0; i < KeyRotation<NW>::N; ++i) {
    const int e = threadIdx.x + 64 * NW * i, oct = e >> 7, c = e & 127;
    const int m16 = c & 15, p = c >> 4, wd = m16 >> 1;
    const int pos = (2 * (2 * (wd & 3) + (p >> 2)) + (wd >> 2)) * 8 + 2 * (p & 3) + (m16 & 1);
    // row_position is its own inverse
    rk[((pos >> 5) * 8 + (oct >> 1)) * 64 + (oct & 1) * 32 + row_position(pos & 31)] = pack_half8(R.r[i]);
  }
  __syncthreads();
  const int l = threadIdx.x & 63;
  cd_h8_t q[8];
#pragma unroll
  for (int kk = 0; kk < 8; ++kk) q[kk] = half_of(x[kk]);
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    cd_f16_t d = splat16(0.0f);
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) d = __builtin_amdgcn_mfma_f32_32x32x16_f16(rk[(8 * t + kk) * 64 + l], q[kk], d, 0, 0, 0);
    d *= kLogit2;
#pragma unroll
    for (int u = 0; u < 2; ++u) Q[2 * t + u] = pack_half8(reinterpret_cast<const float*>(&d) + 8 * u);
  }
  __syncthreads();
}

// O^T <- R_V O^T, each row within fp16's range by a power of two (row_scale). R_V goes through LDS as A
// operands: tile 2 e + o, row m is output channel 64 e + 2 m + o; operand (i, half) takes the channels 32 i + 16 half +
// {4 hh .. + 3, 8 + 4 hh .. + 3} that a lane half holds of tile i. Chunk m of operand op lies at m ^ op (its low bits), so
// that a row's pieces, which differ in operand, spread over the banks.
template <int NW>
__device__ __forceinline__ void unrotate(const float* R, ChunkLds& lds, RowState& st) {
  typedef _Float16 h4 __attribute__((ext_vector_type(4)));
  h4* rv = reinterpret_cast<h4*>(&lds);
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 4096 / (64 * NW); ++i) {
    const int e = threadIdx.x + 64 * NW * i, c = e >> 5, x = e & 31, op = x >> 2;
    const float4 r = *reinterpret_cast<const float4*>(R + (size_t)c * kHeadDim + 4 * x);
    const int t = 2 * (c >> 6) + (c & 1), m = (c & 63) >> 1;
    rv[2 * ((t * 8 + op) * 64 + (x & 1) * 32 + (m ^ op)) + ((x >> 1) & 1)] = h4{(_Float16)r.x, (_Float16)r.y, (_Float16)r.z, (_Float16)r.w};
  }
  __syncthreads();
  const int l = threadIdx.x & 63;
  const RowScale scale = row_scale(row_top(st.O));
  cd_h8_t B[8];
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    const cd_f16_t o = st.O[t] * scale.down;
#pragma unroll
    for (int u = 0; u < 2; ++u) B[2 * t + u] = pack_half8(reinterpret_cast<const float*>(&o) + 8 * u);
  }
#pragma unroll
  for (int t = 0; t < 4; ++t) {
    cd_f16_t d = splat16(0.0f);
#pragma unroll
    for (int op = 0; op < 8; ++op)
      d = __builtin_amdgcn_mfma_f32_32x32x16_f16(reinterpret_cast<cd_h8_t*>(rv)[(t * 8 + op) * 64 + (l ^ op)], B[op], d, 0, 0, 0);
    st.O[t] = d * scale.up;
  }
  __syncthreads();
}

}  // namespace

// Work-group: a piece of a tile of 32 NW rows of one KV head; wave w has rows 32 w .. of it.
template <int NG, int NW, bool TREE>
__global__ __launch_bounds__(64 * NW, 2) void chunk_attn_kernel(ChunkArgs a) {
  __shared__ ChunkLds lds;
  const int H = a.cv.num_kv_heads;
  const int at = quotient((int)blockIdx.x, H), h = (int)blockIdx.x - at * H;
  KeyRotation<NW> R;
  if (a.max_ctx > 0) R.load(a.R_k + (size_t)h * kHeadDim * kHeadDim);  // on its way while the work-group finds its piece
  const Place place = locate<TREE>(a, at, h);
  if (!place.valid) return;
  const Seq seq = place.s;
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = l & 31, hh = l >> 5;
  const int rows = seq.n * a.gq, row_w = place.row0 + 32 * w, tok_w = quotient(min(row_w, rows - 1), a.gq);
  const int nI = int2_units(a, seq, quotient(min(place.row0 + a.bm, rows) - 1, a.gq));
  const int row = row_w + n, rc = min(row, rows - 1), tok = quotient(rc, a.gq);
  // Four waves: one without rows only brings its share of the operands (64 chunks of 2 to 44 tokens over up to 4,000: 144 us,
  // 153 without). Eight: always taken for one with rows, since the second loop costs long chunks 1.5 %.
  const bool live = NW == 8 || row_w < rows;
  RowState st;
  st.m = 0.0f, st.sum = 0.0f, st.thr = kNone;
#pragma unroll
  for (int i = 0; i < 4; ++i) st.O[i] = splat16(0.0f);

  // the row's query: channels 16 kk + 8 hh .. of operand kk (read again for the chunk's own units: the registers are worth more)
  const uint16_t* q = a.q + (seq.start + tok) * a.q_stride + (size_t)(h * a.gq + rc - tok * a.gq) * kHeadDim + 8 * hh;
  auto query = [&](cd_b8_t (&x)[8]) {
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) x[kk] = *reinterpret_cast<const cd_b8_t*>(q + 16 * kk);
  };
  const int i1 = min(place.u1, nI);
  if (place.u0 < i1) {
    cd_b8_t x[8];
    cd_h8_t Q[8];
    query(x);
    auto limit = [&](int t) { return limit_of(a, seq, t); };
    Int2Source<NG, NW> src(a, h, place.b, seq.ctx, w, limit(tok), limit(tok_w), limit(quotient(place.row0, a.gq)));
    src.fetch(place.u0);
    rotate_query<NW>(R, lds, x, Q);
    // (the narrow work-group has no registers to spare)
    attend<typename std::conditional<NW == 8, BasedOps, HalfOps>::type>(src, st, lds, Q, 0.0f, place.u0, i1, live);
    unrotate<NW>(a.R_v + (size_t)h * kHeadDim * kHeadDim, lds, st);
  }

  const int c0 = max(place.u0 - nI, 0), c1 = place.u1 - nI;
  Tree tree{0, 0};
  bool absent = false;  // a row of a token without a path sees nothing
  if constexpr (TREE) {
    tree = tree_of(a, place.b);
    absent = seq.past + tok < 0 || seq.past + tok >= min(tree.count, a.max_tree);
  }
  if (c0 < c1) {
    cd_b8_t Q[8];
    query(Q);
    OwnSource<NW, TREE> src(a, h, TREE ? tree.start : seq.start, TREE ? min(tree.count, a.max_tree) : seq.n, place.row0, w, tok, tok_w);
    src.fetch(c0);
    if constexpr (TREE) {
      int32_t* parents = reinterpret_cast<int32_t*>(&lds);  // (behind unrotate's last barrier nothing is read there)
      if ((int)threadIdx.x < min(tree.count, a.max_tree)) parents[threadIdx.x] = a.parents[tree.start + threadIdx.x];
      __syncthreads();
      src.path = path_of(parents, seq.past + tok, min(tree.count, a.max_tree));
      absent = absent || !has_path(src.path);
      __syncthreads();
    }
    attend<BfOps>(src, st, lds, Q, query_mean(Q, a.mu + (size_t)h * kHeadDim, hh), c0, c1, live);
  }

  // ---- results: register 4 u + v of tile 2 e + o is channel 64 e + 16 u + 8 hh + 2 v + o
  const float all = pair_sum(st.sum);
  if (row >= rows) return;
  if (place.slot < 0) {
    const float inv = all == 0.0f ? 0.0f : 1.0f / all;
    uint16_t* o = a.out + ((size_t)(seq.start + tok) * a.Hq + h * a.gq + row - tok * a.gq) * kHeadDim + 8 * hh;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        uint32_t y[4];
#pragma unroll
        for (int v = 0; v < 4; ++v) {
          y[v] = pack_bf16(st.O[2 * x][4 * q + v] * inv, st.O[2 * x + 1][4 * q + v] * inv);
          if (TREE && absent) y[v] = 0;
        }
        *reinterpret_cast<uint4*>(o + 64 * x + 16 * q) = make_uint4(y[0], y[1], y[2], y[3]);
      }
  } else {
    // partial: bm rows of 128 sums, then their (m, l)
    float* part = a.part + ((size_t)place.slot * H + h) * a.bm * kChunkPartStride;
    const int rt = row - place.row0;
    float* o = part + (size_t)rt * kHeadDim + 8 * hh;
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        float4* d = reinterpret_cast<float4*>(o + 64 * x + 16 * q);
        const cd_f16_t &e = st.O[2 * x], &f = st.O[2 * x + 1];
        d[0] = make_float4(e[4 * q], f[4 * q], e[4 * q + 1], f[4 * q + 1]);
        d[1] = make_float4(e[4 * q + 2], f[4 * q + 2], e[4 * q + 3], f[4 * q + 3]);
      }
    if (hh == 0) reinterpret_cast<float2*>(part + (size_t)a.bm * kHeadDim)[rt] = make_float2(st.thr < 0.0f ? kNone : st.m, TREE && absent ? kAbsent : all);
  }
}

// Block (tile, KV head, 16 rows): thread (row, eight channels) joins the tile's pieces in order, in one pass with the running
// maximum. Bound by latency, so nothing waits for what it need not: the tile is read beside the number of tiles (its place
// exists whether or not it was cut), and four pieces at a time are on their way.
template <bool TREE>
__global__ __launch_bounds__(256) void chunk_merge_kernel(ChunkArgs a) {
  const int t = blockIdx.x, h = blockIdx.y, H = a.cv.num_kv_heads, T = a.head[1];
  const ChunkTile tile = a.tiles[t];
  if (t >= T || tile.pieces <= 1) return;
  const int rt = blockIdx.z * 16 + (threadIdx.x >> 4), c = 8 * (threadIdx.x & 15), row = tile.row0 + rt;
  if (row >= tile.n * a.gq) return;
  const size_t stride = (size_t)H * a.bm * kChunkPartStride, ml_at = (size_t)a.bm * kHeadDim;
  const float* part = a.part + ((size_t)tile.slot * H + h) * a.bm * kChunkPartStride;
  float o[8] = {}, all = 0.0f, top = kNone;
  bool absent = false;
  for (int p0 = 0; p0 < tile.pieces; p0 += 4) {
    float2 ml[4];
    float4 u[4], v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float* x = part + (size_t)min(p0 + i, tile.pieces - 1) * stride;
      ml[i] = reinterpret_cast<const float2*>(x + ml_at)[rt];
      const float4* d = reinterpret_cast<const float4*>(x + (size_t)rt * kHeadDim + c);
      u[i] = d[0], v[i] = d[1];
    }
    float next = top;
#pragma unroll
    for (int i = 0; i < 4; ++i) next = fmaxf(next, ml[i].x);
    const float old = __builtin_amdgcn_exp2f(top - next);
    top = next;
    all *= old;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] *= old;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (p0 + i >= tile.pieces) continue;
      if (TREE) absent |= ml[i].y == kAbsent;
      const float f = __builtin_amdgcn_exp2f(ml[i].x - top);
      all = __builtin_fmaf(ml[i].y, f, all);
      o[0] = __builtin_fmaf(u[i].x, f, o[0]), o[1] = __builtin_fmaf(u[i].y, f, o[1]);
      o[2] = __builtin_fmaf(u[i].z, f, o[2]), o[3] = __builtin_fmaf(u[i].w, f, o[3]);
      o[4] = __builtin_fmaf(v[i].x, f, o[4]), o[5] = __builtin_fmaf(v[i].y, f, o[5]);
      o[6] = __builtin_fmaf(v[i].z, f, o[6]), o[7] = __builtin_fmaf(v[i].w, f, o[7]);
    }
  }
  if (TREE && absent) {  // whatever the other pieces hold
    all = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j] = 0.0f;
  }
  const float inv = all == 0.0f ? 0.0f : 1.0f / all;
  const int tok = quotient(row, a.gq);
  uint16_t* out = a.out + ((size_t)(tile.start + tok) * a.Hq + h * a.gq + row - tok * a.gq) * kHeadDim + c;
  *reinterpret_cast<uint4*>(out) = make_uint4(pack_bf16(o[0] * inv, o[1] * inv), pack_bf16(o[2] * inv, o[3] * inv),
                                              pack_bf16(o[4] * inv, o[5] * inv), pack_bf16(o[6] * inv, o[7] * inv));
}

namespace {

// The plan with kernel `waves` (1: few rows)
ChunkPlan plan_with(int waves, int B, int H, long long seq_rows, long long rows, int max_own, int max_ctx) {
  ChunkPlan p{};
  p.waves = waves;
  p.bm = 32 * p.waves;
  p.resident = num_cus() * (p.waves == 8 ? 1 : 2);
  p.min_piece = p.waves == 1 ? 4 : 2;  // a unit for each wave of the kernel of few rows
  p.piece_units = p.waves == 1 ? 10.0f : 4.0f;
  p.merge_units = p.waves == 1 ? 0.016f : 0.00009f * p.bm;
  const long long per_seq = (seq_rows + p.bm - 1) / p.bm;
  long long tiles = B * per_seq, by_rows = rows / p.bm + B;
  tiles = tiles < by_rows ? tiles : by_rows;
  p.max_tiles = (int)(tiles < 1 ? 1 : tiles);
  // pieces a KV head where tiles are cut: a place on the chip each while the tiles have one, else up to three; never more than
  // the units allow
  const long long most = ((long long)max_ctx + 63) / 64 + ((long long)max_own + 63) / 64, cuts = (most + p.min_piece - 1) / p.min_piece;
  const long long places = (tiles * H <= p.resident ? 1LL : 3LL) * p.resident / H;
  long long cut = places < p.max_tiles * cuts ? places : p.max_tiles * cuts;
  p.max_slots = (int)(cut > 1 ? cut : 1);
  p.max_items = p.max_tiles > p.max_slots ? p.max_tiles : p.max_slots;
  auto up = [](size_t x) { return (x + 255) & ~size_t(255); };
  const size_t listed = B > kChunkWaveSeqs ? (size_t)B : 0;
  size_t off = 0;
  p.off_head = off, off = up(off + 4 * sizeof(int32_t));
  p.off_order = off, off = up(off + listed * sizeof(int32_t));
  p.off_items = off, off = up(off + listed * sizeof(int32_t));
  p.off_starts = off, off = up(off + listed * sizeof(int32_t));
  p.off_tiles = off, off = up(off + (size_t)p.max_tiles * sizeof(ChunkTile));
  p.off_part = off, off = up(off + (size_t)p.max_slots * H * p.bm * kChunkPartStride * sizeof(float));
  p.total = off;
  return p;
}

}  // namespace

ChunkPlan make_chunk_plan(int B, int Hq, int H, int total_q, int max_q, int max_own, int max_ctx) {
  const int gq = Hq / H;
  const long long seq_rows = (long long)max_q * gq, rows = (long long)total_q * gq;
  // The kernel of few rows makes the operands again for every 32 rows, which takes 1.5 of the four waves' time a row. It takes
  // what they would leave more than that empty: 24 sequences of 2 to 20 tokens (32 + 8 heads) over 512 to 16,384: 84 us, with
  // four waves 118; of 2 to 38 157 and 158; 100 of 1 to 40 over up to 2,000 196 and 178.
  // Four waves do the work of eight in 1.1 of the time, but on tiles of half the rows. They take what eight would leave more
  // than that empty: rows a sequence filled up to whole tiles, or half a tile more where the lengths differ. 16 chunks of 17
  // to 100 tokens (32 + 8 heads) over up to 8,000: 100 us, with eight waves 121; of 128 over 2,000: 110 and 97. And prompts with
  // nothing cached (no operands made twice) whose smaller tiles all have a place, since a causal tile's length varies and two
  // share a compute unit, the shortest beside the longest: 500 and 2,011 tokens 23 and 67 us, with eight waves 25 and 71;
  // 4,000, twice what the chip holds at once, 183 and 163.
  auto filled = [&](long long tile) { return rows == seq_rows * B ? (seq_rows + tile - 1) / tile * tile : rows / B + tile / 2; };
  const long long tiles4 = B * ((seq_rows + 127) / 128), rows4 = rows / 128 + B;
  const bool placed = (tiles4 < rows4 ? tiles4 : rows4) * H <= 2LL * num_cus();
  const int waves = seq_rows <= 64 || 3 * filled(32) < 2 * filled(128) ? 1 : seq_rows <= 128 || 11 * filled(128) < 10 * filled(256) || (max_ctx == 0 && placed) ? 4 : 8;
  ChunkPlan p = plan_with(waves, B, H, seq_rows, rows, max_own, max_ctx);
  // a workspace for these bounds is enough for every call within them, whichever kernel that takes
  for (int other : {1, 4, 8})
    if (other == 1 || seq_rows > 16 * other) {
      const size_t need = plan_with(other, B, H, seq_rows, rows, max_own, max_ctx).total;
      p.total = p.total < need ? need : p.total;
    }
  return p;
}

namespace {

template <int NG, int NW, bool TREE>
hipError_t launch_attn(const ChunkArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((chunk_attn_kernel<NG, NW, TREE>), dim3((unsigned)((long long)a.max_items * a.cv.num_kv_heads)), dim3(64 * NW), 0,
                     s, a);
  return hipGetLastError();
}

template <bool TREE>
hipError_t launch_pieces(const ChunkArgs& a, const ChunkPlan& p, hipStream_t s) {
  hipError_t e = hipSuccess;
  if (a.B > kChunkWaveSeqs) {
    hipLaunchKernelGGL(chunk_plan_kernel<TREE>, dim3(1), dim3(kPlanThreads), 0, s, a);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (p.waves == 1)
    e = launch_chunk_few(a, s);
  else if (a.cv.groups == 4)
    e = p.waves == 8 ? launch_attn<4, 8, TREE>(a, s) : launch_attn<4, 4, TREE>(a, s);
  else
    e = p.waves == 8 ? launch_attn<1, 8, TREE>(a, s) : launch_attn<1, 4, TREE>(a, s);
  if (e != hipSuccess) return e;
  if (p.max_slots > 1) {
    hipLaunchKernelGGL(chunk_merge_kernel<TREE>, dim3(p.max_tiles, a.cv.num_kv_heads, p.bm / 16), dim3(256), 0, s, a);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

hipError_t launch_chunk_attention(ChunkArgs a, const ChunkPlan& p, uint8_t* ws, hipStream_t s) {
  a.bm = p.bm;
  a.resident = p.resident;
  a.per_cu = p.waves == 8 ? 1 : 2;
  a.min_piece = p.min_piece;
  a.max_tiles = p.max_tiles;
  a.max_items = p.max_items;
  a.max_slots = p.max_slots;
  a.piece_units = p.piece_units;
  a.merge_units = p.merge_units;
  a.head = reinterpret_cast<int32_t*>(ws + p.off_head);
  a.order = reinterpret_cast<int32_t*>(ws + p.off_order);
  a.item_start = reinterpret_cast<int32_t*>(ws + p.off_items);
  a.tile_start = reinterpret_cast<int32_t*>(ws + p.off_starts);
  a.tiles = reinterpret_cast<ChunkTile*>(ws + p.off_tiles);
  a.part = reinterpret_cast<float*>(ws + p.off_part);
  return !a.parents ? launch_pieces<false>(a, p, s) : launch_pieces<true>(a, p, s);
}

}  // namespace int2kv
