// Attention of few new tokens per sequence (int2kv_chunk_attention): drafted tokens, short turns.
// Bound by the vector ALU that makes operands of the codes (540 instructions and 32 exponentials a wave and unit, 2,900
// cycles; busy 60 % of them all), at a third more than the time of the cache's bytes, so nothing is shared and nothing waited for: the four waves of
// a work-group hold the same 32 rows and take different 64-token units of the context, each with the next unit's records on
// their way to LDS (LDS-DMA) and its own softmax. Codes become matrix operands in the registers they are used from. At the
// end the four partial results meet in LDS, each wave un-rotates the 32 channels of its tile and adds the chunk's own bf16
// tokens to them. 24 sequences of 2 to 8 tokens over 512 to 16,384 cached ones (40 + 8 heads, 141 MB) take 78 us; five tokens
// over 1,011 take 12, most of it waits and the first touch of the code.
#include <type_traits>

#include "append_core.h"
#include "chunk_core.h"

namespace int2kv {

namespace {

constexpr int kFewWaves = 4;
constexpr int kStep = 32;                 // tokens of a step over the chunk's own
constexpr int kStages = 4;                // two units, two stages each
constexpr int kStageBytes = 2 * (1024 + 512);  // codes of two pages, then 512 bytes each of their parameters

struct FewLds {
  union {
    uint8_t stage[kFewWaves][kStages][kStageBytes];
    float o[kFewWaves][4][16][64];        // [wave][tile][register][lane]
  };
  cd_h8_t b[8][64];                       // the rotated queries, then the sums, as operands
  float ml[kFewWaves][3][32];             // the rows' m, sum and largest element
};

}  // namespace

template <int NG>
__global__ __launch_bounds__(64 * kFewWaves, 2) void chunk_few_kernel(ChunkArgs a) {
  using Lay = Rec<NG>;
  __shared__ __align__(16) FewLds lds;
  const int H = a.cv.num_kv_heads;
  const int at = quotient((int)blockIdx.x, H), h = (int)blockIdx.x - at * H;
  const int l = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = l & 31, hh = l >> 5;
  float rk[8][8];  // the wave's columns of R_K: rows 16 kk + 8 hh .. of column 32 w + n
  if (a.max_ctx > 0) {  // on their way while the work-group finds its piece
    const float* R = a.R_k + (size_t)h * kHeadDim * kHeadDim + (size_t)(8 * hh) * kHeadDim + 32 * w + n;
#pragma unroll
    for (int kk = 0; kk < 8; ++kk)
#pragma unroll
      for (int j = 0; j < 8; ++j) rk[kk][j] = R[(size_t)(16 * kk + j) * kHeadDim];
  }
  const Place place = locate(a, at, h);
  if (!place.valid) return;
  const Seq seq = place.s;
  const int rows = seq.n * a.gq, row = place.row0 + n, rc = min(row, rows - 1), tok = quotient(rc, a.gq), tok_tile = quotient(place.row0, a.gq);
  const int nI = int2_units(a, seq, quotient(min(place.row0 + a.bm, rows) - 1, a.gq));
  const int lim = limit_of(a, seq, tok), lim_tile = limit_of(a, seq, tok_tile);  // tokens the row sees, the least of the tile's

  // the row's query: channels 16 kk + 8 hh .. of operand kk (read again for the chunk's own tokens)
  const uint16_t* q = a.q + (seq.start + tok) * a.q_stride + (size_t)(h * a.gq + rc - tok * a.gq) * kHeadDim + 8 * hh;
  auto query = [&](cd_b8_t (&x)[8]) {
#pragma unroll
    for (int kk = 0; kk < 8; ++kk) x[kk] = *reinterpret_cast<const cd_b8_t*>(q + 16 * kk);
  };
  const bool cached = place.u0 < min(place.u1, nI);
  float m = 0.0f, sum = 0.0f, thr = kNone;
  // Behind the un-rotation row m = 8 u + 4 h + v of a wave's tile is channel 32 w + 16 (u / 2) + 8 h + 4 (u % 2) + v, so that a
  // lane's results are eight neighbours at a time; the operand's k order is the channel order the sums lie in
  const int ch = 32 * w + 16 * (n >> 4) + 8 * ((n >> 2) & 1) + 4 * ((n >> 3) & 1) + (n & 3);
  float4 rv[8][2];  // its row of R_V
  {
    cd_f16_t O[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) O[i] = splat16(0.0f);
    // ---- the wave's units: a quarter of the piece's
    const int pages = (seq.ctx + kBlock - 1) / kBlock;
    const int units = max(min(place.u1, nI) - place.u0, 0), s0 = place.u0 + units * w / kFewWaves, s1 = place.u0 + units * (w + 1) / kFewWaves;
    const int32_t* table = a.table + (size_t)place.b * a.max_blocks;
    // lane l: the block of page 4 list0 + l, read for 16 units at a time
    int list0 = 0, list = 0;
    auto load_list = [&](int s) {
      list0 = s;
      const int p = kUnitPages * s + l;
      list = p < pages ? table[p] : -1;
      // taken here, so that the wait for it stands here and not, for all loads on their way, before its uses in the loop
      asm volatile("" : "+v"(list));
    };
    auto good = [&](int id) { return id >= 0 && id < a.cv.num_blocks; };
    auto block = [&](int s, int x) { return __builtin_amdgcn_readlane(list, kUnitPages * (s - list0) + x); };
    const uint32_t stage0 = (uint32_t)(uintptr_t)(&lds.stage[w][0][0]);
    // the records of a unit on their way to its two stages, two pages each
    auto issue = [&](int s) {
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const uint8_t* r[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          const int id = block(s, 2 * half + x);
          r[x] = a.cv.pool + ((size_t)(uint32_t)(good(id) ? id : 0) * H + h) * Lay::kBytes;
        }
        const uint32_t to = stage0 + (uint32_t)(2 * (s & 1) + half) * kStageBytes;
        ap_dma16(r[0] + 16 * l, to);
        ap_dma16(r[1] + 16 * l, to + 1024);
        // a page's 128 NG bytes of parameters; lanes past them read the last 16 again
        ap_dma16((l < 32 ? r[0] : r[1]) + 1024 + min(16 * (l & 31), 128 * NG - 16), to + 2048);
      }
    };
    if (s0 < s1) {
      load_list(s0);
      issue(s0);
      if (s0 + 1 < s1) issue(s0 + 1);
    }
    if (cached) {
      // q R_K with log2(e) / sqrt(128): wave w forms the 32 channels 32 w .. of q' (q is exact in fp16, R_K's elements are
      // rounded to it, 2^-12 of each) and puts them where the products take them
      cd_b8_t Qb[8];
      query(Qb);
      cd_f16_t d = splat16(0.0f);
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) d = HalfOps::mfma(pack_half8(rk[kk]), half_of(Qb[kk]), d);
      // register r: channel 32 w + c, c = 8 (r / 4) + 4 hh + r % 4; channels 16 p + 2 x, + 1 are elements 2 (p % 4), + 1 of
      // operand 2 (x % 4) + p / 4 in lane half x / 4
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        const int p = 2 * w + (r >> 3), x = 4 * ((r >> 2) & 1) + 2 * hh + ((r & 3) >> 1);
        const cd_h2_t y = {(_Float16)(d[r] * kLogit2), (_Float16)(d[r + 1] * kLogit2)};
        reinterpret_cast<uint32_t*>(&lds.b[2 * (x & 3) + (p >> 2)][32 * (x >> 2) + n])[p & 3] = __builtin_bit_cast(uint32_t, y);
      }
      __syncthreads();
    }
    if (s0 < s1) {
      cd_h8_t Q[8];
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) Q[kk] = lds.b[kk][l];
      const int tA = row_token(n & 15), pgA = n >> 4;  // the token (of a half) whose keys this lane's A rows are
      float base = kBias;
      uint32_t found = 0;
      auto whole = [&](int s) {
        return good(block(s, 0)) && good(block(s, 1)) && good(block(s, 2)) && good(block(s, 3)) && kUnit * (s + 1) <= lim_tile;
      };
      // One unit: scores, probabilities, values. PART: some row does not see all of it. SECOND: only the values that are not
      // finite, for the rows that see them
      auto take = [&](int s, auto part_c, auto second_c) {
        constexpr bool part = decltype(part_c)::value, second = decltype(second_c)::value;
        const uint8_t* st = lds.stage[w][2 * (s & 1)];
        uint32_t ok = 15u;
        if constexpr (part) {
#pragma unroll
          for (int x = 0; x < 4; ++x) ok &= good(block(s, x)) ? 15u : ~(1u << x);
        }
        cd_f16_t S[2];
#pragma unroll
        for (int tm = 0; tm < 2; ++tm) {
          const uint8_t* half = st + tm * kStageBytes;
          const cd_u4_t kc = *reinterpret_cast<const cd_u4_t*>(half + 1024 * pgA + 32 * tA + 16 * hh);
          uint32_t km[NG];
#pragma unroll
          for (int g = 0; g < NG; ++g) km[g] = *reinterpret_cast<const uint32_t*>(half + 2048 + 512 * pgA + 4 * NG * tA + 4 * g);
          cd_h2_t ks[NG], kz[NG];
#pragma unroll
          for (int g = 0; g < NG; ++g) ks[g] = both_lo(km[g]), kz[g] = both_hi(km[g]);
          S[tm] = splat16(0.0f);
#pragma unroll
          for (int x = 0; x < 4; ++x) {
            cd_h8_t k[2];
            word_operands<NG>(kc[x], ks, kz, k);
            S[tm] = HalfOps::mfma(k[0], Q[2 * x], S[tm]);
            S[tm] = HalfOps::mfma(k[1], Q[2 * x + 1], S[tm]);
          }
          if constexpr (part) {
#pragma unroll
            for (int i = 0; i < 16; ++i)
              S[tm][i] = ((ok >> (2 * tm + (i >> 3))) & 1) && kUnit * s + 32 * tm + reg_token(i) + 8 * hh < lim ? S[tm][i] : -INFINITY;
          }
        }
        cd_u4_t P[2][2];
        float none = 0.0f;
        if constexpr (!second) settle<HalfOps>(S, base, m, sum, thr, O);
#pragma unroll
        for (int tm = 0; tm < 2; ++tm) soften<HalfOps>(S[tm], base, second ? none : sum, P[tm]);
#pragma unroll
        for (int pg = 0; pg < 4; ++pg) {
          const uint8_t* half = st + (pg >> 1) * kStageBytes;
          const uint8_t* vm = half + 2048 + 512 * (pg & 1) + 16 * hh;
          const cd_u4_t vc = *reinterpret_cast<const cd_u4_t*>(half + 1024 * (pg & 1) + 512 + 32 * (n & 15) + 16 * hh);
          const cd_u4_t p = P[pg >> 1][pg & 1];
          uint32_t word[4];
#pragma unroll
          for (int x = 0; x < 4; ++x) word[x] = vc[x] >> (2 * (n >> 4));
          cd_u4_t s4 = *reinterpret_cast<const cd_u4_t*>(vm + 64 * NG), z4 = *reinterpret_cast<const cd_u4_t*>(vm + 96 * NG);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            if (NG == 4 && i > 0) {
              s4 = *reinterpret_cast<const cd_u4_t*>(vm + 64 * NG + 32 * i);
              z4 = *reinterpret_cast<const cd_u4_t*>(vm + 96 * NG + 32 * i);
            }
            cd_u4_t f;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const uint32_t sv = s4[x], zv = z4[x];  // (copies: a bit cast of a vector's element takes element 0)
              const cd_h2_t code = i == 0   ? land_codes<0>(word[x])
                                   : i == 1 ? land_codes<4>(word[x])
                                   : i == 2 ? land_codes<8>(word[x])
                                            : land_codes<4>(word[x] >> 8);
              f[x] = __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(code, __builtin_bit_cast(cd_h2_t, sv), __builtin_bit_cast(cd_h2_t, zv)));
            }
            if constexpr (part) {
              // tokens that do not exist are zero; values that are not finite are left for the second pass
              int cnt = seq.ctx - (kUnit * s + kBlock * pg);
              cnt = (ok >> pg) & 1 ? cnt : 0;
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                const int tb = 8 * hh + 2 * x;
                f[x] &= (tb < cnt ? 0xFFFFu : 0u) | (tb + 1 < cnt ? 0xFFFF0000u : 0u);
                const uint32_t odd = HalfOps::odd(f[x]);
                found |= odd;
                f[x] &= second ? odd : ~odd;
              }
            }
            if constexpr (!second) {
              O[i] = HalfOps::mfma(__builtin_bit_cast(cd_h8_t, f), __builtin_bit_cast(cd_h8_t, p), O[i]);
            } else {
              for (int t = 0; t < kBlock; ++t) {
                const bool see = ((ok >> pg) & 1) && kUnit * s + kBlock * pg + t < lim;
                const cd_f16_t d = HalfOps::mfma(__builtin_bit_cast(cd_h8_t, only_token(f, t)), __builtin_bit_cast(cd_h8_t, only_token(p, t)), splat16(0.0f));
#pragma unroll
                for (int y = 0; y < 16; ++y) O[i][y] += see ? d[y] : 0.0f;
              }
            }
          }
        }
      };
      // before a unit: it has landed when at most the next one's six loads are on their way; after it: its stages' last
      // readers are done, the unit after next may take them
      auto before = [&](int s) {
        if (s + 1 < s1)
          asm volatile("s_waitcnt vmcnt(6)" ::: "memory");
        else
          asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      };
      auto after = [&](int s) {
        if (s + 2 < s1) {
          if (s + 2 >= list0 + 16) load_list(s + 1);  // units still to be taken keep their place in it
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          issue(s + 2);
        }
      };
      std::true_type yes;
      std::false_type no;
      int s = s0;
      for (; s < s1 && whole(s); ++s) {
        before(s);
        take(s, no, no);
        after(s);
      }
      const int part0 = s;
      for (; s < s1; ++s) {  // the end of the context, or behind a page that does not exist
        before(s);
        take(s, yes, no);
        after(s);
      }
      if (__any(found != 0)) {
        for (s = part0; s < s1; ++s) {  // (the units before them took such values as they are)
          load_list(s);
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          issue(s);
          asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
          take(s, yes, yes);
        }
      }
    }
    if (cached) {
      const float* R = a.R_v + ((size_t)h * kHeadDim + ch) * kHeadDim + 4 * hh;
#pragma unroll
      for (int op = 0; op < 8; ++op) rv[op][0] = *reinterpret_cast<const float4*>(R + 16 * op), rv[op][1] = *reinterpret_cast<const float4*>(R + 16 * op + 8);
    }
    // ---- the waves' results meet
    const float largest = row_top(O);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int r = 0; r < 16; ++r) lds.o[w][i][r][l] = O[i][r];
    sum = pair_sum(sum);
    if (hh == 0) {
      lds.ml[w][0][n] = thr < 0.0f ? kNone : m;
      lds.ml[w][1][n] = sum;
      lds.ml[w][2][n] = largest;
    }
    __syncthreads();
  }
  float top = kNone, all = 0.0f, f[kFewWaves];
#pragma unroll
  for (int x = 0; x < kFewWaves; ++x) top = fmaxf(top, lds.ml[x][0][n]);
#pragma unroll
  for (int x = 0; x < kFewWaves; ++x) {
    f[x] = __builtin_amdgcn_exp2f(lds.ml[x][0][n] - top);
    all = __builtin_fmaf(f[x], lds.ml[x][1][n], all);
  }
  // wave w has the 32 channels of tile w from here on
  cd_f16_t O[1] = {splat16(0.0f)};
  if (cached) {
    float bound = 0.0f;  // of the joined row: every wave, having one tile of it, comes to the same scale
#pragma unroll
    for (int y = 0; y < kFewWaves; ++y) bound = __builtin_fmaf(f[y], lds.ml[y][2][n], bound);
    const RowScale scale = row_scale(bound);
#pragma unroll
    for (int y = 0; y < kFewWaves; ++y) f[y] *= scale.down;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float x = 0.0f;
#pragma unroll
      for (int y = 0; y < kFewWaves; ++y) x = __builtin_fmaf(f[y], lds.o[y][w][r][l], x);
      O[0][r] = x;
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      cd_h8_t b;
#pragma unroll
      for (int j = 0; j < 8; ++j) b[j] = (_Float16)O[0][8 * x + j];
      lds.b[2 * w + x][l] = b;
    }
    __syncthreads();
    cd_f16_t d = splat16(0.0f);
#pragma unroll
    for (int op = 0; op < 8; ++op) {
      const float4 u = rv[op][0], v = rv[op][1];
      const float x[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
      d = HalfOps::mfma(pack_half8(x), lds.b[op][l], d);
    }
    O[0] = d * scale.up;
  }
  m = top == kNone ? 0.0f : top;
  thr = top == kNone ? kNone : kMove;
  sum = hh == 0 ? all : 0.0f;  // pair_sum adds the halves again

  // ---- the chunk's own tokens: every wave has all scores and its tile's values
  const int c0 = max(place.u0 - nI, 0), c1 = place.u1 - nI;
  if (c0 < c1) {
    cd_b8_t Qb[8];
    query(Qb);
    float base = kBias - m - query_mean(Qb, a.mu + (size_t)h * kHeadDim, hh);
    const uint16_t* kb = a.k_new + seq.start * a.k_stride + (size_t)h * kHeadDim + 8 * hh;
    const uint16_t* vb = a.v_new + seq.start * a.v_stride + (size_t)h * kHeadDim + ch;
    const int last = quotient(min(place.row0 + a.bm, rows) - 1, a.gq);  // the tile's last token
    for (int s = c0 * (kUnit / kStep); s < c1 * (kUnit / kStep) && kStep * s <= last; ++s) {
      const uint16_t* kr = kb + min(kStep * s + (n & 16) + row_token(n & 15), seq.n - 1) * a.k_stride;
      cd_h8_t k[8];
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) k[kk] = *reinterpret_cast<const cd_h8_t*>(kr + 16 * kk);
      uint32_t v[2][8];
#pragma unroll
      for (int pg = 0; pg < 2; ++pg)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[pg][j] = vb[min(kStep * s + kBlock * pg + 8 * hh + j, seq.n - 1) * a.v_stride];
      cd_f16_t S[1] = {splat16(0.0f)};
#pragma unroll
      for (int kk = 0; kk < 8; ++kk) S[0] = BfOps::mfma(k[kk], Qb[kk], S[0]);
#pragma unroll
      for (int i = 0; i < 16; ++i) S[0][i] = kStep * s + reg_token(i) + 8 * hh <= tok ? S[0][i] : -INFINITY;
      settle<BfOps>(S, base, m, sum, thr, O);
      cd_u4_t P[2];
      soften<BfOps>(S[0], base, sum, P);
      uint32_t found = 0;
      cd_u4_t y[2], z[2];  // values, and those that are not finite
#pragma unroll
      for (int pg = 0; pg < 2; ++pg)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const int t = kStep * s + kBlock * pg + 8 * hh + 2 * x;
          const uint32_t pair = (t < seq.n ? v[pg][2 * x] : 0u) | (t + 1 < seq.n ? v[pg][2 * x + 1] << 16 : 0u), odd = BfOps::odd(pair);
          found |= odd;
          y[pg][x] = pair & ~odd;
          z[pg][x] = pair & odd;
        }
#pragma unroll
      for (int pg = 0; pg < 2; ++pg) O[0] = BfOps::mfma(__builtin_bit_cast(cd_h8_t, y[pg]), __builtin_bit_cast(cd_b8_t, P[pg]), O[0]);
      if (__any(found != 0)) {
        for (int t = 0; t < kStep; ++t) {
          const bool see = kStep * s + t <= tok;
          const cd_u4_t p = only_token(t < 16 ? P[0] : P[1], t), x = only_token(t < 16 ? z[0] : z[1], t);
          const cd_f16_t d = BfOps::mfma(__builtin_bit_cast(cd_h8_t, x), __builtin_bit_cast(cd_b8_t, p), splat16(0.0f));
#pragma unroll
          for (int i = 0; i < 16; ++i) O[0][i] += see ? d[i] : 0.0f;
        }
      }
    }
  }

  // ---- results: registers 8 x .. 8 x + 7 are channels 32 w + 16 x + 8 hh ..
  all = pair_sum(sum);
  if (row >= rows) return;
  if (place.slot < 0) {
    const float inv = all == 0.0f ? 0.0f : 1.0f / all;
    uint16_t* o = a.out + ((size_t)(seq.start + tok) * a.Hq + h * a.gq + row - tok * a.gq) * kHeadDim + 32 * w + 8 * hh;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      uint32_t y[4];
#pragma unroll
      for (int v = 0; v < 4; ++v) y[v] = pack_bf16(O[0][8 * x + 2 * v] * inv, O[0][8 * x + 2 * v + 1] * inv);
      *reinterpret_cast<uint4*>(o + 16 * x) = make_uint4(y[0], y[1], y[2], y[3]);
    }
  } else {
    float* part = a.part + ((size_t)place.slot * H + h) * a.bm * kChunkPartStride;
    float* o = part + (size_t)n * kHeadDim + 32 * w + 8 * hh;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      float4* d = reinterpret_cast<float4*>(o + 16 * x);
      d[0] = make_float4(O[0][8 * x], O[0][8 * x + 1], O[0][8 * x + 2], O[0][8 * x + 3]);
      d[1] = make_float4(O[0][8 * x + 4], O[0][8 * x + 5], O[0][8 * x + 6], O[0][8 * x + 7]);
    }
    if (w == 0 && hh == 0) reinterpret_cast<float2*>(part + (size_t)a.bm * kHeadDim)[n] = make_float2(thr < 0.0f ? kNone : m, all);
  }
}

hipError_t launch_chunk_few(const ChunkArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)((long long)a.max_items * a.cv.num_kv_heads));
  if (a.cv.groups == 4)
    hipLaunchKernelGGL((chunk_few_kernel<4>), grid, dim3(64 * kFewWaves), 0, s, a);
  else
    hipLaunchKernelGGL((chunk_few_kernel<1>), grid, dim3(64 * kFewWaves), 0, s, a);
  return hipGetLastError();
}

}  // namespace int2kv
