// The tokens of a cache that stay, and their rows' move (int2kv_select_tokens, int2kv_move_tokens).
#include "chunk_core.h"

namespace int2kv {

namespace {

constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;

// A weight as an integer of the same order: zeros of both signs are equal, NaN lies below everything
__device__ __forceinline__ uint32_t order_of(float w) {
  if (w != w) return 0u;
  const uint32_t u = w == 0.0f ? 0u : __float_as_uint(w);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

}  // namespace

namespace {

// Sum of the waves' numbers before this wave, and of all
__device__ __forceinline__ int2 across(const int* waves) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int x = lane < kSelectWaves ? waves[lane] : 0, upto = wave_scan(x);
  return make_int2(__builtin_amdgcn_readlane(upto - x, wave), __builtin_amdgcn_readlane(upto, 63));
}

}  // namespace

// Block: one (sequence, KV head). Thread i has tokens 4 i .. of every 4,096, counted from the 16-byte boundary at or before the
// list; up to 4,096 J tokens are read once and kept in registers, longer lists a span of so many at a time, again in every
// pass. The threshold, the need-th largest key, comes in three passes from histograms of 11, 11 and 10 bits of the keys that
// share the bits so far; then the kept tokens' places are their ranks. Bound by instruction issue: a list of 31,597 tokens takes
// 18 us (keys 1.7, histograms 4.1 and twice 2.0, counts 2.2, places 4.8), 512 lists of up to 32,768 38 us.
template <int J>
__global__ __launch_bounds__(kSelectThreads) void select_tokens_kernel(SelectArgs a) {
  constexpr int kBins = 2048, kStep = 4 * kSelectThreads, kSpan = J * kStep;
  static_assert(J * kSelectWaves <= 128, "two counts a lane");
  __shared__ int bins[kBins], waves[kSelectWaves], found[2], counts[128];
  const int b = blockIdx.x / a.H, h = blockIdx.x - b * a.H, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = min(max(a.lens[b], 0), a.max_ctx), keep = min(len, a.budget);
  const float* w = a.weights + ((size_t)b * a.H + h) * a.stride;
  int32_t* kept = a.kept + ((size_t)b * a.H + h) * a.kept_stride;
  if (h == 0 && tid == 0) a.kept_lens[b] = keep;
  if (len <= a.budget) {
    for (int i = tid; i < len; i += kSelectThreads) kept[i] = i;
    return;
  }
  const int lo = min(a.sink, len), hi = max(lo, len - a.recent);  // lo .. hi - 1 compete for the places that are left
  int need = keep - lo - (len - hi);
  // from the boundary on, a thread's four tokens are one load where all four are the list's
  const int lead = (int)((reinterpret_cast<uintptr_t>(w) >> 2) & 3), end = len + lead;
  uint32_t keys[J][4];
  auto token = [&](int s0, int j) { return s0 + j * kStep + 4 * tid - lead; };  // the first of the thread's
  auto read = [&](int s0) {
    float4 v[J];
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int i = token(s0, j);
      v[j] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      if (i >= 0 && i + 4 <= len)
        v[j] = *reinterpret_cast<const float4*>(w + i);
      else if (i + 4 > 0 && i < len)
        v[j] = make_float4(w[max(i, 0)], w[min(max(i + 1, 0), len - 1)], w[min(max(i + 2, 0), len - 1)], w[min(i + 3, len - 1)]);
    }
#pragma unroll
    for (int j = 0; j < J; ++j)
      keys[j][0] = order_of(v[j].x), keys[j][1] = order_of(v[j].y), keys[j][2] = order_of(v[j].z), keys[j][3] = order_of(v[j].w);
  };
  const bool once = end <= kSpan;
  if (once) read(0);
  for (int i = tid; i < kBins; i += kSelectThreads) bins[i] = 0;
  uint32_t prefix = 0;
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, above_shift = pass == 0 ? 0 : pass == 1 ? 21 : 10;
    const uint32_t mask = pass == 2 ? 1023u : 2047u;
    __syncthreads();
    for (int s0 = 0; s0 < end; s0 += kSpan) {
      if (!once) read(s0);
#pragma unroll
      for (int j = 0; j < J; ++j) {
        if (s0 + j * kStep >= end) break;
        const int i = token(s0, j);
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (i + k >= lo && i + k < hi && (pass == 0 || keys[j][k] >> above_shift == prefix >> above_shift))
            atomicAdd(&bins[(keys[j][k] >> shift) & mask], 1);
      }
    }
    __syncthreads();
    // the bin of the need-th largest: thread t has bins 2047 - 2 t and the next lower one
    const int x = kBins - 1 - 2 * tid, c1 = bins[x], c0 = bins[x - 1];
    bins[x] = bins[x - 1] = 0;
    int upto = wave_scan(c0 + c1);
    if (lane == 63) waves[wave] = upto;
    __syncthreads();
    upto += across(waves).x;
    const int above = upto - c0 - c1;
    if (above < need && need <= upto) {
      const bool upper = need <= above + c1;
      found[0] = upper ? x : x - 1, found[1] = upper ? above : above + c1;
    }
    if (need == 0 && tid == 0) found[0] = mask, found[1] = 0;  // none of them: no key lies above all ones
    __syncthreads();
    prefix |= (uint32_t)found[0] << shift;
    need -= found[1];
  }
  // the keys above `prefix` and the first `need` equal to it, in order. Counts of both are held in one word, above in its lower
  // half (a span has at most 2^15)
  static_assert(kSpan <= 1 << 15, "two counts in a word");
  int above0 = 0, equal0 = 0;  // in the spans before
  for (int s0 = 0; s0 < end; s0 += kSpan) {
    if (!once) read(s0);
    auto flag = [&](int i, uint32_t key) {
      const bool forced = i < lo || i >= hi;
      return i < 0 || i >= len ? 0 : forced || key > prefix ? 1 : key == prefix ? 1 << 16 : 0;
    };
    int before[J];  // of the wave's, in the same step
#pragma unroll
    for (int j = 0; j < J; ++j) {
      const int i = token(s0, j);
      int n = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k) n += flag(i + k, keys[j][k]);
      const int upto = wave_scan(n);
      before[j] = upto - n;
      if (lane == 63) counts[j * kSelectWaves + wave] = upto;
    }
    __syncthreads();
    const int2 two = lane < J * kSelectWaves / 2 ? reinterpret_cast<const int2*>(counts)[lane] : make_int2(0, 0);
    const int upto = wave_scan(two.x + two.y), first = upto - two.x - two.y, second = upto - two.y;
#pragma unroll
    for (int j = 0; j < J; ++j) {
      if (s0 + j * kStep >= end) break;
      const int i = token(s0, j), at = j * kSelectWaves + wave;
      const int past = before[j] + (at & 1 ? __builtin_amdgcn_readlane(second, at >> 1) : __builtin_amdgcn_readlane(first, at >> 1));
      // kept before a token: those above, and of the equal ones as many as there is need for
      int na = above0 + (past & 0xFFFF), ne = equal0 + (int)((uint32_t)past >> 16);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int f = flag(i + k, keys[j][k]);
        if (f == 1 || (f && ne < need)) kept[na + min(ne, need)] = i + k;
        na += f & 1, ne += f >> 16;
      }
    }
    const int all = __builtin_amdgcn_readlane(upto, 63);
    above0 += all & 0xFFFF, equal0 += (int)((uint32_t)all >> 16);
    __syncthreads();
  }
}

hipError_t launch_select_tokens(const SelectArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)(a.B * a.H)), block(kSelectThreads);
  // few keys a thread leave room for two blocks a compute unit: 512 lists of 8,000 tokens 12.8 us, with room for 32 keys 26
  if (a.max_ctx + 3 <= 8 * kSelectThreads)
    hipLaunchKernelGGL(select_tokens_kernel<2>, grid, block, 0, s, a);
  else
    hipLaunchKernelGGL(select_tokens_kernel<8>, grid, block, 0, s, a);
  return hipGetLastError();
}

namespace {

constexpr int kMoveWaves = 4;
constexpr int kStagedWeights = 4 * kBlock;

}  // namespace

// Wave: one page of one KV head of the result. A token's row is 32 bytes of key codes and its parameters, which lie together,
// and two bytes of each of the page's value rows. STAGE 0: from the cache into the result's blocks; 1: from the cache into
// the workspace; 2: from there into the cache. Bound by the pages it touches, whole ones, as a token's values lie in all of a page's
// lines: 4,096 of up to 32,768 tokens, 64 sequences, 8 heads: 1.0 GB in 192 us, 5.2 TB/s.
template <int NG, int STAGE>
__global__ __launch_bounds__(64 * kMoveWaves) void move_tokens_kernel(MoveArgs a) {
  using Lay = Rec<NG>;
  const int H = a.cv.num_kv_heads, l = threadIdx.x & 63;
  const long long item = (long long)blockIdx.x * kMoveWaves + (threadIdx.x >> 6);
  if (item >= (long long)a.B * a.pages * H) return;
  const int h = (int)(item % H), page = (int)(item / H % a.pages), b = (int)(item / H / a.pages);
  const int count = min(min(max(a.kept_lens[b], 0), a.max_kept) - kBlock * page, kBlock);
  if (count <= 0) return;
  const int to = a.out_table[(size_t)b * a.out_max_blocks + page];
  if (to < 0 || to >= a.cv.num_blocks) return;
  // lane t < 16: token t's old place
  const int t = l & 15, token = t < count ? a.kept[((size_t)b * H + h) * a.kept_stride + kBlock * page + t] : -1;
  const bool in_table = token >= 0 && token < (long long)a.max_blocks * kBlock;
  const int block = in_table ? a.table[(size_t)b * a.max_blocks + token / kBlock] : -1;
  const bool good = block >= 0 && block < a.cv.num_blocks;
  const uint32_t mask = (uint32_t)__ballot(good) & 0xFFFFu;  // rows to write
  uint8_t* stage = a.stage + (size_t)item * (Lay::kBytes + kStagedWeights);
  // record and row of token x of the page
  const int record = good ? block : 0, row = STAGE == 2 ? t : token & 15;
  auto from = [&](int x) -> const uint8_t* {
    const int r = __shfl(record, x);
    return STAGE == 2 ? stage : a.cv.pool + ((size_t)r * H + h) * Lay::kBytes;
  };
  uint8_t* dst = STAGE == 1 ? stage : a.cv.pool + ((size_t)to * H + h) * Lay::kBytes;
  // lane 2 t + half: half a row of key codes; lane t: a row of key parameters; lane: tokens 4 (l / 16) .. of value half l % 16;
  // tokens 2 (l / ng2) .. of value parameter row l % ng2
  constexpr int kRows = 2 * NG;
  const int tk = (l >> 1) & 15, rk = __shfl(row, tk);
  const uint8_t* src_k = from(tk);
  uint4 kc = make_uint4(0, 0, 0, 0);
  if (l < 32) kc = *reinterpret_cast<const uint4*>(src_k + 32 * rk + 16 * (l & 1));
  const int rm = __shfl(row, t);
  const uint8_t* src_m = from(t);
  uint32_t km[NG];
  if (l < 16) {
#pragma unroll
    for (int g = 0; g < NG; ++g) km[g] = reinterpret_cast<const uint32_t*>(src_m + Lay::kOffKMeta + 4 * NG * rm)[g];
  }
  uint16_t vc[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int x = 4 * (l >> 4) + i, r = __shfl(row, x);
    vc[i] = *reinterpret_cast<const uint16_t*>(from(x) + kOffVCodes + 32 * t + 2 * r);
  }
  const int vrow = l % kRows, vt = 2 * ((l / kRows) & 7);
  uint16_t vm[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = __shfl(row, vt + i);
    const uint8_t* src = from(vt + i);
    vm[i] = *reinterpret_cast<const uint16_t*>(src + Lay::kOffVScale + 32 * vrow + 2 * r);
  }
  float wt = 0.0f;
  const bool weighs = a.weights && l < 16 && good && token < a.weights_stride;
  if (weighs) wt = STAGE == 2 ? reinterpret_cast<const float*>(stage + Lay::kBytes)[l] : a.weights[((size_t)b * H + h) * a.weights_stride + token];

  if (l < 32 && ((mask >> tk) & 1)) *reinterpret_cast<uint4*>(dst + 16 * l) = kc;
  if (l < 16 && ((mask >> l) & 1)) {
#pragma unroll
    for (int g = 0; g < NG; ++g) reinterpret_cast<uint32_t*>(dst + Lay::kOffKMeta + 4 * NG * l)[g] = km[g];
  }
  const uint32_t mv = (mask >> (4 * (l >> 4))) & 15u, mm = (mask >> vt) & 3u;
  uint16_t* dv = reinterpret_cast<uint16_t*>(dst + kOffVCodes + 32 * t + 8 * (l >> 4));
  if (mv == 15u)
    *reinterpret_cast<uint2*>(dv) = make_uint2(vc[0] | (uint32_t)vc[1] << 16, vc[2] | (uint32_t)vc[3] << 16);
  else
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if ((mv >> i) & 1) dv[i] = vc[i];
  if (l < 8 * kRows) {
    uint16_t* dm = reinterpret_cast<uint16_t*>(dst + Lay::kOffVScale + 32 * vrow + 2 * vt);
    if (mm == 3u)
      *reinterpret_cast<uint32_t*>(dm) = vm[0] | (uint32_t)vm[1] << 16;
    else
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if ((mm >> i) & 1) dm[i] = vm[i];
  }
  if (weighs) {
    if (STAGE == 1)
      reinterpret_cast<float*>(stage + Lay::kBytes)[l] = wt;
    else if (kBlock * page + l < a.out_weights_stride)
      a.out_weights[((size_t)b * H + h) * a.out_weights_stride + kBlock * page + l] = wt;
  }
}

size_t move_stage_bytes(int groups) { return 1024 + 128 * (size_t)groups + kStagedWeights; }

namespace {

template <int NG>
hipError_t launch_move(const MoveArgs& a, bool in_place, hipStream_t s) {
  const dim3 grid((unsigned)(((long long)a.B * a.pages * a.cv.num_kv_heads + kMoveWaves - 1) / kMoveWaves)), block(64 * kMoveWaves);
  if (!in_place) {
    hipLaunchKernelGGL((move_tokens_kernel<NG, 0>), grid, block, 0, s, a);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((move_tokens_kernel<NG, 1>), grid, block, 0, s, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((move_tokens_kernel<NG, 2>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_move_tokens(const MoveArgs& a, bool in_place, hipStream_t s) {
  return a.cv.groups == 4 ? launch_move<4>(a, in_place, s) : launch_move<1>(a, in_place, s);
}

}  // namespace int2kv
