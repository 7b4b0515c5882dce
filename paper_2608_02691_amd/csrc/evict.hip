// The tokens of a cache that stay, and their rows' move (int2kv_select_tokens, int2kv_move_tokens).
#include "common.h"
#include "kernels.h"

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

// Block: one (sequence, KV head). The threshold comes byte by byte from histograms of the keys that share the bytes so far.
__global__ __launch_bounds__(kSelectThreads) void select_tokens_kernel(SelectArgs a) {
  __shared__ int bins[256], waves[kSelectWaves], found[2];
  const int b = blockIdx.x / a.H, h = blockIdx.x - b * a.H, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
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
  uint32_t prefix = 0;
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += kSelectThreads) bins[i] = 0;
    __syncthreads();
    for (int i = lo + tid; i < hi; i += kSelectThreads) {
      const uint32_t k = order_of(w[i]);
      if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&bins[(k >> shift) & 255], 1);
    }
    __syncthreads();
    if (tid == 0) {  // the byte of the need-th largest
      int x = 255, above = 0;
      while (x > 0 && above + bins[x] < need) above += bins[x--];
      found[0] = x, found[1] = above;
    }
    __syncthreads();
    prefix |= (uint32_t)found[0] << shift;
    need -= found[1];
    __syncthreads();
  }
  // the keys above `prefix` and the first `need` equal to it, in order
  int base = 0, ties = 0;
  for (int i0 = 0; i0 < len; i0 += kSelectThreads) {
    const int i = i0 + tid;
    const bool forced = i < lo || i >= hi;
    const uint32_t k = i < len && !forced ? order_of(w[i]) : 0u;
    const bool above = i < len && (forced || k > prefix), equal = i < len && !forced && k == prefix;
    const uint64_t ab = __ballot(above), eb = __ballot(equal), before = (1ull << lane) - 1;
    if (lane == 0) waves[wave] = __popcll(ab) | __popcll(eb) << 16;
    __syncthreads();
    int na = 0, ne = 0, all_a = 0, all_e = 0;
    for (int x = 0; x < kSelectWaves; ++x) {
      const int v = waves[x];
      if (x < wave) na += v & 0xFFFF, ne += v >> 16;
      all_a += v & 0xFFFF, all_e += v >> 16;
    }
    // kept before token i: those above, and of the equal ones as many as there is need for
    const int pa = na + __popcll(ab & before), pe = ties + ne + __popcll(eb & before);
    if (above || (equal && pe < need)) kept[base + pa + min(pe, need) - min(ties, need)] = i;
    base += all_a + min(ties + all_e, need) - min(ties, need);
    ties += all_e;
    __syncthreads();
  }
}

hipError_t launch_select_tokens(const SelectArgs& a, hipStream_t s) {
  hipLaunchKernelGGL(select_tokens_kernel, dim3((unsigned)(a.B * a.H)), dim3(kSelectThreads), 0, s, a);
  return hipGetLastError();
}

namespace {

constexpr int kMoveWaves = 4;
constexpr int kStagedWeights = 4 * kBlock;

}  // namespace

// Wave: one page of one KV head of the result. A token's row is 32 bytes of key codes and its parameters, which lie together,
// and two bytes of each of the page's value rows. STAGE 0: from the cache into the result's blocks; 1: from the cache into
// the workspace; 2: from there into the cache.
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
