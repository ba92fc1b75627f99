// Eviction from a paged cache: of each (sequence, KV head) the first `sink`,
// the last `recent` and the heaviest of the other tokens stay, `budget` in
// all, in their order; their rows go to other pages, one after the other.
//
// select_kernel: one workgroup a (sequence, head). The weight that just stays
// is found digit by digit (11, 11 and 10 bits of the order-preserving bits of
// the weights, a histogram in LDS each), then one pass over the tokens writes
// the ones that stay, ties by the lowest index.
// move_kernel: 128 rows of the new layout a workgroup, as the append. bf16
// rows and codes with a scale per head are copied; with a scale per block a
// new block holds rows of several old ones: its scale is again the smallest
// power of two for its largest value, and the codes are moved by the
// difference of the powers, exact but for what becomes subnormal.
#include <algorithm>
#include <type_traits>

#include "cache.h"

namespace fp2 {

namespace {

constexpr int kThreads = 1024;
constexpr int kBins = 2048;
constexpr int kPer = 4;            // consecutive tokens of a thread
constexpr int kRows = 128;
constexpr int kWaves = 8;

// Bits whose order is that of the numbers; NaN below all, -0 as 0.
__device__ __forceinline__ uint32_t order_of(float x) {
  if (!(x == x)) return 0u;
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int wave_scan(int v, int lane) {   // inclusive
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o, 64);
    if (lane >= o) v += u;
  }
  return v;
}

// Exclusive sum over the workgroup's threads and the total. tot: LDS, one a wave.
__device__ __forceinline__ int block_scan(int v, int* tot, int& total) {
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int incl = wave_scan(v, lane);
  if (lane == 63) tot[w] = incl;
  __syncthreads();
  int before = 0;
  total = 0;
  for (int i = 0; i < kThreads / 64; ++i) {
    before += i < w ? tot[i] : 0;
    total += tot[i];
  }
  __syncthreads();
  return before + incl - v;
}

__global__ __launch_bounds__(kThreads) void select_kernel(CacheProblem p, int budget, int recent,
                                                          const float* __restrict__ weights,
                                                          int64_t stride, float* __restrict__ weights_out,
                                                          int64_t out_stride, int32_t* __restrict__ kept,
                                                          int32_t* __restrict__ cu_out) {
  __shared__ int hist[kBins];
  __shared__ int tot[kThreads / 64];
  __shared__ int s_bin, s_need;
  const int tid = threadIdx.x, lane = tid & 63;
  if (blockIdx.x == 0 && tid < 64) {   // the new lengths
    int base = 0;
    if (lane == 0) cu_out[0] = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 64) {
      const int b = b0 + lane;
      const int n = b < p.batch ? min(p.cuk[b + 1] - p.cuk[b], budget) : 0;
      const int incl = wave_scan(n, lane);
      if (b < p.batch) cu_out[b + 1] = base + incl;
      base += __shfl(incl, 63, 64);
    }
  }
  const int h = blockIdx.x % p.hkv, b = blockIdx.x / p.hkv;
  const int L = ld_uniform(p.cuk, b + 1) - ld_uniform(p.cuk, b);
  const float* wr = weights + ((int64_t)b * p.hkv + h) * stride;
  float* wo = weights_out + ((int64_t)b * p.hkv + h) * out_stride;
  int32_t* kr = kept + ((int64_t)b * p.hkv + h) * budget;
  const int stay = min(L, budget);
  for (int64_t i = stay + tid; i < out_stride; i += kThreads) wo[i] = 0.f;
  for (int i = stay + tid; i < budget; i += kThreads) kr[i] = -1;
  if (L <= budget) {
    for (int i = tid; i < L; i += kThreads) {
      kr[i] = i;
      wo[i] = wr[i];
    }
    return;
  }
  const int lo = min(p.sink, budget), hi = L - recent;   // the tokens between are ranked
  int need = budget - lo - recent;                       // of them stay
  // bits of the weight that just stays, found from the top
  uint32_t edge = 0;
  int left = need;                                       // of those equal to `edge` so far
#pragma unroll 1
  for (int d = 0; d < 3 && need > 0; ++d) {
    const int shift = d == 0 ? 21 : d == 1 ? 10 : 0, bins = d == 2 ? 1024 : 2048;
    const uint32_t above = d == 0 ? 0u : d == 1 ? 0xffe00000u : 0xfffffc00u;
    for (int i = tid; i < bins; i += kThreads) hist[i] = 0;
    __syncthreads();
    for (int i0 = lo + tid; i0 < hi; i0 += 8 * kThreads) {
      float x[8];                        // eight loads in flight
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = i0 + j * kThreads < hi ? wr[i0 + j * kThreads] : 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t u = order_of(x[j]);
        if (i0 + j * kThreads < hi && (u & above) == edge)
          atomicAdd(&hist[(u >> shift) & (bins - 1)], 1);
      }
    }
    __syncthreads();
    // bins from the top, two a thread
    const int b1 = bins - 1 - 2 * tid, n1 = b1 >= 0 ? hist[b1] : 0, n2 = b1 >= 1 ? hist[b1 - 1] : 0;
    int total;
    const int before = block_scan(n1 + n2, tot, total);
    if (before < left && before + n1 >= left) s_bin = b1, s_need = left - before;
    else if (before + n1 < left && before + n1 + n2 >= left) s_bin = b1 - 1, s_need = left - before - n1;
    __syncthreads();
    edge |= (uint32_t)s_bin << shift;
    left = s_need;
    __syncthreads();
  }
  // tokens in order: protected or heavier than the edge, or the first `left` at
  // it. Both are counted by one sum a step, the second kind in the high half.
  int over = 0, equal = 0;               // of the steps before
  float x[kPer], y[kPer];
  auto load = [&](int i0, float (&v)[kPer]) {
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = i0 + kPer * tid + j;
      v[j] = i < L ? wr[i] : 0.f;
    }
  };
  load(0, x);
#pragma unroll 1
  for (int i0 = 0; i0 < L; i0 += kThreads * kPer) {
    load(i0 + kThreads * kPer, y);       // of the next step
    int eq = 0, up = 0;                  // bit masks of this thread's tokens
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const int i = i0 + kPer * tid + j;
      const uint32_t u = order_of(x[j]);
      const bool fixed = i < lo || i >= hi;
      if (i < L && (fixed || (need > 0 && u > edge))) up |= 1 << j;
      else if (i < L && need > 0 && u == edge) eq |= 1 << j;
    }
    int total;
    const int before = block_scan(__popc(up) | __popc(eq) << 16, tot, total);
    int o = over + (before & 0xffff), e = equal + (before >> 16);
#pragma unroll
    for (int j = 0; j < kPer; ++j) {
      const bool is_up = up >> j & 1, is_eq = eq >> j & 1;
      if (is_up || (is_eq && e < left)) {
        const int to = o + min(e, left);
        kr[to] = i0 + kPer * tid + j;
        wo[to] = x[j];
      }
      o += is_up;
      e += is_eq;
    }
    over += total & 0xffff;
    equal += total >> 16;
#pragma unroll
    for (int j = 0; j < kPer; ++j) x[j] = y[j];
  }
}

template <int FORM>
__global__ __launch_bounds__(64 * kWaves) void move_kernel(CacheProblem p, PageMap to, int budget,
                                                           int chunks, const int32_t* __restrict__ kept) {
  constexpr int ESZ = FORM == kCacheBf16 ? 2 : 1;
  __shared__ float s_amax[kWaves];
  int64_t at = blockIdx.x;
  const int h = (int)(at % p.hkv);
  at /= p.hkv;
  const bool is_v = at & 1;
  at >>= 1;
  const int first = (int)(at % chunks) * kRows, b = (int)(at / chunks);
  const int L = ld_uniform(p.cuk, b + 1) - ld_uniform(p.cuk, b);
  const int stay = min(L, budget);
  if (first >= stay) return;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, c = lane & 15;
  uint8_t* pool = is_v ? p.v : p.k;
  uint8_t* scales = is_v ? p.v_block : p.k_block;
  const int64_t rowb = (int64_t)p.hkv * kHeadDim * ESZ, hoff = (int64_t)h * kHeadDim * ESZ;
  const int32_t* kr = kept + ((int64_t)b * p.hkv + h) * budget;
  typedef std::conditional_t<FORM == kCacheBf16, uint4, uint2> row_t;
  row_t x[4];
  float sc[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = first + 16 * w + 4 * i + (lane >> 4);
    x[i] = row_t{};
    sc[i] = 0.f;
    if (r < stay) {
      const int64_t slot = slot_of(p.pm, b, 0, kr[r]);
      x[i] = *(const row_t*)(pool + slot * rowb + hoff + sizeof(row_t) * c);
      if constexpr (FORM == kCacheBlock) sc[i] = block_scale(scales[(slot >> p.sb_shift) * p.hkv + h]);
    }
  }
  float inv = 0.f;
  if constexpr (FORM == kCacheBlock) {
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float y[4], z[4];
      e4m3x4_to_f32(x[i].x, y);
      e4m3x4_to_f32(x[i].y, z);
#pragma unroll
      for (int e = 0; e < 4; ++e) {   // NaN codes do not count
        const float g = fabsf(y[e]), f = fabsf(z[e]);
        amax = fmaxf(amax, g <= 448.f ? g * sc[i] : 0.f);
        amax = fmaxf(amax, f <= 448.f ? f * sc[i] : 0.f);
      }
    }
    amax = wave_max(amax);
    if (lane == 0) s_amax[w] = amax;
    __syncthreads();
    const int wpb = 1 << (p.sb_shift - 4), w0 = w & ~(wpb - 1);
    for (int j = 0; j < wpb; ++j) amax = fmaxf(amax, s_amax[w0 + j]);
    const int byte = scale_byte(amax), tb = first + 16 * w0;
    if (w == w0 && lane == 0 && tb < stay)
      scales[(slot_of(to, b, 0, tb) >> p.sb_shift) * p.hkv + h] = (uint8_t)byte;
    inv = __uint_as_float((uint32_t)(254 - byte) << 23);
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = first + 16 * w + 4 * i + (lane >> 4);
    if (r >= stay) continue;
    row_t v = x[i];
    if constexpr (FORM == kCacheBlock) {
      float y[4], z[4], s[4], t[4];
      e4m3x4_to_f32(v.x, y);
      e4m3x4_to_f32(v.y, z);
#pragma unroll
      for (int e = 0; e < 4; ++e) s[e] = y[e] * sc[i] * inv, t[e] = z[e] * sc[i] * inv;
      v = make_uint2(e4m3x4(y, s), e4m3x4(z, t));
    }
    *(row_t*)(pool + slot_of(to, b, 0, r) * rowb + hoff + sizeof(row_t) * c) = v;
  }
}

}  // namespace

hipError_t launch_cache_evict(const CacheProblem& p, const PageMap& to, int budget, int recent,
                              const float* weights, int64_t stride, float* weights_out,
                              int64_t out_stride, int32_t* kept, int32_t* cu_out, hipStream_t s) {
  const int chunks = (std::min(budget, p.max_kv) + kRows - 1) / kRows;
  const int64_t heads = (int64_t)p.batch * p.hkv, grid = heads * 2 * chunks;
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  select_kernel<<<(unsigned)heads, kThreads, 0, s>>>(p, budget, recent, weights, stride, weights_out,
                                                     out_stride, kept, cu_out);
  if (p.form == kCacheBf16)
    move_kernel<kCacheBf16><<<(unsigned)grid, 64 * kWaves, 0, s>>>(p, to, budget, chunks, kept);
  else if (p.form == kCacheHead)
    move_kernel<kCacheHead><<<(unsigned)grid, 64 * kWaves, 0, s>>>(p, to, budget, chunks, kept);
  else
    move_kernel<kCacheBlock><<<(unsigned)grid, 64 * kWaves, 0, s>>>(p, to, budget, chunks, kept);
  return hipGetLastError();
}

}  // namespace fp2
