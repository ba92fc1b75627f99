// Eviction from a paged cache: of each (sequence, KV head) the first `sink`,
// the last `recent` and the heaviest of the other tokens stay, `budget` in
// all, in their order; their rows go to other pages, one after the other.
//
// select_kernel: one workgroup a (sequence, head). The weight that just stays
// is found digit by digit (11, 11 and 10 bits of the order-preserving bits of
// the weights, a histogram in LDS each), then one more pass writes the tokens
// that stay, ties by the lowest index. What bounds it is a compute unit's vector
// instructions: about 2 us for 16K weights and a pass (40 us for the 57K tokens of
// the longest of 16 sequences), so what need not be looked at is left out, and
// weights of a positive range are told by their own bits.
// move_kernel: a wave takes a run of rows of the new layout of one head, keys
// or values, and the waves beside it the other heads, whose rows lie side by
// side in the new pages and near each other in the old ones. bf16 rows and
// codes with a scale per head are copied; with a scale per block a new block
// holds rows of several old ones: its scale is again the smallest power of two
// for its largest value, and the codes are moved by the difference of the
// powers, exact but for what becomes subnormal. Bound by memory: 4096 rows of 8
// heads and 16 sequences, 270 MB in all, in 53 us (5.1 TB/s).
//
// 16 sequences of 5K to 58K tokens to 4096: 103 us, in bf16 156; one of 2000 to
// 1000: 13 us.
#include <algorithm>
#include <type_traits>

#include "cache.h"

namespace fp2 {

namespace {

constexpr int kThreads = 1024;
constexpr int kSteps = 4;                         // loads of a thread at once, of four tokens each
constexpr int kRound = kSteps * kThreads * 4;     // tokens of them
constexpr int kBins = 2048;
constexpr int kCopies = 4;         // histograms, so that the lanes of a wave seldom meet at a bin
constexpr int kWaves = 8;

// Bits whose order is that of the numbers; NaN below all, -0 as 0.
__device__ __forceinline__ uint32_t order_of(float x) {
  if (!(x == x)) return 0u;
  const uint32_t u = __float_as_uint(x + 0.f);
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Exclusive sum over the workgroup's threads and the total. tot: LDS, one a wave.
__device__ __forceinline__ int block_scan(int v, int* tot, int& total) {
  constexpr int W = kThreads / 64;
  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int incl = wave_scan(v);
  if (lane == 63) tot[w] = incl;
  __syncthreads();
  const int sums = wave_scan(lane < W ? tot[lane] : 0);
  total = __builtin_amdgcn_readlane(sums, W - 1);
  const int before = w ? __shfl(sums, w - 1, 64) : 0;
  __syncthreads();
  return before + incl - v;
}

__global__ __launch_bounds__(kThreads) void select_kernel(CacheProblem p, int budget, int recent,
                                                          const float* __restrict__ weights,
                                                          int64_t stride, float* __restrict__ weights_out,
                                                          int64_t out_stride, int32_t* __restrict__ kept,
                                                          int32_t* __restrict__ cu_out) {
  __shared__ int hist[kCopies][kBins];
  __shared__ int cnt[2][kSteps * kThreads / 64];
  __shared__ int tot[kThreads / 64];
  __shared__ int s_bin, s_need, s_size;
  const int tid = threadIdx.x, lane = tid & 63, w = __builtin_amdgcn_readfirstlane(tid >> 6);
  if (blockIdx.x == 0 && tid < 64) {   // the new lengths
    int base = 0;
    if (lane == 0) cu_out[0] = 0;
    for (int b0 = 0; b0 < p.batch; b0 += 64) {
      const int b = b0 + lane;
      const int n = b < p.batch ? min(p.cuk[b + 1] - p.cuk[b], budget) : 0;
      const int incl = wave_scan(n);
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
  // four weights a load from the 16-byte line that the row starts in: element e
  // of line v is token 4 v + e - skew
  const int skew = (int)((uintptr_t)wr >> 2 & 3), lines = (L + skew + 3) / 4;
  const float4* line = (const float4*)(wr - skew);
  auto load = [&](int v0, float4 (&x)[kSteps]) {
#pragma unroll
    for (int s = 0; s < kSteps; ++s) x[s] = line[min(v0 + s * kThreads + tid, lines - 1)];
  };
  float4 x[kSteps];
  load(0, x);
  const bool once = lines <= kRound / 4;                 // then they are loaded once
  auto at = [](const float4& x, int e) { return e == 0 ? x.x : e == 1 ? x.y : e == 2 ? x.z : x.w; };
  // the first token of a wave's load, and whether all of them are ranked: then
  // none is looked at for its place
  auto begins = [&](int v0, int s) { return 4 * (v0 + s * kThreads + (w << 6)) - skew; };
  auto ranked = [&](int v0, int s) { return begins(v0, s) >= lo && begins(v0, s) + 256 <= hi; };
  // bits of the weight that just stays, found from the top
  uint32_t edge = 0, span = 0;                           // it lies in [edge, edge + span)
  int left = need;                                       // stay of those
  // Weights in a range of positive finite ones are told by their own bits: two
  // operations each, where putting them in order takes seven (one sequence of
  // 100K tokens: 55 us, 61 without).
  constexpr uint32_t kSign = 0x80000000u, kInf = 0x7f800000u;
  bool plain = false;
  auto from_edge = [&](float x, auto own) {              // 0 .. span - 1: in the range
    return own ? __float_as_uint(x) - (edge ^ kSign) : order_of(x) - edge;
  };
#pragma unroll 1
  for (int d = 0; d < 3 && need > 0; ++d) {
    const int shift = d == 0 ? 21 : d == 1 ? 10 : 0, bins = d == 2 ? 1024 : 2048;
    for (int i = tid; i < kCopies * kBins; i += kThreads) hist[0][i] = 0;
    __syncthreads();
#pragma unroll 1
    for (int v0 = 0; v0 < lines; v0 += kRound / 4) {
      if (!once) load(v0, x);
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        auto count = [&](auto inside, auto first, auto own) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int i = 4 * (v0 + s * kThreads + tid) + e - skew;
            const uint32_t u = from_edge(at(x[s], e), own);
            if ((inside || (i >= lo && i < hi)) && (first || u < span))
              atomicAdd(&hist[tid % kCopies][u >> shift], 1);
          }
        };
        using Y = std::true_type;
        using N = std::false_type;
        if (ranked(v0, s)) {
          if (d == 0) count(Y{}, Y{}, N{});
          else if (plain) count(Y{}, N{}, Y{});
          else count(Y{}, N{}, N{});
        } else if (begins(v0, s) < hi) {
          if (d == 0) count(N{}, Y{}, N{});
          else count(N{}, N{}, N{});
        }
      }
    }
    __syncthreads();
    // bins from the top, two a thread
    const int b1 = bins - 1 - 2 * tid;
    int n1 = 0, n2 = 0;
    for (int c = 0; c < kCopies && b1 > 0; ++c) n1 += hist[c][b1], n2 += hist[c][b1 - 1];
    int total;
    const int before = block_scan(n1 + n2, tot, total);
    if (before < left && before + n1 >= left) s_bin = b1, s_need = left - before, s_size = n1;
    else if (before + n1 < left && before + n1 + n2 >= left)
      s_bin = b1 - 1, s_need = left - before - n1, s_size = n2;
    __syncthreads();
    edge += (uint32_t)s_bin << shift;
    span = 1u << shift;
    plain = edge > kSign && edge + span <= (kSign | kInf);
    left = s_need;
    const bool all = s_size == left;     // every weight with these bits stays: no need for the others
    __syncthreads();
    if (all) break;
  }
  // in order: tokens that are protected or heavier than the edge, and the
  // first `left` at it. A round counts both (the second kind in the high half)
  // for every wave and step, and one sum over those gives every place.
  int over = 0, equal = 0;               // of the rounds before
#pragma unroll 1
  for (int v0 = 0, odd = 0; v0 < lines; v0 += kRound / 4, odd ^= 1) {
    if (!once) load(v0, x);
    int up[kSteps], eq[kSteps], incl[kSteps];            // bits of this thread's tokens
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      up[s] = eq[s] = 0;
      auto sort = [&](auto inside, auto own) {
        // heavier: behind the range, up to infinity
        const uint32_t end = own ? kInf - (edge ^ kSign) - span : need > 0 ? ~edge - span : 0u;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = 4 * (v0 + s * kThreads + tid) + e - skew;
          const uint32_t u = from_edge(at(x[s], e), own);
          const bool fixed = !inside && (i < lo || i >= hi), in = inside || (i >= 0 && i < L);
          up[s] |= in && (fixed || (u - span <= end && (own || need > 0))) ? 1 << e : 0;
          eq[s] |= in && !fixed && u < span ? 1 << e : 0;
        }
      };
      if (ranked(v0, s)) {
        if (plain) sort(std::true_type{}, std::true_type{});
        else sort(std::true_type{}, std::false_type{});
      } else if (begins(v0, s) < L) {
        sort(std::false_type{}, std::false_type{});
      }
      incl[s] = wave_scan(__popc(up[s]) | __popc(eq[s]) << 16);
      if (lane == 63) cnt[odd][s * (kThreads / 64) + w] = incl[s];
    }
    __syncthreads();
    static_assert(kSteps * kThreads / 64 == 64, "a lane each");
    const int own = cnt[odd][lane], sum = wave_scan(own), total = __builtin_amdgcn_readlane(sum, 63);
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
      const int before = __shfl(sum - own, s * (kThreads / 64) + w, 64) + incl[s] -
                         (__popc(up[s]) | __popc(eq[s]) << 16);
      int o = over + (before & 0xffff), n = equal + (before >> 16);
      if (!__any(eq[s])) {
        // (most loads)
        const int base = o + min(n, left) , i0 = 4 * (v0 + s * kThreads + tid) - skew;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (up[s] >> e & 1) {
            const int to = base + __popc(up[s] & ((1 << e) - 1));
            kr[to] = i0 + e;
            wo[to] = at(x[s], e);
          }
        continue;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool is_up = up[s] >> e & 1, is_eq = eq[s] >> e & 1;
        if (is_up || (is_eq && n < left)) {
          const int to = o + min(n, left);
          kr[to] = 4 * (v0 + s * kThreads + tid) + e - skew;
          wo[to] = at(x[s], e);
        }
        o += is_up;
        n += is_eq;
      }
    }
    over += total & 0xffff;
    equal += total >> 16;
  }
}

// SB: tokens with one scale (blocks), else 0.
template <int FORM, int SB>
__global__ __launch_bounds__(64 * kWaves) void move_kernel(CacheProblem p, PageMap to, int budget,
                                                           int runs, int64_t total,
                                                           const int32_t* __restrict__ kept) {
  constexpr int ESZ = FORM == kCacheBf16 ? 2 : 1;
  constexpr int RUN = SB > 32 ? SB : 32;         // rows of a wave
  constexpr int LPR = kHeadDim * ESZ / 16;       // lanes of a row, 16 bytes each
  constexpr int RPL = 64 / LPR;                  // rows of a load
  constexpr int N = RUN / RPL;
  int64_t at = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (at >= total) return;
  const int h = (int)(at % p.hkv);
  at /= p.hkv;
  const bool is_v = at & 1;
  at >>= 1;
  const int first = (int)(at % runs) * RUN, b = (int)(at / runs);
  const int stay = min(ld_uniform(p.cuk, b + 1) - ld_uniform(p.cuk, b), budget);
  if (first >= stay) return;
  const int lane = threadIdx.x & 63, c = lane % LPR, r0 = lane / LPR;
  const int64_t rowb = (int64_t)p.hkv * kHeadDim * ESZ, hoff = (int64_t)h * kHeadDim * ESZ + 16 * c;
  const int32_t* kr = kept + ((int64_t)b * p.hkv + h) * budget;
  // slots of the rows: every lane looks up some, the loads below ask it
  constexpr int LOOK = (RUN + 63) / 64;
  int64_t from[LOOK], dest[LOOK];
#pragma unroll
  for (int i = 0; i < LOOK; ++i) {
    const int r = min(first + 64 * i + lane, stay - 1);
    from[i] = slot_of(p.pm, b, 0, kr[r]);
    dest[i] = slot_of(to, b, 0, r);
  }
  uint8_t* pool = is_v ? p.v : p.k;
  uint8_t* scales = is_v ? p.v_block : p.k_block;
  i32x4_t x[N];   // (a vector, not the struct: a copied struct would be kept in LDS)
  uint32_t old[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int r = RPL * i + r0;
    const int64_t slot = __shfl(from[RPL * i / 64], r & 63, 64);
    x[i] = *(const i32x4_t*)(pool + slot * rowb + hoff);
    if constexpr (FORM == kCacheBlock) old[i] = scales[(slot >> p.sb_shift) * p.hkv + h];
  }
  if constexpr (FORM == kCacheBlock) {
    constexpr int PER = SB / RPL;              // loads of a block
    float amax[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const uint32_t d[4] = {(uint32_t)x[i][0], (uint32_t)x[i][1], (uint32_t)x[i][2], (uint32_t)x[i][3]};
      float m = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float y[4];
        e4m3x4_to_f32(d[j], y);
#pragma unroll
        for (int e = 0; e < 4; ++e) m = fmaxf(m, fabsf(y[e]));   // a NaN is left out
      }
      // rows behind the last repeat it: they change no maximum
      amax[i] = m * block_scale(old[i]);
    }
    int byte = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (i % PER == 0) {
        float m = amax[i];
#pragma unroll
        for (int j = 1; j < PER; ++j) m = fmaxf(m, amax[i + j]);
        byte = scale_byte(wave_max(m));
        const int64_t slot = __shfl(dest[RPL * i / 64], RPL * i & 63, 64);
        if (lane == 0 && first + RPL * i < stay)
          scales[(slot >> p.sb_shift) * p.hkv + h] = (uint8_t)byte;
      }
      // What a code is times: 2^(old - new), which leaves at most 448. Codes that are not
      // 0 need at most 2^17 for that; a row of zeros may come with any scale, and its
      // power is held finite (below, 2^-126 leaves zeros too).
      const float f = block_scale((uint32_t)min(max((int)old[i] - byte + 127, 1), 254));
      // converted once more: kept from above they would take 16 registers a load
      uint32_t d[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) d[j] = (uint32_t)pinned((int)x[i][j]);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float y[4];
        e4m3x4_to_f32(d[j], y);
        const uint32_t nan = ((d[j] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;   // top bits of NaN codes
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0] * f, y[1] * f, 0, false);
        w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2] * f, y[3] * f, w, true);
        d[j] = ((uint32_t)w & ~((nan >> 7) * 0xffu)) | (nan - (nan >> 7));
      }
      x[i] = (i32x4_t){(int)d[0], (int)d[1], (int)d[2], (int)d[3]};
    }
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int r = RPL * i + r0;
    const int64_t slot = __shfl(dest[RPL * i / 64], r & 63, 64);
    if (first + r < stay) *(i32x4_t*)(pool + slot * rowb + hoff) = x[i];
  }
}

template <int FORM, int SB>
hipError_t launch(const CacheProblem& p, const PageMap& to, int budget, int recent, const float* weights,
                  int64_t stride, float* weights_out, int64_t out_stride, int32_t* kept, int32_t* cu_out,
                  hipStream_t s) {
  constexpr int RUN = SB > 32 ? SB : 32;
  const int runs = (std::min(budget, p.max_kv) + RUN - 1) / RUN;
  const int64_t heads = (int64_t)p.batch * p.hkv;
  const int64_t total = heads * 2 * runs, grid = (total + kWaves - 1) / kWaves;
  if (!launchable(heads, kThreads) || !launchable(grid, 64 * kWaves)) return hipErrorInvalidValue;
  select_kernel<<<(unsigned)heads, kThreads, 0, s>>>(p, budget, recent, weights, stride, weights_out,
                                                     out_stride, kept, cu_out);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  move_kernel<FORM, SB><<<(unsigned)grid, 64 * kWaves, 0, s>>>(p, to, budget, runs, total, kept);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_evict(const CacheProblem& p, const PageMap& to, int budget, int recent,
                              const float* weights, int64_t stride, float* weights_out,
                              int64_t out_stride, int32_t* kept, int32_t* cu_out, hipStream_t s) {
  auto run = [&](auto f) {
    return f(p, to, budget, recent, weights, stride, weights_out, out_stride, kept, cu_out, s);
  };
  if (p.form == kCacheBf16) return run(launch<kCacheBf16, 0>);
  if (p.form == kCacheHead) return run(launch<kCacheHead, 0>);
  return p.sb_shift == 4   ? run(launch<kCacheBlock, 16>)
         : p.sb_shift == 5 ? run(launch<kCacheBlock, 32>)
         : p.sb_shift == 6 ? run(launch<kCacheBlock, 64>)
                           : run(launch<kCacheBlock, 128>);
}

}  // namespace fp2
