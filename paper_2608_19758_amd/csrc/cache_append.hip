// New tokens' keys and values into a paged cache, in its type.
//
// A workgroup takes 128 consecutive tokens of one sequence, one head and keys
// or values: wave w rows 16 w .. 16 w + 15, four rows a load, 16 bytes a lane.
// bf16 rows are copied; with a scale per head the codes are e4m3(x / scale).
//
// With a scale per block of tokens (16 to 128, so blocks never leave the
// workgroup) the block's largest finite value decides: 2^e, e =
// ceil(log2(amax / 448)), read off the bits of amax. A power of two makes
// x 2^-e exact, so a code is rounded once. Where a block already holds tokens
// its scale never falls; if it grows by 2^n their codes are taken times 2^-n,
// which rounds again only what becomes subnormal.
//
// Bound by memory: 256 + 128 bytes a token and head, keys and values each. 32768
// tokens of 8 heads with scales of 64 tokens take 48 us (4.2 TB/s), into a bf16
// cache 57 us (4.7).
//
// Few new tokens a sequence (a decode step) leave most of such a workgroup idle,
// and starting them is what bounds the call; there a wave has a sequence's head
// to itself: one token of 8 sequences takes 4.1 us (4.5 in workgroups of 128
// rows), of 256 sequences 6.8 (21), of 1024 14 (71).
#include "cache.h"

namespace fp2 {

namespace {

constexpr int kRows = 128;     // tokens per workgroup
constexpr int kWaves = 8;
constexpr int kFew = 16;       // new tokens of a sequence that a wave takes alone (of one: 4.7 us both ways)

__device__ __forceinline__ void unpack8(uint4 w, float (&x)[8]) {
  const uint32_t d[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(d[i] << 16);
    x[2 * i + 1] = __uint_as_float(d[i] & 0xffff0000u);
  }
}

__device__ __forceinline__ uint2 codes8(const float (&x)[8], const float (&y)[8]) {
  const float a[4] = {x[0], x[1], x[2], x[3]}, b[4] = {x[4], x[5], x[6], x[7]};
  const float c[4] = {y[0], y[1], y[2], y[3]}, d[4] = {y[4], y[5], y[6], y[7]};
  return make_uint2(e4m3x4(a, c), e4m3x4(b, d));
}

// Codes of eight values times a power of two.
__device__ __forceinline__ uint2 shrunk8(uint2 old, float shrink) {
  float x[4], y[4], z[4], u[4];
  e4m3x4_to_f32(old.x, x);
  e4m3x4_to_f32(old.y, z);
#pragma unroll
  for (int e = 0; e < 4; ++e) y[e] = x[e] * shrink, u[e] = z[e] * shrink;
  return make_uint2(e4m3x4(x, y), e4m3x4(z, u));
}

template <int FORM>
__global__ __launch_bounds__(64 * kWaves) void append_kernel(CacheProblem p,
                                                             const uint16_t* __restrict__ k_new,
                                                             const uint16_t* __restrict__ v_new,
                                                             int chunks) {
  __shared__ float s_amax[kWaves];
  __shared__ int s_byte[kWaves];
  int64_t at = blockIdx.x;
  const int h = (int)(at % p.hkv);
  at /= p.hkv;
  const bool is_v = at & 1;
  at >>= 1;
  const int ck = (int)(at % chunks), b = (int)(at / chunks);
  const int q0 = ld_uniform(p.cu, b), n = ld_uniform(p.cu, b + 1) - q0;
  const int64_t tok0 = ld_uniform(p.cuk, b);
  const int L = ld_uniform(p.cuk, b + 1) - (int)tok0;
  const int P = L - n;                        // tokens before the new ones
  const int first = (P / kRows + ck) * kRows;
  if (n <= 0 || first >= L) return;

  const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
  const int c = lane & 15;
  const uint16_t* src = is_v ? v_new : k_new;
  uint8_t* pool = is_v ? p.v : p.k;
  const int64_t rowb = (int64_t)p.hkv * kHeadDim;       // elements of a token
  const int64_t hoff = (int64_t)h * kHeadDim + 8 * c;
  int t[4];
  uint4 raw[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    t[i] = first + 16 * w + 4 * i + (lane >> 4);
    raw[i] = make_uint4(0, 0, 0, 0);
    if (t[i] >= P && t[i] < L)
      raw[i] = *(const uint4*)(src + ((int64_t)q0 + t[i] - P) * rowb + hoff);
  }
  if constexpr (FORM == kCacheBf16) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (t[i] >= P && t[i] < L)
        *(uint4*)((uint16_t*)pool + slot_of(p.pm, b, tok0, t[i]) * rowb + hoff) = raw[i];
  } else if constexpr (FORM == kCacheHead) {
    const float scale = ld_uniform(is_v ? p.v_head : p.k_head, h);
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (t[i] >= P && t[i] < L) {
        float x[8], y[8];
        unpack8(raw[i], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x[e] / scale;
        *(uint2*)(pool + slot_of(p.pm, b, tok0, t[i]) * rowb + hoff) = codes8(x, y);
      }
  } else {
    // largest finite value of the wave's new tokens, then of its block's waves
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float x[8];
      unpack8(raw[i], x);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float a = fabsf(x[e]);
        amax = fmaxf(amax, a < INFINITY ? a : 0.f);
      }
    }
    amax = wave_max(amax);
    const int wpb = 1 << (p.sb_shift - 4);              // waves per block
    const int w0 = w & ~(wpb - 1);
    const int tb = first + 16 * w0, te = tb + (1 << p.sb_shift);   // the block's tokens
    const bool touched = te > P && tb < L;
    uint8_t* sp = nullptr;
    int before = 0;                                     // byte of a block that holds tokens
    if (w == w0 && touched) {
      sp = (is_v ? p.v_block : p.k_block) +
           (slot_of(p.pm, b, tok0, tb) >> p.sb_shift) * p.hkv + h;
      if (tb < P) before = *sp;
    }
    if (lane == 0) {
      s_amax[w] = amax;
      if (w == w0) s_byte[w] = before;
    }
    __syncthreads();
    if (!touched) return;
    for (int j = 0; j < wpb; ++j) amax = fmaxf(amax, s_amax[w0 + j]);
    before = s_byte[w0];
    const int byte = max(scale_byte(amax), before);
    if (sp && lane == 0) *sp = (uint8_t)byte;
    const float inv = __uint_as_float((uint32_t)(254 - byte) << 23);   // 2^-e
    // 2^-n for codes that were there; nothing to do for them where n is 0
    const bool grows = tb < P && byte > before;
    const float shrink = grows ? __uint_as_float((uint32_t)max(127 - (byte - before), 0) << 23) : 1.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (t[i] >= L || (t[i] < P && !grows)) continue;
      uint2* row = (uint2*)(pool + slot_of(p.pm, b, tok0, t[i]) * rowb + hoff);
      if (t[i] >= P) {
        float x[8], y[8];
        unpack8(raw[i], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = x[e] * inv;
        *row = codes8(x, y);
      } else {
        *row = shrunk8(*row, shrink);
      }
    }
  }
}

// At most kFew new tokens a sequence: a wave takes one head of a sequence, keys
// or values, and the waves beside it the other heads. The tokens lie in at most
// two blocks, one after the other; the codes that a block held are read only if
// its scale grows.
template <int FORM>
__global__ __launch_bounds__(64 * kWaves) void append_few_kernel(CacheProblem p,
                                                                 const uint16_t* __restrict__ k_new,
                                                                 const uint16_t* __restrict__ v_new,
                                                                 int64_t total) {
  int64_t at = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (at >= total) return;
  const int h = (int)(at % p.hkv);
  at /= p.hkv;
  const bool is_v = at & 1;
  const int b = (int)(at >> 1);
  const int q0 = ld_uniform(p.cu, b), n = ld_uniform(p.cu, b + 1) - q0;
  const int64_t tok0 = ld_uniform(p.cuk, b);
  const int L = ld_uniform(p.cuk, b + 1) - (int)tok0, P = L - n;
  if (n <= 0) return;
  const int lane = threadIdx.x & 63, c = lane & 15, r0 = lane >> 4;
  const uint16_t* src = is_v ? v_new : k_new;
  uint8_t* pool = is_v ? p.v : p.k;
  const int64_t rowb = (int64_t)p.hkv * kHeadDim;       // elements of a token
  const int64_t hoff = (int64_t)h * kHeadDim + 8 * c;
  const int size = FORM == kCacheBlock ? 1 << p.sb_shift : kFew;
  float scale = 1.f;
  if constexpr (FORM == kCacheHead) scale = ld_uniform(is_v ? p.v_head : p.k_head, h);
#pragma unroll 1
  for (int from = P; from < L;) {
    // the new tokens from .. to - 1 of a block
    const int first = FORM == kCacheBlock ? from & -size : from, to = min(first + size, L);
    uint4 raw[kFew / 4];
#pragma unroll
    for (int i = 0; i < kFew / 4; ++i) {
      const int t = from + 4 * i + r0;
      raw[i] = make_uint4(0, 0, 0, 0);
      if (t < to) raw[i] = *(const uint4*)(src + ((int64_t)q0 + t - P) * rowb + hoff);
    }
    float inv = 1.f;
    if constexpr (FORM == kCacheBlock) {
      uint8_t* sp = (is_v ? p.v_block : p.k_block) + (slot_of(p.pm, b, tok0, first) >> p.sb_shift) * p.hkv + h;
      const int before = first < P ? *sp : 0;           // byte of a block that holds tokens
      float amax = 0.f;
#pragma unroll
      for (int i = 0; i < kFew / 4; ++i) {
        float x[8];
        unpack8(raw[i], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float a = fabsf(x[e]);
          amax = fmaxf(amax, a < INFINITY ? a : 0.f);
        }
      }
      const int byte = __builtin_amdgcn_readfirstlane(max(scale_byte(wave_max(amax)), before));
      if (lane == 0) *sp = (uint8_t)byte;
      inv = __uint_as_float((uint32_t)(254 - byte) << 23);   // 2^-e
      if (first < P && byte > before) {
        const float shrink = __uint_as_float((uint32_t)max(127 - (byte - before), 0) << 23);
#pragma unroll 4
        for (int t = first + r0; t < P; t += 4) {
          uint2* row = (uint2*)(pool + slot_of(p.pm, b, tok0, t) * rowb + hoff);
          *row = shrunk8(*row, shrink);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < kFew / 4; ++i) {
      const int t = from + 4 * i + r0;
      if (t >= to) continue;
      const int64_t slot = slot_of(p.pm, b, tok0, t);
      if constexpr (FORM == kCacheBf16) {
        *(uint4*)((uint16_t*)pool + slot * rowb + hoff) = raw[i];
      } else {
        float x[8], y[8];
        unpack8(raw[i], x);
#pragma unroll
        for (int e = 0; e < 8; ++e) y[e] = FORM == kCacheHead ? x[e] / scale : x[e] * inv;
        *(uint2*)(pool + slot * rowb + hoff) = codes8(x, y);
      }
    }
    from = to;
  }
}

template <int FORM>
hipError_t launch(const CacheProblem& p, const uint16_t* k_new, const uint16_t* v_new, hipStream_t s) {
  if (p.max_new <= kFew) {
    const int64_t total = (int64_t)p.batch * 2 * p.hkv, grid = (total + kWaves - 1) / kWaves;
    if (!launchable(grid, 64 * kWaves)) return hipErrorInvalidValue;
    append_few_kernel<FORM><<<(unsigned)grid, 64 * kWaves, 0, s>>>(p, k_new, v_new, total);
    return hipGetLastError();
  }
  // tokens of a sequence lie in at most this many runs of kRows
  const int chunks = (p.max_new + kRows - 2) / kRows + 1;
  const int64_t grid = (int64_t)p.batch * chunks * 2 * p.hkv;
  if (!launchable(grid, 64 * kWaves)) return hipErrorInvalidValue;
  append_kernel<FORM><<<(unsigned)grid, 64 * kWaves, 0, s>>>(p, k_new, v_new, chunks);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_cache_append(const CacheProblem& p, const uint16_t* k_new, const uint16_t* v_new,
                               hipStream_t s) {
  return p.form == kCacheBf16   ? launch<kCacheBf16>(p, k_new, v_new, s)
         : p.form == kCacheHead ? launch<kCacheHead>(p, k_new, v_new, s)
                                : launch<kCacheBlock>(p, k_new, v_new, s);
}

}  // namespace fp2
