// Kernels of the paged KV cache's operators (internal to the library).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "common.h"

namespace fp2 {

enum CacheForm : int32_t {
  kCacheBf16 = 0,    // bf16 rows
  kCacheHead = 1,    // e4m3 codes, one fp32 scale per head
  kCacheBlock = 2    // e4m3 codes, one power-of-two scale per (block of tokens, head)
};

// What every kernel of these operators reads of a call.
struct CacheProblem {
  const uint16_t* q;        // [new tokens, Hq, d] bf16
  const int32_t* cu;        // [batch + 1] new tokens (queries)
  const int32_t* cuk;       // [batch + 1] tokens in the cache, the new ones included
  uint8_t* k;               // [slots, Hkv, d] bf16 or codes
  uint8_t* v;
  PageMap pm;
  const float* k_head;      // kCacheHead: [Hkv]
  const float* v_head;
  uint8_t* k_block;         // kCacheBlock: [slots / sb, Hkv], 2^(byte - 127)
  uint8_t* v_block;
  int32_t batch, hq, hkv, g;
  int32_t form;
  int32_t sb_shift;         // log2 of the tokens per scale
  int32_t sink, window;     // window >= 1; without one: sink 0, window 2^30
  int32_t max_new, max_kv;  // bounds of the lengths
  int32_t splits;           // 0: by the work of the call, n: n parts
  float scale_log2;         // softmax scale * log2(e)
  int32_t heads;            // few rows: heads that the waves of a workgroup take side by side
};

constexpr int kNoWindow = 1 << 30;

// Exponent bytes of a scale 2^(byte - 127): those of fp32.
__device__ __forceinline__ float block_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// A scale is kept in [2^-100, 2^118]: 448 times the largest is a finite bf16,
// and the smallest code times the smallest a normal one.
constexpr int kMinScaleByte = 127 - 100, kMaxScaleByte = 127 + 118;

// The scale of a head's scores (base 2). Never 0, which a masked score, minus
// infinity, would make NaN; at 2^-126 the scores of queries up to 2^80 are below 2^-30.
template <int FORM>
__device__ __forceinline__ float score_scale(const CacheProblem& p, int h) {
  if constexpr (FORM != kCacheHead) return p.scale_log2;
  else return fmaxf(p.scale_log2 * ld_uniform(p.k_head, h), 0x1p-126f);
}

// Byte of the scale for values of at most amax (finite, >= 0): the smallest
// power of two that is at least amax / 448. 448 = 0.875 * 2^9, so it is read
// off the bits of amax = 1.m * 2^x: 2^(x - 8) where 1.m <= 1.75, else twice
// that. Below 2^-92 the lower bound holds.
__device__ __forceinline__ int scale_byte(float amax) {
  const uint32_t u = __float_as_uint(amax);
  const int e = (int)(u >> 23) - 8 + ((u & 0x7fffff) > 0x600000);
  return min(max(e, kMinScaleByte), kMaxScaleByte);
}

// Four values as e4m3 codes (nearest, ties to even, held within +-448) from
// x = the values in units of the scale; NaN where the value itself, `raw`, is
// infinite or NaN.
__device__ __forceinline__ uint32_t e4m3x4(const float (&raw)[4], const float (&x)[4]) {
  float y[4];
  uint32_t bad = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool fin = fabsf(raw[i]) < INFINITY;
    bad |= fin ? 0u : 0x7fu << (8 * i);
    y[i] = fin ? __builtin_amdgcn_fmed3f(x[i], -448.f, 448.f) : 0.f;
  }
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
  w = __builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
  return (uint32_t)w | bad;
}

// Four codes as floats.
__device__ __forceinline__ void e4m3x4_to_f32(uint32_t w, float (&x)[4]) {
  const f32x2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false);
  const f32x2_t hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = lo[0]; x[1] = lo[1]; x[2] = hi[0]; x[3] = hi[1];
}

// Inclusive sum over the lanes of a wave, by the vector ALU's lane shifts (six
// exchanges through LDS take some six times as long).
__device__ __forceinline__ int wave_scan(int v) {
#define FP2_STEP(ctrl, rows) v += __builtin_amdgcn_update_dpp(0, v, ctrl, rows, 0xf, false)
  FP2_STEP(0x111, 0xf);   // row_shr 1, 2, 4, 8: within 16 lanes
  FP2_STEP(0x112, 0xf);
  FP2_STEP(0x114, 0xf);
  FP2_STEP(0x118, 0xf);
  FP2_STEP(0x142, 0xa);   // row_bcast 15: the second and fourth row take the row before
  FP2_STEP(0x143, 0xc);   // row_bcast 31: the upper half takes the lower one
#undef FP2_STEP
  return v;
}

// Keeps the compiler from computing many masks (a pair of scalar registers
// each) before it uses the first: x is needed here.
template <class T>
__device__ __forceinline__ T pinned(T x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Whether a launch of so many workgroups may be made: HIP counts its threads in
// 32 bits. Asked for every kernel of a call before the first of them.
inline bool launchable(int64_t groups, int threads) { return groups * threads < 1ll << 32; }

// Partial outputs of sequences whose keys are cut into parts.
struct CachePartials {
  float* o;                 // [slots, rows, d]
  float* ml;                // [slots, rows, 2] {running maximum (base 2), denominator}
  int32_t* at;              // few rows, equal shares: [batch, 2] {first share, parts} of a sequence;
                            // cross attention of many rows: what each workgroup leaves to join
};

// At most this many packed rows (new tokens times heads of a group) a sequence
// go to the kernels of few rows, which read each key once for all of them. With
// 64 rows attention over 30K tokens takes 36 us there and 57 as a short prompt,
// of 8 sequences 99 and 285; with 900 tokens both take 25.
constexpr int kFewRows = 64;

// Slots, and packed rows of each, of the partial outputs of a call.
void cache_decode_partials(const CacheProblem& p, int64_t* slots, int* rows);
void cache_extend_partials(const CacheProblem& p, int64_t* slots, int* rows);

// Floats of the partial weights of a call.
int64_t cache_weights_partials(const CacheProblem& p);

// hipErrorInvalidValue, and nothing launched, where the call is too large for it.
hipError_t launch_cache_append(const CacheProblem& p, const uint16_t* k_new, const uint16_t* v_new,
                               hipStream_t s);
hipError_t launch_cache_decode(const CacheProblem& p, const CachePartials& part, uint16_t* out,
                               float* lse, hipStream_t s, bool cross = false);
hipError_t launch_cache_extend(const CacheProblem& p, const CachePartials& part, uint16_t* out,
                               float* lse, hipStream_t s);
hipError_t launch_cache_weights(const CacheProblem& p, const float* lse, const float* in, float* out,
                                int64_t stride, float* part, hipStream_t s);
hipError_t launch_cache_evict(const CacheProblem& p, const PageMap& to, int budget, int recent,
                              const float* weights, int64_t stride, float* weights_out,
                              int64_t out_stride, int32_t* kept, int32_t* cu_out, hipStream_t s);

}  // namespace fp2
