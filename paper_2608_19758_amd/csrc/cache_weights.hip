// The attention weight that cached tokens received of a call's queries: for
// each KV head, the sum over the new tokens and the g query heads of
// exp(scale q.k - lse), with the log-sum-exp that the attention returned.
//
// A workgroup takes 256 keys of a (sequence, head), a wave 64 of them as the
// A operand of S^T = K Q^T (v_mfma_f32_32x32x16_bf16), which stay in registers
// while the packed query rows that see them pass by, 32 at a time, through
// LDS. A lane then holds query l % 32 and 32 keys and adds its probabilities
// in fp32; at the end the 32 sums of a lane are exchanged and added over the
// lanes, half of them a step (31 exchanges). Each sum has one writer: no
// atomics, and the same result in every run.
//
// Few rows: bound by the keys' bytes. Prompts: by the products and the
// exponentials, half of the attention's work.
#include "cache.h"

namespace fp2 {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kWaves = 4;
constexpr int kKeys = 64;                 // of a wave
constexpr int kRows = 32;                 // packed query rows of a step

__device__ __forceinline__ int place(int r, int c) { return r * 16 + (c ^ (r & 15)); }

struct Shared {
  uint4 q[2][kRows * 16];
  float lse[2][kRows];
};

template <int FORM>
__global__ __launch_bounds__(64 * kWaves) void weights_kernel(CacheProblem p,
                                                              const float* __restrict__ lse,
                                                              const float* in, float* out,
                                                              int64_t stride) {
  constexpr bool kBf16 = FORM == kCacheBf16;
  constexpr int ESZ = kBf16 ? 2 : 1;
  __shared__ Shared sh;
  int64_t at = blockIdx.x;
  const int h = (int)(at % p.hkv);
  at /= p.hkv;
  const int b = (int)(at % p.batch), c0 = (int)(at / p.batch) * kWaves * kKeys;
  const int64_t tok0 = ld_uniform(p.cuk, b);
  const int L = ld_uniform(p.cuk, b + 1) - (int)tok0;
  if (c0 >= L) return;
  const int q0 = ld_uniform(p.cu, b), Lq = ld_uniform(p.cu, b + 1) - q0;
  const int P = L - Lq, rows = Lq * p.g;

  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const int k0 = c0 + kKeys * w;              // the wave's first key

  // rows of the workgroup's keys: from the first that lies at or behind them
  // to the last whose window reaches them (all where they are first tokens)
  const int kend = min(c0 + kWaves * kKeys, L) - 1;
  const int i_lo = max(c0 - P, 0);
  const int i_hi = c0 < p.sink ? Lq - 1 : min((int64_t)Lq - 1, (int64_t)kend + p.window - 1 - P);
  const int t_lo = i_lo * p.g / kRows, t_hi = i_hi >= i_lo ? (i_hi * p.g + p.g - 1) / kRows + 1 : t_lo;

  float acc[32];
#pragma unroll
  for (int i = 0; i < 32; ++i) acc[i] = 0.f;

  if (t_lo < t_hi) {
    const int64_t rowb = (int64_t)p.hkv * kHeadDim * ESZ;
    const uint8_t* K = p.k + (int64_t)h * kHeadDim * ESZ;
    bf16x8_t a[2][8];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      const int64_t slot = slot_of(p.pm, b, tok0, min(k0 + 32 * u + l32, L - 1));
      const uint8_t* row = K + slot * rowb;
      if constexpr (kBf16) {
#pragma unroll
        for (int s = 0; s < 8; ++s)
          a[u][s] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(row + 32 * s + 16 * half));
      } else {
        float sc = 1.f;
        if constexpr (FORM == kCacheBlock) sc = block_scale(p.k_block[(slot >> p.sb_shift) * p.hkv + h]);
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint4 x = *(const uint4*)(row + 32 * j + 16 * half);
          const uint32_t d[4] = {x.x, x.y, x.z, x.w};
          b2 y[8];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            y[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)d[i], sc, false);
            y[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)d[i], sc, true);
          }
          const b2 y0[4] = {y[0], y[1], y[2], y[3]}, y1[4] = {y[4], y[5], y[6], y[7]};
          a[u][2 * j] = __builtin_bit_cast(bf16x8_t, y0);
          a[u][2 * j + 1] = __builtin_bit_cast(bf16x8_t, y1);
        }
      }
    }
    const float cs = p.scale_log2 * (FORM == kCacheHead ? ld_uniform(p.k_head, h) : 1.f);

    // staging: thread -> row tid / 8 of a step, two 16-byte chunks
    const int r = tid >> 3, c = 2 * (tid & 7);
    uint4 x[2];
    float ls = 0.f;
    auto load = [&](int t) {
      const int pr = min(kRows * t + r, rows - 1);
      const uint16_t* src = p.q + ((int64_t)(q0 + pr / p.g) * p.hq + h * p.g + pr % p.g) * kHeadDim;
      x[0] = *(const uint4*)(src + 8 * c);
      x[1] = *(const uint4*)(src + 8 * c + 8);
      if (tid < kRows) {
        const int pl = min(kRows * t + tid, rows - 1);
        ls = lse[(int64_t)(q0 + pl / p.g) * p.hq + h * p.g + pl % p.g] * kLog2e;
      }
    };
    auto write = [&](int t) {
      sh.q[t & 1][place(r, c)] = x[0];
      sh.q[t & 1][place(r, c + 1)] = x[1];
      if (tid < kRows) sh.lse[t & 1][tid] = ls;
    };
    load(t_lo);
    write(t_lo);
    if (t_lo + 1 < t_hi) load(t_lo + 1);
#pragma unroll 1
    for (int t = t_lo; t < t_hi; ++t) {
      lds_barrier();
      if (t + 1 < t_hi) write(t + 1);
      if (t + 2 < t_hi) load(t + 2);
      const int pr = kRows * t + l32;
      const int pos = pr < rows ? P + pr / p.g : -1;     // a row past the last sees nothing
      const int first = P + kRows * t / p.g, last = P + min(kRows * t + kRows, rows) / p.g;
      if (last < k0) continue;                           // (uniform) none of the wave's keys is seen
      const float ref = sh.lse[t & 1][l32];
      f32x16_t s[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) s[u] = f32x16_t{};
#pragma unroll
      for (int st = 0; st < 8; ++st) {
        // dimensions 16 st + 8 half of bf16 keys, 32 (st / 2) + 16 half + 8 (st % 2) of codes
        const int ch = kBf16 ? 2 * st + half : 4 * (st >> 1) + 2 * half + (st & 1);
        const bf16x8_t q = __builtin_bit_cast(bf16x8_t, sh.q[t & 1][place(l32, ch)]);
#pragma unroll
        for (int u = 0; u < 2; ++u)
          s[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(a[u][st], q, s[u], 0, 0, 0);
      }
      const bool masked = k0 + kKeys - 1 > first || kRows * t + kRows > rows ||
                          (k0 <= last - p.window && k0 + kKeys > p.sink);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          float v = fast_exp2(fmaf(s[u][e], cs, -ref));
          if (masked) {
            const int key = k0 + 32 * u + 8 * (e >> 2) + 4 * half + (e & 3);
            v = key <= pos && (key < p.sink || key > pos - p.window) ? v : 0.f;
          }
          acc[16 * u + e] += v;
        }
    }
  }
  // sums over the 32 lanes of a half: lane l32 keeps that of element l32
#pragma unroll
  for (int n = 16; n > 0; n >>= 1) {
    const bool up = l32 & n;
#pragma unroll
    for (int j = 0; j < n; ++j) {
      const float send = up ? acc[j] : acc[j + n], keep = up ? acc[j + n] : acc[j];
      acc[j] = keep + __shfl_xor(send, n, 64);
    }
  }
  const int u = l32 >> 4, e = l32 & 15;
  const int key = k0 + 32 * u + 8 * (e >> 2) + 4 * half + (e & 3);
  if (key < L) {
    const int64_t to = ((int64_t)b * p.hkv + h) * stride + key;
    out[to] = (in ? in[to] : 0.f) + acc[0];
  }
}

}  // namespace

hipError_t launch_cache_weights(const CacheProblem& p, const float* lse, const float* in, float* out,
                                int64_t stride, hipStream_t s) {
  const int64_t grid = (int64_t)p.batch * p.hkv * ((p.max_kv + kWaves * kKeys - 1) / (kWaves * kKeys));
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  if (p.form == kCacheBf16)
    weights_kernel<kCacheBf16><<<(unsigned)grid, 64 * kWaves, 0, s>>>(p, lse, in, out, stride);
  else if (p.form == kCacheHead)
    weights_kernel<kCacheHead><<<(unsigned)grid, 64 * kWaves, 0, s>>>(p, lse, in, out, stride);
  else
    weights_kernel<kCacheBlock><<<(unsigned)grid, 64 * kWaves, 0, s>>>(p, lse, in, out, stride);
  return hipGetLastError();
}

}  // namespace fp2
