// New tokens' queries, keys and values in one pass: queries and keys turned by
// their positions, keys and values written into a paged cache in its type.
//
// A workgroup takes a run of 64 consecutive tokens of one sequence (128 where a
// scale stands for as many), works out their turns once in LDS and goes through
// its heads with them, a wave a head: queries out, keys and values to their
// slots. With a scale per block of tokens the block lies in one wave, so its
// largest value is a wave's maximum; 2^e, e = ceil(log2(amax / 448)) of the
// turned keys, makes x 2^-e exact and a code is rounded once, from fp32. Where a
// block holds tokens already its scale never falls; if it grows their codes are
// rounded again.
//
// Bound by memory: 256 bytes a row in, 256 or 128 out.
//
// Few new tokens a sequence (a decode step): a wave has one head of a sequence
// to itself and works its turns out in registers.
#include "rotary_rows.h"

namespace fp2 {

namespace {

constexpr int kWaves = 8;
constexpr int kFew = 16;       // new tokens of a sequence that a wave takes alone

struct New {
  const uint16_t* k;
  const uint16_t* v;
  int64_t k_stride, v_stride;
  const int32_t* positions;   // of the new tokens; null: their indexes in the sequence
};

// A sequence's part of the call.
struct Seq {
  int b, q0, n, L, P;
  int64_t tok0;
  __device__ __forceinline__ Seq(const CacheProblem& p, int b_) : b(b_) {
    q0 = ld_uniform(p.cu, b);
    n = ld_uniform(p.cu, b + 1) - q0;
    tok0 = ld_uniform(p.cuk, b);
    L = ld_uniform(p.cuk, b + 1) - (int)tok0;
    P = L - n;
  }
  __device__ __forceinline__ int64_t row(int t) const { return (int64_t)q0 + t - P; }
  __device__ __forceinline__ int position(const New& x, int t) const { return x.positions ? x.positions[row(t)] : t; }
};

// Codes of a lane's sixteen values times a power of two.
__device__ __forceinline__ void shrink16(uint32_t (&w)[4], float by) {
  float x[16], y[16];
  unpack16(w, x);
#pragma unroll
  for (int e = 0; e < 16; ++e) y[e] = x[e] * by;
  pack16(x, y, w);
}
__device__ __forceinline__ void shrink_row(uint8_t* row, int lane, float by) {
  uint4* at = (uint4*)(row + 16 * (lane & 7));
  uint32_t w[4] = {at->x, at->y, at->z, at->w};
  shrink16(w, by);
  *at = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ float power_down(int from, int to) {   // 2^(from - to), to >= from
  return __uint_as_float((uint32_t)max(127 - (to - from), 0) << 23);
}

// SB: tokens of a scale (kCacheBlock), else 0.
template <int FORM, int SB, int PLACE>
__global__ __launch_bounds__(64 * kWaves) void append_rotary_kernel(CacheProblem p, Rotary r, RotaryRows q, New x,
                                                                    int chunks, int groups) {
  constexpr int TOK = SB == 128 ? 128 : 64;      // tokens of a workgroup
  constexpr int RUN = SB > 32 ? SB : 32;         // tokens whose loads a wave has in flight
  constexpr int N = RUN / kPass;
  constexpr int ESZ = FORM == kCacheBf16 ? 2 : 1;
  __shared__ TurnTable<TOK> table;
  __shared__ int64_t s_slot[TOK];
  int64_t at = blockIdx.x;
  const int group = (int)(at % groups);
  at /= groups;
  const int ck = (int)(at % chunks);
  const Seq s(p, (int)(at / chunks));
  const int first = (s.P / TOK + ck) * TOK;
  if (s.n <= 0 || first >= s.L) return;
  table.fill(r, 64 * kWaves, [&](int i) { return s.position(x, min(max(first + i, s.P), s.L - 1)); });
  for (int i = threadIdx.x; i < TOK; i += 64 * kWaves) s_slot[i] = slot_of(p.pm, s.b, s.tok0, min(first + i, s.L - 1));
  __syncthreads();

  const int lane = threadIdx.x & 63, r0 = lane / kLaneRow;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const LaneRow<PLACE> l(lane, r.dim);
  const int64_t rowb = (int64_t)p.hkv * kHeadDim;
  const int jobs = 2 * p.hkv + q.heads;
#pragma unroll 1
  for (int j = group * kWaves + w; j < jobs; j += groups * kWaves) {
    const bool is_q = j >= 2 * p.hkv, is_v = !is_q && j >= p.hkv;
    const int h = is_q ? j - 2 * p.hkv : is_v ? j - p.hkv : j;
    const uint16_t* src = (is_q ? q.x : is_v ? x.v : x.k) + h * kHeadDim;
    const int64_t stride = is_q ? q.x_stride : is_v ? x.v_stride : x.k_stride;
    uint8_t* pool = (is_v ? p.v : p.k) + h * kHeadDim * ESZ;
#pragma unroll 1
    for (int g = 0; g < TOK; g += RUN) {
      if (first + g >= s.L || first + g + RUN <= s.P) continue;
      uint32_t raw[N][8];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int t = first + g + kPass * i + r0;
        load_part(l, src + s.row(min(max(t, s.P), s.L - 1)) * stride, raw[i]);
      }
      if (is_q) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int k = g + kPass * i + r0, t = first + k;
          Turns y;
          table.get(k, l.c, y);
          turn_and_store(l, y, raw[i], q, s.row(t), h, t >= s.P && t < s.L);
        }
        continue;
      }
      auto values = [&](int i, float (&z)[16]) {   // of pass i, turned
        unpack16(raw[i], z);
        if (!is_v) {
          Turns y;
          table.get(g + kPass * i + r0, l.c, y);
          turn16(l, y, z);
        }
      };
      if constexpr (FORM != kCacheBlock) {
        float scale = 1.f;
        if constexpr (FORM == kCacheHead) scale = ld_uniform(is_v ? p.v_head : p.k_head, h);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int k = g + kPass * i + r0, t = first + k;
          float z[16];
          values(i, z);
          if (t < s.P || t >= s.L) continue;
          uint8_t* row = pool + s_slot[k] * rowb * ESZ;
          if constexpr (FORM == kCacheBf16) {
            uint32_t c[8];
            pack16(z, c);
            store_part(l, (uint16_t*)row, c);
          } else {
            float u[16];
            uint32_t c[4];
#pragma unroll
            for (int e = 0; e < 16; ++e) u[e] = z[e] / scale;
            pack16(z, u, c);
            store_part(l, row, c);
          }
        }
      } else {
        constexpr int PER = SB / kPass;              // passes of a block
#pragma unroll
        for (int i0 = 0; i0 < N; i0 += PER) {
          const int kb = g + kPass * i0, tb = first + kb;   // the block's first token
          if (tb >= s.L || tb + SB <= s.P) continue;
          uint8_t* sp = (is_v ? p.v_block : p.k_block) + (s_slot[kb] >> p.sb_shift) * p.hkv + h;
          const int before = tb < s.P ? *sp : 0;     // byte of a block that holds tokens
          float amax = 0.f;
#pragma unroll
          for (int i = i0; i < i0 + PER; ++i) {      // (rows outside the new tokens repeat one of them)
            float z[16];
            values(i, z);
            amax = fmaxf(amax, largest16(z));
          }
          const int byte = __builtin_amdgcn_readfirstlane(max(scale_byte(wave_max(amax)), before));
          if (lane == 0) *sp = (uint8_t)byte;
          const float inv = __uint_as_float((uint32_t)(254 - byte) << 23);   // 2^-e
          if (tb < s.P && byte > before) {
            const float by = power_down(before, byte);
            for (int t = tb + r0; t < min(s.P, tb + SB); t += kPass)
              shrink_row(pool + s_slot[t - first] * rowb, lane, by);
          }
#pragma unroll
          for (int i = i0; i < i0 + PER; ++i) {
            const int k = g + kPass * i + r0, t = first + k;
            float z[16], u[16];
            uint32_t c[4];
            // turned once more: kept from above the values would take 16 registers a pass
#pragma unroll
            for (int e = 0; e < 8; ++e) raw[i][e] = (uint32_t)pinned((int)raw[i][e]);
            values(i, z);
#pragma unroll
            for (int e = 0; e < 16; ++e) u[e] = z[e] * inv;
            pack16(z, u, c);
            if (t >= s.P && t < s.L) store_part(l, pool + s_slot[k] * rowb, c);
          }
        }
      }
    }
  }
}

// At most kFew new tokens a sequence. They lie in at most two blocks, one after
// the other; the codes that a block held are read only if its scale grows.
template <int FORM, int PLACE>
__global__ __launch_bounds__(64 * kWaves) void append_rotary_few_kernel(CacheProblem p, Rotary r, RotaryRows q, New x,
                                                                        int64_t total) {
  constexpr int ESZ = FORM == kCacheBf16 ? 2 : 1;
  constexpr int N = kFew / kPass;
  const int64_t at = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (at >= total) return;
  const int jobs = 2 * p.hkv + q.heads, j = (int)(at % jobs);
  const Seq s(p, (int)(at / jobs));
  if (s.n <= 0) return;
  const bool is_q = j >= 2 * p.hkv, is_v = !is_q && j >= p.hkv;
  const int h = is_q ? j - 2 * p.hkv : is_v ? j - p.hkv : j;
  const int lane = threadIdx.x & 63, r0 = lane / kLaneRow;
  const uint16_t* src = (is_q ? q.x : is_v ? x.v : x.k) + h * kHeadDim;
  const int64_t stride = is_q ? q.x_stride : is_v ? x.v_stride : x.k_stride;
  const int64_t rowb = (int64_t)p.hkv * kHeadDim;
  uint8_t* pool = (is_v ? p.v : p.k) + h * kHeadDim * ESZ;
  const LaneRow<PLACE> l(lane, r.dim);
  const Freqs freqs = l.freqs(r);
  const int size = FORM == kCacheBlock && !is_q ? 1 << p.sb_shift : kFew;
  float scale = 1.f;
  if constexpr (FORM == kCacheHead)
    if (!is_q) scale = ld_uniform(is_v ? p.v_head : p.k_head, h);
#pragma unroll 1
  for (int from = s.P; from < s.L;) {
    // the new tokens from .. to - 1 of a block
    const int first = FORM == kCacheBlock && !is_q ? from & -size : from, to = min(min(first + size, s.L), from + kFew);
    float z[N][16];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (from + kPass * i >= to) break;
      const int t = min(from + kPass * i + r0, to - 1);
      uint32_t raw[8];
      load_part(l, src + s.row(t) * stride, raw);
      if (!is_v) {
        Turns y;
        l.turns(r, freqs, s.position(x, t), y);
        if (is_q) {
          turn_and_store(l, y, raw, q, s.row(t), h, from + kPass * i + r0 < to);
          continue;
        }
        unpack16(raw, z[i]);
        turn16(l, y, z[i]);
      } else {
        unpack16(raw, z[i]);
      }
    }
    if (!is_q) {
      float inv = 1.f;
      if constexpr (FORM == kCacheBlock) {
        uint8_t* sp = (is_v ? p.v_block : p.k_block) + (slot_of(p.pm, s.b, s.tok0, first) >> p.sb_shift) * p.hkv + h;
        const int before = first < s.P ? *sp : 0;       // byte of a block that holds tokens
        float amax = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          if (from + kPass * i >= to) break;
          amax = fmaxf(amax, largest16(z[i]));
        }
        const int byte = __builtin_amdgcn_readfirstlane(max(scale_byte(wave_max(amax)), before));
        if (lane == 0) *sp = (uint8_t)byte;
        inv = __uint_as_float((uint32_t)(254 - byte) << 23);   // 2^-e
        if (first < s.P && byte > before) {
          const float by = power_down(before, byte);
#pragma unroll 4
          for (int t = first + r0; t < s.P; t += kPass) shrink_row(pool + slot_of(p.pm, s.b, s.tok0, t) * rowb, lane, by);
        }
      }
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int t = from + kPass * i + r0;
        if (t >= to) continue;
        uint8_t* row = pool + slot_of(p.pm, s.b, s.tok0, t) * rowb * ESZ;
        if constexpr (FORM == kCacheBf16) {
          uint32_t c[8];
          pack16(z[i], c);
          store_part(l, (uint16_t*)row, c);
        } else {
          float u[16];
          uint32_t c[4];
#pragma unroll
          for (int e = 0; e < 16; ++e) u[e] = FORM == kCacheHead ? z[i][e] / scale : z[i][e] * inv;
          pack16(z[i], u, c);
          store_part(l, row, c);
        }
      }
    }
    from = to;
  }
}

template <int FORM, int SB, int PLACE>
hipError_t launch(const CacheProblem& p, const Rotary& r, const RotaryRows& q, const New& x, hipStream_t s) {
  const int jobs = 2 * p.hkv + q.heads;
  if (p.max_new <= kFew) {
    const int64_t total = (int64_t)p.batch * jobs, grid = (total + kWaves - 1) / kWaves;
    if (!launchable(grid, 64 * kWaves)) return hipErrorInvalidValue;
    append_rotary_few_kernel<FORM, PLACE><<<(unsigned)grid, 64 * kWaves, 0, s>>>(p, r, q, x, total);
    return hipGetLastError();
  }
  constexpr int TOK = SB == 128 ? 128 : 64;
  // tokens of a sequence lie in at most this many runs of TOK
  const int chunks = (p.max_new + TOK - 2) / TOK + 1;
  // heads are dealt to several workgroups where the runs alone would not fill the chip twice
  int groups = 1;
  while (groups * kWaves < jobs && (int64_t)p.batch * chunks * groups < 512) groups *= 2;
  const int64_t grid = (int64_t)p.batch * chunks * groups;
  if (!launchable(grid, 64 * kWaves)) return hipErrorInvalidValue;
  append_rotary_kernel<FORM, SB, PLACE><<<(unsigned)grid, 64 * kWaves, 0, s>>>(p, r, q, x, chunks, groups);
  return hipGetLastError();
}

template <int PLACE>
hipError_t launch_form(const CacheProblem& p, const Rotary& r, const RotaryRows& q, const New& x, hipStream_t s) {
  if (p.form == kCacheBf16) return launch<kCacheBf16, 0, PLACE>(p, r, q, x, s);
  if (p.form == kCacheHead) return launch<kCacheHead, 0, PLACE>(p, r, q, x, s);
  return p.sb_shift == 4   ? launch<kCacheBlock, 16, PLACE>(p, r, q, x, s)
         : p.sb_shift == 5 ? launch<kCacheBlock, 32, PLACE>(p, r, q, x, s)
         : p.sb_shift == 6 ? launch<kCacheBlock, 64, PLACE>(p, r, q, x, s)
                           : launch<kCacheBlock, 128, PLACE>(p, r, q, x, s);
}

}  // namespace

hipError_t launch_cache_append_rotary(const CacheProblem& p, const Rotary& r, bool interleaved, const RotaryRows& q,
                                      const uint16_t* k_new, int64_t k_stride, const uint16_t* v_new, int64_t v_stride,
                                      const int32_t* positions, hipStream_t s) {
  const New x{k_new, v_new, k_stride, v_stride, positions};
  const PairPlace place = place_of(r.dim, interleaved);
  return place == kPairs    ? launch_form<kPairs>(p, r, q, x, s)
         : place == kHalves ? launch_form<kHalves>(p, r, q, x, s)
                            : launch_form<kOdd>(p, r, q, x, s);
}

}  // namespace fp2
