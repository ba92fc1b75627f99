// Tokens of a paged cache read back as bf16 rows, and moved to other pages or
// positions.
//
// Both take a run of tokens of one sequence and head, keys or values, a wave
// each, eight lanes a row; the waves beside it take the other heads of the same
// tokens, so memory is read in long runs. What a wave turns keys by is worked
// out in registers: for a run that moves as one, once; else for each row.
//
// Moving: keys of codes with a scale per head keep the scale (a turn is linear:
// the codes' numbers are turned and rounded again, held within +-448); a block
// with a scale of its own gets the one that its turned keys need, and each code
// is rounded once, from fp32. Rows that are not turned are copied, codes and
// scales. A wave holds whole blocks before it writes, so the pages may be the
// same (in place).
//
// Bound by memory: 128 or 256 bytes a row in, and 256 (reading) or as many out.
#include <type_traits>

#include "rotary_rows.h"

namespace fp2 {

namespace {

constexpr int kWaves = 8;

// ---- reading

template <int FORM, int PLACE, bool TURN>
__global__ __launch_bounds__(64 * kWaves) void read_kernel(CacheProblem p, Rotary r, const int32_t* __restrict__ positions,
                                                           uint16_t* __restrict__ k_out, uint16_t* __restrict__ v_out,
                                                           int runs, int64_t total) {
  constexpr int RUN = 32, N = RUN / kPass;
  constexpr int ESZ = FORM == kCacheBf16 ? 2 : 1;
  typedef std::conditional_t<FORM == kCacheBf16, uint16_t, uint8_t> elem_t;
  int64_t at = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (at >= total) return;
  const int h = (int)(at % p.hkv);
  at /= p.hkv;
  const int kinds = (k_out != nullptr) + (v_out != nullptr);
  const bool is_v = !k_out || (kinds == 2 && (at & 1));
  at /= kinds;
  const int b = (int)(at / runs), i0 = (int)(at % runs) * RUN;
  const int q0 = ld_uniform(p.cu, b), n = ld_uniform(p.cu, b + 1) - q0;
  const int L = ld_uniform(p.cuk, b + 1) - ld_uniform(p.cuk, b), P = L - n;
  if (i0 >= n) return;
  const int lane = threadIdx.x & 63, r0 = lane / kLaneRow;
  const LaneRow<PLACE> l(lane, r.dim);
  const int64_t slot_l = slot_of(p.pm, b, 0, P + min(i0 + (lane & (RUN - 1)), n - 1));
  const uint8_t* pool = is_v ? p.v : p.k;
  const uint8_t* scales = is_v ? p.v_block : p.k_block;
  uint16_t* out = is_v ? v_out : k_out;
  uint32_t raw[N][4 * ESZ], byte[N];
  int pos[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int64_t slot = __shfl(slot_l, kPass * i + r0, 64);
    load_part(l, (const elem_t*)pool + (slot * p.hkv + h) * kHeadDim, raw[i]);
    if constexpr (FORM == kCacheBlock) byte[i] = scales[(slot >> p.sb_shift) * p.hkv + h];
    const int t = min(i0 + kPass * i + r0, n - 1);
    pos[i] = !TURN || is_v ? 0 : positions ? positions[(int64_t)q0 + t] : P + t;
  }
  Freqs freqs{};
  if (TURN && !is_v) freqs = l.freqs(r);
  float scale = 1.f;
  if constexpr (FORM == kCacheHead) scale = ld_uniform(is_v ? p.v_head : p.k_head, h);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int t = i0 + kPass * i + r0;
    if (t >= n) continue;
    uint16_t* row = out + (((int64_t)q0 + t) * p.hkv + h) * kHeadDim;
    if constexpr (FORM == kCacheBf16 && !TURN) {
      store_part(l, row, raw[i]);
    } else {
      float x[16];
      unpack16(raw[i], x);
      if constexpr (FORM == kCacheHead || FORM == kCacheBlock) {
        const float by = FORM == kCacheHead ? scale : block_scale(byte[i]);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] *= by;
      }
      if (TURN && !is_v) {
        Turns y;
        l.turns(r, freqs, pos[i], y);
        turn16(l, y, x);
      }
      uint32_t c[8];
      pack16(x, c);
      store_part(l, row, c);
    }
  }
}

// ---- moving

// SB: tokens of a scale (kCacheBlock), else 0. TURN: 0 rows as they are, 1 a
// sequence's head moves as one, 2 every token by its own number of positions.
template <int FORM, int SB, int PLACE, int TURN>
__global__ __launch_bounds__(64 * kWaves) void move_tokens_kernel(CacheProblem p, Rotary r, Moves m, PageMap to, int kinds,
                                                                  int runs, int64_t total) {
  constexpr int RUN = SB > 32 ? SB : 32, N = RUN / kPass;
  constexpr int ESZ = FORM == kCacheBf16 ? 2 : 1;
  typedef std::conditional_t<FORM == kCacheBf16, uint16_t, uint8_t> elem_t;
  int64_t at = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (at >= total) return;
  const int h = (int)(at % p.hkv);
  at /= p.hkv;
  const bool is_v = kinds == 2 && (at & 1);
  at /= kinds;
  const int b = (int)(at / runs), first = (int)(at % runs) * RUN;
  const int L = ld_uniform(p.cuk, b + 1) - ld_uniform(p.cuk, b);
  if (first >= L) return;
  const int lane = threadIdx.x & 63, r0 = lane / kLaneRow;
  // slots of the rows: every lane looks up some, the loads below ask it
  constexpr int LOOK = (RUN + 63) / 64;
  int64_t from[LOOK], dest[LOOK];
#pragma unroll
  for (int i = 0; i < LOOK; ++i) {
    const int t = min(first + 64 * i + (RUN < 64 ? lane & (RUN - 1) : lane), L - 1);
    from[i] = slot_of(p.pm, b, 0, t);
    dest[i] = to.table ? slot_of(to, b, 0, t) : from[i];
  }
  uint8_t* pool = is_v ? p.v : p.k;
  uint8_t* scales = is_v ? p.v_block : p.k_block;
  const LaneRow<PLACE> l(lane, r.dim);
  uint32_t raw[N][4 * ESZ], old[N];
  int by[N];
  const int64_t mh = TURN && !is_v ? b * m.batch + h * m.head : 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int64_t slot = __shfl(from[kPass * i / 64], (kPass * i + r0) & 63, 64);
    load_part(l, (const elem_t*)pool + (slot * p.hkv + h) * kHeadDim, raw[i]);
    if constexpr (FORM == kCacheBlock) old[i] = scales[(slot >> p.sb_shift) * p.hkv + h];
    if constexpr (TURN == 2) by[i] = is_v ? 0 : m.by[mh + min(first + kPass * i + r0, L - 1) * m.token];
  }
  auto row_at = [&](int i) {
    const int64_t slot = __shfl(dest[kPass * i / 64], (kPass * i + r0) & 63, 64);
    return (elem_t*)pool + (slot * p.hkv + h) * kHeadDim;
  };
  if (TURN == 0 || is_v) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      elem_t* row = row_at(i);
      if (first + kPass * i + r0 < L) store_part(l, row, raw[i]);
      if constexpr (FORM == kCacheBlock) {
        const int64_t slot = __shfl(dest[kPass * i / 64], kPass * i & 63, 64);
        if (kPass * i % SB == 0 && lane == 0 && first + kPass * i < L)
          scales[(slot >> p.sb_shift) * p.hkv + h] = (uint8_t)old[i];
      }
    }
    return;
  }
  if constexpr (TURN != 0) {
    const Freqs freqs = l.freqs(r);
    Turns one;
    if constexpr (TURN == 1) l.turns(r, freqs, m.by[mh], one);
    auto values = [&](int i, float (&x)[16]) {   // of pass i, turned; with a scale per head in units of it
      unpack16(raw[i], x);
      if constexpr (FORM == kCacheBlock) {
        const float f = block_scale(old[i]);
#pragma unroll
        for (int e = 0; e < 16; ++e) x[e] *= f;
      }
      if constexpr (TURN == 1) {
        turn16(l, one, x);
      } else {
        Turns y;
        l.turns(r, freqs, by[i], y);
        turn16(l, y, x);
      }
    };
    if constexpr (FORM != kCacheBlock) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        float x[16];
        uint32_t c[4 * ESZ];
        values(i, x);
        if constexpr (FORM == kCacheBf16) pack16(x, c);
        else pack16(x, x, c);
        elem_t* row = row_at(i);
        if (first + kPass * i + r0 < L) store_part(l, row, c);
      }
    } else {
      constexpr int PER = SB / kPass;
#pragma unroll
      for (int i0 = 0; i0 < N; i0 += PER) {
        float amax = 0.f;
#pragma unroll
        for (int i = i0; i < i0 + PER; ++i) {       // (rows behind the last repeat it)
          float x[16];
          values(i, x);
          amax = fmaxf(amax, largest16(x));
        }
        const int byte = __builtin_amdgcn_readfirstlane(scale_byte(wave_max(amax)));
        const int64_t slot = __shfl(dest[kPass * i0 / 64], kPass * i0 & 63, 64);
        if (lane == 0 && first + kPass * i0 < L) scales[(slot >> p.sb_shift) * p.hkv + h] = (uint8_t)byte;
        const float inv = __uint_as_float((uint32_t)(254 - byte) << 23);   // 2^-e
#pragma unroll
        for (int i = i0; i < i0 + PER; ++i) {
          float x[16], u[16];
          uint32_t c[4];
          // turned once more: kept from above the values would take 16 registers a pass
#pragma unroll
          for (int e = 0; e < 4; ++e) raw[i][e] = (uint32_t)pinned((int)raw[i][e]);
          values(i, x);
#pragma unroll
          for (int e = 0; e < 16; ++e) u[e] = x[e] * inv;
          pack16(x, u, c);
          elem_t* row = row_at(i);
          if (first + kPass * i + r0 < L) store_part(l, row, c);
        }
      }
    }
  }
}

template <int FORM, int PLACE, bool TURN>
hipError_t launch_read(const CacheProblem& p, const Rotary& r, const int32_t* positions, uint16_t* k_out, uint16_t* v_out,
                       hipStream_t s) {
  const int runs = (p.max_new + 31) / 32, kinds = (k_out != nullptr) + (v_out != nullptr);
  const int64_t total = (int64_t)p.batch * runs * kinds * p.hkv, grid = (total + kWaves - 1) / kWaves;
  if (!launchable(grid, 64 * kWaves)) return hipErrorInvalidValue;
  read_kernel<FORM, PLACE, TURN><<<(unsigned)grid, 64 * kWaves, 0, s>>>(p, r, positions, k_out, v_out, runs, total);
  return hipGetLastError();
}

template <int FORM, int SB, int PLACE, int TURN>
hipError_t launch_move(const CacheProblem& p, const Rotary& r, const Moves& m, const PageMap& to, hipStream_t s) {
  constexpr int RUN = SB > 32 ? SB : 32;
  const int runs = (p.max_kv + RUN - 1) / RUN, kinds = to.table ? 2 : 1;
  const int64_t total = (int64_t)p.batch * runs * kinds * p.hkv, grid = (total + kWaves - 1) / kWaves;
  if (!launchable(grid, 64 * kWaves)) return hipErrorInvalidValue;
  move_tokens_kernel<FORM, SB, PLACE, TURN><<<(unsigned)grid, 64 * kWaves, 0, s>>>(p, r, m, to, kinds, runs, total);
  return hipGetLastError();
}

template <int PLACE, int TURN>
hipError_t launch_move_form(const CacheProblem& p, const Rotary& r, const Moves& m, const PageMap& to, hipStream_t s) {
  if (p.form == kCacheBf16) return launch_move<kCacheBf16, 0, PLACE, TURN>(p, r, m, to, s);
  if (p.form == kCacheHead) return launch_move<kCacheHead, 0, PLACE, TURN>(p, r, m, to, s);
  return p.sb_shift == 4   ? launch_move<kCacheBlock, 16, PLACE, TURN>(p, r, m, to, s)
         : p.sb_shift == 5 ? launch_move<kCacheBlock, 32, PLACE, TURN>(p, r, m, to, s)
         : p.sb_shift == 6 ? launch_move<kCacheBlock, 64, PLACE, TURN>(p, r, m, to, s)
                           : launch_move<kCacheBlock, 128, PLACE, TURN>(p, r, m, to, s);
}

}  // namespace

hipError_t launch_cache_read(const CacheProblem& p, const Rotary& r, bool interleaved, const int32_t* positions,
                             uint16_t* k_out, uint16_t* v_out, hipStream_t s) {
  auto go = [&](auto form) {
    constexpr int FORM = decltype(form)::value;
    if (!r.turns) return launch_read<FORM, kPairs, false>(p, r, positions, k_out, v_out, s);
    const PairPlace place = place_of(r.dim, interleaved);
    return place == kPairs    ? launch_read<FORM, kPairs, true>(p, r, positions, k_out, v_out, s)
           : place == kHalves ? launch_read<FORM, kHalves, true>(p, r, positions, k_out, v_out, s)
                              : launch_read<FORM, kOdd, true>(p, r, positions, k_out, v_out, s);
  };
  return p.form == kCacheBf16   ? go(std::integral_constant<int, kCacheBf16>{})
         : p.form == kCacheHead ? go(std::integral_constant<int, kCacheHead>{})
                                : go(std::integral_constant<int, kCacheBlock>{});
}

hipError_t launch_cache_move(const CacheProblem& p, const Rotary& r, bool interleaved, const Moves& m, const PageMap& to,
                             hipStream_t s) {
  if (!r.turns) return launch_move_form<kPairs, 0>(p, r, m, to, s);
  const PairPlace place = place_of(r.dim, interleaved);
  if (m.token == 0)
    return place == kPairs    ? launch_move_form<kPairs, 1>(p, r, m, to, s)
           : place == kHalves ? launch_move_form<kHalves, 1>(p, r, m, to, s)
                              : launch_move_form<kOdd, 1>(p, r, m, to, s);
  return place == kPairs    ? launch_move_form<kPairs, 2>(p, r, m, to, s)
         : place == kHalves ? launch_move_form<kHalves, 2>(p, r, m, to, s)
                            : launch_move_form<kOdd, 2>(p, r, m, to, s);
}

}  // namespace fp2
