// What the kernels for few query rows of a sequence share: the tiles of keys
// that the rows see, and how a call's tiles are dealt to workgroups.
#pragma once
#include "cache.h"

namespace fp2 {

namespace {

constexpr int kTile = 32;        // keys per wave and step
constexpr int kParts = 1024;     // parts that a call's keys are cut for: four workgroups a compute unit
constexpr int kMinTiles = 16;    // tiles of a part, at least

// Tiles of a sequence that some row sees: `sinks` leading ones, then those
// from `from` on.
struct Tiles {
  int sinks, from, n;
};

// With `all`, every tile of the sequence.
__device__ __forceinline__ Tiles tiles_of(const CacheProblem& p, int Lq, int L, bool all = false) {
  Tiles t{0, 0, 0};
  if (all) t.n = (L + kTile - 1) / kTile;
  if (all || Lq <= 0 || L <= 0) return t;
  const int lo = max(L - Lq - p.window + 1, 0);
  t.sinks = (min(p.sink, L) + kTile - 1) / kTile;
  t.from = max(lo / kTile, t.sinks);
  t.n = t.sinks + max((L - 1) / kTile - t.from + 1, 0);
  return t;
}

__device__ __forceinline__ int wave_scan(int v, int lane) {   // inclusive
  for (int o = 1; o < 64; o <<= 1) {
    const int u = __shfl_up(v, o, 64);
    if (lane >= o) v += u;
  }
  return v;
}

struct Unit {
  int b, h, part, parts, slot;   // slot: first partial slot of the unit, if parts > 1
};

// The `item`-th (sequence, part, head) of the call, or, with by_unit, the
// unit (sequence, head) of that number. Wave-uniform; false past the last.
template <bool BY_UNIT>
__device__ __forceinline__ bool find_item(const CacheProblem& p, int item, Unit& out,
                                          bool all = false) {
  const int lane = threadIdx.x & 63;
  auto tiles_at = [&](int b) {
    return b < p.batch ? tiles_of(p, p.cu[b + 1] - p.cu[b], p.cuk[b + 1] - p.cuk[b], all).n : 0;
  };
  int64_t total = 0;   // tiles of the call
  int cut = 0;         // tiles of a part
  const int n0 = tiles_at(lane);
  if (p.splits == 0) {
    for (int b0 = 0; b0 < p.batch; b0 += 64) {
      int64_t s = b0 ? tiles_at(b0 + lane) : n0;
      for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
      total += s;
    }
    total *= p.hkv;
    cut = max((int)((total + kParts - 1) / kParts), kMinTiles);
  }
  int items = 0, slots = 0;
  for (int b0 = 0; b0 < p.batch; b0 += 64) {
    const int n = b0 ? tiles_at(b0 + lane) : n0;
    const int parts = p.splits ? min(p.splits, n) : (n + cut - 1) / cut;
    const int mine = BY_UNIT ? (b0 + lane < p.batch ? p.hkv : 0) : parts * p.hkv;
    const int own_slots = parts > 1 ? parts * p.hkv : 0;
    const int incl = wave_scan(mine, lane), sincl = wave_scan(own_slots, lane);
    const uint64_t hit = __ballot(items + incl > item);
    if (hit) {
      const int l = __ffsll((unsigned long long)hit) - 1;
      const int local = item - items - __shfl(incl - mine, l, 64);
      out.b = b0 + l;
      out.parts = __shfl(parts, l, 64);
      out.h = local % p.hkv;
      out.part = local / p.hkv;
      out.slot = slots + __shfl(sincl - own_slots, l, 64) + out.h * out.parts;
      out.b = __builtin_amdgcn_readfirstlane(out.b);
      out.h = __builtin_amdgcn_readfirstlane(out.h);
      out.part = __builtin_amdgcn_readfirstlane(out.part);
      out.parts = __builtin_amdgcn_readfirstlane(out.parts);
      out.slot = __builtin_amdgcn_readfirstlane(out.slot);
      return true;
    }
    items += __shfl(incl, 63, 64);
    slots += __shfl(sincl, 63, 64);
  }
  return false;
}

__device__ __forceinline__ bf16x8_t codes_to_bf16(uint32_t a, uint32_t b, float s) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  const b2 x[4] = {__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)a, s, false),
                   __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)a, s, true),
                   __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)b, s, false),
                   __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)b, s, true)};
  return __builtin_bit_cast(bf16x8_t, x);
}

// 16-row tiles of the bound of the rows of a sequence.
inline int row_tiles(const CacheProblem& p) {
  const int rows = p.max_new * p.g;
  return rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
}

}  // namespace

}  // namespace fp2
