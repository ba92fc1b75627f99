// What the kernels for few query rows of a sequence share: the tiles of keys
// that the rows see, and how a call's tiles are dealt to workgroups.
#pragma once
#include "cache.h"

namespace fp2 {

namespace {

constexpr int kTile = 32;        // keys per wave and step
constexpr int kFewWaves = 8;     // waves of a workgroup
constexpr int kFewGroups = 256;  // workgroups that a call is dealt to: one a compute unit
constexpr int kWholeTiles = 16;  // sequences of at most as many are not cut, if there are many

// Tiles of a sequence that some row sees: `sinks` leading ones, then those
// from `from` on.
struct Tiles {
  int sinks, from, n;
};

__device__ __forceinline__ Tiles tiles_of(const CacheProblem& p, int Lq, int L) {
  Tiles t{0, 0, 0};
  if (Lq <= 0 || L <= 0) return t;
  const int lo = max(L - Lq - p.window + 1, 0);
  t.sinks = (min(p.sink, L) + kTile - 1) / kTile;
  t.from = max(lo / kTile, t.sinks);
  t.n = t.sinks + max((L - 1) / kTile - t.from + 1, 0);
  return t;
}

// Whether the query at `pos` sees `key`.
__device__ __forceinline__ bool sees(const CacheProblem& p, int pos, int key) {
  return (uint32_t)(key - pos + p.window - 1) < (uint32_t)p.window || (key < p.sink && key <= pos);
}

// Keeps the compiler from computing many masks (a pair of scalar registers
// each) before it uses the first: x is needed here.
template <class T>
__device__ __forceinline__ T pinned(T x) {
  asm volatile("" : "+v"(x));
  return x;
}

// The heads of a token lie side by side in the pool, so the waves of a
// workgroup take different heads of the same tokens where they can: memory is
// then read in runs of heads x 128 codes (reading a pool of 8 heads this way
// reaches 6.2 TB/s, with the heads in different workgroups 5.5). `heads` of a
// workgroup's waves are heads, `rows` halves or quarters of the query rows, and
// the others (`keys`) alternate tiles of the same head.
struct WaveSplit {
  int heads, rows, keys;
};
inline __host__ __device__ WaveSplit wave_split(const CacheProblem& p, int rows) {
  int heads = kFewWaves / rows;
  while (p.hkv % heads) heads >>= 1;
  return WaveSplit{heads, rows, kFewWaves / rows / heads};
}

// The tiles of a call, one sequence after the other, form a line, which is cut
// into equal shares; a workgroup takes one share of its heads, so that all have
// the same work whatever the lengths. A share may hold the end of one
// sequence, whole ones, and the start of another. With kv_splits n >= 1 every
// sequence is cut into at most n shares of its own instead.
struct Share {
  int lo, hi;       // tiles of the line
  int b;            // sequence of the first
  int base;         // and where that one starts
  int len;          // tiles of a share (kv_splits 0)
  int q0, Lq, L;    // the sequence's first query and its lengths
};

// Short sequences, by the bounds of the call, are taken whole if they are
// enough to fill the chip: there is nothing to even out, and nothing to join.
inline CacheProblem dealt(CacheProblem p, int rows) {
  const int64_t a = p.max_kv, b = (int64_t)p.window + p.max_new + p.sink;
  if (p.splits == 0 && (a < b ? a : b) / kTile + 3 <= kWholeTiles &&
      (int64_t)p.batch * (p.hkv / wave_split(p, rows).heads) >= kFewGroups)
    p.splits = 1;
  return p;
}

// Shares of the line.
inline __host__ __device__ int shares_of(const CacheProblem& p, int rows) {
  const int groups = p.hkv / wave_split(p, rows).heads;
  return p.splits ? p.batch * p.splits : (kFewGroups + groups - 1) / groups;
}

__device__ __forceinline__ int lane_value(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

// Share `index` of the call, or, with BY_SEQ, sequence `index` (lo .. hi then
// are all its tiles). Wave-uniform; false where there is none. A call has
// fewer than 2^31 tiles (the host's check).
template <bool BY_SEQ>
__device__ __forceinline__ bool find_share(const CacheProblem& p, int shares, int index, Share& out) {
  const int lane = threadIdx.x & 63;
  int q0, Lq, L;
  auto tiles_at = [&](int b) {
    q0 = Lq = L = 0;
    if (b < p.batch) {
      q0 = p.cu[b];
      Lq = p.cu[b + 1] - q0;
      L = p.cuk[b + 1] - p.cuk[b];
    }
    return tiles_of(p, Lq, L).n;
  };
  auto take = [&](int l) {
    out.q0 = lane_value(q0, l);
    out.Lq = lane_value(Lq, l);
    out.L = lane_value(L, l);
  };
  if (p.splits) {
    const int b = BY_SEQ ? index : index / p.splits, part = BY_SEQ ? 0 : index % p.splits;
    const int n = lane_value(tiles_at(b), 0);
    const int parts = BY_SEQ ? 1 : min(p.splits, n);
    if (part >= parts) return false;
    out.lo = (int)((int64_t)n * part / parts);
    out.hi = (int)((int64_t)n * (part + 1) / parts);
    out.b = b;
    out.base = out.len = 0;
    take(0);
    return out.lo < out.hi;
  }
  // tiles before each sequence, 64 of them at a time; up to 64 are looked at once
  auto scan = [&](int n) {
    for (int o = 1; o < 64; o <<= 1) {
      const int u = __shfl_up(n, o, 64);
      if (lane >= o) n += u;
    }
    return n;
  };
  int n = tiles_at(lane), incl = scan(n), total = lane_value(incl, 63);
  for (int b0 = 64; b0 < p.batch; b0 += 64) {
    int s = tiles_at(b0 + lane);
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    total += __builtin_amdgcn_readfirstlane(s);
  }
  out.len = max((int)(((int64_t)total + shares - 1) / shares), 1);
  out.lo = (int)min((int64_t)index * out.len, (int64_t)total);
  out.hi = (int)min((int64_t)out.lo + out.len, (int64_t)total);
  if (!BY_SEQ && out.lo >= out.hi) return false;
  int before = 0;
  for (int b0 = 0; b0 < p.batch; b0 += 64) {
    if (p.batch > 64) {
      n = tiles_at(b0 + lane);
      incl = before + scan(n);
    }
    const uint64_t hit = __ballot(BY_SEQ ? b0 + lane == index : incl > out.lo);
    if (hit) {
      const int l = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)hit) - 1);
      const int nl = lane_value(n, l);
      out.b = b0 + l;
      out.base = lane_value(incl, l) - nl;
      take(l);
      if (BY_SEQ) out.lo = out.base, out.hi = out.base + nl;
      return out.lo < out.hi;
    }
    before = lane_value(incl, 63);
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

}  // namespace

}  // namespace fp2
