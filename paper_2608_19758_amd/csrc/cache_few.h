// What the kernels for few query rows of a sequence share: the tiles of keys
// that the rows see, and how a call's tiles are dealt to workgroups.
#pragma once
#include "cache.h"

namespace fp2 {

namespace {

constexpr int kTile = 32;        // keys per wave and step
constexpr int kFewGroups = 256;  // workgroups that a call is dealt to: one a compute unit
constexpr int kWholeTiles = 48;  // sequences of at most as many (half of it in bf16) are not cut

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

// The heads of a token lie side by side in the pool, so the waves of a
// workgroup take up to `heads` different heads of the same tokens, and memory
// is read in runs of heads x 128 codes (reading a pool of 8 heads this way
// reaches 6.2 TB/s, with the heads in different workgroups 5.5); the other
// waves alternate tiles. Short sequences, by the bounds of the call, are taken whole, with
// fewer heads a workgroup where those would not fill the chip: joining parts
// is a second kernel and costs about 8 us, a compute unit reads some 100 KB in
// that time. 64 sequences of 1000 visible tokens take 30 us whole and 42 cut,
// one of 617 tokens in bf16 12 and 15, of 1500 in codes 14 both ways.
inline CacheProblem dealt(CacheProblem p, int heads) {
  p.heads = heads;
  while (p.hkv % p.heads) p.heads >>= 1;
  const int64_t a = p.max_kv, b = (int64_t)p.window + p.max_new + p.sink;
  if (p.splits == 0 && (a < b ? a : b) / kTile + 3 <= kWholeTiles >> (p.form == kCacheBf16)) {
    p.splits = 1;
    while (p.heads > 1 && (int64_t)p.batch * (p.hkv / p.heads) < kFewGroups) p.heads >>= 1;
  }
  return p;
}

// Shares of the line.
inline __host__ __device__ int shares_of(const CacheProblem& p) {
  const int groups = p.hkv / p.heads;
  return p.splits ? p.batch * p.splits : (kFewGroups + groups - 1) / groups;
}

__device__ __forceinline__ int lane_value(int v, int lane) { return __builtin_amdgcn_readlane(v, lane); }

// Share `index` of the call. Wave-uniform; false where there is none. A call has
// fewer than 2^31 tiles (the host's check).
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
    const int b = index / p.splits, part = index % p.splits;
    const int n = lane_value(tiles_at(b), 0);
    const int parts = min(p.splits, n);
    if (part >= parts) return false;
    out.lo = (int)((int64_t)n * part / parts);
    out.hi = (int)((int64_t)n * (part + 1) / parts);
    out.b = b;
    out.base = out.len = 0;
    take(0);
    return out.lo < out.hi;
  }
  // tiles before each sequence, 64 of them at a time; up to 64 are looked at once
  int n = tiles_at(lane), incl = wave_scan(n), total = lane_value(incl, 63);
  if (p.batch > 64) {
    int more = 0;
#pragma unroll 4
    for (int b0 = 64; b0 < p.batch; b0 += 64) more += tiles_at(b0 + lane);
    total += lane_value(wave_scan(more), 63);
  }
  out.len = max((int)(((int64_t)total + shares - 1) / shares), 1);
  out.lo = (int)min((int64_t)index * out.len, (int64_t)total);
  out.hi = (int)min((int64_t)out.lo + out.len, (int64_t)total);
  if (out.lo >= out.hi) return false;
  int before = 0;
  for (int b0 = 0; b0 < p.batch; b0 += 64) {
    if (p.batch > 64) {
      n = tiles_at(b0 + lane);
      incl = before + wave_scan(n);
    }
    const uint64_t hit = __ballot(incl > out.lo);
    if (hit) {
      const int l = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)hit) - 1);
      out.b = b0 + l;
      out.base = lane_value(incl, l) - lane_value(n, l);
      take(l);
      return true;
    }
    before = lane_value(incl, 63);
  }
  return false;
}

// Where the keys of a tile lie: the pages of its two groups of 16 and the
// places in them (GROUPED), or the page and place of key lane % 32. The table's
// entries are kept as loaded and used a tile later, so that nothing waits for
// them. Keys past the sequence stand on valid ones.
struct Where {
  int page[2], off[2];
  __device__ __forceinline__ int64_t slot(const PageMap& pm, int u) const {
    return (int64_t)page[u] * pm.page + off[u];
  }
};
template <bool GROUPED>
__device__ __forceinline__ Where where_at(const PageMap& pm, const int32_t* table, int tile, int last, int lane) {
  Where a;
  const int t0 = kTile * tile;
#pragma unroll
  for (int u = 0; u < (GROUPED ? 2 : 1); ++u) {
    const int t = !GROUPED ? min(t0 + (lane & 31), last) : u && t0 + 16 > last ? t0 : t0 + 16 * u;
    const int pg = pm.shift >= 0 ? t >> pm.shift : t / pm.page;
    a.page[u] = GROUPED ? ld_uniform(table, pg) : table[pg];
    a.off[u] = t - pg * pm.page;
  }
  return a;
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
