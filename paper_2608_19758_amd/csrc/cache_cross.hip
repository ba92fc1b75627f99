// Attention of many query rows over a paged cache whose keys they all see: cross
// attention to an encoder's states, or to a prefix that requests share.
//
// A unit is a (sequence, KV head, run of 256 / g queries): 256 packed rows, the
// g query heads of a token side by side, 32 rows a wave. Keys come in tiles of
// 64, from the pool to registers and on to LDS as bf16 (codes are converted
// there, once for all waves, with the power of two of their block; a scale per
// head multiplies the scores and the output).
//
// Per tile and wave: S^T = K Q^T and O^T += V^T P^T on
// v_mfma_f32_32x32x16_bf16; a lane holds query l % 32 and 32 keys, so the
// probabilities go into the second product as they are, and the transposing
// LDS reads give V^T. The running maximum moves when a score passes it by more
// than 2^8. Probabilities are rounded to bf16 for the product, the matrix
// cores' type (half a step of 2^-8 each); sums, maxima and outputs are fp32.
//
// Two groups of four waves, one of each on every SIMD, take turns: while one
// has the matrix cores (scores of the next tile, values of this one) the other
// has the vector ALUs (probabilities, and the next tiles from registers to LDS).
// Tiles have three places in LDS, since the groups are a phase apart. The matrix
// operands are read kAhead products ahead.
//
// The tiles of all units form a line that is dealt to the workgroups in equal
// shares, one workgroup a compute unit, each working its own out from the lengths
// (on the device only). Units that lie in several shares are joined by
// join_kernel. With kv_splits every unit is cut into so many parts instead.
//
// 4096 queries of 32 heads over 30001 keys: 1.80 ms, 1.12 PFLOP/s. Bound by power:
// the matrix cores are busy 56% of the cycles, the vector ALUs 54%, at 1.67 GHz. 8
// sequences of 100 to 800 queries over 900 to 4000 keys: 165 to 185 us, of which 16
// are the join, and 8 each piece of a unit's start and end.
#include <algorithm>

#include "rotary_rows.h"

namespace fp2 {

namespace {

constexpr float kLn2f = 0.69314718055994530942f;
constexpr int kStep = 64;        // keys per tile
constexpr int kWaves = 8;
constexpr int kRows = 32 * kWaves;
constexpr int kMaxParts = 32;
constexpr int kShares = kCrossCuts;  // workgroups that run at a time, one a compute unit
constexpr int kXcds = 8;         // dies, each with a cache of its own, that workgroups go to in turn
constexpr int kMinShare = 4;     // length of a share, at least (one unit of 16 tiles: 21 us, with 8 30)
// Tiles that a unit's start and end take as long as. 24 sequences of 100 to 3000 queries over 100 to 9000 keys: 854 us,
// with 0 1996, with 8 892.
constexpr int kUnit = 4;
constexpr int kAhead = 5;        // products that operands are read ahead (600 queries over 4000 keys: 67 us, with 3 71, with 7 68)
constexpr float kTau = 8.0f;
constexpr float kNoRef = -1e30f;

typedef __attribute__((address_space(3))) i16x4_t lds_i16x4_t;
typedef __attribute__((address_space(3))) char lds_char_t;

// 16-byte chunk c of row r is kept at these places, so that the operand reads
// of an instruction spread over all LDS banks.
__device__ __forceinline__ int kplace(int r, int c) { return r * 16 + (c ^ (r & 15)); }
__device__ __forceinline__ int vplace(int r, int c) { return r * 16 + (c ^ (4 * (r & 3))); }

__device__ __forceinline__ float other_half_max(float v) {   // over lanes l and l ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// A sequence: its queries, its keys, and how many units a head has and tiles a unit.
struct Seq {
  int q0, n, L, units, tiles;
  __device__ __forceinline__ Seq(const CacheProblem& p, int b) {
    q0 = ld_uniform(p.cu, b);
    n = max(ld_uniform(p.cu, b + 1) - q0, 0);
    L = max(ld_uniform(p.cuk, b + 1) - ld_uniform(p.cuk, b), 0);
    units = (int)(((int64_t)n * p.g + kRows - 1) / kRows);
    tiles = max((L + kStep - 1) / kStep, 1);     // without keys one, which writes what comes of none
  }
};

// A unit counts as its tiles and kUnit more, about the time that its start and
// end take (as one, where the call's units have few tiles and none is cut); of a
// sequence its units, head by head, lie one behind the other.
__device__ __forceinline__ int64_t line_of(const CacheProblem& p, int cuts, int b, int64_t& units) {   // (any lane's b; 0 past the batch)
  units = 0;
  if (b >= p.batch) return 0;
  const int n = max(p.cu[b + 1] - p.cu[b], 0), L = max(p.cuk[b + 1] - p.cuk[b], 0);
  units = ((int64_t)n * p.g + kRows - 1) / kRows * p.hkv;
  return units * (cuts ? max((L + kStep - 1) / kStep, 1) + kUnit : 1);
}

__device__ __forceinline__ int64_t wave_sum_to(int64_t v) {   // inclusive, over the lanes before
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int64_t x = __shfl_up(v, o, 64);
    v += lane >= o ? x : 0;
  }
  return v;
}
__device__ __forceinline__ int64_t lane_value(int64_t v, int lane) {
  return (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)v, lane) |
         (int64_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32;
}

// What a workgroup takes of the line: lo .. hi - 1, from sequence b on, which starts at `base`.
struct Share {
  int index, b;
  int64_t lo, hi, base, len;
};
__device__ __forceinline__ bool find_share(const CacheProblem& p, int cuts, Share& s) {
  // every lane adds up a run of sequences, the first of which lie as far apart
  const int lane = threadIdx.x & 63, run = (p.batch + 63) / 64;
  int64_t own = 0, units = 0, u;
#pragma unroll 4
  for (int i = 0; i < run; ++i) {
    const int b = lane * run + i;
    own += line_of(p, cuts, b, u);
    units += u;
  }
  const int64_t to = wave_sum_to(own), total = lane_value(to, 63);
  units = lane_value(wave_sum_to(units), 63);
  // short units are left whole while there are workgroups for them
  const int64_t most = min(max(units, total / kMinShare), (int64_t)gridDim.x);
  s.len = max((total + most - 1) / max(most, (int64_t)1), (int64_t)1);
  // neighbours in the line share keys, so they go to one die
  const int shares = (int)((total + s.len - 1) / s.len), each = (shares + kXcds - 1) / kXcds;
  s.index = blockIdx.x % kXcds * each + blockIdx.x / kXcds;
  if ((int)(blockIdx.x / kXcds) >= each || s.index >= shares) return false;
  s.lo = s.index * s.len;
  s.hi = min(s.lo + s.len, total);
  // the lane whose run holds the first, and the sequence of the run
  const int l = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)__ballot(to > s.lo)) - 1);
  s.base = lane_value(to - own, l);
  s.b = l * run;
  for (const int end = min(s.b + run, p.batch); run > 1 && s.b < end; s.b += 64) {
    const int64_t one = s.b + lane < end ? line_of(p, cuts, s.b + lane, u) : 0, upto = s.base + wave_sum_to(one);
    const uint64_t hit = __ballot(upto > s.lo);
    if (hit) {
      const int k = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)hit) - 1);
      s.b += k;
      s.base = lane_value(upto - one, k);
      break;
    }
    s.base = lane_value(upto, 63);
  }
  return true;
}

// A unit that a workgroup's share starts and does not end (parts 0: none), for the join.
struct Cut {
  int b, h, unit;
  int parts;        // and the share's index, from bit 16 on
};

struct Shared {
  i32x4_t k[3][kStep * 16];
  i32x4_t v[3][kStep * 16];
};

// Tiles lo .. hi - 1 of a unit; slot: of the partial results, or -1 where they are all.
// GROUPED: pages hold a multiple of 8 tokens, so the rows of a tile that a wave
// stages together lie one after the other and their address is uniform (scalar).
template <int FORM, bool GROUPED>
__device__ __forceinline__ void segment(const CacheProblem& p, const CachePartials& part, Shared& sh, int b, int h, int unit,
                                        const Seq& q, int lo, int hi, int64_t slot, uint16_t* __restrict__ out,
                                        float* __restrict__ lse) {
  constexpr bool kBf16 = FORM == kCacheBf16;
  constexpr int ESZ = kBf16 ? 2 : 1;
  constexpr int NJ = kBf16 ? 2 : 1;              // rows of a tile per thread
  constexpr int TPR = kBf16 ? 16 : 8;            // threads of a row, 16 bytes each
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const int pr = 32 * w + l32;                   // packed row
  const int i0 = unit * (kRows / p.g), rows = min(kRows / p.g, q.n - i0) * p.g;
  const int hq = h * p.g + pr % p.g;
  const bool valid = pr < rows;
  const int64_t qrow = (int64_t)(q.q0 + i0 + min(pr, rows - 1) / p.g) * p.hq + hq;
  if (q.L <= 0) {                                // no keys: zeros, and minus infinity
    if (!valid) return;
    for (int d = 64 * half; d < 64 * half + 64; d += 8)
      *(uint4*)(out + qrow * kHeadDim + d) = make_uint4(0, 0, 0, 0);
    if (lse && half == 0) lse[qrow] = -INFINITY;
    return;
  }

  bf16x8_t qb[8];
#pragma unroll
  for (int ds = 0; ds < 8; ++ds)
    qb[ds] = __builtin_bit_cast(bf16x8_t, *(const i32x4_t*)(p.q + qrow * kHeadDim + 16 * ds + 8 * half));
  f32x16_t o[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) o[dt] = f32x16_t{};
  float m = kNoRef, l = 0.f;
  const float cs = score_scale<FORM>(p, h);
  float vsc = 1.f;
  if constexpr (FORM == kCacheHead) vsc = ld_uniform(p.v_head, h);

  // ---- staging
  const int64_t rowb = (int64_t)p.hkv * kHeadDim * ESZ;
  const int64_t hoff = (int64_t)h * kHeadDim * ESZ;
  const int c = tid % TPR, r0 = tid / TPR;       // this thread's chunk and first row of a tile
  struct Regs {
    i32x4_t x[NJ];
    uint32_t scale;
  };
  // Where the wave's rows of a tile lie (GROUPED), or this thread's: the table's
  // entries as loaded (used a tile later, so that nothing waits for them) and the
  // places in the pages. Keys past the sequence stand on valid ones.
  constexpr int GROUP = 64 / TPR;                // rows that a wave loads at once
  struct Where {
    int page[NJ], off[NJ];
  };
  const int32_t* table = p.pm.table + (int64_t)b * p.pm.stride;
  auto where = [&](int i) {
    Where a;
    const int k0 = kStep * min(i, hi - 1);       // past the end the last tile again
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int t = GROUPED ? min(k0 + GROUP * w + 32 * j, (q.L - 1) & -GROUP) : min(k0 + r0 + 32 * j, q.L - 1);
      const int pg = p.pm.shift >= 0 ? t >> p.pm.shift : t / p.pm.page;
      a.page[j] = GROUPED ? ld_uniform(table, pg) : table[pg];
      a.off[j] = t - pg * p.pm.page;
    }
    return a;
  };
  const uint32_t roff = (uint32_t)((GROUPED ? lane / TPR : 0) * rowb + 16 * c);   // this thread's place behind its address
  auto load = [&](const uint8_t* pool, const uint8_t* scales, const Where& a, Regs& x) {
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int64_t s = (int64_t)a.page[j] * p.pm.page + a.off[j];
      x.x[j] = *(const i32x4_t*)(pool + s * rowb + hoff + roff);
      if constexpr (FORM == kCacheBlock) x.scale = scales[(s >> p.sb_shift) * p.hkv + h];
    }
  };
  auto widen = [](const Regs& x, i32x4_t (&y)[2]) {   // 16 codes -> 16 bf16
    const float s = FORM == kCacheBlock ? block_scale(x.scale) : 1.f;
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const b2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x.x[0][i], s, false);
      const b2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x.x[0][i], s, true);
      y[i >> 1][2 * (i & 1)] = __builtin_bit_cast(int, a);
      y[i >> 1][2 * (i & 1) + 1] = __builtin_bit_cast(int, b);
    }
  };
  auto write_k = [&](i32x4_t* to, const Regs& x) {
    i32x4_t y[2];
    if constexpr (kBf16) y[0] = x.x[0], y[1] = x.x[NJ - 1];
    else widen(x, y);
#pragma unroll
    for (int j = 0; j < 2; ++j) to[kplace(kBf16 ? r0 + 32 * j : r0, kBf16 ? c : 2 * c + j)] = y[j];
  };
  auto write_v = [&](i32x4_t* to, int i, const Regs& x) {
    i32x4_t y[2];
    if constexpr (kBf16) y[0] = x.x[0], y[1] = x.x[NJ - 1];
    else widen(x, y);
    // values behind the last key (the pool holds anything there) must not meet zero probabilities
    const int k0 = kStep * min(i, hi - 1);
    if (k0 + kStep > q.L) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (k0 + r0 + (kBf16 ? 32 * j : 0) >= q.L) y[j] = i32x4_t{};
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) to[vplace(kBf16 ? r0 + 32 * j : r0, kBf16 ? c : 2 * c + j)] = y[j];
  };

  // operands of the products: 32 keys uu by 16 dimensions ds; and of V^T 16 keys
  // kg by 32 dimensions dt, where place i' of lane half H is key 16 kg + 8 (i' / 4)
  // + 4 H + i' % 4
  auto kread = [&](const i32x4_t* kt, int uu, int ds) {
    return __builtin_bit_cast(bf16x8_t, kt[kplace(32 * uu + l32, 2 * ds + half)]);
  };
  const int g16 = lane >> 4, i16 = lane & 15;
  auto vread = [&](const i32x4_t* vt, int kg, int dt) {
    i16x4_t rd[2];
#pragma unroll
    for (int tt = 0; tt < 2; ++tt) {
      const int key = 16 * kg + 8 * tt + 4 * (g16 >> 1) + (i16 >> 2);
      const int d = 32 * dt + 16 * (g16 & 1) + 4 * (i16 & 3);
      const int byte = vplace(key, d >> 3) * 16 + (d & 7) * 2;
      rd[tt] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4_t*)((lds_char_t*)vt + byte));
    }
    const i32x2_t a = __builtin_bit_cast(i32x2_t, rd[0]), b = __builtin_bit_cast(i32x2_t, rd[1]);
    return __builtin_bit_cast(bf16x8_t, (i32x4_t){a[0], a[1], b[0], b[1]});
  };

  // the maximum that scores become probabilities against moves when one passes it by more than kTau
  auto move_max = [&](const f32x16_t (&s)[2]) {
    float mx = -INFINITY;
#pragma unroll
    for (int uu = 0; uu < 2; ++uu)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[uu][e]);
    mx = other_half_max(mx) * cs;
    const bool up = mx > m + kTau;
    if (__any(up)) {
      const float mn = up ? mx : m, f = fast_exp2(m - mn);
      m = mn;
      l *= f;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[dt][e] *= f;
    }
  };
  // probabilities of the scores, rounded to bf16 for the product; their sum is of the unrounded ones
  auto exponentials = [&](const f32x16_t (&s)[2], uint32_t (&pw)[16]) {
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int uu = 0; uu < 2; ++uu)
#pragma unroll
      for (int e = 0; e < 16; e += 2) {
        const float a = fast_exp2(fmaf(s[uu][e], cs, -m)), b = fast_exp2(fmaf(s[uu][e + 1], cs, -m));
        sum[e & 2] += a;
        sum[(e & 2) + 1] += b;
        pw[8 * uu + e / 2] = pack_bf16x2(a, b);
      }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  };
  auto mask = [&](int k0, f32x16_t (&s)[2]) {    // element e of s[uu] is key k0 + 32 uu + 8 (e / 4) + 4 half + e % 4
#pragma unroll
    for (int uu = 0; uu < 2; ++uu)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = k0 + 32 * uu + 8 * (e >> 2) + 4 * half + (e & 3);
        s[uu][e] = pinned(key < q.L ? s[uu][e] : -INFINITY);
      }
  };

  auto phase = [] {
    __builtin_amdgcn_sched_barrier(0);
    lds_barrier();
    __builtin_amdgcn_sched_barrier(0);
  };
  Regs kregs, vregs;
  f32x16_t s[2];
  uint32_t pw[16];
  Where at = where(lo + 1), vat = where(lo + 2);
  {
    Regs k0, k1, v0;             // of the first two tiles
    const Where first = where(lo);
    load(p.k, p.k_block, first, k0);
    load(p.k, p.k_block, at, k1);
    load(p.v, p.v_block, first, v0);
    load(p.v, p.v_block, at, vregs);
    load(p.k, p.k_block, vat, kregs);
    at = where(lo + 3);
    lds_barrier();               // the segment before is done with the places
    write_k(sh.k[0], k0);
    write_k(sh.k[1], k1);
    write_v(sh.v[0], lo, v0);
  }
  i32x4_t *kw = sh.k[2], *kr = sh.k[1], *kx = sh.k[0];   // to write, to read next, the other
  i32x4_t *vw = sh.v[1], *vr = sh.v[0], *vx = sh.v[2];
  phase();
  if (w >= kWaves / 2) phase();
#pragma unroll
  for (int uu = 0; uu < 2; ++uu) {
    s[uu] = f32x16_t{};
#pragma unroll
    for (int ds = 0; ds < 8; ++ds)
      s[uu] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kread(sh.k[0], uu, ds), qb[ds], s[uu], 0, 0, 0);
  }
#pragma unroll 1
  for (int i = lo; i < hi; ++i) {
    phase();
    write_k(kw, kregs);          // tile i + 2
    write_v(vw, i + 1, vregs);
    load(p.k, p.k_block, at, kregs);
    load(p.v, p.v_block, vat, vregs);
    vat = at;
    at = where(i + 4);
    if (kStep * i + kStep > q.L) mask(kStep * i, s);
    move_max(s);
    exponentials(s, pw);
    phase();
    // 16 products of the next tile's scores, then 16 of this one's values
    bf16x8_t f[kAhead];
    auto fetch = [&](int n) { return n < 16 ? kread(kr, n & 1, n >> 1) : vread(vr, (n - 16) >> 2, n & 3); };
#pragma unroll
    for (int n = 0; n < kAhead; ++n) f[n] = fetch(n);
#pragma unroll
    for (int n = 0; n < 32; ++n) {
      const bf16x8_t x = f[n % kAhead];
      if (n < 16) {
        const int uu = n & 1, ds = n >> 1;
        s[uu] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, qb[ds], ds ? s[uu] : f32x16_t{}, 0, 0, 0);
      } else {
        const int kg = (n - 16) >> 2, dt = n & 3;
        const i32x4_t pb = {(int)pw[4 * kg], (int)pw[4 * kg + 1], (int)pw[4 * kg + 2], (int)pw[4 * kg + 3]};
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, __builtin_bit_cast(bf16x8_t, pb), o[dt], 0, 0, 0);
      }
      if (n + kAhead < 32) f[n % kAhead] = fetch(n + kAhead);
      __builtin_amdgcn_sched_barrier(0);
    }
    i32x4_t* t = kr;
    kr = kw, kw = kx, kx = t;
    t = vr;
    vr = vw, vw = vx, vx = t;
  }
  if (w < kWaves / 2) phase();

  // ---- output
  l += __shfl_xor(l, 32, 64);
  if (slot >= 0) {
    if (!valid) return;
    const int64_t row = slot * kRows + pr;
#pragma unroll
    for (int dt = 0; dt < 4; ++dt)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *(float4*)(part.o + row * kHeadDim + 32 * dt + 8 * i + 4 * half) =
            make_float4(o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]);
    if (half == 0) *(float2*)(part.ml + 2 * row) = make_float2(m, l);
    return;
  }
  const float inv = vsc / l;
  uint16_t* orow = out + qrow * kHeadDim;
  // the lane halves hold alternate groups of four columns: exchanged in pairs
  // so that a store carries 16 bytes
#pragma unroll
  for (int dt = 0; dt < 4; ++dt)
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      uint32_t a[2], b[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const auto r = __builtin_amdgcn_permlane32_swap(
            pack_bf16x2(o[dt][4 * i + 2 * k] * inv, o[dt][4 * i + 2 * k + 1] * inv),
            pack_bf16x2(o[dt][4 * i + 4 + 2 * k] * inv, o[dt][4 * i + 5 + 2 * k] * inv), false, false);
        a[k] = r[0];
        b[k] = r[1];
      }
      if (valid) *(uint4*)(orow + 32 * dt + 8 * (i + half)) = make_uint4(a[0], a[1], b[0], b[1]);
    }
  if (lse && valid && half == 0) lse[qrow] = (m + fast_log2(l)) * kLn2f;
}

// Equal shares of the line. A share leaves what it has of a unit that started
// before it in slot 2 index, of one that goes on behind it in slot 2 index + 1.
// cuts 0: units are left whole.
template <int FORM, bool GROUPED>
__global__ __launch_bounds__(64 * kWaves, 1) void cross_kernel(CacheProblem p, CachePartials part, int cuts,
                                                               uint16_t* __restrict__ out, float* __restrict__ lse) {
  __shared__ Shared sh;
  Cut cut{0, 0, 0, 0};
  Share s;
  const bool any = find_share(p, cuts, s);
  int64_t pos = any ? s.lo : 0;
#pragma unroll 1
  while (any && pos < s.hi) {
    const Seq q(p, s.b);
    const int64_t off = pos - s.base, each = cuts ? q.tiles + kUnit : 1, all = q.units * each * p.hkv;
    if (off >= all) {
      ++s.b;
      s.base += all;
      continue;
    }
    const int64_t at = off / each, start = s.base + at * each;   // the unit among the sequence's, head by head
    const int h = (int)(at / q.units), unit = (int)(at % q.units);
    const int lo = (int)max(pos - start - kUnit, (int64_t)0);
    const int hi = cuts ? (int)min(s.hi - start - kUnit, (int64_t)q.tiles) : q.tiles;
    pos = min(start + each, s.hi);
    if (lo >= hi) continue;                      // no tile of it in this share
    const bool whole = lo == 0 && hi == q.tiles;
    segment<FORM, GROUPED>(p, part, sh, s.b, h, unit, q, lo, hi, whole ? -1 : 2 * (int64_t)s.index + (lo == 0), out, lse);
    if (lo == 0 && !whole) cut = Cut{s.b, h, unit, ((int)((start + each - 1) / s.len) - s.index + 1) | s.index << 16};
  }
  if (cuts && threadIdx.x == 0) *(int4*)(part.at + 4 * blockIdx.x) = make_int4(cut.b, cut.h, cut.unit, cut.parts);
}

// kv_splits: every unit in up to `parts` parts of its own.
template <int FORM, bool GROUPED>
__global__ __launch_bounds__(64 * kWaves, 1) void split_kernel(CacheProblem p, CachePartials part, int units, int parts,
                                                               uint16_t* __restrict__ out, float* __restrict__ lse) {
  __shared__ Shared sh;
  const int nbh = p.batch * p.hkv, bh = blockIdx.x % nbh, at = blockIdx.x / nbh;
  const int sp = at % parts, unit = at / parts, b = bh / p.hkv, h = bh % p.hkv;
  const Seq q(p, b);
  const int n = min(parts, q.tiles);
  if (unit >= q.units || sp >= n) return;
  const int lo = (int)((int64_t)q.tiles * sp / n), hi = (int)((int64_t)q.tiles * (sp + 1) / n);
  segment<FORM, GROUPED>(p, part, sh, b, h, unit, q, lo, hi, n > 1 ? ((int64_t)unit * nbh + bh) * parts + sp : -1, out, lse);
}

// Joins the parts of a unit that was cut: a workgroup takes eight packed rows, 32
// lanes each. units 0: the unit that each workgroup's share started; else those of every
// sequence, `parts` slots each.
__global__ __launch_bounds__(256) void join_kernel(CacheProblem p, CachePartials part, int units, int parts,
                                                   uint16_t* __restrict__ out, float* __restrict__ lse) {
  constexpr int per = kRows / 8;
  const int index = blockIdx.x / per;
  int b, h, unit, n;
  int64_t first, next;           // the first part's slot, and the second's; then one after the other by `step`
  int step = 1;
  if (units == 0) {
    const int4 cut = *(const int4*)(part.at + 4 * index);
    b = cut.x, h = cut.y, unit = cut.z, n = cut.w & 0xffff;
    first = 2 * (int64_t)(cut.w >> 16) + 1;
    next = first + 1;
    step = 2;
    if (n <= 1) return;
  } else {
    const int nbh = p.batch * p.hkv, bh = index % nbh;
    b = bh / p.hkv, h = bh % p.hkv, unit = index / nbh;
    first = (int64_t)index * parts;
    next = first + 1;
  }
  const Seq q(p, b);
  if (units != 0) {
    n = min(parts, q.tiles);
    if (n <= 1 || unit >= q.units) return;
  }
  const int first_q = unit * (kRows / p.g), rows = min(kRows / p.g, q.n - first_q) * p.g;
  const int pr = 8 * (blockIdx.x % per) + (threadIdx.x >> 5), d = 4 * (threadIdx.x & 31);
  if (pr >= rows) return;
  auto row = [&](int i) { return (i == 0 ? first : next + (int64_t)step * (i - 1)) * kRows + pr; };
  // eight parts a step, their loads in flight together (29 queries over 9280 keys, in 30 or 31
  // parts a unit, take 31.6 us; with the loads of four in flight 33.1)
  float mm = kNoRef, l = 0.f;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
  for (int i0 = 0; i0 < n; i0 += 8) {
    float2 ml[8];
    float4 y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t at = row(min(i0 + j, n - 1));          // past the end the last part again, for nothing
      ml[j] = *(const float2*)(part.ml + 2 * at);
      y[j] = *(const float4*)(part.o + at * kHeadDim + d);
    }
    float mn = mm;
#pragma unroll
    for (int j = 0; j < 8; ++j) mn = fmaxf(mn, ml[j].x);
    const float f = fast_exp2(mm - mn);
    mm = mn;
    l *= f;
    a.x *= f, a.y *= f, a.z *= f, a.w *= f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (i0 + j >= n) break;
      const float g = fast_exp2(ml[j].x - mm);
      l += g * ml[j].y;
      a.x += g * y[j].x, a.y += g * y[j].y, a.z += g * y[j].z, a.w += g * y[j].w;
    }
  }
  const float inv = (p.form == kCacheHead ? ld_uniform(p.v_head, h) : 1.f) / l;
  const int64_t at = (int64_t)(q.q0 + first_q + pr / p.g) * p.hq + h * p.g + pr % p.g;
  *(uint2*)(out + at * kHeadDim + d) =
      make_uint2(pack_bf16x2(a.x * inv, a.y * inv), pack_bf16x2(a.z * inv, a.w * inv));
  if (lse && d == 0) lse[at] = (mm + fast_log2(l)) * kLn2f;
}

int64_t units_of(const CacheProblem& p) { return ((int64_t)p.max_new * p.g + kRows - 1) / kRows; }
int tiles_of(const CacheProblem& p) { return std::max((p.max_kv + kStep - 1) / kStep, 1); }

// Whether units are cut. A second piece, and parts to join, cost as long as some eight tiles; and the more
// workgroups have a unit each, the less there is to gain. Whole and cut: 16 units of 8 tiles 21.9 and 22.9 us,
// of 16 34 and 26; 64 of 12 29.7 and 31.2, of 24 49 and 38; 128 of 16 38 and 45, of 36 72 and 66; 256 of 24 65 and
// 68. Of more than fit at once the lengths differ, and a workgroup has as many units as the next: 320 of 12 62 and 68,
// 768 109 and 107.
bool cut(const CacheProblem& p) {
  const int64_t units = (int64_t)p.batch * p.hkv * units_of(p);
  return tiles_of(p) > (units <= kShares ? 8 + units / 16 : 12);
}

// Workgroups of the equal shares, whole dies' worth: as many as the call's bounds allow. Which of them
// have a share the lengths say.
int shares_of(const CacheProblem& p) {
  const int64_t units = (int64_t)p.batch * p.hkv * units_of(p), line = units * (tiles_of(p) + kUnit);
  const int64_t most = std::min<int64_t>(kShares, std::max(units, line / kMinShare));
  return (int)((most + kXcds - 1) / kXcds * kXcds);
}

int parts_of(const CacheProblem& p) { return std::min(std::min(p.splits, tiles_of(p)), kMaxParts); }

template <int FORM, bool GROUPED>
hipError_t launch(const CacheProblem& p, const CachePartials& part, uint16_t* out, float* lse, hipStream_t s) {
  if (p.splits == 0) {
    const int grid = shares_of(p);
    const bool cuts = cut(p);
    cross_kernel<FORM, GROUPED><<<grid, 64 * kWaves, 0, s>>>(p, part, cuts, out, lse);
    if (cuts) join_kernel<<<grid * (kRows / 8), 256, 0, s>>>(p, part, 0, 0, out, lse);
    return hipGetLastError();
  }
  const int parts = parts_of(p);
  const int64_t units = (int64_t)p.batch * p.hkv * units_of(p), joins = units * (kRows / 8);
  if (!launchable(units * parts, 64 * kWaves) || (parts > 1 && !launchable(joins, 256))) return hipErrorInvalidValue;
  split_kernel<FORM, GROUPED><<<(unsigned)(units * parts), 64 * kWaves, 0, s>>>(p, part, (int)units_of(p), parts, out, lse);
  if (parts > 1) join_kernel<<<(unsigned)joins, 256, 0, s>>>(p, part, (int)units_of(p), parts, out, lse);
  return hipGetLastError();
}

template <int FORM>
hipError_t launch_pages(const CacheProblem& p, const CachePartials& part, uint16_t* out, float* lse, hipStream_t s) {
  // scales of blocks imply pages of a multiple of 16 tokens
  if constexpr (FORM == kCacheBlock) return launch<FORM, true>(p, part, out, lse, s);
  else return p.pm.page % 8 == 0 ? launch<FORM, true>(p, part, out, lse, s) : launch<FORM, false>(p, part, out, lse, s);
}

}  // namespace

void cache_cross_partials(const CacheProblem& p, int64_t* slots, int* rows) {
  *rows = kRows;
  if (p.splits == 0) *slots = cut(p) ? 2 * (int64_t)shares_of(p) : 0;
  else *slots = parts_of(p) > 1 ? (int64_t)p.batch * p.hkv * units_of(p) * parts_of(p) : 0;
}

hipError_t launch_cache_cross(const CacheProblem& p, const CachePartials& part, uint16_t* out, float* lse, hipStream_t s) {
  return p.form == kCacheBf16   ? launch_pages<kCacheBf16>(p, part, out, lse, s)
         : p.form == kCacheHead ? launch_pages<kCacheHead>(p, part, out, lse, s)
                                : launch_pages<kCacheBlock>(p, part, out, lse, s);
}

}  // namespace fp2
