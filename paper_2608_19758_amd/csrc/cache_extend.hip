// Attention of many query rows (prompts and chunks of them) over a paged
// cache: causal, over the first `sink` tokens and the last `window` ones.
//
// A unit is a (sequence, KV head, run of 256 / g positions): 256 packed rows,
// the g query heads of a position side by side, 32 rows a wave. Its visible
// keys come in tiles of 64 and only those are visited. A tile goes from the
// pool to registers and on to LDS as bf16 (codes are converted there, once for
// all waves, with the power of two of their block; a scale per head multiplies
// the scores and the output), two stages deep: while a tile is computed the
// next one is written and the one after that is on its way.
//
// Per tile and wave: S^T = K Q^T and O^T += V^T P^T on
// v_mfma_f32_32x32x16_bf16; a lane holds query l % 32 and 32 keys, so the
// probabilities go into the second product as they are, and the transposing
// LDS reads give V^T. The running maximum moves when a score passes it by more
// than 2^8. Probabilities are rounded to bf16 for the product, the matrix
// cores' type (half a step of 2^-8 each); sums, maxima and outputs are fp32.
//
// Bound by the products and, beside them, a step's chain of exponentials: a
// prompt of 32K tokens, 32 heads, window 4096, takes 2.10 ms from codes with
// scales of 64 tokens (0.98 PFLOP/s; a large bf16 matrix product reaches 1.22)
// and 2.34 from a bf16 cache, whose tiles take twice the loads.
//
// Calls of few units cut each unit's tiles into equal parts, joined by
// join_kernel. From 129 units on none is cut, and a unit of few rows (a single
// token beside a chunk) goes through all its keys alone.
#include <algorithm>

#include "cache.h"

namespace fp2 {

namespace {

constexpr float kLn2f = 0.69314718055994530942f;
constexpr int kStep = 64;        // keys per tile
constexpr int kWaves = 8;
constexpr int kRows = 32 * kWaves;
constexpr int kMaxParts = 32;
constexpr int kChip = 256;       // workgroups that run at a time, one a compute unit
constexpr int kMinTiles = 4;     // tiles of a part, at least
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

struct Tiles {
  int sinks, from, n;   // `sinks` leading tiles, then those from `from` on
};
__device__ __forceinline__ Tiles tiles_of(const CacheProblem& p, int first, int last) {
  Tiles t;
  t.sinks = (min(p.sink, last + 1) + kStep - 1) / kStep;
  t.from = max(max(first - p.window + 1, 0) / kStep, t.sinks);
  t.n = t.sinks + max(last / kStep - t.from + 1, 0);
  return t;
}

// A wave's unit, or false past the sequence.
struct Unit {
  int b, h, I, index;
  int q0, Lq, L;
  int64_t tok0;
  int i0, first, last;
};
__device__ __forceinline__ bool unit_at(const CacheProblem& p, int nq, int units_before, int bh, Unit& u) {
  u.I = nq - 1 - units_before;   // the longest rows first
  u.b = bh / p.hkv;
  u.h = bh % p.hkv;
  u.index = units_before * p.batch * p.hkv + bh;
  u.q0 = ld_uniform(p.cu, u.b);
  u.Lq = ld_uniform(p.cu, u.b + 1) - u.q0;
  u.tok0 = ld_uniform(p.cuk, u.b);
  u.L = ld_uniform(p.cuk, u.b + 1) - (int)u.tok0;
  const int np = kRows / p.g;
  u.i0 = u.I * np;
  if (u.i0 >= u.Lq) return false;
  u.first = u.L - u.Lq + u.i0;
  u.last = u.L - u.Lq + min(u.i0 + np, u.Lq) - 1;
  return true;
}

__device__ __forceinline__ bool sees(const CacheProblem& p, int pos, int key) {
  return key <= pos && (key < p.sink || key > pos - p.window);
}

// Infinities and NaN of eight bf16 values set to zero; whether there were any.
__device__ __forceinline__ bool drop_odd(uint4& v) {
  uint32_t d[4] = {v.x, v.y, v.z, v.w};
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if ((d[i] & 0x7f800000u) == 0x7f800000u) d[i] &= 0xffffu, bad = true;
    if ((d[i] & 0x7f80u) == 0x7f80u) d[i] &= 0xffff0000u, bad = true;
  }
  v = make_uint4(d[0], d[1], d[2], d[3]);
  return bad;
}

struct Shared {
  uint4 k[2][kStep * 16];
  uint4 v[2][kStep * 16];
  int bad[4];               // a tile's values had infinities or NaN that some row does not see
};

// FORM: the cache's type. WIDE: pages hold a multiple of 64 tokens, so a tile
// lies in one and its address is uniform (scalar). The prompt above in bf16: 2.34
// ms, from pages of 48 tokens 2.6.
template <int FORM, bool WIDE>
__global__ __launch_bounds__(64 * kWaves, 1) void extend_kernel(CacheProblem p, CachePartials part,
                                                                int nq, int parts,
                                                                uint16_t* __restrict__ out,
                                                                float* __restrict__ lse) {
  constexpr bool kBf16 = FORM == kCacheBf16;
  constexpr int ESZ = kBf16 ? 2 : 1;
  constexpr int NJ = kBf16 ? 2 : 1;              // rows of a tile per thread
  constexpr int TPR = kBf16 ? 16 : 8;            // threads of a row, 16 bytes each
  __shared__ Shared sh;
  const int nbh = p.batch * p.hkv;
  const int rem = blockIdx.x % (nbh * parts);
  Unit u;
  if (!unit_at(p, nq, blockIdx.x / (nbh * parts), rem % nbh, u)) return;
  const int sp = rem / nbh;
  const Tiles tl = tiles_of(p, u.first, u.last);
  const int nsp = min(parts, tl.n);
  if (sp >= nsp) return;
  const int lo = (int)((int64_t)tl.n * sp / nsp), hi = (int)((int64_t)tl.n * (sp + 1) / nsp);
  auto key0_at = [&](int i) { return kStep * (i < tl.sinks ? i : tl.from + i - tl.sinks); };

  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const int pr = 32 * w + l32;                   // packed row
  const int pos = u.first + pr / p.g;
  const int hq = u.h * p.g + pr % p.g;
  const bool valid = pos <= u.last;
  const int wfirst = u.first + 32 * w / p.g, wlast = u.first + (32 * w + 31) / p.g;
  const int64_t qrow = (int64_t)(u.q0 + u.i0 + min(pr / p.g, u.last - u.first)) * p.hq + hq;

  bf16x8_t qb[8];
#pragma unroll
  for (int ds = 0; ds < 8; ++ds)
    qb[ds] = __builtin_bit_cast(bf16x8_t, *(const uint4*)(p.q + qrow * kHeadDim + 16 * ds + 8 * half));
  f32x16_t o[4];
#pragma unroll
  for (int dt = 0; dt < 4; ++dt) o[dt] = f32x16_t{};
  float m = kNoRef, l = 0.f;
  const float cs = score_scale<FORM>(p, u.h);
  float vsc = 1.f;
  if constexpr (FORM == kCacheHead) vsc = ld_uniform(p.v_head, u.h);

  // ---- staging
  const int64_t rowb = (int64_t)p.hkv * kHeadDim * ESZ;
  const int64_t hoff = (int64_t)u.h * kHeadDim * ESZ;
  const int c = tid % TPR, r0 = tid / TPR;       // this thread's chunk and first row of a tile
  struct Regs {
    uint4 k[NJ], v[NJ];
    uint32_t ks, vs;
  };
  // Where a tile lies (WIDE), or this thread's rows of it: the table's entries
  // as loaded (used a tile later, so that nothing waits for them) and the places
  // in the pages. Keys past the sequence stand on valid ones.
  struct Where {
    int page[NJ], off[NJ];
  };
  const int32_t* table = p.pm.table + (int64_t)u.b * p.pm.stride;
  auto where = [&](int i) {
    Where a;
    const int k0 = key0_at(min(i, hi - 1));      // past the end the last tile again
#pragma unroll
    for (int j = 0; j < NJ; ++j) {
      const int t = WIDE ? k0 : min(k0 + r0 + 32 * j, u.L - 1);
      const int pg = p.pm.shift >= 0 ? t >> p.pm.shift : t / p.pm.page;
      a.page[j] = WIDE ? ld_uniform(table, pg) : table[pg];
      a.off[j] = t - pg * p.pm.page;
    }
    return a;
  };
  const uint32_t roff = (uint32_t)(r0 * rowb + 16 * c);                  // WIDE: this thread's place in a tile
  const uint32_t soff = (uint32_t)((r0 >> p.sb_shift) * p.hkv);          // and its scale's among the tile's
  auto load = [&](const Where& a, Regs& x) {
    if constexpr (WIDE) {
      const int64_t s0 = (int64_t)a.page[0] * p.pm.page + a.off[0];
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        const int64_t at = (s0 + 32 * j) * rowb + hoff;
        x.k[j] = *(const uint4*)(p.k + at + roff);
        x.v[j] = *(const uint4*)(p.v + at + roff);
      }
      if constexpr (FORM == kCacheBlock) {
        const int64_t at = (s0 >> p.sb_shift) * p.hkv + u.h;
        x.ks = (p.k_block + at)[soff];
        x.vs = (p.v_block + at)[soff];
      }
    } else {
      int64_t s[NJ];
#pragma unroll
      for (int j = 0; j < NJ; ++j) {
        s[j] = (int64_t)a.page[j] * p.pm.page + a.off[j];
        const int64_t at = s[j] * rowb + hoff + 16 * c;
        x.k[j] = *(const uint4*)(p.k + at);
        x.v[j] = *(const uint4*)(p.v + at);
      }
      if constexpr (FORM == kCacheBlock) {
        const int64_t at = (s[0] >> p.sb_shift) * p.hkv + u.h;
        x.ks = p.k_block[at];
        x.vs = p.v_block[at];
      }
    }
  };
  auto widen = [](uint4 x, uint32_t byte, uint4 (&y)[2]) {   // 16 codes -> 16 bf16
    const float s = FORM == kCacheBlock ? block_scale(byte) : 1.f;
    const uint32_t d[4] = {x.x, x.y, x.z, x.w};
    uint32_t z[8];
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const b2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)d[i], s, false);
      const b2 b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)d[i], s, true);
      z[2 * i] = __builtin_bit_cast(uint32_t, a);
      z[2 * i + 1] = __builtin_bit_cast(uint32_t, b);
    }
    y[0] = make_uint4(z[0], z[1], z[2], z[3]);
    y[1] = make_uint4(z[4], z[5], z[6], z[7]);
  };
  auto write_k = [&](int i, const Regs& x) {
    uint4 y[2];
    if constexpr (kBf16) y[0] = x.k[0], y[1] = x.k[NJ - 1];
    else widen(x.k[0], x.ks, y);
#pragma unroll
    for (int j = 0; j < 2; ++j)
      sh.k[i & 1][kplace(kBf16 ? r0 + 32 * j : r0, kBf16 ? c : 2 * c + j)] = y[j];
  };
  auto write_v = [&](int i, const Regs& x) {
    uint4 y[2];
    if constexpr (kBf16) y[0] = x.v[0], y[1] = x.v[NJ - 1];
    else widen(x.v[0], x.vs, y);
    // values that no row of the unit sees (the pool holds anything there) must
    // not meet zero probabilities; nor infinities and NaN that only some see
    const int k0 = key0_at(min(i, hi - 1));
    if (k0 + kStep - 1 > u.first || (k0 <= u.last - p.window && k0 + kStep > p.sink)) {
      bool bad = false;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int key = k0 + r0 + (kBf16 ? 32 * j : 0);
        const bool any = key <= u.last && (key < p.sink || key > u.first - p.window);
        const bool all = key <= u.first && (key < p.sink || key > u.last - p.window);
        if (!any) y[j] = make_uint4(0, 0, 0, 0);
        else if (!all) bad |= drop_odd(y[j]);
      }
      if (bad && i < hi) sh.bad[i & 3] = 1;
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
      sh.v[i & 1][vplace(kBf16 ? r0 + 32 * j : r0, kBf16 ? c : 2 * c + j)] = y[j];
  };

  // V^T fragment of 16 keys kg and output tile dt: place i' of lane half H is
  // key 16 kg + 8 (i' / 4) + 4 H + i' % 4
  const int g16 = lane >> 4, i16 = lane & 15;
  auto vread = [&](const uint4* vt, int kg, int dt) {
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

  // scores of tile i: element e of s[uu] is key k0 + 32 uu + 8 (e / 4) + 4 half + e % 4
  auto qk = [&](int i, f32x16_t (&s)[2]) {
    const uint4* kt = sh.k[i & 1];
#pragma unroll
    for (int uu = 0; uu < 2; ++uu) {
      s[uu] = f32x16_t{};
#pragma unroll
      for (int ds = 0; ds < 8; ++ds)
        s[uu] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
            __builtin_bit_cast(bf16x8_t, kt[kplace(32 * uu + l32, 2 * ds + half)]), qb[ds], s[uu], 0, 0, 0);
    }
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
  auto exponentials = [&](f32x16_t (&s)[2]) {
    float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int uu = 0; uu < 2; ++uu)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[uu][e] = fast_exp2(fmaf(s[uu][e], cs, -m));
        sum[e & 3] += s[uu][e];
      }
    l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
  };
  auto pv = [&](int i, const f32x16_t (&s)[2]) {
    const uint4* vt = sh.v[i & 1];
#pragma unroll
    for (int kg = 0; kg < 4; ++kg) {
      uint32_t pw[4];
#pragma unroll
      for (int q = 0; q < 4; ++q)
        pw[q] = pack_bf16x2(s[kg >> 1][8 * (kg & 1) + 2 * q], s[kg >> 1][8 * (kg & 1) + 2 * q + 1]);
      const bf16x8_t pb = __builtin_bit_cast(bf16x8_t, make_uint4(pw[0], pw[1], pw[2], pw[3]));
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
        o[dt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vread(vt, kg, dt), pb, o[dt], 0, 0, 0);
    }
  };
  auto masked = [&](int k0) {
    return k0 + kStep - 1 > wfirst || (k0 <= wlast - p.window && k0 + kStep > p.sink);
  };
  auto mask = [&](int k0, f32x16_t (&s)[2]) {
#pragma unroll
    for (int uu = 0; uu < 2; ++uu)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = k0 + 32 * uu + 8 * (e >> 2) + 4 * half + (e & 3);
        s[uu][e] = pinned(sees(p, pos, key) ? s[uu][e] : -INFINITY);
      }
  };
  // rare: what drop_odd took, to the rows that see it
  auto add_odd = [&](int k0) {
#pragma unroll 1
    for (int k = 0; k < kStep; ++k) {
      const int key = k0 + k;
      const bool any = key <= u.last && (key < p.sink || key > u.first - p.window);
      const bool all = key <= u.first && (key < p.sink || key > u.last - p.window);
      if (!any || all) continue;
      const uint8_t* row = p.v + slot_of(p.pm, u.b, u.tok0, key) * rowb + hoff;
#pragma unroll
      for (int dt = 0; dt < 4; ++dt)
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int d = 32 * dt + 8 * (e >> 2) + 4 * half + (e & 3);
          float x;
          if constexpr (kBf16) x = bf16_to_f32(((const uint16_t*)row)[d]);
          else x = (row[d] & 0x7f) == 0x7f ? __uint_as_float(0x7fc00000u) : 0.f;
          o[dt][e] += pinned(!(fabsf(x) < INFINITY) && sees(p, pos, key) ? x : 0.f);
        }
    }
  };

  // Keys run one tile ahead of values: the scores of the next tile are computed
  // while the exponentials of this one run on the vector ALUs (in one block, behind
  // the branch that moves the maximum: 2.10 ms, with the scores before it 2.13).
  Regs regs;
  if (tid < 4) sh.bad[tid] = 0;
  __syncthreads();
  Where at = where(lo + 1);
  load(where(lo), regs);
  write_k(lo, regs);
  write_v(lo, regs);
  load(at, regs);
  at = where(lo + 2);
  lds_barrier();
  f32x16_t s[2], t[2];
  qk(lo, s);
  write_k(lo + 1, regs);
  // tile i, whose scores are in x, and the scores of the next one into y
  auto step = [&](int i, f32x16_t (&x)[2], f32x16_t (&y)[2]) {
    lds_barrier();   // keys of tile i + 1 and values of tile i are there; all are done with those before
    if (tid == 0) sh.bad[(i + 2) & 3] = 0;   // read last for tile i - 2, written next for i + 2
    // (past the end the last tile is staged again)
    write_v(i + 1, regs);
    load(at, regs);
    at = where(i + 3);
    const int k0 = key0_at(i);
    if (masked(k0)) mask(k0, x);
    move_max(x);
    qk(i + 1, y);
    exponentials(x);
    pv(i, x);
    if (sh.bad[i & 3]) add_odd(k0);
    write_k(i + 2, regs);
  };
#pragma unroll 1
  for (int i = lo; i < hi; i += 2) {
    step(i, s, t);
    if (i + 1 >= hi) break;
    step(i + 1, t, s);
  }

  // ---- output
  l += __shfl_xor(l, 32, 64);
  if (nsp > 1) {
    if (!valid) return;
    const int64_t row = ((int64_t)u.index * parts + sp) * kRows + pr;
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

// Joins the parts of each unit: a workgroup takes eight packed rows, 32 lanes each.
__global__ __launch_bounds__(256) void join_kernel(CacheProblem p, CachePartials part, int nq, int parts,
                                                   uint16_t* __restrict__ out, float* __restrict__ lse) {
  const int nbh = p.batch * p.hkv, per = kRows / 8;
  const int unit = blockIdx.x / per;
  Unit u;
  if (!unit_at(p, nq, unit / nbh, unit % nbh, u)) return;
  const int nsp = min(parts, tiles_of(p, u.first, u.last).n);
  const int pr = 8 * (blockIdx.x % per) + (threadIdx.x >> 5), d = 4 * (threadIdx.x & 31);
  if (nsp <= 1 || u.first + pr / p.g > u.last) return;
  const int64_t row0 = (int64_t)u.index * parts * kRows + pr;
  float mm = kNoRef;
  for (int s = 0; s < nsp; ++s) mm = fmaxf(mm, part.ml[2 * (row0 + (int64_t)s * kRows)]);
  float l = 0.f;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s = 0; s < nsp; ++s) {
    const int64_t row = row0 + (int64_t)s * kRows;
    const float2 ml = *(const float2*)(part.ml + 2 * row);
    const float4 y = *(const float4*)(part.o + row * kHeadDim + d);
    const float f = fast_exp2(ml.x - mm);
    l += f * ml.y;
    a.x += f * y.x, a.y += f * y.y, a.z += f * y.z, a.w += f * y.w;
  }
  const float inv = (p.form == kCacheHead ? ld_uniform(p.v_head, u.h) : 1.f) / l;
  const int64_t at = (int64_t)(u.q0 + u.i0 + pr / p.g) * p.hq + u.h * p.g + pr % p.g;
  *(uint2*)(out + at * kHeadDim + d) =
      make_uint2(pack_bf16x2(a.x * inv, a.y * inv), pack_bf16x2(a.z * inv, a.w * inv));
  if (lse && d == 0) lse[at] = (mm + fast_log2(l)) * kLn2f;
}

int query_tiles(const CacheProblem& p) { return (p.max_new * p.g + kRows - 1) / kRows; }

// Parts of a unit: as many as fill the chip, of at least kMinTiles tiles. 256
// tokens behind 30000 take 156 us, and 896 whole; 256 behind 1000 28 us, with
// parts of 8 tiles or more 36.
int parts_for(const CacheProblem& p) {
  const int64_t units = (int64_t)p.batch * p.hkv * query_tiles(p);
  const int64_t seen = std::min<int64_t>(p.max_kv, (int64_t)p.window + kRows / p.g + p.sink);
  const int tiles = (int)(seen / kStep) + 3;
  if (p.splits) return std::min(std::min(p.splits, tiles), kMaxParts);
  const int64_t fill = kChip / std::max<int64_t>(units, 1);
  return (int)std::max<int64_t>(1, std::min<int64_t>({fill, tiles / kMinTiles, kMaxParts}));
}

template <int FORM>
hipError_t launch(const CacheProblem& p, const CachePartials& part, uint16_t* out, float* lse,
                  hipStream_t s) {
  const int nq = query_tiles(p), parts = parts_for(p);
  const int64_t units = (int64_t)p.batch * p.hkv * nq;
  const int64_t joins = units * (kRows / 8);
  if (!launchable(units * parts, 64 * kWaves) || (parts > 1 && !launchable(joins, 256)))
    return hipErrorInvalidValue;
  const dim3 grid((unsigned)(units * parts)), threads(64 * kWaves);
  if (p.pm.page % kStep == 0)
    extend_kernel<FORM, true><<<grid, threads, 0, s>>>(p, part, nq, parts, out, lse);
  else
    extend_kernel<FORM, false><<<grid, threads, 0, s>>>(p, part, nq, parts, out, lse);
  if (parts > 1) join_kernel<<<(unsigned)joins, 256, 0, s>>>(p, part, nq, parts, out, lse);
  return hipGetLastError();
}

}  // namespace

void cache_extend_partials(const CacheProblem& p, int64_t* slots, int* rows) {
  const int parts = parts_for(p);
  *slots = parts > 1 ? (int64_t)p.batch * p.hkv * query_tiles(p) * parts : 0;
  *rows = kRows;
}

hipError_t launch_cache_extend(const CacheProblem& p, const CachePartials& part, uint16_t* out,
                               float* lse, hipStream_t s) {
  return p.form == kCacheBf16   ? launch<kCacheBf16>(p, part, out, lse, s)
         : p.form == kCacheHead ? launch<kCacheHead>(p, part, out, lse, s)
                                : launch<kCacheBlock>(p, part, out, lse, s);
}

}  // namespace fp2
