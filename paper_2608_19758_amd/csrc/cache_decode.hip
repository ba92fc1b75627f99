// Attention of few query rows over a paged cache: single tokens, drafted
// tokens, short tails. Causal, over the first `sink` tokens and the last
// `window` ones.
//
// A unit is a (sequence, KV head): its rows are the new tokens times the g
// query heads that share the head's keys, at most 64 (16 NT). The keys are
// read once for all of them, so the call is bound by memory, 2 * 128 bytes a
// key and head in 8 bits, twice that in bf16.
//
// * Work: the visible keys of a sequence come in tiles of 32. All tiles of the
//   call are dealt to the workgroups in equal shares (each works its own out
//   from the lengths, which are on the device only); combine_kernel joins
//   sequences that lie in several shares. The waves of a workgroup take
//   different heads of the same tokens; where there are fewer heads they
//   alternate tiles and join in LDS.
// * A wave goes from global memory to the matrix cores without LDS.
//   S^T = K Q^T on v_mfma_f32_16x16x32_bf16: A holds 16 keys, and which of the
//   128 dimensions stands at which place of a product is free, so four lanes
//   load 64 adjacent bytes of a row. A lane then holds query l % 16 and keys
//   4 (l / 16) + i of two groups of 16: these eight are the B operand of
//   O^T += V^T P^T if the values come in that order. A lane loads eight
//   dimensions of those eight keys (16 lanes a row) and turns the 8 x 8 block
//   by byte permutes; row r of A is then dimension 8 r + t of product t.
// * Codes become bf16 exactly, with the block's power of two in the
//   conversion; a scale per head multiplies the scores and the output.
// * The running maximum m of a row moves only when a score passes it by more
//   than 2^8, so most tiles have no exchange between lanes. Probabilities are
//   rounded to bf16 for the product, the matrix cores' type (half a step of 2^-8
//   each); sums, maxima and outputs are fp32.
//
// One token of each of 32 sequences of 1.3K to 112K tokens, 8 heads of 4: 274 us
// in codes (5.5 TB/s), 525 in bf16 (5.7); one sequence of 128K 63 us, of which 9
// are the join; 64 with windows of 4096 tokens 92 us. 8 drafted tokens and 8
// heads a group (64 rows), 8 sequences: 96 us (3.2 TB/s); there a wave alone on
// its SIMD has products and exponentials one after the other.
#include <algorithm>
#include <type_traits>

#include "cache_few.h"

namespace fp2 {

namespace {

constexpr float kLn2f = 0.69314718055994530942f;
constexpr float kTau = 8.0f;
constexpr float kNoRef = -1e30f; // maximum of a row that saw no key

// A tile as it comes from memory.
template <int FORM>
struct Raw {
  static constexpr bool kBf16 = FORM == kCacheBf16;
  uint4 k[2][kBf16 ? 4 : 2];                               // keys r and 16 + r, 16 bytes a chunk
  std::conditional_t<kBf16, uint4, uint2> v[8];            // eight keys, eight dimensions
  uint32_t ks[2], vs[2];                                   // kCacheBlock: scale bytes of the groups
};

// Infinities and NaN among packed values, with no compare a value: adding the
// lowest exponent bit (bf16), or one (codes), to a magnitude carries into the
// sign's place only from them. The top bit of each odd value is returned.
__device__ __forceinline__ uint32_t odd_bf16(uint32_t x) {
  return ((x & 0x7f807f80u) + 0x00800080u) & 0x80008000u;
}
__device__ __forceinline__ uint32_t odd_codes(uint32_t x) {
  return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u;
}
__device__ __forceinline__ bool odd_values(uint4 v) {
  return (odd_bf16(v.x) | odd_bf16(v.y) | odd_bf16(v.z) | odd_bf16(v.w)) != 0;
}
__device__ __forceinline__ bool odd_values(uint2 v) { return (odd_codes(v.x) | odd_codes(v.y)) != 0; }
// The values with those set to zero.
__device__ __forceinline__ uint4 even_values(uint4 v) {
  auto f = [](uint32_t x) { return x & ~((odd_bf16(x) >> 15) * 0xffffu); };
  return make_uint4(f(v.x), f(v.y), f(v.z), f(v.w));
}
__device__ __forceinline__ uint2 even_values(uint2 v) {
  auto f = [](uint32_t x) { return x & ~((odd_codes(x) >> 7) * 0xffu); };
  return make_uint2(f(v.x), f(v.y));
}
// fp32 bits of value e of the eight where it is odd, else zero.
__device__ __forceinline__ uint32_t odd_value(uint4 v, int e) {
  const uint32_t d = e < 2 ? v.x : e < 4 ? v.y : e < 6 ? v.z : v.w, o = odd_bf16(d) >> 15;
  return e & 1 ? d & ((o >> 16) * 0xffff0000u) : (d << 16) & ((o & 1) * 0xffff0000u);
}
__device__ __forceinline__ uint32_t odd_value(uint2 v, int e) {
  return ((odd_codes(e < 4 ? v.x : v.y) >> (8 * (e & 3) + 7)) & 1) * 0x7fc00000u;
}

// FORM: the cache's type. NT: 16-row tiles of query rows of a wave. RH: waves
// that share the rows. W: waves (many registers a wave: four, one a SIMD).
// GROUPED: pages hold a multiple of 16 tokens, so the 16 keys of a group lie one
// after the other and their address is uniform (scalar); otherwise every key has
// its own (8 sequences of 64 rows: 99 us, with pages of 24 tokens 108).
template <int FORM, int NT, int RH, int W, bool GROUPED>
__global__ __launch_bounds__(64 * W, W / 4) void decode_kernel(CacheProblem p, CachePartials part,
                                                               int shares, uint16_t* __restrict__ out,
                                                               float* __restrict__ lse) {
  constexpr bool kBf16 = FORM == kCacheBf16;
  constexpr int ESZ = kBf16 ? 2 : 1;
  constexpr int KC = kBf16 ? 4 : 2;            // 16-byte chunks of a key per lane
  constexpr int LDR = kHeadDim + 4;            // LDS row, padded against bank conflicts
  __shared__ float s_o[W][16][LDR];
  __shared__ float s_ml[W][16][2];
  const int groups = p.hkv / p.heads, index = blockIdx.x / groups;
  const int units = p.heads * RH, KS = W / units;   // (head, half of the rows): how many waves alternate its tiles
  Share sh;
  if (!find_share(p, shares, index, sh)) return;

  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.x % groups * p.heads + w % p.heads;
  const int ks = w / units;                    // place among the head's tiles
  const int rb = RH == 1 ? 0 : w / p.heads % RH * 16 * NT;   // the wave's first packed row
  const int c16 = lane & 15, kg = lane >> 4;
  const float cs = score_scale<FORM>(p, h);
  float vsc = 1.f;
  if constexpr (FORM == kCacheHead) vsc = ld_uniform(p.v_head, h);
  const int64_t rowb = (int64_t)p.hkv * kHeadDim * ESZ;
  const int64_t hoff = (int64_t)h * kHeadDim * ESZ;
  const uint8_t* K = p.k + hoff;
  const uint8_t* V = p.v + hoff;
  const uint32_t koff = (uint32_t)(c16 * rowb + 16 * kg);
  const uint32_t voff = (uint32_t)(4 * kg * rowb + 8 * ESZ * c16);

  int b = sh.b, base = sh.base;
#pragma unroll 1
  for (bool again = false;; again = true) {
  if (again) {
    sh.q0 = ld_uniform(p.cu, b);
    sh.Lq = ld_uniform(p.cu, b + 1) - sh.q0;
    sh.L = ld_uniform(p.cuk, b + 1) - ld_uniform(p.cuk, b);
  }
  const int q0 = sh.q0, Lq = sh.Lq, L = sh.L;
  const int first = L - Lq, last = L - 1;      // positions of the first and the last row
  const int rows = Lq * p.g;
  const Tiles tl = tiles_of(p, Lq, L);
  const int lo = max(sh.lo, base) - base, hi = min(sh.hi, base + tl.n) - base;
  auto tile_at = [&](int i) { return i < tl.sinks ? i : tl.from + i - tl.sinks; };
  if (lo < hi) {

  // queries: the B operand of score product s holds, for lane group kg, eight
  // of the dimensions that the key operand holds there
  bf16x8_t qb[NT][4];
  int pos[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = rb + 16 * nt + c16;
    pos[nt] = first + r / p.g;
    const uint16_t* qrow = p.q + ((int64_t)(q0 + min(r / p.g, Lq - 1)) * p.hq + h * p.g + r % p.g) *
                                     kHeadDim;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int d = kBf16 ? 32 * s + 8 * kg : 64 * (s >> 1) + 16 * kg + 8 * (s & 1);
      uint4 x = *(const uint4*)(qrow + d);
      if (r >= rows) x = make_uint4(0, 0, 0, 0);
      qb[nt][s] = __builtin_bit_cast(bf16x8_t, x);
    }
  }
  f32x4_t o[NT][8];
  float m[NT], l[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
#pragma unroll
    for (int t = 0; t < 8; ++t) o[nt][t] = f32x4_t{};
    m[nt] = kNoRef;
    l[nt] = 0.f;
  }

  const int32_t* table = p.pm.table + (int64_t)b * p.pm.stride;
  auto where = [&](int tile) { return where_at<GROUPED>(p.pm, table, tile, last, lane); };
  typedef std::conditional_t<kBf16, uint4, uint2> vrow_t;
  auto load = [&](const Where& a, Raw<FORM>& x, uint32_t on) {   // on: ~0, or 0 to read one row over and over
    if constexpr (GROUPED) {
      const int64_t slot[2] = {a.slot(p.pm, 0), a.slot(p.pm, 1)};
      if constexpr (FORM == kCacheBlock) {   // before the rows: loads come back in order
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int64_t at = (slot[u] >> p.sb_shift) * p.hkv + h;
          x.ks[u] = p.k_block[at];
          x.vs[u] = p.v_block[at];
        }
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint8_t* kb = K + slot[u] * rowb;
#pragma unroll
        for (int c = 0; c < KC; ++c) x.k[u][c] = *(const uint4*)(kb + ((koff & on) + 64u * c));
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint8_t* vb = V + slot[u] * rowb;
#pragma unroll
        for (int e = 0; e < 4; ++e) x.v[4 * u + e] = *(const vrow_t*)(vb + e * rowb + (voff & on));
      }
    } else {
      const int slot = (int)a.slot(p.pm, 0);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint8_t* kb = K + (int64_t)__shfl(slot, 16 * u + c16, 64) * rowb + 16 * kg;
#pragma unroll
        for (int c = 0; c < KC; ++c) x.k[u][c] = *(const uint4*)(kb + 64 * c);
#pragma unroll
        for (int e = 0; e < 4; ++e)
          x.v[4 * u + e] = *(const vrow_t*)(V + (int64_t)__shfl(slot, 16 * u + 4 * kg + e, 64) * rowb +
                                            8 * ESZ * c16);
      }
    }
  };

  // the maximum that scores become probabilities against moves when one passes it by more than kTau
  auto move_max = [&](int nt, const f32x4_t (&s)[2]) {
    float mx = -INFINITY;
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[u][i]);
    mx *= cs;
    if (__any(mx > m[nt] + kTau)) {
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float mn = mx > m[nt] + kTau ? mx : m[nt];
      const float f = fast_exp2(m[nt] - mn);
      m[nt] = mn;
      l[nt] *= f;
#pragma unroll
      for (int t = 0; t < 8; ++t) o[nt][t] *= f;
    }
  };

  auto step = [&](int tile, Raw<FORM>& x) {
    const int t0 = kTile * tile;
    // keys that some row does not see: behind the first row, or before the
    // last row's window and not among the first tokens
    const bool masked = t0 + kTile - 1 > first ||
                        (t0 <= last - p.window && t0 + kTile > p.sink);
    f32x4_t s[NT][2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      bf16x8_t a[4];
      if constexpr (kBf16) {
#pragma unroll
        for (int c = 0; c < 4; ++c) a[c] = __builtin_bit_cast(bf16x8_t, x.k[u][c]);
      } else {
        const float sc = FORM == kCacheBlock ? block_scale(x.ks[u]) : 1.f;
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          a[2 * c] = codes_to_bf16(x.k[u][c].x, x.k[u][c].y, sc);
          a[2 * c + 1] = codes_to_bf16(x.k[u][c].z, x.k[u][c].w, sc);
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        s[nt][u] = f32x4_t{};
#pragma unroll
        for (int c = 0; c < 4; ++c)
          s[nt][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[c], qb[nt][c], s[nt][u], 0, 0, 0);
      }
    }
    if (masked) {
      // element i of group u is key t0 + 16 u + 4 kg + i
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            s[nt][u][i] = sees(p, pos[nt], t0 + 16 * u + 4 * kg + i) ? s[nt][u][i] : -INFINITY;
            s[nt][u][i] = pinned(s[nt][u][i]);
          }
      // values that no row sees (the pool holds anything there) must not meet
      // the zero probabilities; nor infinities and NaN that some row does not see
      if constexpr (FORM == kCacheBlock) {   // (a scale of 255 makes NaN of zeros)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          const int key = t0 + 16 * u;
          if (key > last || (key >= p.sink && key + 15 <= first - p.window)) x.vs[u] = 127;
        }
      }
      bool bad = false;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int key = t0 + 16 * (e >> 2) + 4 * kg + (e & 3);
        const bool any = key <= last && (key < p.sink || key > first - p.window);
        if (!any) x.v[e] = vrow_t{};
        bad |= odd_values(x.v[e]);
        x.v[e].x = pinned(x.v[e].x);
      }
      if (Lq > 1 && __any(bad)) {
        // rare: such values are added to the rows that see them by hand, infinities
        // (codes have none) once the maximum is this tile's: times the factor of its
        // move, which may be 0, they would become NaN
        if constexpr (kBf16) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) move_max(nt, s[nt]);
        }
#pragma unroll 1
        for (int k = 0; k < kTile; ++k) {
          const int key = t0 + k;
          if (key > last || !(key < p.sink || key > first - p.window)) continue;
          const uint8_t* row = V + slot_of(p.pm, b, 0, key) * rowb;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const vrow_t v = *(const vrow_t*)(row + (32 * kg + 8 * i) * ESZ);
            if (!odd_values(v)) continue;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
              const uint32_t see = sees(p, pos[nt], key) ? ~0u : 0u;
#pragma unroll
              for (int t = 0; t < 8; ++t) {
                o[nt][t][i] += __uint_as_float(odd_value(v, t) & see);
                o[nt][t][i] = pinned(o[nt][t][i]);
              }
            }
          }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x.v[e] = even_values(x.v[e]);
          x.v[e].x = pinned(x.v[e].x);
        }
      }
    }
    // values: pair (2p, 2p + 1) of keys, dimension 8 c16 + t -> word p of
    // product t's A operand
    uint32_t va[8][4];
    if constexpr (kBf16) {
#pragma unroll
      for (int pr = 0; pr < 4; ++pr) {
        const uint4 a = x.v[2 * pr], b = x.v[2 * pr + 1];
        const uint32_t ad[4] = {a.x, a.y, a.z, a.w}, bd[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          va[2 * t][pr] = __builtin_amdgcn_perm(bd[t], ad[t], 0x05040100u);
          va[2 * t + 1][pr] = __builtin_amdgcn_perm(bd[t], ad[t], 0x07060302u);
        }
      }
    } else {
#pragma unroll
      for (int pr = 0; pr < 4; ++pr) {
        const float sc = FORM == kCacheBlock ? block_scale(x.vs[pr >> 1]) : 1.f;
        const uint2 a = x.v[2 * pr], b = x.v[2 * pr + 1];
        const uint32_t ad[2] = {a.x, a.y}, bd[2] = {b.x, b.y};
#pragma unroll
        for (int t = 0; t < 4; ++t) {   // bytes a0 b0 a1 b1 of two dimensions
          const uint32_t y = __builtin_amdgcn_perm(bd[t >> 1], ad[t >> 1],
                                                   t & 1 ? 0x07030602u : 0x05010400u);
          typedef __bf16 b2 __attribute__((ext_vector_type(2)));
          const b2 y0 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)y, sc, false);
          const b2 y1 = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)y, sc, true);
          va[2 * t][pr] = __builtin_bit_cast(uint32_t, y0);
          va[2 * t + 1][pr] = __builtin_bit_cast(uint32_t, y1);
        }
      }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      move_max(nt, s[nt]);
      float e[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) e[i] = fast_exp2(fmaf(s[nt][i >> 2][i & 3], cs, -m[nt]));
      l[nt] += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
      const bf16x8_t pb = __builtin_bit_cast(
          bf16x8_t, make_uint4(pack_bf16x2(e[0], e[1]), pack_bf16x2(e[2], e[3]),
                               pack_bf16x2(e[4], e[5]), pack_bf16x2(e[6], e[7])));
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const bf16x8_t a = __builtin_bit_cast(bf16x8_t, make_uint4(va[t][0], va[t][1], va[t][2], va[t][3]));
        o[nt][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, pb, o[nt][t], 0, 0, 0);
      }
    }
  };

  // The next tile's rows are on their way while a tile is computed. Loads are
  // never left out (past the end they repeat a row): behind a load that may not
  // have been issued the compiler can only wait for all of them.
  if (lo + ks < hi) {
    Raw<FORM> r0, r1;
    auto where_to = [&](int i) { return where(tile_at(min(i, hi - 1))); };
    load(where_to(lo + ks), r0, ~0u);
    Where a0 = where_to(lo + ks + KS), a1;
#pragma unroll 1
    for (int i = lo + ks; i < hi; i += 2 * KS) {
      load(a0, r1, i + KS < hi ? ~0u : 0u);
      a1 = where_to(i + 2 * KS);
      step(tile_at(i), r0);
      load(a1, r0, i + 2 * KS < hi ? ~0u : 0u);
      a0 = where_to(i + 3 * KS);
      if (i + KS < hi) step(tile_at(i + KS), r1);
    }
  }

  // A sequence in several shares leaves its part in slot 2 * share, if it
  // started in an earlier one, or 2 * share + 1 (kv_splits: the share's own).
  const bool split = p.splits ? hi - lo < tl.n : base < sh.lo || base + tl.n > sh.hi;
  if (!p.splits && base >= sh.lo && threadIdx.x == 0 && blockIdx.x % groups == 0) {   // for the join
    part.at[2 * b] = index;
    part.at[2 * b + 1] = (base + tl.n - 1) / sh.len - index + 1;
  }
  const int64_t slot = (p.splits ? (int64_t)index : 2 * (int64_t)index + (base >= sh.lo)) * p.hkv;
  // eight values of packed row pr of head hh, from dimension d on
  auto put = [&](int hh, int pr, int d, float mm, float ll, float4 x, float4 y) {
    if (split) {
      const int64_t at = (slot + hh) * (16 * NT * RH) + pr;
      *(float4*)(part.o + at * kHeadDim + d) = x;
      *(float4*)(part.o + at * kHeadDim + d + 4) = y;
      if (d == 0) *(float2*)(part.ml + 2 * at) = make_float2(mm, ll);
    } else {
      const float inv = vsc / ll;
      const int64_t at = (int64_t)(q0 + pr / p.g) * p.hq + hh * p.g + pr % p.g;
      *(uint4*)(out + at * kHeadDim + d) =
          make_uint4(pack_bf16x2(x.x * inv, x.y * inv), pack_bf16x2(x.z * inv, x.w * inv),
                     pack_bf16x2(y.x * inv, y.y * inv), pack_bf16x2(y.z * inv, y.w * inv));
      if (lse && d == 0) lse[at] = (mm + fast_log2(ll)) * kLn2f;
    }
  };
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    l[nt] += __shfl_xor(l[nt], 16, 64);
    l[nt] += __shfl_xor(l[nt], 32, 64);
    const int pr = rb + 16 * nt + c16;
    if (KS == 1) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (pr < rows)
          put(h, pr, 32 * kg + 8 * i, m[nt], l[nt],
              make_float4(o[nt][0][i], o[nt][1][i], o[nt][2][i], o[nt][3][i]),
              make_float4(o[nt][4][i], o[nt][5][i], o[nt][6][i], o[nt][7][i]));
      continue;
    }
    if (16 * nt >= rows) continue;
    // the waves of a head, joined 16 rows at a time
    if (nt || again) __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float* d = &s_o[w][c16][32 * kg + 8 * i];
      *(float4*)d = make_float4(o[nt][0][i], o[nt][1][i], o[nt][2][i], o[nt][3][i]);
      *(float4*)(d + 4) = make_float4(o[nt][4][i], o[nt][5][i], o[nt][6][i], o[nt][7][i]);
    }
    if (kg == 0) {
      s_ml[w][c16][0] = m[nt];
      s_ml[w][c16][1] = l[nt];
    }
    __syncthreads();
    // the ks-th of them joins that share of the pieces of eight dimensions
    const int w0 = w % units, stepw = units;
    for (int x = 64 * ks + lane; x < 16 * 16; x += 64 * KS) {
      const int r = x >> 4, d = 8 * (x & 15), jr = rb + 16 * nt + r;
      if (jr >= rows) continue;
      float mm = kNoRef;
      for (int v = 0; v < KS; ++v) mm = fmaxf(mm, s_ml[w0 + v * stepw][r][0]);
      float ll = 0.f;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f), c = a;
      for (int v = 0; v < KS; ++v) {
        const float* src = &s_o[w0 + v * stepw][r][d];
        const float f = fast_exp2(s_ml[w0 + v * stepw][r][0] - mm);
        const float4 y = *(const float4*)src, z = *(const float4*)(src + 4);
        ll += f * s_ml[w0 + v * stepw][r][1];
        a.x += f * y.x, a.y += f * y.y, a.z += f * y.z, a.w += f * y.w;
        c.x += f * z.x, c.y += f * z.y, c.z += f * z.z, c.w += f * z.w;
      }
      put(h, jr, d, mm, ll, a, c);
    }
  }
  }
  base += tl.n;
  if (p.splits || base >= sh.hi) break;
  ++b;
  }
}

// Joins the parts of the units that were cut. Where a sequence's parts lie the
// workgroup that took its start left in the workspace (looked for among the
// lengths again, 2000 sequences of 1000 tokens take 1495 us instead of 767, 128 of
// 8000 416 instead of 401). A workgroup takes one packed row, groups of 32 lanes
// the parts in turn, eight of them a step with all their loads in flight; the
// groups are joined in LDS.
__global__ __launch_bounds__(1024) void combine_kernel(CacheProblem p, CachePartials part,
                                                      int rows_cap, int max_rows,
                                                      uint16_t* __restrict__ out,
                                                      float* __restrict__ lse) {
  __shared__ float s_m[32], s_l[32];
  __shared__ float4 s_a[32][32];
  const int pr = blockIdx.x % max_rows, bh = blockIdx.x / max_rows;
  const int b = bh / p.hkv, h = bh % p.hkv;
  const int q0 = ld_uniform(p.cu, b), Lq = ld_uniform(p.cu, b + 1) - q0;
  if (pr >= Lq * p.g) return;
  const int tiles = tiles_of(p, Lq, ld_uniform(p.cuk, b + 1) - ld_uniform(p.cuk, b)).n;
  if (tiles <= 0) return;
  // the sequence's parts: slots `s0`, then every second share's (kv_splits:
  // its own shares')
  int parts;
  int64_t s0, step;
  if (p.splits) {
    parts = min(p.splits, tiles);
    s0 = (int64_t)b * p.splits;
    step = 1;
  } else {
    parts = ld_uniform(part.at, 2 * b + 1);
    s0 = 2 * (int64_t)ld_uniform(part.at, 2 * b);   // the first part, one slot further
    step = 2;
  }
  if (parts <= 1) return;
  const int odd = p.splits ? 0 : 1;
  // row `pr` of part i, among the rows of all slots
  auto row = [&](int i) { return ((s0 + step * i + (i ? 0 : odd)) * p.hkv + h) * rows_cap + pr; };
  const int tid = threadIdx.x, grp = tid >> 5, d = tid & 31;
  const int groups = blockDim.x >> 5;
  float m = kNoRef, l = 0.f;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
  for (int i0 = grp; i0 < parts; i0 += 8 * groups) {
    float2 x[8];
    float4 y[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int64_t at = row(min(i0 + j * groups, parts - 1));
      x[j] = *(const float2*)(part.ml + 2 * at);
      y[j] = *(const float4*)(part.o + at * kHeadDim + 4 * d);
    }
    float mn = m;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      x[j].x = i0 + j * groups < parts ? x[j].x : -INFINITY;
      mn = fmaxf(mn, x[j].x);
    }
    const float f = fast_exp2(m - mn);
    m = mn;
    l *= f;
    a.x *= f, a.y *= f, a.z *= f, a.w *= f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if (i0 + j * groups >= parts) break;
      const float g = fast_exp2(x[j].x - m);
      l += g * x[j].y;
      a.x += g * y[j].x, a.y += g * y[j].y, a.z += g * y[j].z, a.w += g * y[j].w;
    }
  }
  if (d == 0) s_m[grp] = m, s_l[grp] = l;
  s_a[grp][d] = a;
  __syncthreads();
  if (tid >= 32) return;
#pragma unroll 8
  for (int i = 0; i < groups; ++i) m = fmaxf(m, s_m[i]);
  l = 0.f;
  a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 8
  for (int i = 0; i < groups; ++i) {   // (8 or 32)
    const float g = fast_exp2(s_m[i] - m);
    const float4 y = s_a[i][d];
    l += g * s_l[i];
    a.x += g * y.x, a.y += g * y.y, a.z += g * y.z, a.w += g * y.w;
  }
  const float inv = (p.form == kCacheHead ? ld_uniform(p.v_head, h) : 1.f) / l;
  const int64_t at = (int64_t)(q0 + pr / p.g) * p.hq + h * p.g + pr % p.g;
  *(uint2*)(out + at * kHeadDim + 4 * d) =
      make_uint2(pack_bf16x2(a.x * inv, a.y * inv), pack_bf16x2(a.z * inv, a.w * inv));
  if (lse && d == 0) lse[at] = (m + fast_log2(l)) * kLn2f;
}

// Rows that a workgroup holds: 16, 32 or 64.
int rows_cap(const CacheProblem& p) {
  const int rows = p.max_new * p.g;
  return rows <= 16 ? 16 : rows <= 32 ? 32 : 64;
}

// Heads that a workgroup takes side by side: many for long runs of memory, few
// for few partial results, of which it leaves one for each head and row. 8
// sequences of 5K to 38K tokens, codes, 32 rows: 78 us with 4 heads, 95 with 8;
// 64 rows: 101 us with 2, 105 with 4.
int heads_for(const CacheProblem& p) { return 128 / rows_cap(p); }

template <int FORM, int NT, int RH, int W, bool GROUPED>
hipError_t launch(const CacheProblem& problem, const CachePartials& part, uint16_t* out, float* lse,
                  hipStream_t s) {
  const CacheProblem p = dealt(problem, heads_for(problem));
  const int shares = shares_of(p), max_rows = p.max_new * p.g;
  const int64_t grid = (int64_t)shares * (p.hkv / p.heads);
  const int64_t joins = (int64_t)p.batch * p.hkv * max_rows;
  // few joins have many parts each, and a compute unit to themselves: 32 joins
  // of a sequence of 128K take 63 us with the attention, 69 with 256 threads;
  // 4096 of 8 sequences 100, and 122 with 1024
  const int threads = joins <= kFewGroups ? 1024 : 256;
  if (!launchable(grid, 64 * W) || (p.splits != 1 && !launchable(joins, threads))) return hipErrorInvalidValue;
  decode_kernel<FORM, NT, RH, W, GROUPED><<<(unsigned)grid, 64 * W, 0, s>>>(p, part, shares, out, lse);
  if (p.splits == 1) return hipGetLastError();
  combine_kernel<<<(unsigned)joins, threads, 0, s>>>(p, part, 16 * NT * RH, max_rows, out, lse);
  return hipGetLastError();
}

// Waves of a workgroup: a tile of bf16 keys takes twice the registers of one
// of codes. 64 rows need a wave's 512 registers; in bf16 not even those hold
// them, and two waves share them (145 us, 170 with spilled registers; in codes
// 108 instead of 101).
template <int FORM, bool GROUPED>
hipError_t launch_rows(const CacheProblem& p, const CachePartials& part, uint16_t* out, float* lse,
                       hipStream_t s) {
  constexpr bool kBf16 = FORM == kCacheBf16;
  const int rows = rows_cap(p);
  return rows == 16   ? launch<FORM, 1, 1, 8, GROUPED>(p, part, out, lse, s)
         : rows == 32 ? launch<FORM, 2, 1, kBf16 ? 4 : 8, GROUPED>(p, part, out, lse, s)
                      : launch<FORM, kBf16 ? 2 : 4, kBf16 ? 2 : 1, 4, GROUPED>(p, part, out, lse, s);
}

template <int FORM>
hipError_t launch_pages(const CacheProblem& p, const CachePartials& part, uint16_t* out, float* lse,
                        hipStream_t s) {
  // scales of blocks imply pages of a multiple of 16 tokens
  if constexpr (FORM == kCacheBlock) return launch_rows<FORM, true>(p, part, out, lse, s);
  else if (p.pm.page % 16 == 0) return launch_rows<FORM, true>(p, part, out, lse, s);
  else return launch_rows<FORM, false>(p, part, out, lse, s);
}

}  // namespace

void cache_decode_partials(const CacheProblem& problem, int64_t* slots, int* rows) {
  const CacheProblem p = dealt(problem, heads_for(problem));
  *slots = p.splits == 1 ? 0 : (int64_t)shares_of(p) * (p.splits ? 1 : 2) * p.hkv;
  *rows = rows_cap(p);
}

hipError_t launch_cache_decode(const CacheProblem& p, const CachePartials& part, uint16_t* out,
                               float* lse, hipStream_t s) {
  return p.form == kCacheBf16   ? launch_pages<kCacheBf16>(p, part, out, lse, s)
         : p.form == kCacheHead ? launch_pages<kCacheHead>(p, part, out, lse, s)
                                : launch_pages<kCacheBlock>(p, part, out, lse, s);
}

}  // namespace fp2
