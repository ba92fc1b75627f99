// The attention weight that cached tokens received of a call's queries: for
// each KV head, the sum over the new tokens and the g query heads of
// exp(scale q.k - lse), with the log-sum-exp that the attention returned. Each
// sum has one writer: no atomics, and the same result in every run.
//
// few_kernel: at most 64 packed rows a sequence, bound by the keys' bytes. As
// in the attention of few rows, the call's tiles are dealt in equal shares and a
// wave takes tiles of 32 keys from global memory to the matrix cores; a lane then
// holds one query and eight keys, whose sums over the 16 lanes of a group take
// eight exchanges. One token of 16 sequences of 9K to 60K tokens, 8 heads of 4:
// 111 us (4.4 TB/s).
//
// many_kernel: a workgroup takes 256 keys, a wave 64 of them as the B operand
// of S = Q K^T (v_mfma_f32_32x32x16_bf16), which stay in registers while the
// packed query rows that see them pass by, 32 at a time, through LDS. A lane
// holds two keys with 16 queries each, whose probabilities it adds in fp32; its
// sums take two registers (with keys as rows they took 32). Bound by the
// products and the exponentials, half of the attention's work: 8101 tokens of 32
// heads, bf16, take 330 us (0.82 PFLOP/s). Where the keys alone do not fill the
// chip the rows are cut into segments too, whose sums sum_kernel adds in their
// order.
#include <algorithm>

#include "cache_few.h"

namespace fp2 {

namespace {

constexpr float kLog2e = 1.44269504088896340736f;
constexpr int kFewWaves = 8;              // waves of a workgroup (few rows)
constexpr int kWaves = 4;                 // (many rows)
constexpr int kCopy = 4096;               // entries of a workgroup's turn in the copy
constexpr int kKeys = 64;                 // of a wave (many rows)
constexpr int kChunk = kWaves * kKeys;
constexpr int kRows = 32;                 // packed query rows of a step
constexpr int kFill = 8192;               // workgroups that fill the chip evenly
constexpr int kMaxSegs = 64;
constexpr int kMinSteps = 8;              // steps of a segment, at least

template <int FORM, int NT, bool GROUPED>
__global__ __launch_bounds__(64 * kFewWaves) void few_kernel(CacheProblem p, const float* __restrict__ lse,
                                                          const float* in, float* out, int64_t stride,
                                                          int shares) {
  constexpr bool kBf16 = FORM == kCacheBf16;
  constexpr int ESZ = kBf16 ? 2 : 1;
  constexpr int KC = kBf16 ? 4 : 2;            // 16-byte chunks of a key per lane
  const int groups = p.hkv / p.heads, index = blockIdx.x / groups, KS = kFewWaves / p.heads;
  if (index >= shares) {   // not in place: what no query sees, and what lies past the sequences
    const int64_t turn = blockIdx.x - (int64_t)shares * groups, per = (stride + kCopy - 1) / kCopy;
    const int64_t row = turn / per, from = turn % per * kCopy;
    const int sb = (int)(row / p.hkv);
    const int Ls = ld_uniform(p.cuk, sb + 1) - ld_uniform(p.cuk, sb);
    const Tiles t = tiles_of(p, ld_uniform(p.cu, sb + 1) - ld_uniform(p.cu, sb), Ls);
    // tiles sinks .. until - 1 are unseen, and the entries from Ls on
    const int until = t.n ? t.from : (Ls + kTile - 1) / kTile;
    for (int64_t j = from + threadIdx.x; j < min(from + kCopy, stride); j += 64 * kFewWaves)
      if (j >= Ls || (j / kTile >= t.sinks && j / kTile < until))
        out[row * stride + j] = in ? in[row * stride + j] : 0.f;
    return;
  }
  Share sh;
  if (!find_share(p, shares, index, sh)) return;
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int h = blockIdx.x % groups * p.heads + w % p.heads, ks = w / p.heads;
  const int c16 = lane & 15, kg = lane >> 4;
  const float cs = score_scale<FORM>(p, h);
  const int64_t rowb = (int64_t)p.hkv * kHeadDim * ESZ;
  const uint8_t* K = p.k + (int64_t)h * kHeadDim * ESZ;
  const uint32_t koff = (uint32_t)(c16 * rowb + 16 * kg);
  // key of a tile that this lane writes
  const int mine = 16 * (c16 >> 3) + 4 * kg + ((c16 >> 1) & 3);

  int b = sh.b, base = sh.base;
#pragma unroll 1
  for (bool again = false;; again = true) {
  if (again) {
    sh.q0 = ld_uniform(p.cu, b);
    sh.Lq = ld_uniform(p.cu, b + 1) - sh.q0;
    sh.L = ld_uniform(p.cuk, b + 1) - ld_uniform(p.cuk, b);
  }
  const int q0 = sh.q0, Lq = sh.Lq, L = sh.L;
  const int first = L - Lq, last = L - 1, rows = Lq * p.g;
  const Tiles tl = tiles_of(p, Lq, L);
  const int lo = max(sh.lo, base) - base, hi = min(sh.hi, base + tl.n) - base;
  auto tile_at = [&](int i) { return i < tl.sinks ? i : tl.from + i - tl.sinks; };
  const int64_t wrow = ((int64_t)b * p.hkv + h) * stride;
  const float* old_row = (in ? in : out) + wrow;   // loaded in any case, used where there is one

  bf16x8_t qb[NT][4];
  int pos[NT];
  float ref[NT];
#pragma unroll
  for (int nt = 0; nt < NT; ++nt) {
    const int r = 16 * nt + c16;
    pos[nt] = r < rows ? first + r / p.g : -1;        // a row past the last sees nothing
    ref[nt] = 0.f;
    const int64_t qrow = (int64_t)(q0 + r / p.g) * p.hq + h * p.g + r % p.g;
    if (r < rows) ref[nt] = lse[qrow] * kLog2e;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      const int d = kBf16 ? 32 * s + 8 * kg : 64 * (s >> 1) + 16 * kg + 8 * (s & 1);
      uint4 x = make_uint4(0, 0, 0, 0);
      if (r < rows) x = *(const uint4*)(p.q + qrow * kHeadDim + d);
      qb[nt][s] = __builtin_bit_cast(bf16x8_t, x);
    }
  }
  struct Raw {
    uint4 k[2][KC];
    uint32_t ks[2];
    float old;
  };
  const int32_t* table = p.pm.table + (int64_t)b * p.pm.stride;
  auto where = [&](int tile) { return where_at<GROUPED>(p.pm, table, tile, last, lane); };
  auto load = [&](int tile, const Where& at, Raw& x, uint32_t on) {   // on: ~0, or 0 to read one row over and over
    x.old = old_row[min(kTile * tile + mine, last)];
    if constexpr (GROUPED) {
      const int64_t s[2] = {at.slot(p.pm, 0), at.slot(p.pm, 1)};
      // the scales first: loads come back in order
      if constexpr (FORM == kCacheBlock) {
#pragma unroll
        for (int u = 0; u < 2; ++u) x.ks[u] = p.k_block[(s[u] >> p.sb_shift) * p.hkv + h];
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint8_t* kb = K + s[u] * rowb;
#pragma unroll
        for (int c = 0; c < KC; ++c) x.k[u][c] = *(const uint4*)(kb + ((koff & on) + 64u * c));
      }
    } else {
      const int slot = (int)at.slot(p.pm, 0);
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const uint8_t* kb = K + (int64_t)__shfl(slot, 16 * u + c16, 64) * rowb + 16 * kg;
#pragma unroll
        for (int c = 0; c < KC; ++c) x.k[u][c] = *(const uint4*)(kb + 64 * c);
      }
    }
  };
  auto step = [&](int tile, const Raw& x) {
    const int t0 = kTile * tile;
    float sum[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) sum[i] = 0.f;
    {
      const bool masked = t0 + kTile - 1 > first || rows < 16 * NT ||
                          (t0 <= last - p.window && t0 + kTile > p.sink);
      bf16x8_t a[2][4];
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        if constexpr (kBf16) {
#pragma unroll
          for (int c = 0; c < 4; ++c) a[u][c] = __builtin_bit_cast(bf16x8_t, x.k[u][c]);
        } else {
          const float sc = FORM == kCacheBlock ? block_scale(x.ks[u]) : 1.f;
#pragma unroll
          for (int c = 0; c < 2; ++c) {
            a[u][2 * c] = codes_to_bf16(x.k[u][c].x, x.k[u][c].y, sc);
            a[u][2 * c + 1] = codes_to_bf16(x.k[u][c].z, x.k[u][c].w, sc);
          }
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        f32x4_t s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          s[u] = f32x4_t{};
#pragma unroll
          for (int c = 0; c < 4; ++c)
            s[u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a[u][c], qb[nt][c], s[u], 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i >> 2][i & 3] = fast_exp2(fmaf(s[i >> 2][i & 3], cs, -ref[nt]));
        if (masked) {   // behind the exponentials: lse may be NaN or infinite too
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const int key = t0 + 16 * (i >> 2) + 4 * kg + (i & 3);
            s[i >> 2][i & 3] = sees(p, pos[nt], key) ? s[i >> 2][i & 3] : 0.f;
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) sum[i] += s[i >> 2][i & 3];
      }
    }
    // over the 16 lanes of a group: lanes 2 i and 2 i + 1 end with element i
#pragma unroll
    for (int n = 4; n > 0; n >>= 1) {
      const bool up = c16 & (2 * n);
#pragma unroll
      for (int j = 0; j < n; ++j) {
        const float send = up ? sum[j] : sum[j + n], keep = up ? sum[j + n] : sum[j];
        sum[j] = keep + __shfl_xor(send, 2 * n, 64);
      }
    }
    sum[0] += __shfl_xor(sum[0], 1, 64);
    if (!(c16 & 1) && t0 + mine <= last) out[wrow + t0 + mine] = (in ? x.old : 0.f) + sum[0];
  };

  // a tile ahead, with loads never left out (past the end they repeat a
  // row): behind a load that may not have been issued the compiler can only
  // wait for all of them
  if (lo + ks < hi) {
    Raw r0, r1;
    const int end = hi - 1;
    auto tile_to = [&](int i) { return tile_at(min(i, end)); };
    load(tile_at(lo + ks), where(tile_at(lo + ks)), r0, ~0u);
    Where a0 = where(tile_to(lo + ks + KS)), a1;
#pragma unroll 1
    for (int i = lo + ks; i < hi; i += 2 * KS) {
      load(tile_to(i + KS), a0, r1, i + KS < hi ? ~0u : 0u);
      a1 = where(tile_to(i + 2 * KS));
      step(tile_at(i), r0);
      load(tile_to(i + 2 * KS), a1, r0, i + 2 * KS < hi ? ~0u : 0u);
      a0 = where(tile_to(i + 3 * KS));
      if (i + KS < hi) step(tile_at(i + KS), r1);
    }
  }
  base += tl.n;
  if (p.splits || base >= sh.hi) break;
  ++b;
  }
}

__device__ __forceinline__ int place(int r, int c) { return r * 16 + (c ^ (r & 15)); }

struct Shared {
  uint4 q[2][kRows * 16];
  float lse[2][kRows];
};

// Steps of rows, [from, to), that see some of the keys c0 .. c0 + kChunk - 1.
struct Steps {
  int from, to;
};
__device__ __forceinline__ Steps steps_of(const CacheProblem& p, int c0, int Lq, int L) {
  // from the first query at or behind the keys to the last whose window
  // reaches them (all where first tokens are among them)
  const int P = L - Lq, kend = min(c0 + kChunk, L) - 1;
  const int i_lo = max(c0 - P, 0);
  const int i_hi = c0 < p.sink ? Lq - 1 : (int)min((int64_t)Lq - 1, (int64_t)kend + p.window - 1 - P);
  const int from = i_lo * p.g / kRows;
  return Steps{from, i_hi >= i_lo ? (i_hi * p.g + p.g - 1) / kRows + 1 : from};
}

// segs == 1: sums join `in` and go to `out`; else to part[seg][sequence, head][key].
template <int FORM>
__global__ __launch_bounds__(64 * kWaves, 3) void many_kernel(CacheProblem p,
                                                              const float* __restrict__ lse,
                                                              const float* in, float* out,
                                                              int64_t stride, float* part, int segs,
                                                              int seg_steps, int chunks) {
  constexpr bool kBf16 = FORM == kCacheBf16;
  constexpr int ESZ = kBf16 ? 2 : 1;
  __shared__ Shared sh;
  int64_t at = blockIdx.x;             // the first keys are seen by most rows: they come first
  const int h = (int)(at % p.hkv);
  at /= p.hkv;
  const int b = (int)(at % p.batch);
  at /= p.batch;
  const int seg = (int)(at % segs), c0 = (int)(at / segs) * kChunk;
  const int64_t tok0 = ld_uniform(p.cuk, b);
  const int L = ld_uniform(p.cuk, b + 1) - (int)tok0;
  if (c0 >= L) {                       // past the sequence, not in place
    if (segs == 1 && in != out) {
      const int64_t to = ((int64_t)b * p.hkv + h) * stride + c0 + threadIdx.x;
      if (c0 + threadIdx.x < stride) out[to] = in ? in[to] : 0.f;
    }
    return;
  }
  const int q0 = ld_uniform(p.cu, b), Lq = ld_uniform(p.cu, b + 1) - q0;
  const int P = L - Lq, rows = Lq * p.g;
  const Steps st = steps_of(p, c0, Lq, L);
  const int from = max(st.from, seg * seg_steps), to = min(st.to, (seg + 1) * seg_steps);
  if (segs > 1 && from >= to) return;

  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, l32 = lane & 31;
  const int k0 = c0 + kKeys * w;              // the wave's first key
  float acc[2] = {0.f, 0.f};

  if (from < to) {
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
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint4 x = *(const uint4*)(row + 32 * j + 16 * half);
          a[u][2 * j] = codes_to_bf16(x.x, x.y, sc);
          a[u][2 * j + 1] = codes_to_bf16(x.z, x.w, sc);
        }
      }
    }
    const float cs = score_scale<FORM>(p, h);

    // staging: thread -> row tid / 8 of a step, two 16-byte chunks; g is a power of two
    const int r = tid >> 3, c = 2 * (tid & 7);
    const int gs = __builtin_ctz(p.g), gm = p.g - 1;
    const uint16_t* Q = p.q + ((int64_t)q0 * p.hq + h * p.g) * kHeadDim;
    const float* Z = lse + (int64_t)q0 * p.hq + h * p.g;
    uint4 x0, x1;
    float ls = 0.f;
#define LOAD(t)                                                                              \
  do {                                                                                       \
    const int pr = min(kRows * (t) + r, rows - 1);                                           \
    const uint16_t* src = Q + ((int64_t)(pr >> gs) * p.hq + (pr & gm)) * kHeadDim + 8 * c;   \
    x0 = *(const uint4*)src;                                                                 \
    x1 = *(const uint4*)(src + 8);                                                           \
    if (tid < kRows) {                                                                       \
      const int pl = min(kRows * (t) + tid, rows - 1);                                       \
      ls = Z[(int64_t)(pl >> gs) * p.hq + (pl & gm)] * kLog2e;                               \
    }                                                                                        \
  } while (0)
#define STORE(t)                                                                             \
  do {                                                                                       \
    sh.q[(t) & 1][place(r, c)] = x0;                                                         \
    sh.q[(t) & 1][place(r, c + 1)] = x1;                                                     \
    if (tid < kRows) sh.lse[(t) & 1][tid] = ls;                                              \
  } while (0)
    LOAD(from);
    STORE(from);
    if (from + 1 < to) LOAD(from + 1);
#pragma unroll 1
    for (int t = from; t < to; ++t) {
      lds_barrier();
      if (t + 1 < to) STORE(t + 1);
      if (t + 2 < to) LOAD(t + 2);
      const int first = P + ((kRows * t) >> gs), last = P + ((min(kRows * t + kRows, rows) - 1) >> gs);
      if (last < k0) continue;                           // (uniform) none of the wave's keys is seen
      f32x16_t s[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) s[u] = f32x16_t{};
#pragma unroll
      for (int d = 0; d < 8; ++d) {
        // dimensions 16 d + 8 half of bf16 keys, 32 (d / 2) + 16 half + 8 (d % 2) of codes
        const int ch = kBf16 ? 2 * d + half : 4 * (d >> 1) + 2 * half + (d & 1);
        const bf16x8_t q = __builtin_bit_cast(bf16x8_t, sh.q[t & 1][place(l32, ch)]);
#pragma unroll
        for (int u = 0; u < 2; ++u)
          s[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q, a[u][d], s[u], 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 z = *(const float4*)&sh.lse[t & 1][8 * i + 4 * half];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          s[u][4 * i] = fast_exp2(fmaf(s[u][4 * i], cs, -z.x));
          s[u][4 * i + 1] = fast_exp2(fmaf(s[u][4 * i + 1], cs, -z.y));
          s[u][4 * i + 2] = fast_exp2(fmaf(s[u][4 * i + 2], cs, -z.z));
          s[u][4 * i + 3] = fast_exp2(fmaf(s[u][4 * i + 3], cs, -z.w));
        }
      }
      // element e is row 8 (e / 4) + 4 half + e % 4 of the step, key k0 + 32 u + l32;
      // masked behind the exponentials: lse may be NaN or infinite too
      if (k0 + kKeys - 1 > first || kRows * t + kRows > rows ||
          (k0 <= last - p.window && k0 + kKeys > p.sink)) {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int pr = kRows * t + 8 * (e >> 2) + 4 * half + (e & 3);
          const int pos = pr < rows ? P + (pr >> gs) : -1;   // a row past the last sees nothing
#pragma unroll
          for (int u = 0; u < 2; ++u)
            s[u][e] = pinned(sees(p, pos, k0 + 32 * u + l32) ? s[u][e] : 0.f);
        }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int u = 0; u < 2; ++u)
          acc[u] += (s[u][4 * i] + s[u][4 * i + 1]) + (s[u][4 * i + 2] + s[u][4 * i + 3]);
    }
#undef LOAD
#undef STORE
  }
  // the halves of a wave hold other rows of the same keys; each keeps one of the two
  acc[0] += __shfl_xor(acc[0], 32, 64);
  acc[1] += __shfl_xor(acc[1], 32, 64);
  const float sum = half ? acc[1] : acc[0];
  const int key = k0 + lane;
  const int64_t bh = (int64_t)b * p.hkv + h;
  if (segs > 1) {
    part[((int64_t)seg * p.batch * p.hkv + bh) * ((int64_t)chunks * kChunk) + key] = sum;
  } else if (key < L || (in != out && key < stride)) {
    out[bh * stride + key] = (in ? in[bh * stride + key] : 0.f) + (key < L ? sum : 0.f);
  }
}

// The segments' sums of a key, in their order.
__global__ __launch_bounds__(kChunk) void sum_kernel(CacheProblem p, const float* in, float* out,
                                                     int64_t stride, const float* __restrict__ part,
                                                     int segs, int seg_steps, int chunks) {
  const int bh = blockIdx.x % (p.batch * p.hkv), c0 = blockIdx.x / (p.batch * p.hkv) * kChunk;
  const int b = bh / p.hkv;
  const int L = ld_uniform(p.cuk, b + 1) - ld_uniform(p.cuk, b);
  const int key = c0 + threadIdx.x;
  if (key >= (in != out ? stride : (int64_t)L)) return;
  const Steps st = steps_of(p, c0, ld_uniform(p.cu, b + 1) - ld_uniform(p.cu, b), L);
  float sum = 0.f;
  const int s0 = st.from / seg_steps, s1 = key < L ? min((st.to + seg_steps - 1) / seg_steps, segs) : s0;
  if (st.from < st.to) {
#pragma unroll 8
    for (int s = s0; s < s1; ++s)
      sum += part[((int64_t)s * p.batch * p.hkv + bh) * ((int64_t)chunks * kChunk) + key];
  }
  const int64_t to = (int64_t)bh * stride + key;
  out[to] = (in ? in[to] : 0.f) + sum;
}

int chunks_of(const CacheProblem& p) { return (p.max_kv + kChunk - 1) / kChunk; }

// Segments of the rows, and steps of each. Workgroups differ much in work (the
// first keys are seen by all rows), so many small ones fill the chip evenly: 8101
// tokens take 333 us with 8192 of them, 537 with 1024, 1010 without segments; 500
// tokens 21 and 79.
int segments(const CacheProblem& p, int* steps) {
  const int all = (int)(((int64_t)p.max_new * p.g + kRows - 1) / kRows);
  const int64_t groups = std::max<int64_t>(1, (int64_t)p.batch * p.hkv * chunks_of(p));
  const int segs = (int)std::max<int64_t>(1, std::min<int64_t>({kFill / groups, all / kMinSteps, kMaxSegs}));
  *steps = (all + segs - 1) / segs;
  return segs;
}

bool few_rows(const CacheProblem& p) { return (int64_t)p.max_new * p.g <= kFewRows; }

template <int FORM>
hipError_t launch_few(const CacheProblem& problem, const float* lse, const float* in, float* out,
                      int64_t stride, hipStream_t s) {
  const CacheProblem p = dealt(problem, kFewWaves);
  const int shares = shares_of(p), rows = p.max_new * p.g;
  const int nt = rows <= 16 ? 1 : rows <= 32 ? 2 : 4;
  const int64_t copies = in != out ? (int64_t)p.batch * p.hkv * ((stride + kCopy - 1) / kCopy) : 0;
  const int64_t grid = (int64_t)shares * (p.hkv / p.heads) + copies;
  if (!launchable(grid, 64 * kFewWaves)) return hipErrorInvalidValue;
  const dim3 g((unsigned)grid), t(64 * kFewWaves);
  if (FORM == kCacheBlock || p.pm.page % 16 == 0) {
    if (nt == 1) few_kernel<FORM, 1, true><<<g, t, 0, s>>>(p, lse, in, out, stride, shares);
    else if (nt == 2) few_kernel<FORM, 2, true><<<g, t, 0, s>>>(p, lse, in, out, stride, shares);
    else few_kernel<FORM, 4, true><<<g, t, 0, s>>>(p, lse, in, out, stride, shares);
  } else if constexpr (FORM != kCacheBlock) {
    if (nt == 1) few_kernel<FORM, 1, false><<<g, t, 0, s>>>(p, lse, in, out, stride, shares);
    else if (nt == 2) few_kernel<FORM, 2, false><<<g, t, 0, s>>>(p, lse, in, out, stride, shares);
    else few_kernel<FORM, 4, false><<<g, t, 0, s>>>(p, lse, in, out, stride, shares);
  }
  return hipGetLastError();
}

template <int FORM>
hipError_t launch(const CacheProblem& p, const float* lse, const float* in, float* out, int64_t stride,
                  float* part, hipStream_t s) {
  if (few_rows(p)) return launch_few<FORM>(p, lse, in, out, stride, s);
  int steps;
  const int segs = segments(p, &steps), chunks = chunks_of(p);
  // not in place, the entries past the sequences are written too
  const int64_t all = in != out ? (stride + kChunk - 1) / kChunk : chunks;
  const int64_t groups = (int64_t)p.batch * p.hkv * (segs > 1 ? chunks : all);
  const int64_t sums = (int64_t)p.batch * p.hkv * all;
  if (all > 0x7fffffff / kChunk || !launchable(groups * segs, 64 * kWaves) ||
      (segs > 1 && !launchable(sums, kChunk)))
    return hipErrorInvalidValue;
  many_kernel<FORM><<<(unsigned)(groups * segs), 64 * kWaves, 0, s>>>(p, lse, in, out, stride, part, segs,
                                                                      steps, chunks);
  if (segs > 1)
    sum_kernel<<<(unsigned)sums, kChunk, 0, s>>>(p, in, out, stride, part, segs, steps,
                                                                    chunks);
  return hipGetLastError();
}

}  // namespace

int64_t cache_weights_partials(const CacheProblem& p) {
  int steps;
  const int segs = few_rows(p) ? 1 : segments(p, &steps);
  return segs > 1 ? (int64_t)segs * p.batch * p.hkv * chunks_of(p) * kChunk : 0;
}

hipError_t launch_cache_weights(const CacheProblem& p, const float* lse, const float* in, float* out,
                                int64_t stride, float* part, hipStream_t s) {
  return p.form == kCacheBf16   ? launch<kCacheBf16>(p, lse, in, out, stride, part, s)
         : p.form == kCacheHead ? launch<kCacheHead>(p, lse, in, out, stride, part, s)
                                : launch<kCacheBlock>(p, lse, in, out, stride, part, s);
}

}  // namespace fp2
