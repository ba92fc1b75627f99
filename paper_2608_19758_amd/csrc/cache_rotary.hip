// New tokens' queries, keys and values in one pass: queries and keys turned by
// their positions, keys and values written into a paged cache in its type.
//
// A wave of queries takes eight tokens and several heads, and works its turns out
// once for them. A wave of keys or values takes 32 tokens of a head; where a scale
// stands for 64 or 128 tokens two or four waves share the block and its largest
// value, through LDS. 2^e, e = ceil(log2(amax / 448)) of the turned keys, makes
// x 2^-e exact, and a code is rounded once, from the fp32 that the wave holds.
// Where a block holds tokens already its scale never falls; if it grows their
// codes are rounded again.
//
// Bound by memory: 256 bytes a row in, 256 or 128 out. 32768 tokens of 32 and 8
// heads, scales of 64: 165 us (4.4 TB/s).
//
// Few new tokens a sequence: a wave has one head of a sequence to itself, or, of up to
// four tokens, several heads. One token of 32 sequences, scales of 16: 4.9 us, which
// are a launch, the lengths, the page, the block's scale, one after the other; of
// 1024 sequences 9.7 (with a head a wave 49), four of 256 9.7 (17).
#include <type_traits>

#include "cache_runs.h"
#include "rotary_rows.h"

namespace fp2 {

namespace {

constexpr int kWaves = 8;
// New tokens of a sequence that a wave takes alone, at most: eight rows, or with
// registers for 16 tokens, or for 32 (64 sequences of 8: 6.9 us, with those for 16
// 7.2; 256 of 16: 24, with those for 32 29; 256 of 32: 55, dealt out as many 132).
// 64 tokens in a wave: 26 us instead of 31 for 64 sequences, 13 instead of 9 for one.
constexpr int kFew = 16, kSome = 32;

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

// Codes of a row times a power of two (at most 1).
__device__ __forceinline__ void shrink_row(uint8_t* row, int lane, float by) {
  uint4* at = (uint4*)(row + 16 * (lane & 7));
  uint32_t w[4] = {at->x, at->y, at->z, at->w};
  float x[16];
  unpack16(w, x);
#pragma unroll
  for (int e = 0; e < 16; ++e) x[e] *= by;
  codes16(x, w);
  *at = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ float power_down(int from, int to) {   // 2^(from - to), to >= from
  return __uint_as_float((uint32_t)max(127 - (to - from), 0) << 23);
}

// Queries: heads h0 .. h1 - 1 of eight new tokens, from the i0-th on.
template <int PLACE>
__device__ __forceinline__ void turn_queries(const CacheProblem& p, const Rotary& r, const RotaryRows& q, const New& x,
                                             int b, int64_t i0, int h0, int h1) {
  constexpr int kAhead = 4;                      // heads whose loads are in flight
  const Seq s(p, b);
  if (i0 >= s.n) return;
  const int lane = threadIdx.x & 63, t = s.P + min((int)i0 + lane / kLaneRow, s.n - 1);
  const bool there = i0 + lane / kLaneRow < s.n;
  const LaneRow<PLACE> l(lane, r.dim);
  const int64_t row = s.row(t);
  Turns<PLACE> y;
  l.turns(r, l.freqs(r), s.position(x, t), y);
#pragma unroll 1
  for (int h = h0; h < h1; h += kAhead) {
    uint32_t w[kAhead][8];
#pragma unroll
    for (int i = 0; i < kAhead; ++i)             // past the end the last head again
      load_part(l, q.x + row * q.x_stride + min(h + i, h1 - 1) * kHeadDim, w[i]);
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
      if (h + i < h1) turn_and_store(l, y, w[i], q, row, h + i, there);
  }
}

// 32 new tokens of a head, keys or values, of the block (of 32 PARTS tokens) that is
// the run-th with new tokens. Every wave of the workgroup takes part.
template <int FORM, int SB, int PLACE>
__device__ __forceinline__ void append_step(const CacheProblem& p, const Rotary& r, const New& x, float* s_amax, bool is_v,
                                            bool on, int b, int h, int w, int part, int64_t run) {
  constexpr int PARTS = SB > 32 ? SB / 32 : 1;   // waves of a block
  constexpr int TOK = 32 * PARTS;
  constexpr int N = 32 / kPass;
  constexpr int ESZ = FORM == kCacheBf16 ? 2 : 1;
  const Seq s(p, b);
  const int64_t block64 = ((int64_t)(s.P / TOK) + run) * TOK;
  on = on && s.n > 0 && block64 < s.L;
  const int block = on ? (int)block64 : 0, first = block + 32 * part;
  const bool mine = on && first < s.L && first + 32 > s.P;     // some of the wave's own tokens are new
  const int lane = threadIdx.x & 63, r0 = lane / kLaneRow;
  const LaneRow<PLACE> l(lane, r.dim);
  const uint16_t* src = (is_v ? x.v : x.k) + h * kHeadDim;
  const int64_t stride = is_v ? x.v_stride : x.k_stride, rowb = (int64_t)p.hkv * kHeadDim;
  uint8_t* pool = (is_v ? p.v : p.k) + h * kHeadDim * ESZ;
  float z[N][16];
  int64_t slot_l = 0;                            // of token first + lane % 32
  if (mine) {
    uint32_t raw[N][8];
    int pos[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {                // (rows that are not new repeat one that is)
      const int t = min(max(first + kPass * i + r0, s.P), s.L - 1);
      load_part(l, src + s.row(t) * stride, raw[i]);
      pos[i] = is_v ? 0 : s.position(x, t);
    }
    slot_l = slot_of(p.pm, s.b, s.tok0, min(first + (lane & 31), s.L - 1));
    if (is_v) {
#pragma unroll
      for (int i = 0; i < N; ++i) unpack16(raw[i], z[i]);
    } else {
      const Freqs<PLACE> freqs = l.freqs(r);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        turned16_at(l, r, freqs, pos[i], raw[i], z[i]);
      }
    }
  }
  auto store = [&](int i, auto&& convert) {      // pass i in the cache's type
    const int t = first + kPass * i + r0;
    const int64_t slot = __shfl(slot_l, kPass * i + r0, 64);
    uint32_t c[4 * ESZ];
    convert(z[i], c);
    if (t >= s.P && t < s.L) store_part(l, (std::conditional_t<ESZ == 2, uint16_t, uint8_t>*)pool + slot * rowb, c);
  };
  if constexpr (FORM == kCacheBf16) {
    if (!mine) return;
#pragma unroll
    for (int i = 0; i < N; ++i) store(i, [](const float (&v)[16], uint32_t (&c)[8]) { pack16(v, c); });
  } else if constexpr (FORM == kCacheHead) {
    if (!mine) return;
    const Divisor d(ld_uniform(is_v ? p.v_head : p.k_head, h));
#pragma unroll
    for (int i = 0; i < N; ++i) store(i, [&](const float (&v)[16], uint32_t (&c)[4]) { codes16_by(v, d, c); });
  } else {
    constexpr int BLOCKS = SB == 16 ? 2 : 1, PER = N / BLOCKS;   // of a wave, and passes of each
    float amax[BLOCKS];
#pragma unroll
    for (int k = 0; k < BLOCKS; ++k) {
      amax[k] = 0.f;
      if (mine) {
#pragma unroll
        for (int i = PER * k; i < PER * (k + 1); ++i) amax[k] = fmaxf(amax[k], largest16(z[i]));
        amax[k] = wave_max(amax[k]);
        if (!(amax[k] < INFINITY)) {             // (rare: infinities do not count)
          amax[k] = 0.f;
#pragma unroll
          for (int i = PER * k; i < PER * (k + 1); ++i) amax[k] = fmaxf(amax[k], largest16_finite(z[i]));
          amax[k] = wave_max(amax[k]);
        }
      }
    }
    // bytes of blocks that hold tokens, read before the barrier: behind it the first wave of a block writes its own
    uint8_t* sp[BLOCKS];
    int before[BLOCKS];
#pragma unroll
    for (int k = 0; k < BLOCKS; ++k) {
      const int tb = PARTS > 1 ? block : first + SB * k;         // the block's first token
      sp[k] = nullptr;
      before[k] = 0;
      if (!on || tb >= s.L || tb + SB <= s.P) continue;
      sp[k] = (is_v ? p.v_block : p.k_block) + (slot_of(p.pm, s.b, s.tok0, tb) >> p.sb_shift) * p.hkv + h;
      if (tb < s.P) before[k] = __builtin_amdgcn_readfirstlane((int)*sp[k]);
    }
    if constexpr (PARTS > 1) {
      if (lane == 0) s_amax[w] = amax[0];
      __syncthreads();
#pragma unroll
      for (int j = 0; j < PARTS; ++j) amax[0] = fmaxf(amax[0], s_amax[w - part + j]);
    }
    if (!on) return;
#pragma unroll
    for (int k = 0; k < BLOCKS; ++k) {
      const int tb = PARTS > 1 ? block : first + SB * k;
      if (!sp[k]) continue;
      const int byte = __builtin_amdgcn_readfirstlane(max(scale_byte(amax[k]), before[k]));
      if (tb < s.P && byte > before[k]) {        // the wave's share of the codes that were there
        const float by = power_down(before[k], byte);
        const int from = PARTS > 1 ? first : tb;
        for (int t = from + r0; t < min(s.P, from + (PARTS > 1 ? 32 : SB)); t += kPass)
          shrink_row(pool + slot_of(p.pm, s.b, s.tok0, t) * rowb, lane, by);
      }
      if (mine) {
        const float inv = __uint_as_float((uint32_t)(254 - byte) << 23);   // 2^-e
#pragma unroll
        for (int i = PER * k; i < PER * (k + 1); ++i) {
#pragma unroll
          for (int e = 0; e < 16; ++e) z[i][e] *= inv;
          if (byte < kMaxScaleByte) store(i, [](const float (&v)[16], uint32_t (&c)[4]) { codes16(v, c); });
          else store(i, [](const float (&v)[16], uint32_t (&c)[4]) { codes16_held(v, c); });
        }
      }
      if (part == 0 && lane == 0) *sp[k] = (uint8_t)byte;
    }
  }
}

// SB: tokens of a scale (kCacheBlock), else 0. Workgroups below `kv` take equal
// shares of the keys and values, the others of the queries, `heads` heads at a time.
template <int FORM, int SB, int PLACE>
__global__ __launch_bounds__(64 * kWaves) void append_rotary_kernel(CacheProblem p, Rotary r, RotaryRows q, New x,
                                                                    Steps steps, int kv, int heads) {
  constexpr int PARTS = SB > 32 ? SB / 32 : 1, WIDE = kWaves / PARTS, SHIFT = PARTS == 4 ? 7 : PARTS == 2 ? 6 : 5;
  __shared__ float s_amax[2][kWaves];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if ((int)blockIdx.x >= kv) {
    Runs<3, 1> line(p.cu, p.batch);
    const int groups = (q.heads + heads - 1) / heads;
    const int64_t items = line.total() * groups, waves = (int64_t)(gridDim.x - kv) * kWaves;
    const int64_t wave = (int64_t)(blockIdx.x - kv) * kWaves + w, lo = items * wave / waves, hi = items * (wave + 1) / waves;
    int64_t slot = lo / groups;
    int g = (int)(lo - slot * groups);
#pragma unroll 1
    for (int64_t i = lo; i < hi; ++i) {
      const int64_t pass = line.seek(slot);
      turn_queries<PLACE>(p, r, q, x, line.b, pass * kPass, g * heads, min((g + 1) * heads, q.heads));
      if (++g == groups) g = 0, ++slot;
    }
    return;
  }
  const int part = PARTS > 1 ? w % PARTS : 0, place = w / PARTS;
  Runs<SHIFT, 2> line(p.cu, p.batch);
  const int64_t slots = line.total(), all = steps_in(steps, WIDE, slots);
  const int64_t lo = all * blockIdx.x / kv, hi = all * (blockIdx.x + 1) / kv;
  const int per = steps.groups * steps.kinds, each = WIDE / steps.heads;
  int64_t set = lo / per;                        // of `each` slots
  int rest = (int)(lo - set * per);
#pragma unroll 1
  for (int64_t i = lo; i < hi; ++i) {
    const int h = rest % steps.groups * steps.heads + place % steps.heads;
    const int64_t slot = set * each + place / steps.heads;
    const int64_t run = line.seek(min(slot, slots - 1));
    append_step<FORM, SB, PLACE>(p, r, x, s_amax[i & 1], rest >= steps.groups, slot < slots && h < p.hkv, line.b, h, w, part,
                                 run);
    if (++rest == per) rest = 0, ++set;
  }
}

// At most T (1, 2, 4, 8) new tokens a sequence: a wave takes all of them and 8 / T
// heads of its queries, keys or values. They lie in at most two blocks; the codes that
// the first one held are read only if its scale grows.
template <int FORM, int PLACE, int T>
__global__ __launch_bounds__(64 * kWaves) void append_rotary_rows_kernel(CacheProblem p, Rotary r, RotaryRows q, New x,
                                                                         int64_t total) {
  typedef std::conditional_t<FORM == kCacheBf16, uint16_t, uint8_t> elem_t;
  constexpr int HEADS = kPass / T;
  const int64_t at = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (at >= total) return;
  const int kv = (p.hkv + HEADS - 1) / HEADS, jobs = 2 * kv + (q.heads + HEADS - 1) / HEADS, j = (int)(at % jobs);
  const Seq s(p, (int)(at / jobs));
  if (s.n <= 0) return;
  const bool is_q = j >= 2 * kv, is_v = !is_q && j >= kv;
  const int h0 = HEADS * (is_q ? j - 2 * kv : is_v ? j - kv : j), heads = is_q ? q.heads : p.hkv;
  const int lane = threadIdx.x & 63, r0 = lane / kLaneRow, i = r0 % T;   // rows of a head lie side by side
  const int h = min(h0 + r0 / T, heads - 1), t = min(s.P + i, s.L - 1);
  const bool there = h0 + r0 / T < heads && i < s.n;
  const LaneRow<PLACE> l(lane, r.dim);
  const int64_t row = s.row(t);
  uint32_t raw[8];
  load_part(l, (is_q ? q.x + row * q.x_stride : is_v ? x.v + row * x.v_stride : x.k + row * x.k_stride) + h * kHeadDim, raw);
  float z[16];
  if (is_v) unpack16(raw, z);
  else turned16_at(l, r, l.freqs(r), s.position(x, t), raw, z);
  uint32_t c[4], w[8];
  if (is_q) {
    const int64_t to = row * q.out_stride + h * kHeadDim;
    if (q.scale) {
      codes16_by(z, Divisor(q.scale[h]), c);
      if (there) store_part(l, q.out + to, c);
    } else {
      pack16(z, w);
      if (there) store_part(l, (uint16_t*)q.out + to, w);
    }
    return;
  }
  elem_t* pool = (elem_t*)(is_v ? p.v : p.k);
  const int64_t slot = slot_of(p.pm, s.b, s.tok0, t);
  elem_t* to = pool + (slot * p.hkv + h) * kHeadDim;
  if constexpr (FORM == kCacheBf16) {
    pack16(z, w);
    if (there) store_part(l, to, w);
  } else if constexpr (FORM == kCacheHead) {
    codes16_by(z, Divisor((is_v ? p.v_head : p.k_head)[h]), c);
    if (there) store_part(l, to, c);
  } else {
    const int first = t & -(1 << p.sb_shift);
    uint8_t* sp = (is_v ? p.v_block : p.k_block) + (slot >> p.sb_shift) * p.hkv + h;
    const int before = first < s.P ? *sp : 0;            // byte of a block that holds tokens
    auto over = [](float m, int from, int to) {          // the largest of lanes that differ in these bits
      for (int o = from; o < to; o *= 2) m = fmaxf(m, __shfl_xor(m, o, 64));
      return m;
    };
    float amax = over(largest16(z), 1, kLaneRow);        // of the row
    if (__any(!(amax < INFINITY))) {                     // (rare: infinities do not count)
      const float finite = over(largest16_finite(z), 1, kLaneRow);
      amax = amax < INFINITY ? amax : finite;
    }
    if constexpr (T > 1) {                               // of the row's block
      const bool one = first <= s.P;
      const float a = over(one ? amax : 0.f, kLaneRow, kLaneRow * T), b = over(one ? 0.f : amax, kLaneRow, kLaneRow * T);
      amax = one ? a : b;
    }
    const int byte = max(scale_byte(amax), before);
    const float inv = __uint_as_float((uint32_t)(254 - byte) << 23);   // 2^-e
#pragma unroll
    for (int e = 0; e < 16; ++e) z[e] *= inv;
    if (__any(byte >= kMaxScaleByte)) codes16_held(z, c);
    else codes16(z, c);
    if (there) store_part(l, to, c);
    if (there && l.c == 0 && t == max(first, s.P)) *sp = (uint8_t)byte;
    // the whole wave takes the heads whose first block's scale grew, one after the other
    const int held = s.P & -(1 << p.sb_shift);
    for (uint64_t grew = __ballot(there && l.c == 0 && i == 0 && first < s.P && byte > before); grew; grew &= grew - 1) {
      const int from = __ffsll((unsigned long long)grew) - 1;
      const float by = power_down(__builtin_amdgcn_readlane(before, from), __builtin_amdgcn_readlane(byte, from));
      elem_t* head = pool + (h0 + from / (kLaneRow * T)) * kHeadDim;
#pragma unroll 4
      for (int u = held + r0; u < s.P; u += kPass)
        shrink_row(head + slot_of(p.pm, s.b, s.tok0, u) * p.hkv * kHeadDim, lane, by);
    }
  }
}

// At most MOST new tokens a sequence: a wave takes a head. They lie in at most three
// blocks, one after the other; the codes that a block held are read only if its scale grows.
template <int FORM, int PLACE, int MOST>
__global__ __launch_bounds__(64 * kWaves) void append_rotary_few_kernel(CacheProblem p, Rotary r, RotaryRows q, New x,
                                                                        int64_t total) {
  constexpr int ESZ = FORM == kCacheBf16 ? 2 : 1;
  constexpr int N = MOST / kPass;
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
  const Freqs<PLACE> freqs = l.freqs(r);
  const int size = FORM == kCacheBlock && !is_q ? 1 << p.sb_shift : MOST;
  float scale = 1.f;
  if constexpr (FORM == kCacheHead)
    if (!is_q) scale = ld_uniform(is_v ? p.v_head : p.k_head, h);
#pragma unroll 1
  for (int from = s.P; from < s.L;) {
    // the new tokens from .. to - 1 of a block
    const int first = FORM == kCacheBlock && !is_q ? from & -size : from, to = min(min(first + size, s.L), from + MOST);
    float z[N][16];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (from + kPass * i >= to) break;
      const int t = min(from + kPass * i + r0, to - 1);
      uint32_t raw[8];
      load_part(l, src + s.row(t) * stride, raw);
      if (is_q) {
        Turns<PLACE> y;
        l.turns(r, freqs, s.position(x, t), y);
        turn_and_store(l, y, raw, q, s.row(t), h, from + kPass * i + r0 < to);
      } else if (!is_v) {
        turned16_at(l, r, freqs, s.position(x, t), raw, z[i]);
      } else {
        unpack16(raw, z[i]);
      }
    }
    if (!is_q) {
      float inv = 1.f;
      bool held = false;
      if constexpr (FORM == kCacheBlock) {
        uint8_t* sp = (is_v ? p.v_block : p.k_block) + (slot_of(p.pm, s.b, s.tok0, first) >> p.sb_shift) * p.hkv + h;
        const int before = first < s.P ? *sp : 0;       // byte of a block that holds tokens
        float amax = 0.f;
#pragma unroll
        for (int i = 0; i < N; ++i) {
          if (from + kPass * i >= to) break;
          amax = fmaxf(amax, largest16(z[i]));
        }
        amax = wave_max(amax);
        if (!(amax < INFINITY)) {                       // (rare: infinities do not count)
          amax = 0.f;
#pragma unroll
          for (int i = 0; i < N; ++i)
            if (from + kPass * i < to) amax = fmaxf(amax, largest16_finite(z[i]));
          amax = wave_max(amax);
        }
        const int byte = __builtin_amdgcn_readfirstlane(max(scale_byte(amax), before));
        held = byte >= kMaxScaleByte;
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
          uint32_t c[4];
          if constexpr (FORM == kCacheHead) {
            codes16_by(z[i], Divisor(scale), c);
          } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) z[i][e] *= inv;
            if (held) codes16_held(z[i], c);
            else codes16(z[i], c);
          }
          store_part(l, row, c);
        }
      }
    }
    from = to;
  }
}

template <int FORM, int SB, int PLACE>
hipError_t launch(const CacheProblem& p, const Rotary& r, const RotaryRows& q, const New& x, hipStream_t s) {
  if (p.max_new <= kSome) {
    const int each = p.max_new == 1 ? 8 : p.max_new == 2 ? 4 : p.max_new <= 4 ? 2 : 1;   // heads of a wave
    const int64_t total = (int64_t)p.batch * (2 * ((p.hkv + each - 1) / each) + (q.heads + each - 1) / each);
    const int64_t grid = (total + kWaves - 1) / kWaves;
    if (!launchable(grid, 64 * kWaves)) return hipErrorInvalidValue;
    auto go = [&](auto kernel) {
      kernel<<<(unsigned)grid, 64 * kWaves, 0, s>>>(p, r, q, x, total);
      return hipGetLastError();
    };
    return each == 8           ? go(append_rotary_rows_kernel<FORM, PLACE, 1>)
           : each == 4         ? go(append_rotary_rows_kernel<FORM, PLACE, 2>)
           : each == 2         ? go(append_rotary_rows_kernel<FORM, PLACE, 4>)
           : p.max_new <= 8    ? go(append_rotary_rows_kernel<FORM, PLACE, 8>)
           : p.max_new <= kFew ? go(append_rotary_few_kernel<FORM, PLACE, kFew>)
                               : go(append_rotary_few_kernel<FORM, PLACE, kSome>);
  }
  constexpr int PARTS = SB > 32 ? SB / 32 : 1, TOK = 32 * PARTS, WIDE = kWaves / PARTS;
  const Steps steps = steps_of(p.hkv, WIDE, 2);
  // a workgroup for each step that there can be, at most 2048, eight a compute unit: with 8192 32K tokens take
  // 181 us instead of 171. With two workgroups a sequence too few 40 tokens of 8 take 14.6 us, so 9.3.
  const int64_t slots = (int64_t)p.batch * ((p.max_new + TOK - 1) / TOK + 2);
  const int64_t kv = grid_for(steps_in(steps, WIDE, slots), 2048);
  // query heads of a wave: many share the turns, few fill the chip where tokens are few (32 heads:
  // 2000 tokens 15.2 us with 4, 15.5 with 8, 21.2 with 1; 16384 96 with 8, 101 with 16, 144 with 1)
  const int64_t passes = (int64_t)p.batch * (p.max_new / kPass + 1);
  int heads = 8;
  while (heads > 1 && passes * ((q.heads + heads - 1) / heads) < 512) heads >>= 1;
  const int64_t queries = grid_for((passes * ((q.heads + heads - 1) / heads) + kWaves - 1) / kWaves, 2048);
  append_rotary_kernel<FORM, SB, PLACE><<<(unsigned)(kv + (q.heads ? queries : 0)), 64 * kWaves, 0, s>>>(p, r, q, x, steps,
                                                                                                  (int)kv, heads);
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
