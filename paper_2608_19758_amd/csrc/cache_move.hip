// Tokens of a paged cache read back as bf16 rows, and moved to other pages or
// positions. Eight lanes a row, a wave a head at a time; the waves beside it take
// the other heads of the same tokens, so memory is read in long runs.
//
// Reading: a wave takes 16 tokens and several heads, the loads of two (bf16) or four
// (codes) of them at once, and works out what it turns keys back by once for them.
//
// Moving: a wave takes 32 tokens of a head. Keys of codes with a scale per head
// keep the scale (a turn is linear: the codes' numbers are turned and rounded
// again, held within +-448); a block with a scale of its own gets the one that its
// turned keys need, and each code is rounded once, from the fp32 that the wave
// holds. Where a scale stands for 64 or 128 tokens two or four waves share the
// block and its largest value, through LDS. Rows that are not turned are copied,
// codes and scales. All that is read of a block is read before it is written, so
// the pages may be the same (in place).
//
// Bound by memory: 128 or 256 bytes a row in, and 256 (reading) or as many out. 398K
// tokens of 8 heads, scales of 64, read and turned back: 481 us (5.1 TB/s); 186K
// moved to other pages, scales of 64: 171 (4.4 TB/s: rows of 1 KB at places of their
// own); 1000 tokens of every head's own 10, 2001 read 6.8. With a number of positions
// for each head and token a row has 64 turns of its own, and the vector ALUs are busy
// 75% of the time: the same 186K 220 us (a scale a head 239, bf16 319 as with one number).
#include <algorithm>
#include <type_traits>

#include "cache_runs.h"
#include "rotary_rows.h"

namespace fp2 {

namespace {

constexpr int kWaves = 8;

// ---- reading

constexpr int kReadShift = 4, kReadTokens = 1 << kReadShift;

template <int FORM, int PLACE, bool TURN>
__device__ __forceinline__ void read_heads(const CacheProblem& p, const Rotary& r, const int32_t* positions, bool is_v,
                                           uint16_t* out, int b, int run, int h0, int h1) {
  constexpr int N = kReadTokens / kPass, AHEAD = FORM == kCacheBf16 ? 2 : 4;
  constexpr int ESZ = FORM == kCacheBf16 ? 2 : 1;
  typedef std::conditional_t<FORM == kCacheBf16, uint16_t, uint8_t> elem_t;
  const int q0 = ld_uniform(p.cu, b), n = ld_uniform(p.cu, b + 1) - q0;
  const int L = ld_uniform(p.cuk, b + 1) - ld_uniform(p.cuk, b), P = L - n;
  // runs start at multiples of 16 in the sequence, so that one lies in one block
  const int first = (P / kReadTokens + run) * kReadTokens;
  if (n <= 0 || first >= L) return;
  const int lane = threadIdx.x & 63, r0 = lane / kLaneRow;
  const LaneRow<PLACE> l(lane, r.dim);
  int64_t slot[N];
  Turns<PLACE> y[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int t = min(max(first + kPass * i + r0, P), L - 1);
    slot[i] = slot_of(p.pm, b, 0, t);
    if constexpr (TURN) l.turns(r, l.freqs(r), positions ? positions[(int64_t)q0 + t - P] : t, y[i]);
  }
  const elem_t* pool = (const elem_t*)(is_v ? p.v : p.k);
  const uint8_t* scales = is_v ? p.v_block : p.k_block;
#pragma unroll 1
  for (int h = h0; h < h1; h += AHEAD) {
    uint32_t raw[AHEAD][N][4 * ESZ], byte[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      const int hh = min(h + j, h1 - 1);         // past the end the last head again
      if constexpr (FORM == kCacheBlock) byte[j] = scales[(slot[0] >> p.sb_shift) * p.hkv + hh];
#pragma unroll
      for (int i = 0; i < N; ++i) load_part(l, pool + (slot[i] * p.hkv + hh) * kHeadDim, raw[j][i]);
    }
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (h + j >= h1) break;
      float by = 1.f;
      if constexpr (FORM == kCacheHead) by = ld_uniform(is_v ? p.v_head : p.k_head, h + j);
      if constexpr (FORM == kCacheBlock) by = block_scale(byte[j]);
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const int t = first + kPass * i + r0;
        uint32_t c[8];
        if constexpr (FORM == kCacheBf16 && !TURN) {
#pragma unroll
          for (int e = 0; e < 8; ++e) c[e] = raw[j][i][e];
        } else {
          float x[16];                           // codes are turned in units of their scale
          if constexpr (TURN) turned16(l, y[i], raw[j][i], x);
          else unpack16(raw[j][i], x);
          if constexpr (FORM != kCacheBf16) {
#pragma unroll
            for (int e = 0; e < 16; ++e) x[e] *= by;
          }
          pack16(x, c);
        }
        if (t >= P && t < L) store_part(l, out + (((int64_t)q0 + t - P) * p.hkv + h + j) * kHeadDim, c);
      }
    }
  }
}

// Waves take equal shares of the line of (run, keys or values, `heads` heads).
template <int FORM, int PLACE, bool TURN>
__global__ __launch_bounds__(64 * kWaves) void read_kernel(CacheProblem p, Rotary r, const int32_t* __restrict__ positions,
                                                           uint16_t* k_out, uint16_t* v_out, int heads) {
  Runs<kReadShift, 2> line(p.cu, p.batch);
  const int groups = (p.hkv + heads - 1) / heads, kinds = (k_out != nullptr) + (v_out != nullptr), per = groups * kinds;
  const int64_t items = line.total() * per, waves = (int64_t)gridDim.x * kWaves;
  const int64_t wave = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t lo = items * wave / waves, hi = items * (wave + 1) / waves;
  int64_t slot = lo / per;
  int rest = (int)(lo - slot * per);
#pragma unroll 1
  for (int64_t i = lo; i < hi; ++i) {
    const int h0 = rest % groups * heads, h1 = min(h0 + heads, p.hkv);
    const bool is_v = !k_out || rest >= groups;
    const int run = (int)line.seek(slot);
    if (is_v) read_heads<FORM, kPairs, false>(p, r, nullptr, true, v_out, line.b, run, h0, h1);
    else read_heads<FORM, PLACE, TURN>(p, r, positions, false, k_out, line.b, run, h0, h1);
    if (++rest == per) rest = 0, ++slot;
  }
}

// ---- moving

// Rows as they are, with their scales: 32 tokens of a head. SB: tokens of a scale, else 0.
template <int FORM, int SB>
__device__ __forceinline__ void copy_rows(const CacheProblem& p, const PageMap& to, bool is_v, int b, int h, int first, int L) {
  constexpr int ESZ = FORM == kCacheBf16 ? 2 : 1, N = 32 / kPass;
  typedef std::conditional_t<FORM == kCacheBf16, uint16_t, uint8_t> elem_t;
  const int lane = threadIdx.x & 63, r0 = lane / kLaneRow;
  const LaneRow<kPairs> l(lane, kHeadDim);
  elem_t* pool = (elem_t*)(is_v ? p.v : p.k);
  uint8_t* scales = is_v ? p.v_block : p.k_block;
  const int64_t from_l = slot_of(p.pm, b, 0, min(first + (lane & 31), L - 1));
  const int64_t dest_l = slot_of(to, b, 0, min(first + (lane & 31), L - 1));
  uint32_t raw[N][4 * ESZ], byte[2] = {0, 0};
#pragma unroll
  for (int i = 0; i < N; ++i) load_part(l, pool + (__shfl(from_l, kPass * i + r0, 64) * p.hkv + h) * kHeadDim, raw[i]);
  constexpr int BLOCKS = SB == 16 ? 2 : SB > 0 ? 1 : 0;
#pragma unroll
  for (int k = 0; k < BLOCKS; ++k) byte[k] = scales[(__shfl(from_l, SB * k & 31, 64) >> p.sb_shift) * p.hkv + h];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    elem_t* row = pool + (__shfl(dest_l, kPass * i + r0, 64) * p.hkv + h) * kHeadDim;
    if (first + kPass * i + r0 < L) store_part(l, row, raw[i]);
  }
#pragma unroll
  for (int k = 0; k < BLOCKS; ++k) {
    const int64_t slot = __shfl(dest_l, SB * k & 31, 64);
    if (lane == 0 && first + SB * k < L && first % (SB > 0 ? SB : 1) == 0)
      scales[(slot >> p.sb_shift) * p.hkv + h] = (uint8_t)byte[k];
  }
}

// 32 tokens of a head, from `first` on. SB: tokens of a scale (kCacheBlock), else 0.
// TURN: 0 rows as they are, 1 a sequence's head moves as one, 2 every token by its
// own number of positions. Every wave of the workgroup takes part (`there` or not).
template <int FORM, int SB, int PLACE, int TURN>
__device__ __forceinline__ void move_step(const CacheProblem& p, const Rotary& r, const Moves& m, const PageMap& to,
                                          float* s_amax, bool is_v, bool there, int b, int h, int w, int part, int first) {
  constexpr int PARTS = SB > 32 ? SB / 32 : 1;   // waves of a block
  constexpr int N = 32 / kPass;
  constexpr int ESZ = FORM == kCacheBf16 ? 2 : 1;
  typedef std::conditional_t<FORM == kCacheBf16, uint16_t, uint8_t> elem_t;
  const int L = ld_uniform(p.cuk, b + 1) - ld_uniform(p.cuk, b);
  const bool mine = there && first < L, turned = TURN && !is_v;
  if (mine && !turned) copy_rows<FORM, SB>(p, to, is_v, b, h, first, L);
  if constexpr (TURN != 0) {
    if (PARTS == 1 && !(mine && turned)) return;
    const int lane = threadIdx.x & 63, r0 = lane / kLaneRow;
    const LaneRow<PLACE> l(lane, r.dim);
    elem_t* pool = (elem_t*)p.k;
    float x[N][16];
    int64_t dest_l = 0;
    int old[2] = {0, 0};                         // scale bytes of a wave's blocks
    constexpr int BLOCKS = SB == 16 ? 2 : 1, PER = N / BLOCKS;
    if (mine && turned) {
      const int64_t from_l = slot_of(p.pm, b, 0, min(first + (lane & 31), L - 1));
      dest_l = to.table ? slot_of(to, b, 0, min(first + (lane & 31), L - 1)) : from_l;
      const int64_t mh = b * m.batch + h * m.head;
      uint32_t raw[N][4 * ESZ];
      int by[N];
#pragma unroll
      for (int i = 0; i < N; ++i) {
        load_part(l, pool + (__shfl(from_l, kPass * i + r0, 64) * p.hkv + h) * kHeadDim, raw[i]);
        by[i] = TURN == 2 ? m.by[mh + min(first + kPass * i + r0, L - 1) * m.token] : 0;
      }
      if constexpr (FORM == kCacheBlock) {
#pragma unroll
        for (int k = 0; k < BLOCKS; ++k)
          old[k] = __builtin_amdgcn_readfirstlane(
              (int)p.k_block[(__shfl(from_l, SB * k & 31, 64) >> p.sb_shift) * p.hkv + h]);
      }
      const Freqs<PLACE> freqs = l.freqs(r);
      Turns<PLACE> y;
      if constexpr (TURN == 1) l.turns(r, freqs, m.by[mh], y);
#pragma unroll
      for (int i = 0; i < N; ++i) {              // codes are turned in units of their scale
        if constexpr (TURN == 2) turned16_at(l, r, freqs, by[i], raw[i], x[i]);
        else turned16(l, y, raw[i], x[i]);
      }
    }
    auto store = [&](int i, const uint32_t (&c)[4 * ESZ]) {
      elem_t* row = pool + (__shfl(dest_l, kPass * i + r0, 64) * p.hkv + h) * kHeadDim;
      if (first + kPass * i + r0 < L) store_part(l, row, c);
    };
    if constexpr (FORM == kCacheBf16) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        uint32_t c[8];
        pack16(x[i], c);
        store(i, c);
      }
    } else if constexpr (FORM == kCacheHead) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        uint32_t c[4];
        codes16_held(x[i], c);
        store(i, c);
      }
    } else {
      float amax[BLOCKS];
#pragma unroll
      for (int k = 0; k < BLOCKS; ++k) {
        amax[k] = 0.f;
        if (!(mine && turned)) continue;
#pragma unroll
        for (int i = PER * k; i < PER * (k + 1); ++i) amax[k] = fmaxf(amax[k], largest16(x[i]));   // (codes have no infinities)
        amax[k] = wave_max(amax[k]);
      }
      if constexpr (PARTS > 1) {
        if (lane == 0) s_amax[w] = amax[0];
        __syncthreads();
        if (!(mine && turned)) return;
#pragma unroll
        for (int j = 0; j < PARTS; ++j) amax[0] = fmaxf(amax[0], s_amax[w - part + j]);
      }
#pragma unroll
      for (int k = 0; k < BLOCKS; ++k) {
        const int byte = __builtin_amdgcn_readfirstlane(scale_byte(amax[k] * block_scale((uint32_t)old[k])));
        const int64_t slot = __shfl(dest_l, SB * k & 31, 64);
        // 2^(old - new), which leaves at most 448 of the largest; held finite for rows of zeros, which may
        // come with any scale
        const float f = block_scale((uint32_t)min(max(old[k] - byte + 127, 1), 254));
#pragma unroll
        for (int i = PER * k; i < PER * (k + 1); ++i) {
          uint32_t c[4];
#pragma unroll
          for (int e = 0; e < 16; ++e) x[i][e] *= f;
          if (byte < kMaxScaleByte) codes16(x[i], c);
          else codes16_held(x[i], c);
          store(i, c);
        }
        if (part == 0 && lane == 0 && first + SB * k < L) p.k_block[(slot >> p.sb_shift) * p.hkv + h] = (uint8_t)byte;
      }
    }
  }
}

template <int FORM, int SB, int PLACE, int TURN>
__global__ __launch_bounds__(64 * kWaves) void move_tokens_kernel(CacheProblem p, Rotary r, Moves m, PageMap to,
                                                                  Steps steps) {
  constexpr int PARTS = SB > 32 ? SB / 32 : 1;   // waves of a block
  constexpr int WIDE = kWaves / PARTS, SHIFT = PARTS == 4 ? 7 : PARTS == 2 ? 6 : 5;
  __shared__ float s_amax[2][kWaves];
  const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int part = PARTS > 1 ? w % PARTS : 0, place = w / PARTS;
  Runs<SHIFT, 1> line(p.cuk, p.batch);
  const int64_t slots = line.total(), all = steps_in(steps, WIDE, slots);
  const int64_t lo = all * blockIdx.x / gridDim.x, hi = all * (blockIdx.x + 1) / gridDim.x;
  const int per = steps.groups * steps.kinds, each = WIDE / steps.heads;
  int64_t set = lo / per;                        // of `each` slots
  int rest = (int)(lo - set * per);
#pragma unroll 1
  for (int64_t i = lo; i < hi; ++i) {
    const int h = rest % steps.groups * steps.heads + place % steps.heads;
    const bool is_v = rest >= steps.groups;
    const int64_t slot = set * each + place / steps.heads;
    const bool there = slot < slots && h < p.hkv;
    const int run = (int)line.seek(min(slot, slots - 1));
    move_step<FORM, SB, PLACE, TURN>(p, r, m, to, s_amax[i & 1], is_v, there, line.b, h, w, part, (run * PARTS + part) * 32);
    if (++rest == per) rest = 0, ++set;
  }
}

template <int FORM, int PLACE, bool TURN>
hipError_t launch_read(const CacheProblem& p, const Rotary& r, const int32_t* positions, uint16_t* k_out, uint16_t* v_out,
                       hipStream_t s) {
  // the most runs that the bounds allow
  const int64_t runs = (int64_t)p.batch * ((p.max_new >> kReadShift) + 2);
  const int kinds = (k_out != nullptr) + (v_out != nullptr);
  // heads of a wave: many share the turns, few fill the chip where tokens are few (8 heads: 2000 tokens 8.5 us with
  // one a wave, 12.7 with eight; 20000 25.7 with four, 27.5 with eight, 45.8 with one; 200000 261 with eight, 441)
  int heads = std::min(8, p.hkv);
  while (heads > 1 && runs * kinds * ((p.hkv + heads - 1) / heads) < 4096) heads >>= 1;
  // (200000 tokens: with 2048 workgroups at most 272 us)
  const int64_t grid = grid_for((runs * kinds * ((p.hkv + heads - 1) / heads) + kWaves - 1) / kWaves, 8192);
  read_kernel<FORM, PLACE, TURN><<<(unsigned)grid, 64 * kWaves, 0, s>>>(p, r, positions, k_out, v_out, heads);
  return hipGetLastError();
}

template <int FORM, int SB, int PLACE, int TURN>
hipError_t launch_move(const CacheProblem& p, const Rotary& r, const Moves& m, const PageMap& to, hipStream_t s) {
  constexpr int PARTS = SB > 32 ? SB / 32 : 1, TOK = 32 * PARTS, WIDE = kWaves / PARTS;
  const Steps steps = steps_of(p.hkv, WIDE, to.table ? 2 : 1);
  // (200000 tokens: 189 us, with 8192 workgroups at most 199)
  const int64_t grid = grid_for(steps_in(steps, WIDE, (int64_t)p.batch * (p.max_kv / TOK + 1)), 2048);
  move_tokens_kernel<FORM, SB, PLACE, TURN><<<(unsigned)grid, 64 * kWaves, 0, s>>>(p, r, m, to, steps);
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
