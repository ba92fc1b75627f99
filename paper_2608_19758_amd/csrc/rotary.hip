// Rotary positions of queries and keys: rows of heads turned by their tokens'
// positions, bf16 in, bf16 or e4m3 codes with a scale per head out.
//
// A wave takes eight tokens, eight lanes a row, works out its turns once (in
// registers) and goes through `run` heads with them, four heads' loads in
// flight. Bound by memory: 256 bytes a row in, 256 or 128 out; a turn is some 35
// instructions, shared by the heads. 16384 tokens of 32 heads, to codes, and of
// eight of keys: 53 us (5.0 TB/s); 8 tokens 4.5, a launch and three loads that wait
// for each other.
#include <algorithm>

#include "rotary_rows.h"

namespace fp2 {

namespace {

constexpr int kWaves = 4;
constexpr int kAhead = 4;         // heads whose loads are in flight

template <int PLACE>
__global__ __launch_bounds__(64 * kWaves) void rotary_kernel(Rotary r, int64_t tokens,
                                                             const int32_t* __restrict__ positions,
                                                             RotaryRows q, RotaryRows k, int run, int runs,
                                                             int64_t total) {
  const int64_t at = (int64_t)blockIdx.x * kWaves + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (at >= total) return;
  const int lane = threadIdx.x & 63, heads = q.heads + k.heads;
  const int h0 = (int)(at % runs) * run, h1 = min(h0 + run, heads);
  const int64_t token = at / runs * kPass + lane / kLaneRow;
  const bool there = token < tokens;
  const int64_t t = there ? token : tokens - 1;
  const LaneRow<PLACE> l(lane, r.dim);
  Turns<PLACE> y;
  l.turns(r, l.freqs(r), positions[t], y);
#pragma unroll 1
  for (int h = h0; h < h1; h += kAhead) {
    uint32_t w[kAhead][8];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int hh = min(h + i, h1 - 1);     // past the end the last head again
      const RotaryRows& x = hh < q.heads ? q : k;
      load_part(l, x.x + t * x.x_stride + (hh < q.heads ? hh : hh - q.heads) * kHeadDim, w[i]);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int hh = h + i;
      if (hh >= h1) break;
      if (hh < q.heads) turn_and_store(l, y, w[i], q, t, hh, there);
      else turn_and_store(l, y, w[i], k, t, hh - q.heads, there);
    }
  }
}

// Heads of a wave: many share the turns, few fill the chip where tokens are few (40
// heads: 512 tokens 5.8 us with one a wave, 6.7 with eight; 16384 bf16 tokens 107
// with one, 67 with eight, 76 with 16).
int run_for(int64_t tokens, int heads) {
  const int64_t passes = (tokens + kPass - 1) / kPass;
  int run = 8;
  while (run > 1 && passes * ((heads + run - 1) / run) < 2048) run >>= 1;
  return std::min(run, heads);
}

}  // namespace

hipError_t launch_rotary(const Rotary& r, bool interleaved, int64_t tokens, const int32_t* positions, const RotaryRows& q,
                         const RotaryRows& k, hipStream_t s) {
  const int heads = q.heads + k.heads, run = run_for(tokens, heads), runs = (heads + run - 1) / run;
  const int64_t total = (tokens + kPass - 1) / kPass * runs, grid = (total + kWaves - 1) / kWaves;
  if (!launchable(grid, 64 * kWaves)) return hipErrorInvalidValue;
  auto go = [&](auto kernel) {
    kernel<<<(unsigned)grid, 64 * kWaves, 0, s>>>(r, tokens, positions, q, k, run, runs, total);
    return hipGetLastError();
  };
  const PairPlace place = place_of(r.dim, interleaved);
  return place == kPairs ? go(rotary_kernel<kPairs>) : place == kHalves ? go(rotary_kernel<kHalves>) : go(rotary_kernel<kOdd>);
}

}  // namespace fp2
