// How the kernels that go through a call's tokens share them out (internal to the
// library).
#pragma once
#include "cache.h"

namespace fp2 {

namespace {

// Runs of 2^SHIFT tokens of each sequence, one sequence behind the other, in a
// line of slots. Lengths are known on the device only, and a grid by their bounds
// would be mostly empty where they are ragged (an empty workgroup takes 1.7 ns),
// so a bounded grid deals the line to its workgroups in equal shares, each in one piece
// (every n-th step instead: 222 us for the move of 186K tokens that takes 177). Sequence b
// has the slots from cu[b] / 2^SHIFT + EXTRA b on: EXTRA more than its tokens fill,
// for the runs that its ends cut; a few slots have no tokens.
template <int SHIFT, int EXTRA>
struct Runs {
  const int32_t* cu;
  int batch, b;
  int64_t at, next;         // slots of sequence b
  __device__ __forceinline__ Runs(const int32_t* cu_, int batch_) : cu(cu_), batch(batch_), b(-1), at(0), next(0) {}
  __device__ __forceinline__ int64_t start(int i) const { return (int64_t)(cu[i] >> SHIFT) + (int64_t)EXTRA * i; }
  __device__ __forceinline__ int64_t total() const {
    return (int64_t)(ld_uniform(cu, batch) >> SHIFT) + (int64_t)EXTRA * batch;
  }
  // Index of a slot among its sequence's, which becomes b. The slots that a wave asks for do not fall.
  // Every lane of the wave takes part: 64 sequences are looked at at once.
  __device__ __forceinline__ int64_t seek(int64_t slot) {
    if (b < 0 || slot >= next) {
      const int lane = threadIdx.x & 63;
      int lo = max(b, 0), hi = batch;
      while (true) {
        const int step = (hi - lo + 63) / 64, i = lo + lane * step;
        const uint64_t before = __ballot(i < hi && start(i) <= slot);
        lo += max(__popcll(before) - 1, 0) * step;
        hi = min(lo + step, hi);
        if (step == 1) break;
      }
      b = __builtin_amdgcn_readfirstlane(lo);
      at = (int64_t)(ld_uniform(cu, b) >> SHIFT) + (int64_t)EXTRA * b;
      next = (int64_t)(ld_uniform(cu, b + 1) >> SHIFT) + (int64_t)EXTRA * (b + 1);
    }
    return slot - at;
  }
};

// What one step of a workgroup takes: WIDE pairs of a slot and a head side by
// side, `heads` heads (a power of two) of WIDE / heads slots; the heads of a slot
// come in `groups` steps of each of `kinds` (keys, values).
struct Steps {
  int heads, groups, kinds;
};
inline Steps steps_of(int hkv, int wide, int kinds) {
  Steps s{1, 0, kinds};
  while (s.heads < wide && s.heads < hkv) s.heads *= 2;
  s.groups = (hkv + s.heads - 1) / s.heads;
  return s;
}
// Steps of a line of `slots`.
inline __host__ __device__ int64_t steps_in(const Steps& s, int wide, int64_t slots) {
  const int each = wide / s.heads;
  return (slots + each - 1) / each * s.groups * s.kinds;
}

// Workgroups of a call whose line has at most `bound` steps: several times what
// runs at once, so that the ends even out.
inline int64_t grid_for(int64_t bound, int64_t most) { return bound < most ? bound : most; }

}  // namespace

}  // namespace fp2
