// Rows that are turned outside the cache (internal to the library).
#pragma once
#include "rotary.h"

namespace fp2 {

// Rows [tokens, heads, 128] with heads side by side, in and out.
struct RotaryRows {
  const uint16_t* x;        // bf16
  int64_t x_stride;         // elements between tokens
  uint8_t* out;             // bf16, or codes where scale is given
  int64_t out_stride;
  const float* scale;       // [heads]
  int32_t heads;
};

namespace {

// A lane's part of row (token t, head h), turned and stored.
template <int PLACE>
__device__ __forceinline__ void turn_and_store(const LaneRow<PLACE>& l, const Turns<PLACE>& y, const uint32_t (&w)[8],
                                               const RotaryRows& to, int64_t t, int h, bool there) {
  float x[16];
  turned16(l, y, w, x);
  const int64_t at = t * to.out_stride + h * kHeadDim;
  if (to.scale) {
    uint32_t c[4];
    codes16_by(x, Divisor(ld_uniform(to.scale, h)), c);
    if (there) store_part(l, to.out + at, c);
  } else {
    uint32_t b[8];
    pack16(x, b);
    if (there) store_part(l, (uint16_t*)to.out + at, b);
  }
}

}  // namespace

// hipErrorInvalidValue, and nothing launched, where the call is too large for it.
hipError_t launch_rotary(const Rotary& r, bool interleaved, int64_t tokens, const int32_t* positions, const RotaryRows& q,
                         const RotaryRows& k, hipStream_t s);
hipError_t launch_cache_append_rotary(const CacheProblem& p, const Rotary& r, bool interleaved, const RotaryRows& q,
                                      const uint16_t* k_new, int64_t k_stride, const uint16_t* v_new, int64_t v_stride,
                                      const int32_t* positions, hipStream_t s);
// r.turns null: rows as they are.
hipError_t launch_cache_read(const CacheProblem& p, const Rotary& r, bool interleaved, const int32_t* positions,
                             uint16_t* k_out, uint16_t* v_out, hipStream_t s);

// Positions that each token's keys are turned by, with strides in elements (0: the same for all).
struct Moves {
  const int32_t* by;
  int64_t batch, head, token;
};
// to.table null: in place, keys only. r.turns null: rows as they are.
hipError_t launch_cache_move(const CacheProblem& p, const Rotary& r, bool interleaved, const Moves& moves, const PageMap& to,
                             hipStream_t s);
constexpr int kCrossCuts = 256;      // units that a cross attention cuts, at most (16 bytes each behind its partial outputs)
hipError_t launch_cache_cross(const CacheProblem& p, const CachePartials& part, uint16_t* out, float* lse, hipStream_t s);
void cache_cross_partials(const CacheProblem& p, int64_t* slots, int* rows);

}  // namespace fp2
