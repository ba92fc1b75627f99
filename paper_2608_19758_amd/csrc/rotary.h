// Rotary positions: the angles, and how a wave holds and turns rows of a head
// (device helpers of the kernels that turn queries and keys).
//
// The pair (x, y) of a row at position n becomes a (x cos t - y sin t,
// x sin t + y cos t), t = f_i n. The frequencies come as fractions of a turn in
// 64-bit fixed point, F_i = 2^64 f_i / 2 pi, so n F_i modulo 2^64 is the exact
// fraction of a turn at any position: two 32-bit multiplications, no table of
// positions and no argument reduction. In fp32 an angle of 10^6 radians would
// be off by up to 2^-5.
//
// Eight lanes hold a row of 128, 16 elements each as eight pairs; a pass of a
// wave is eight rows. Where the pairs lie:
//   kPairs   dimensions (2 i, 2 i + 1); a lane's 16 elements are adjacent
//   kHalves  (i, i + dim / 2), dim a multiple of 16: two runs of eight elements
//   kOdd     the same for any even dim: element by element
// Dimensions from dim on stand in pairs too, which are left as they are (not
// turned by 0: an infinity would make NaN of its neighbour).
#pragma once
#include "cache.h"

namespace fp2 {

struct Rotary {
  const uint64_t* turns;    // [dim / 2]
  int32_t dim;
  int32_t inverse;          // turns backwards
  float scale;              // a
};

enum PairPlace : int32_t { kPairs = 0, kHalves = 1, kOdd = 2 };

inline PairPlace place_of(int dim, bool interleaved) { return interleaved ? kPairs : dim % 16 ? kOdd : kHalves; }

namespace {

constexpr int kPairsOfRow = kHeadDim / 2;
constexpr int kLaneRow = 8;       // lanes of a row
constexpr int kPass = 8;          // rows of a pass
constexpr int kPer = 8;           // pairs of a lane

// Top 32 bits of n F modulo 2^64.
__device__ __forceinline__ uint32_t phase_at(int n, uint64_t f) {
  const uint32_t lo = (uint32_t)f, u = (uint32_t)n;
  return u * (uint32_t)(f >> 32) + __umulhi(u, lo) - (n < 0 ? lo : 0u);
}

// Cosine and sine of a fraction of a turn. To the nearest quarter, then Taylor
// polynomials on +-pi/4: their rests are below 2^-25 (x^10 / 10!) and 2^-29
// (x^11 / 11!), the rounding of the argument and of the terms 2^-23 in all.
__device__ __forceinline__ float2 cos_sin(uint32_t phase) {
  const uint32_t quarter = (phase + 0x20000000u) >> 30;
  const float x = (float)(int)(phase - (quarter << 30)) * 1.4629180792671596e-09f;   // 2 pi / 2^32
  const float x2 = x * x;
  float c = fmaf(x2, 2.48015873e-5f, -1.38888889e-3f);
  c = fmaf(x2, c, 4.16666667e-2f);
  c = fmaf(x2, c, -0.5f);
  c = fmaf(x2, c, 1.f);
  float s = fmaf(x2, 2.75573192e-6f, -1.98412698e-4f);
  s = fmaf(x2, s, 8.33333333e-3f);
  s = fmaf(x2, s, -1.66666667e-1f);
  s = fmaf(x2 * x, s, x);
  const float a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  return make_float2((quarter + 1) & 2 ? -a : a, quarter & 2 ? -b : b);
}

__device__ __forceinline__ float2 turn_at(const Rotary& r, int n, uint64_t f) {
  const float2 t = cos_sin(phase_at(n, f));
  return make_float2(t.x * r.scale, (r.inverse ? -t.y : t.y) * r.scale);
}

// A lane's eight frequencies and turns.
struct Freqs {
  uint64_t f[kPer];
};
struct Turns {
  float2 t[kPer];
};

// What lane c (of the eight) holds of a row. `turned` pairs of its eight: the first ones.
template <int PLACE>
struct LaneRow {
  int c, dim;
  int at[2];        // kPairs, kHalves: first elements of its two runs of eight
  int turned;
  __device__ __forceinline__ LaneRow(int lane, int dim_) : c(lane & 7), dim(dim_) {
    turned = min(max(dim / 2 - kPer * c, 0), kPer);
    if constexpr (PLACE == kPairs) at[0] = 16 * c, at[1] = 16 * c + 8;
    else if (turned) at[0] = 8 * c, at[1] = dim / 2 + 8 * c;
    else at[0] = 16 * c, at[1] = 16 * c + 8;      // dim + 16 (c - dim / 16)
  }
  // elements of pair e (kOdd)
  __device__ __forceinline__ int2 pair(int e) const {
    const int i = kPer * c + e, h = dim / 2;
    return i < h ? make_int2(i, i + h) : make_int2(2 * i, 2 * i + 1);
  }
  __device__ __forceinline__ Freqs freqs(const Rotary& r) const {
    Freqs y;
#pragma unroll
    for (int e = 0; e < kPer; ++e) y.f[e] = e < turned ? r.turns[kPer * c + e] : 0;
    return y;
  }
  // The turns of the lane's pairs at position n.
  __device__ __forceinline__ void turns(const Rotary& r, const Freqs& f, int n, Turns& y) const {
#pragma unroll
    for (int e = 0; e < kPer; ++e) y.t[e] = turn_at(r, n, f.f[e]);
  }
};

// A lane's part of a row as it comes: 16 bf16 (eight words) or 16 codes (four).
// kPairs, kOdd: word by word the pairs; kHalves: the first run, then the second.
template <int PLACE, class T>
__device__ __forceinline__ void load_part(const LaneRow<PLACE>& l, const T* row, uint32_t (&w)[4 * sizeof(T)]) {
  if constexpr (PLACE == kOdd) {
#pragma unroll
    for (int i = 0; i < 4 * (int)sizeof(T); ++i) w[i] = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int2 d = l.pair(e);
      if constexpr (sizeof(T) == 2) w[e] = (uint32_t)row[d.x] | (uint32_t)row[d.y] << 16;
      else w[e / 2] |= ((uint32_t)row[d.x] | (uint32_t)row[d.y] << 8) << (16 * (e & 1));
    }
  } else if constexpr (sizeof(T) == 2) {
    const uint4 a = *(const uint4*)(row + l.at[0]), b = *(const uint4*)(row + l.at[1]);
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
  } else if constexpr (PLACE == kPairs) {
    const uint4 a = *(const uint4*)(row + l.at[0]);
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
  } else {
    const uint2 a = *(const uint2*)(row + l.at[0]), b = *(const uint2*)(row + l.at[1]);
    w[0] = a.x, w[1] = a.y, w[2] = b.x, w[3] = b.y;
  }
}
template <int PLACE, class T>
__device__ __forceinline__ void store_part(const LaneRow<PLACE>& l, T* row, const uint32_t (&w)[4 * sizeof(T)]) {
  if constexpr (PLACE == kOdd) {
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int2 d = l.pair(e);
      if constexpr (sizeof(T) == 2) {
        row[d.x] = (T)w[e];
        row[d.y] = (T)(w[e] >> 16);
      } else {
        row[d.x] = (T)(w[e / 2] >> (16 * (e & 1)));
        row[d.y] = (T)(w[e / 2] >> (16 * (e & 1) + 8));
      }
    }
  } else if constexpr (sizeof(T) == 2) {
    *(uint4*)(row + l.at[0]) = make_uint4(w[0], w[1], w[2], w[3]);
    *(uint4*)(row + l.at[1]) = make_uint4(w[4], w[5], w[6], w[7]);
  } else if constexpr (PLACE == kPairs) {
    *(uint4*)(row + l.at[0]) = make_uint4(w[0], w[1], w[2], w[3]);
  } else {
    *(uint2*)(row + l.at[0]) = make_uint2(w[0], w[1]);
    *(uint2*)(row + l.at[1]) = make_uint2(w[2], w[3]);
  }
}

// Sixteen values in the order of the words.
__device__ __forceinline__ void unpack16(const uint32_t (&w)[8], float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
  }
}
__device__ __forceinline__ void unpack16(const uint32_t (&w)[4], float (&x)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float y[4];
    e4m3x4_to_f32(w[i], y);
#pragma unroll
    for (int e = 0; e < 4; ++e) x[4 * i + e] = y[e];
  }
}
__device__ __forceinline__ void pack16(const float (&x)[16], uint32_t (&w)[8]) {
#pragma unroll
  for (int i = 0; i < 8; ++i) w[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
}
// as codes: y = the values in units of the scale, x the values themselves (their infinities and NaN count)
__device__ __forceinline__ void pack16(const float (&x)[16], const float (&y)[16], uint32_t (&w)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float a[4] = {x[4 * i], x[4 * i + 1], x[4 * i + 2], x[4 * i + 3]};
    const float b[4] = {y[4 * i], y[4 * i + 1], y[4 * i + 2], y[4 * i + 3]};
    w[i] = e4m3x4(a, b);
  }
}

template <int PLACE>
__device__ __forceinline__ void turn16(const LaneRow<PLACE>& l, const Turns& t, float (&v)[16]) {
#pragma unroll
  for (int e = 0; e < kPer; ++e) {
    const int i = PLACE == kHalves ? e : 2 * e, j = PLACE == kHalves ? 8 + e : 2 * e + 1;
    const float x = v[i], y = v[j];
    const bool on = PLACE == kHalves ? l.turned > 0 : e < l.turned;
    v[i] = on ? fmaf(x, t.t[e].x, -(y * t.t[e].y)) : x;
    v[j] = on ? fmaf(x, t.t[e].y, y * t.t[e].x) : y;
  }
}

__device__ __forceinline__ float largest16(const float (&x)[16]) {   // of the finite ones
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const float a = fabsf(x[e]);
    m = fmaxf(m, a < INFINITY ? a : 0.f);
  }
  return m;
}

// The turns of a run of tokens in LDS, computed once for all heads: lane c of a
// row finds its eight in four reads of 16 bytes, side by side with the other
// lanes'.
template <int TOKENS>
struct TurnTable {
  float4 t[TOKENS][kPer / 2][kLaneRow];
  // position(i) of the run's token i; every thread of the workgroup takes part
  template <class F>
  __device__ __forceinline__ void fill(const Rotary& r, int threads, F position) {
    for (int i = threadIdx.x; i < TOKENS * kPairsOfRow; i += threads) {
      const int f = i % kPairsOfRow;
      if (2 * f >= r.dim) continue;
      const float2 y = turn_at(r, position(i / kPairsOfRow), r.turns[f]);
      ((float2*)&t[i / kPairsOfRow][f % kPer / 2][f / kPer])[f & 1] = y;
    }
  }
  __device__ __forceinline__ void get(int token, int c, Turns& y) const {
#pragma unroll
    for (int j = 0; j < kPer / 2; ++j) {
      const float4 a = t[token][j][c];
      y.t[2 * j] = make_float2(a.x, a.y);
      y.t[2 * j + 1] = make_float2(a.z, a.w);
    }
  }
};

}  // namespace

}  // namespace fp2
