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
//   kOdd     the same for any even dim: a lane's 16 elements are adjacent, and
//            their partners come through LDS
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
  float eighth, rest;       // a pi / 4, in two parts
};
inline Rotary make_rotary(const uint64_t* turns, int dim, bool inverse, double scale) {
  const double eighth = scale * 0.785398163397448309616;
  return Rotary{turns, dim, inverse, (float)scale, (float)eighth, (float)(eighth - (float)eighth)};
}

enum PairPlace : int32_t { kPairs = 0, kHalves = 1, kOdd = 2 };

inline PairPlace place_of(int dim, bool interleaved) {
  return interleaved || dim == 2 ? kPairs : dim % 16 ? kOdd : kHalves;
}

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

// Cosine and sine of a fraction of a turn, times a. A quarter of a turn about the
// nearest multiple of one is left of it, f in [-1, 1) eighths: sin(pi/4 f) = f S(f^2)
// and cos(pi/4 f) = C(f^2), with the coefficients of least largest error (2^-29.6 and
// 2^-34). With a = 1 they are off by at most 2^-23.7, as a rule (rms) by 2^-25.8 over 2^24
// fractions, so that a turn is as near as one with rounded sines. The hardware's own
// sine and cosine are off by up to 2^-22.3, and twice as many codes come out on the
// other side of a border with them.
__device__ __forceinline__ float2 turn_at(const Rotary& r, int n, uint64_t turns) {
  const uint32_t phase = phase_at(n, turns);
  const float f = (float)(int)(phase << 2) * 0x1p-31f, z = f * f;
  const float s2 = z * fmaf(z, fmaf(z, -3.58772584e-5f, 2.48987197e-3f), -8.07453673e-2f);   // S - pi/4
  const float c2 = fmaf(z, fmaf(z, fmaf(z, 3.53133465e-6f, -3.25942008e-4f), 1.58543278e-2f), -3.08425136e-1f);
  const float s = fmaf(f, r.eighth, f * fmaf(r.scale, s2, r.rest));
  const float c = fmaf(r.scale * z, c2, r.scale);
  const uint32_t q = phase + (1u << 29), odd = q << 1;     // quarter: the top two bits of q
  const float x = (int)odd < 0 ? s : c, y = (int)odd < 0 ? c : s;
  return make_float2(__uint_as_float(__float_as_uint(x) ^ ((q ^ odd) & 0x80000000u)),
                     __uint_as_float(__float_as_uint(y) ^ ((r.inverse ? ~q : q) & 0x80000000u)));
}

// A lane's frequencies and turns: of eight pairs, or (kOdd) of its sixteen elements.
template <int PLACE>
struct Freqs {
  uint64_t f[PLACE == kOdd ? 1 : kPer];          // (kOdd: read again where they are needed)
};
template <int PLACE>
struct Turns {
  float2 t[PLACE == kOdd ? 2 * kPer : kPer];
};

// What lane c (of the eight) holds of a row. `turned` pairs of its eight: the first ones.
template <int PLACE>
struct LaneRow {
  int c, dim;
  int at[2];        // first elements of its two runs of eight
  int turned;
  __device__ __forceinline__ LaneRow(int lane, int dim_) : c(lane & 7), dim(dim_) {
    turned = min(max(dim / 2 - kPer * c, 0), kPer);
    if (PLACE == kHalves && turned) at[0] = 8 * c, at[1] = dim / 2 + 8 * c;
    else at[0] = 16 * c, at[1] = 16 * c + 8;      // (halves: dim + 16 (c - dim / 16))
  }
  __device__ __forceinline__ Freqs<PLACE> freqs(const Rotary& r) const {
    Freqs<PLACE> y{};
    if constexpr (PLACE != kOdd) {
#pragma unroll
      for (int e = 0; e < kPer; ++e) y.f[e] = e < turned ? r.turns[kPer * c + e] : 0;
    }
    return y;
  }
  // The turns of the lane's pairs, or elements, at position n.
  __device__ __forceinline__ void turns(const Rotary& r, const Freqs<PLACE>& f, int n, Turns<PLACE>& y) const {
    if constexpr (PLACE != kOdd) {
#pragma unroll
      for (int e = 0; e < kPer; ++e) y.t[e] = turn_at(r, n, f.f[e]);
    } else {
#pragma unroll
      for (int e = 0; e < 2 * kPer; ++e) y.t[e] = element_turn(r, n, e);
    }
  }
  // kOdd: element e becomes itself times .x plus its partner times .y: x cos - y sin of the first, y cos + x sin of
  // the second (past dim anything)
  __device__ __forceinline__ float2 element_turn(const Rotary& r, int n, int e) const {
    const int h = dim / 2, j = 16 * c + e;
    const float2 t = turn_at(r, n, r.turns[j < h ? j : j < dim ? j - h : 0]);
    return make_float2(t.x, j < h ? -t.y : t.y);
  }
};

// A lane's part of a row as it comes: 16 bf16 (eight words) or 16 codes (four).
// kPairs, kOdd: in the row's order; kHalves: the first run, then the second.
template <int PLACE, class T>
__device__ __forceinline__ void load_part(const LaneRow<PLACE>& l, const T* row, uint32_t (&w)[4 * sizeof(T)]) {
  if constexpr (sizeof(T) == 2) {
    const uint4 a = *(const uint4*)(row + l.at[0]), b = *(const uint4*)(row + l.at[1]);
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
  } else if constexpr (PLACE != kHalves) {
    const uint4 a = *(const uint4*)(row + l.at[0]);
    w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w;
  } else {
    const uint2 a = *(const uint2*)(row + l.at[0]), b = *(const uint2*)(row + l.at[1]);
    w[0] = a.x, w[1] = a.y, w[2] = b.x, w[3] = b.y;
  }
}
template <int PLACE, class T>
__device__ __forceinline__ void store_part(const LaneRow<PLACE>& l, T* row, const uint32_t (&w)[4 * sizeof(T)]) {
  if constexpr (sizeof(T) == 2) {
    *(uint4*)(row + l.at[0]) = make_uint4(w[0], w[1], w[2], w[3]);
    *(uint4*)(row + l.at[1]) = make_uint4(w[4], w[5], w[6], w[7]);
  } else if constexpr (PLACE != kHalves) {
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

// Values in units of a scale, at most 448 if finite, as codes (nearest, ties to
// even). The conversion makes NaN codes of infinities and NaN.
__device__ __forceinline__ void codes16(const float (&x)[16], uint32_t (&w)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i], x[4 * i + 1], 0, false);
    w[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[4 * i + 2], x[4 * i + 3], lo, true);
  }
}
// The same for values that may be larger, held within +-448.
__device__ __forceinline__ void codes16_held(const float (&x)[16], uint32_t (&w)[4]) {
  float y[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) y[e] = fabsf(x[e]) < INFINITY ? __builtin_amdgcn_fmed3f(x[e], -448.f, 448.f) : x[e];
  codes16(y, w);
}

// x / scale, correctly rounded, held within +-448, as codes: the product with the
// scale's inverse (held at 1024, so that nothing overflows), corrected by its
// remainder; a division takes ten instructions. Scales whose inverse or
// remainders leave fp32's normal range are divided by.
struct Divisor {
  float scale, inv;
  bool fast;
  __device__ __forceinline__ explicit Divisor(float s)
      : scale(s), inv(1.f / s), fast(s > 0x1p-90f && s < 0x1p90f) {}
};
__device__ __forceinline__ void codes16_by(const float (&x)[16], const Divisor& d, uint32_t (&w)[4]) {
  float y[16];
  if (d.fast) {
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float q = __builtin_amdgcn_fmed3f(x[e] * d.inv, -1024.f, 1024.f);
      y[e] = fmaf(fmaf(-q, d.scale, x[e]), d.inv, q);
    }
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) y[e] = x[e] / d.scale;
  }
#pragma unroll
  for (int e = 0; e < 16; ++e)
    y[e] = fabsf(x[e]) < INFINITY ? __builtin_amdgcn_fmed3f(y[e], -448.f, 448.f) : x[e];
  codes16(y, w);
}

// The partners of a lane's sixteen elements, by way of LDS (kOdd): every lane of
// the wave leaves its part of a row there and reads the elements dim / 2 further
// or before. Rows lie four words apart from a multiple of the banks.
template <int N>
__device__ __forceinline__ void partners16(const LaneRow<kOdd>& l, const uint32_t (&w)[N], float (&v)[16]) {
  constexpr int kMostWaves = 8, ROW = 8 * N + 4, ESZ = N / 4;   // words of a row, bytes of an element
  __shared__ __align__(16) uint32_t s_rows[kMostWaves][kPass][ROW];
  uint32_t* row = s_rows[threadIdx.x >> 6][(threadIdx.x & 63) / kLaneRow];
  // (one wave's traffic, which LDS takes in order; the fences keep the compiler to it)
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
#pragma unroll
  for (int i = 0; i < N; i += 4) *(uint4*)(row + N * l.c + i) = make_uint4(w[i], w[i + 1], w[i + 2], w[i + 3]);
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
  const int h = l.dim / 2;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const int j = 16 * l.c + e, at = j < h ? j + h : j < l.dim ? j - h : j;
    if constexpr (ESZ == 2) v[e] = __uint_as_float((uint32_t)((const uint16_t*)row)[at] << 16);
    else v[e] = __builtin_amdgcn_cvt_f32_fp8(((const uint8_t*)row)[at], 0);
  }
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A lane's values, turned. Every lane of the wave takes part.
template <int PLACE, int N>
__device__ __forceinline__ void turned16(const LaneRow<PLACE>& l, const Turns<PLACE>& t, const uint32_t (&w)[N], float (&v)[16]) {
  unpack16(w, v);
  if constexpr (PLACE == kOdd) {
    float p[16];
    partners16(l, w, p);
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = 16 * l.c + e < l.dim ? fmaf(v[e], t.t[e].x, p[e] * t.t[e].y) : v[e];
  } else {
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int i = PLACE == kHalves ? e : 2 * e, j = PLACE == kHalves ? 8 + e : 2 * e + 1;
      const float x = v[i], y = v[j];
      const bool on = PLACE == kHalves ? l.turned > 0 : e < l.turned;
      v[i] = on ? fmaf(x, t.t[e].x, -(y * t.t[e].y)) : x;
      v[j] = on ? fmaf(x, t.t[e].y, y * t.t[e].x) : y;
    }
  }
}

// The same at position n, for one row: its turns are not kept (sixteen would not fit beside what is).
template <int PLACE, int N>
__device__ __forceinline__ void turned16_at(const LaneRow<PLACE>& l, const Rotary& r, const Freqs<PLACE>& f, int n,
                                            const uint32_t (&w)[N], float (&v)[16]) {
  if constexpr (PLACE == kOdd) {
    float p[16];
    __builtin_amdgcn_sched_barrier(0);
    partners16(l, w, p);
    unpack16(w, v);
#pragma unroll
    for (int e = 0; e < 16; ++e) {
      const float2 t = l.element_turn(r, n, e);
      v[e] = 16 * l.c + e < l.dim ? fmaf(v[e], t.x, p[e] * t.y) : v[e];
    }
    __builtin_amdgcn_sched_barrier(0);
  } else {
    Turns<PLACE> t;
    l.turns(r, f, n, t);
    turned16(l, t, w, v);
  }
}

__device__ __forceinline__ float largest16(const float (&x)[16]) {   // NaN is left out, infinities are not
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) m = fmaxf(m, fabsf(x[e]));
  return m;
}
__device__ __forceinline__ float largest16_finite(const float (&x)[16]) {
  float m = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) m = fmaxf(m, fabsf(x[e]) < INFINITY ? fabsf(x[e]) : 0.f);
  return m;
}

}  // namespace

}  // namespace fp2
