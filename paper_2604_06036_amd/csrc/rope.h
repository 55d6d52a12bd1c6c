// Angles of rotary embedding.  Internal to the library.
#pragma once

#include <math.h>

#include "common.h"

namespace cs {

constexpr int kRopeMaxPairs = 128;       // head_dim <= 256

// theta_i = base^(-2i/head_dim), evaluated on the host, and which positional component drives pair i.
struct RopeAngles {
  double theta[kRopeMaxPairs];
  const int32_t* __restrict__ pos;             // [rows], or [rows][3] with axis_of_pair; nullptr: no rotation
  const uint8_t* __restrict__ axis_of_pair;    // [head_dim / 2] values 0..2
};

// (64 powers: about 1 us of the host.)
inline void rope_angles(RopeAngles* r, const int32_t* pos, const uint8_t* axis_of_pair, float base, int head_dim) {
  for (int i = 0; i < kRopeMaxPairs; ++i) r->theta[i] = i < head_dim / 2 ? pow(static_cast<double>(base), -2.0 * i / head_dim) : 0.0;
  r->pos = pos;
  r->axis_of_pair = axis_of_pair;
}

// Cosine and sine of an angle in double precision, rounded to single: reduced by multiples of pi/2 (two parts, fused),
// then the Taylor series to where the next term is below 2^-53 on [-pi/4, pi/4].  Rows that are held in 4 bits need it:
// a cosine one unit off would now and then round an element of a row to another code than the formula's.
__device__ __forceinline__ void sincos_rounded(double ang, float* sn, float* cn) {
  const double k = rint(ang * 0.63661977236758134);
  double r = fma(-k, 1.5707963267948966, ang);
  r = fma(-k, 6.123233995736766e-17, r);
  const double z = r * r;
  double s = 1.0 / 355687428096000.0;                                   // 1/17!
  s = fma(s, z, -1.0 / 1307674368000.0);
  s = fma(s, z, 1.0 / 6227020800.0);
  s = fma(s, z, -1.0 / 39916800.0);
  s = fma(s, z, 1.0 / 362880.0);
  s = fma(s, z, -1.0 / 5040.0);
  s = fma(s, z, 1.0 / 120.0);
  s = fma(s, z, -1.0 / 6.0);
  s = fma(s * z, r, r);
  double c = 1.0 / 20922789888000.0;                                    // 1/16!
  c = fma(c, z, -1.0 / 87178291200.0);
  c = fma(c, z, 1.0 / 479001600.0);
  c = fma(c, z, -1.0 / 3628800.0);
  c = fma(c, z, 1.0 / 40320.0);
  c = fma(c, z, -1.0 / 720.0);
  c = fma(c, z, 1.0 / 24.0);
  c = fma(c, z, -0.5);
  c = fma(c, z, 1.0);
  const int quad = static_cast<int>(static_cast<long long>(k)) & 3;
  const float sf = static_cast<float>(s), cf = static_cast<float>(c);
  const float sq = (quad & 1) ? cf : sf, cq = (quad & 1) ? sf : cf;
  *sn = (quad & 2) ? -sq : sq;
  *cn = ((quad + 1) & 2) ? -cq : cq;
}

// cos / sin of N pairs from `first` on, for row `row`.
template <int N>
__device__ __forceinline__ void rope_row(const RopeAngles& r, int64_t row, int first, float* cn, float* sn) {
  int p0, p1 = 0, p2 = 0;
  if (r.axis_of_pair) {
    p0 = r.pos[row * 3];
    p1 = r.pos[row * 3 + 1];
    p2 = r.pos[row * 3 + 2];
  } else {
    p0 = r.pos[row];
  }
#pragma unroll
  for (int i = 0; i < N; ++i) {
    int p = p0;
    if (r.axis_of_pair) {
      const int axis = r.axis_of_pair[first + i];
      p = axis == 0 ? p0 : axis == 1 ? p1 : p2;
    }
    sincos_rounded(static_cast<double>(p) * r.theta[first + i], &sn[i], &cn[i]);
  }
}

// One pair, turned: products and their sum are rounded one by one (single precision, not fused), so that the rows a
// 4-bit cache holds are those of the formula in single precision, whoever evaluates it.
__device__ __forceinline__ void rope_turn(float a, float b, float c, float s, float* ra, float* rb) {
#pragma clang fp contract(off)
  const float ac = a * c, bs = b * s, bc = b * c, as = a * s;
  *ra = ac - bs;
  *rb = bc + as;
}

}  // namespace cs
