// Rotary positions: device code shared by rope.hip and kvcache.hip.
//
// A workgroup first takes cosine and sine (times mscale) of its rows' pairs
// into LDS in fp64, each once for all heads of the row, then rotates in fp64
// and rounds once.  The angle pos * inv_freq is an fp64 product: at position
// 10^6 an fp32 angle would be off by 0.06 radian.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/w4a8.h"

namespace w4a8 {

// Pairs of a workgroup's LDS table (16 KB).
constexpr int ROPE_PAIRS = 1024;

struct RopeArgs {
  const double *inv_freq;
  const int32_t *pos;
  int half;          // n_rot / 2; 0: no rotation
  int interleaved;
  double mscale;
};

inline RopeArgs rope_args(const w4a8_rope *r) {
  RopeArgs a = {};
  if (r) {
    a.inv_freq = r->inv_freq;
    a.pos = r->pos;
    a.half = (int)(r->n_rot / 2);
    a.interleaved = r->layout == W4A8_ROPE_INTERLEAVED;
    a.mscale = (double)r->mscale;
  }
  return a;
}

// Host checks of a w4a8_rope for heads of D elements.
int rope_check(const w4a8_rope *rope, int64_t D);

// Sine and cosine of an fp64 angle to about 2^-53, for any angle that is
// itself known that well: less a multiple n of pi/2 in two parts (the fused
// difference is exact to its rounding), then the Taylor series over
// |r| <= pi/4, whose first terms left out are r^17/17! < 2^-54 and r^18/18!.
// (The library's sincos carries its reduction of huge angles along: three times
// the registers.)
__device__ __forceinline__ void rope_sincos(double a, double &s, double &c) {
  const double n = rint(a * 0.63661977236758134308);       // 2 / pi
  double r = fma(-n, 1.57079632679489655800, a);           // pi / 2 to 53 bits
  r = fma(-n, 6.12323399573676603587e-17, r);              // and what is left of it
  const double z = r * r;
  double p = -1.0 / 1307674368000.0;                       // 1 / 15!, with its sign
  p = fma(p, z, 1.0 / 6227020800.0);
  p = fma(p, z, -1.0 / 39916800.0);
  p = fma(p, z, 1.0 / 362880.0);
  p = fma(p, z, -1.0 / 5040.0);
  p = fma(p, z, 1.0 / 120.0);
  p = fma(p, z, -1.0 / 6.0);
  const double sr = fma(p * z, r, r);
  double q = 1.0 / 20922789888000.0;                       // 1 / 16!
  q = fma(q, z, -1.0 / 87178291200.0);
  q = fma(q, z, 1.0 / 479001600.0);
  q = fma(q, z, -1.0 / 3628800.0);
  q = fma(q, z, 1.0 / 40320.0);
  q = fma(q, z, -1.0 / 720.0);
  q = fma(q, z, 1.0 / 24.0);
  q = fma(q, z, -0.5);
  const double cr = fma(q, z, 1.0);
  const int k = (int)(n - 4.0 * floor(n * 0.25));          // quadrant
  const double x = k & 1 ? cr : sr, y = k & 1 ? sr : cr;
  s = k & 2 ? -x : x;
  c = (k + 1) & 2 ? -y : y;
}

// cs[i * half + p] = (cos, sin) * mscale of row t0 + i, pair p (all threads).
__device__ __forceinline__ void rope_table(const RopeArgs &r, double2 *cs, int64_t t0, int rows) {
  for (int i = threadIdx.x; i < rows * r.half; i += blockDim.x) {
    const int row = i / r.half, p = i - row * r.half;
    const double a = (double)r.pos[t0 + row] * r.inv_freq[p];
    double s, c;
    rope_sincos(a, s, c);
    cs[i] = make_double2(c * r.mscale, s * r.mscale);
  }
}

__device__ __forceinline__ float2 rope_pair(float xa, float xb, double2 cs) {
  const double a = (double)xa, b = (double)xb;
  return make_float2((float)(a * cs.x - b * cs.y), (float)(b * cs.x + a * cs.y));
}

// How a head of D elements falls into units that one thread rotates, so that
// both elements of every pair are read and written by the same thread (which
// makes in-place calls safe): with `vec` 16-byte units (half layout: two of
// them half a rotation apart, then the plain ones; interleaved: one), else
// single pairs, then single elements.
struct RopeUnits {
  int vec, units;
  __host__ __device__ RopeUnits(int half, int interleaved, int D) {
    vec = interleaved ? (half % 2 == 0) : (half % 4 == 0);
    units = !vec ? D - half : interleaved ? D / 4 : D / 4 - half / 4;
  }
};

// A unit's first element, and its pairs' other halves (else the same again).
__device__ __forceinline__ int2 rope_unit_at(const RopeArgs &r, int u) {
  if (r.interleaved) return make_int2(4 * u, 4 * u);
  const int nr = r.half / 4, d = u < nr ? 4 * u : 2 * r.half + 4 * (u - nr);
  return make_int2(d, u < nr ? d + r.half : d);
}

// Stores unit u with `vec`, loaded as a and b from rope_unit_at.
__device__ __forceinline__ void rope_unit_turn(const RopeArgs &r, float4 a, float4 b, float *y,
                                               const double2 *cs, int u) {
  const int2 at = rope_unit_at(r, u);
  if (!r.interleaved) {
    if (u < r.half / 4) {
      const float2 p0 = rope_pair(a.x, b.x, cs[4 * u]), p1 = rope_pair(a.y, b.y, cs[4 * u + 1]),
                   p2 = rope_pair(a.z, b.z, cs[4 * u + 2]), p3 = rope_pair(a.w, b.w, cs[4 * u + 3]);
      *reinterpret_cast<float4 *>(y + at.y) = make_float4(p0.y, p1.y, p2.y, p3.y);
      a = make_float4(p0.x, p1.x, p2.x, p3.x);
    }
  } else if (2 * u < r.half) {
    const float2 p0 = rope_pair(a.x, a.y, cs[2 * u]), p1 = rope_pair(a.z, a.w, cs[2 * u + 1]);
    a = make_float4(p0.x, p0.y, p1.x, p1.y);
  }
  *reinterpret_cast<float4 *>(y + at.x) = a;
}

__device__ __forceinline__ void rope_unit(const RopeArgs &r, RopeUnits ru, const float *x, float *y,
                                          const double2 *cs, int u) {
  if (ru.vec && !r.interleaved && u < r.half / 4) {
    const float4 a = *reinterpret_cast<const float4 *>(x + 4 * u);
    const float4 b = *reinterpret_cast<const float4 *>(x + 4 * u + r.half);
    rope_unit_turn(r, a, b, y, cs, u);
  } else if (ru.vec) {
    const float4 a = *reinterpret_cast<const float4 *>(x + rope_unit_at(r, u).x);
    rope_unit_turn(r, a, a, y, cs, u);
  } else if (u < r.half) {
    const int ia = r.interleaved ? 2 * u : u, ib = r.interleaved ? 2 * u + 1 : u + r.half;
    const float2 p = rope_pair(x[ia], x[ib], cs[u]);
    y[ia] = p.x;
    y[ib] = p.y;
  } else {
    y[u + r.half] = x[u + r.half];
  }
}

// Elements d .. d + 3 of a rotated head, d = 4 e4, from a, the elements as they
// are, and b: in the half layout their pairs' other halves, where that is one
// quad (half % 4 == 0), from d + rope_other(r, d).
__device__ __forceinline__ int rope_other(const RopeArgs &r, int d) {
  return r.interleaved || d >= 2 * r.half ? 0 : d < r.half ? r.half : -r.half;
}
__device__ __forceinline__ void rope_four_turn(const RopeArgs &r, float4 a, float4 b,
                                               const double2 *cs, int e4, float v[4]) {
  const int d = 4 * e4;
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
  if (d >= 2 * r.half) return;
  if (r.interleaved) {
#pragma unroll
    for (int i = 0; i < 4; i += 2)
      if (d + i < 2 * r.half) {
        const float2 p = rope_pair(v[i], v[i + 1], cs[(d + i) / 2]);
        v[i] = p.x;
        v[i + 1] = p.y;
      }
  } else {                           // first half a cos - b sin, second b sin + a cos
    const float o[4] = {b.x, b.y, b.z, b.w};
    const double sign = d < r.half ? -1.0 : 1.0;
    const double2 *c = cs + (d < r.half ? d : d - r.half);
#pragma unroll
    for (int i = 0; i < 4; i++)
      v[i] = (float)((double)v[i] * c[i].x + (double)o[i] * (sign * c[i].y));
  }
}
// The same where a quad's other halves are not one quad.
__device__ __forceinline__ void rope_four(const RopeArgs &r, const float *x, const double2 *cs,
                                          int e4, float v[4]) {
  const int d = 4 * e4;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const int k = d + i;
    if (k >= 2 * r.half) v[i] = x[k];
    else if (r.interleaved) v[i] = k % 2 ? rope_pair(x[k - 1], x[k], cs[k / 2]).y
                                         : rope_pair(x[k], x[k + 1], cs[k / 2]).x;
    else if (k < r.half) v[i] = rope_pair(x[k], x[k + r.half], cs[k]).x;
    else v[i] = rope_pair(x[k - r.half], x[k], cs[k - r.half]).y;
  }
}

}  // namespace w4a8
