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

// cs[i * half + p] = (cos, sin) * mscale of row t0 + i, pair p (all threads).
__device__ __forceinline__ void rope_table(const RopeArgs &r, double2 *cs, int64_t t0, int rows) {
  for (int i = threadIdx.x; i < rows * r.half; i += blockDim.x) {
    const int row = i / r.half, p = i - row * r.half;
    const double a = (double)r.pos[t0 + row] * r.inv_freq[p];
    double s, c;
    sincos(a, &s, &c);
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

__device__ __forceinline__ void rope_unit(const RopeArgs &r, RopeUnits ru, const float *x, float *y,
                                          const double2 *cs, int u) {
  if (ru.vec && !r.interleaved) {
    const int nr = r.half / 4;
    if (u < nr) {
      const float4 a = *reinterpret_cast<const float4 *>(x + 4 * u);
      const float4 b = *reinterpret_cast<const float4 *>(x + 4 * u + r.half);
      const float2 p0 = rope_pair(a.x, b.x, cs[4 * u]), p1 = rope_pair(a.y, b.y, cs[4 * u + 1]),
                   p2 = rope_pair(a.z, b.z, cs[4 * u + 2]), p3 = rope_pair(a.w, b.w, cs[4 * u + 3]);
      *reinterpret_cast<float4 *>(y + 4 * u) = make_float4(p0.x, p1.x, p2.x, p3.x);
      *reinterpret_cast<float4 *>(y + 4 * u + r.half) = make_float4(p0.y, p1.y, p2.y, p3.y);
    } else {
      const int d = 2 * r.half + 4 * (u - nr);
      *reinterpret_cast<float4 *>(y + d) = *reinterpret_cast<const float4 *>(x + d);
    }
  } else if (ru.vec) {
    float4 a = *reinterpret_cast<const float4 *>(x + 4 * u);
    if (2 * u < r.half) {
      const float2 p0 = rope_pair(a.x, a.y, cs[2 * u]), p1 = rope_pair(a.z, a.w, cs[2 * u + 1]);
      a = make_float4(p0.x, p0.y, p1.x, p1.y);
    }
    *reinterpret_cast<float4 *>(y + 4 * u) = a;
  } else if (u < r.half) {
    const int ia = r.interleaved ? 2 * u : u, ib = r.interleaved ? 2 * u + 1 : u + r.half;
    const float2 p = rope_pair(x[ia], x[ib], cs[u]);
    y[ia] = p.x;
    y[ib] = p.y;
  } else {
    y[u + r.half] = x[u + r.half];
  }
}

// Elements 4 * e4 .. + 3 of the rotated head (reads the pairs' other halves
// from x; for out-of-place use).
__device__ __forceinline__ void rope_four(const RopeArgs &r, const float *x, const double2 *cs,
                                          int e4, float v[4]) {
  const float4 t = reinterpret_cast<const float4 *>(x)[e4];
  v[0] = t.x; v[1] = t.y; v[2] = t.z; v[3] = t.w;
  const int d = 4 * e4;
  if (d >= 2 * r.half) return;
  if (r.interleaved) {
#pragma unroll
    for (int i = 0; i < 4; i += 2)
      if (d + i < 2 * r.half) {
        const float2 p = rope_pair(v[i], v[i + 1], cs[(d + i) / 2]);
        v[i] = p.x;
        v[i + 1] = p.y;
      }
  } else {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int k = d + i;
      if (k < r.half) v[i] = rope_pair(v[i], x[k + r.half], cs[k]).x;
      else if (k < 2 * r.half) v[i] = rope_pair(x[k - r.half], v[i], cs[k - r.half]).y;
    }
  }
}

}  // namespace w4a8
