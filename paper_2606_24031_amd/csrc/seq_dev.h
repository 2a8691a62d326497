// The plan of the recurrent operators (w4a8_seqs): its host checks, and how a
// kernel finds a sequence's rows and state slots.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "w4a8_host.h"

namespace w4a8 {

// Plan arrays as a kernel takes them (src and dst may be null).
struct Seqs {
  const int32_t *cu, *src, *dst;
  int64_t n_slots;
  int B, T;
};

inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }

inline int seqs_sizes(const w4a8_seqs *q, int64_t T) {
  if (!q) return W4A8_ENULL;
  if (q->B < 0 || q->n_slots < 0 || T < 0) return W4A8_ESHAPE;
  if (q->B >= (1 << 20) || q->n_slots >= ((int64_t)1 << 31) || T >= ((int64_t)1 << 31))
    return W4A8_ERANGE;
  return W4A8_OK;
}
inline int seqs_pointers(const w4a8_seqs *q) {
  if (q->B > 0 && !q->cu_rows) return W4A8_ENULL;
  if (!aligned4(q->cu_rows) || !aligned4(q->src) || !aligned4(q->dst)) return W4A8_EALIGN;
  return W4A8_OK;
}
inline Seqs seqs_args(const w4a8_seqs *q, int64_t T) {
  return Seqs{q->cu_rows, q->src, q->dst, q->n_slots, (int)q->B, (int)T};
}

// First row of sequence b (its end is that of b + 1), within the call's rows
// whatever the array holds.
__device__ __forceinline__ int seq_begin(const Seqs &q, int b) { return min(max(q.cu[b], 0), q.T); }

// The sequence that row t lies in: the last b with cu[b] <= t; -1 or B where
// none has it.
__device__ __forceinline__ int seq_of(const Seqs &q, int t) {
  int lo = -1, hi = q.B + 1;               // cu[lo] <= t < cu[hi], cu[-1] and cu[B + 1] at the ends
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (q.cu[m] <= t) lo = m; else hi = m;
  }
  return lo;
}

// State slots of sequence b, -1 for none.
__device__ __forceinline__ int64_t seq_src(const Seqs &q, int b) {
  const int s = q.src ? q.src[b] : b;
  return s >= 0 && s < q.n_slots ? s : -1;
}
__device__ __forceinline__ int64_t seq_dst(const Seqs &q, int b) {
  const int s = q.dst ? q.dst[b] : q.src ? q.src[b] : b;
  return s >= 0 && s < q.n_slots ? s : -1;
}

}  // namespace w4a8
