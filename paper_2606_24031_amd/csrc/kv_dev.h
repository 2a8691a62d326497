// The paged 4-bit cache: layout and plan helpers shared by kvcache.hip and
// attn.hip (see w4a8.h for the layout).
//
// A tile is stored in the order in which attention reads it into matrix
// operands: a lane's share of a 64-token page is one 16-byte load a block,
// whole wave instructions are 1 KB contiguous, and neither side transposes.
// K: lane l takes payload dword l / 16 of tokens l % 16 + 16 i.  V: lane l
// takes payload byte l % 16 (elements l % 16 and + 16) of tokens
// 4 (l / 16) + e + 16 i, e in the order 0 2 1 3 so that one mask picks the
// pair (0, 1) and, eight bits down, (2, 3) into 16-bit halves.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "w4a8_dev.h"

namespace w4a8 {

constexpr int KV_PAGE = W4A8_KV_PAGE;

__host__ __device__ constexpr int kv_scale_bytes(bool sym) { return sym ? 4 : 2; }
__host__ __device__ constexpr int64_t kv_tile_bytes(int D, bool sym) {
  return (int64_t)(D / 32) * (1024 + KV_PAGE * kv_scale_bytes(sym));
}
__host__ __device__ constexpr int kv_k_dword(int b, int c, int t) {
  return b * 256 + c * 64 + (t % 16) * 4 + t / 16;
}
__host__ __device__ constexpr int kv_v_byte(int b, int j, int t) {
  return b * 1024 + (t % 16) / 4 * 256 + j * 16 + t / 16 * 4 + ((t & 1) << 1 | (t >> 1 & 1));
}
__host__ __device__ constexpr int kv_scale_at(int b, int t) {
  return b * KV_PAGE + (t % 16) / 4 * 16 + t / 16 * 4 + t % 4;
}

// The cache's and attention's quantizers take a block's scale as the product
// amax * fl(1/7) or amax * fl(1/127), at most an ulp from the quotient of the
// block formats' own quantizers: one multiply where a correctly rounded
// division is a dozen instructions, in a prologue that every run of pages
// repeats.  (Q4_0's m / -8 is exact either way.)
__device__ __forceinline__ float kv_amax8(const float v[4]) {
  return max8(fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3]))));
}
__device__ __forceinline__ uint32_t kv_q4_sym_block8(const float v[4], float &d) {
  d = kv_amax8(v) * (1.0f / 7.0f);
  return q4_sym_codes(v, d);
}
// 8-bit codes of a query's block; d: its scale (a fp16 number, or with SYM
// any), whose reciprocal the codes are taken with.
template <bool SYM>
__device__ __forceinline__ uint32_t kv_q8_block8(const float v[4], float &d) {
  d = kv_amax8(v) * (1.0f / 127.0f);
  if (!SYM) d = f16_bits_to_f32(f32_to_f16_bits(d));
  const float id = SYM ? sym_inverse(d) : d != 0.0f ? 1.0f / d : 0.0f;
  uint32_t packed = 0;
#pragma unroll
  for (int i = 0; i < 4; i++) {
    const int c = id == 0.0f ? 0 : round_clamp(v[i] * id, 127);
    packed |= ((uint32_t)c & 0xFFu) << (8 * i);
  }
  return packed;
}

// Device view of a plan.
struct KvPlan {
  uint8_t *k, *v;
  const int32_t *pages, *len, *cu;
  int64_t n_pages;
  int max_pages, B, NKV;
};

inline KvPlan kv_plan(const w4a8_kv *kv) {
  return {reinterpret_cast<uint8_t *>(kv->k_pages), reinterpret_cast<uint8_t *>(kv->v_pages),
          kv->page_table, kv->kv_len, kv->cu_rows, kv->n_pages, (int)kv->max_pages, (int)kv->B,
          (int)kv->NKV};
}

// Sizes and format only / sizes, pointers and alignment.
int kv_check_sizes(const w4a8_kv *kv);
int kv_check(const w4a8_kv *kv);

__device__ __forceinline__ int64_t kv_clamp_row(int v, int64_t T) {
  return v < 0 ? 0 : (v > T ? T : v);
}

// The sequence that holds row r and the row's token, found by one wave: 64
// entries of cu_rows are probed at once, so up to 64 sequences take one load
// round and 4096 two.  Returns -1 (token -1) for a row of no sequence.
__device__ __forceinline__ int kv_find(const KvPlan &p, int64_t T, int64_t r, int &token) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = p.B;
  token = -1;
  while (n > 64) {
    const int step = (n + 63) / 64, at = lane * step;
    const bool ok = at < n && kv_clamp_row(p.cu[lo + at], T) <= r;
    const int k = __popcll(__ballot(ok)) - 1;
    if (k < 0) return -1;
    lo += k * step;
    n = min(step, n - k * step);
  }
  int c0 = 0, c1 = 0, len = 0;
  if (lane < n) {
    c0 = p.cu[lo + lane];
    c1 = p.cu[lo + lane + 1];
    len = p.len[lo + lane];
  }
  const int k = __popcll(__ballot(lane < n && kv_clamp_row(c0, T) <= r)) - 1;
  if (k < 0) return -1;
  const int64_t r0 = kv_clamp_row(__builtin_amdgcn_readlane(c0, k), T);
  const int64_t r1 = kv_clamp_row(__builtin_amdgcn_readlane(c1, k), T);
  if (r < r0 || r >= r1) return -1;
  // counted from the sequence's own end, which may lie past the call's rows
  const int64_t t = (int64_t)__builtin_amdgcn_readlane(len, k) -
                    ((int64_t)__builtin_amdgcn_readlane(c1, k) - r);
  token = t < 0 || t >= (int64_t)p.max_pages * KV_PAGE ? -1 : (int)t;
  return lo + k;
}

}  // namespace w4a8
