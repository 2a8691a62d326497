// Softmax attention over the paged 4-bit cache (Sec. 2.2: 10 of the 40 blocks
// are softmax attention with grouped query heads; Sec. 3.2 runs it in one
// pass with a running maximum and sum).
//
// A work item is a tile of 4 to 32 query rows of one KV head of a sequence (row
// f of a sequence: token f / G, head f % G of the group), times a run of pages
// when the rows alone would leave compute units idle; the last workgroup to
// finish, or a second launch, then joins the runs' partial results, in their
// order whoever is last.  A workgroup of AW waves takes AW pages of 64 keys a
// step:
//   scores   each wave its own page.  S^T = K Q^T: one
//            v_mfma_i32_16x16x32_i8 per 16 keys, 16 rows and block of 32, K
//            codes straight from the page (a 16-byte load a lane and block), Q
//            codes from LDS.  The accumulator starts at 0x4B400000, so the
//            int32 result read as a float is 1.5 2^23 + 16 s; with the row's
//            fp16 scale d_q one FMA gives 16 s d_q rounded once, the second
//            adds it times d_k.
//   softmax  base 2 with a running maximum per row, exchanged between the
//            waves through LDS; sums rescaled only on steps where some row's
//            maximum grows.  fp32.  The probabilities go to LDS, as each
//            lane holds them.
//   values   each wave its own block of 32 columns (of PS sets of the step's
//            pages where there are more waves than blocks): O^T += V^T W^T
//            with W = p d_v.  V codes are small integers, exact in fp16; W
//            goes in as hi + lo, two fp16 halves (22 bits; one fp16 or bf16
//            would be off by 2^-12 or 2^-9, more than everything else here
//            together).  d_v is scaled by a power of two, kept per wave, to
//            put the largest value scale met so far just below 2^15, so halves
//            do not overflow; fp16's smallest step is then 2^-26 of any scale's
//            as long as the scales lie within 2^13 of each other.  Where they
//            do not, a key of a huge scale that a row does not see, or gives no
//            probability, would push the row's other products off fp16's end:
//            from that step on the wave takes each row's products by a power
//            of two of the row's own (vexp WIDE).
// Scores by keys and values by columns: a wave's sums are 32 columns, not D,
// so registers leave room for two and more waves a SIMD, the code stays small
// (a short decode is bound by fetching it once) and no sums are exchanged at
// the end.  The lane layout of the score product's result (row l % 16, keys
// 4 (l / 16) + e + 16 i) is the one the value product wants for W, so a lane
// reads back from LDS what the same lane of another wave wrote.
// Bound: long decodes by HBM (36 bytes a key and 32 columns of K and V, read
// once for a tile's rows: for a group's heads up to 8 in small calls, 16 or 32
// in larger ones, again for the rest) and by VALU issue, which is close behind:
// 48 rows of 32 heads of 128 over up to 6000 keys take 52 us, 3.9 TB/s; one of
// 16 heads of 256 over 131072 keys 28 us, 19 of them the runs, 4.0 TB/s.
// Prompts by VALU issue, 94 % of a large one's cycles (2 x 2048 rows over 8192
// keys, 32 heads of 128: 803 us, 430 TFLOP/s): the two scaling operations a
// score and block and the three that make W's halves.  Short calls by their chain of
// launch, plan, page ids, pages and join (one row over 948 keys: 12 us).
#include <algorithm>
#include <cfloat>
#include <cmath>
#include <numeric>

#include "kv_dev.h"
#include "share_dev.h"
#include "w4a8_dev.h"
#include "w4a8_host.h"

namespace w4a8 {

namespace {

constexpr int TARGET = 768;           // runs wanted: three workgroups a compute unit
constexpr int AW = 4, AT = 64 * AW;   // waves of a workgroup; pages of a step
constexpr int GROUP = 16;             // runs joined at a time
constexpr int JT = 1024;              // threads of the joining kernel
constexpr int SLOTS_MAX = 2 * TARGET; // most runs of split items
// Value scales that a wave's two halves serve: from 2^-UNDER to 2^OVER times
// the first step's largest, none of 2^127 and more; others are wide.
constexpr int UNDER = 8, OVER = 5, WIDE = 128;
constexpr float FAR = 4194304.0f;     // 2^22: half a unit in the last place is 2^-3 below it
constexpr int64_t COUNTERS = (2 * SLOTS_MAX * 4 + 255) / 256 * 256;   // bytes before the partial results
static_assert(SLOTS_MAX / GROUP / GROUP <= GROUP, "two levels of joins");

typedef int v4i __attribute__((ext_vector_type(4)));
typedef uint32_t __attribute__((may_alias)) word;    // raw access to LDS of other types
typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));

struct AttnArgs {
  KvPlan p;
  const float *q;
  int64_t qs;
  float *out, *lse;
  int64_t T;
  int NH, G;
  float k;          // |scale| * log2(e) / 16, 1 for 0
  float sign;       // of scale: -1, 0 or 1
  int window;       // 0: none
  int *count;       // arrivals: [SLOTS_MAX] of a group of runs, [SLOTS_MAX] of an item's groups
  float *part;      // partial results, `slots` of them
  int slots;
  int64_t ids;      // runs at most
  int fused;        // the last workgroups join, not a second launch
  float inv_G;      // 1 / G
};

// What a sequence asks for.
struct Seq {
  int r0;           // its first row
  int qlen, pos;    // rows, the first one's token
  int lo, pages;    // first page any row sees, pages from there on
  int tiles;
  bool falls;       // cu_rows decrease here
};

template <int RT_>
__device__ __forceinline__ Seq seq_of(const AttnArgs &a, int s) {
  Seq r;
  const int c0 = a.p.cu[s], c1 = a.p.cu[s + 1], T = (int)a.T;
  const int r0 = min(max(c0, 0), T), r1 = min(max(c1, 0), T);
  r.falls = c1 < c0;
  r.r0 = r0;
  r.qlen = max(r1 - r0, 0);
  // (no tokens are as good as fewer than none, and no call has the 2^30 rows
  // that would lead from below to token 0: nothing here or in a row's keys
  // leaves 32 bits where cu_rows do not decrease)
  r.pos = max(max(a.p.len[s], 0) - (int)((uint32_t)c1 - (uint32_t)r0), -(1 << 30));
  const int hi = min(r.pos + r.qlen, a.p.max_pages * KV_PAGE);
  r.lo = a.window > 0 && r.pos >= a.window ? (r.pos - a.window + 1) / KV_PAGE : 0;
  const int end = (hi + KV_PAGE - 1) / KV_PAGE;
  r.pages = r.qlen > 0 && hi > 0 && end > r.lo ? end - r.lo : 0;
  r.tiles = (int)(((uint32_t)r.qlen * a.G + RT_ - 1) / RT_);
  return r;
}

// Inclusive scan of a wave's values by DPP moves.
template <int CTRL, int ROWS_, typename T_> __device__ __forceinline__ T_ dpp_or_0(T_ x) {
  const int v = __builtin_bit_cast(int, x);
  return __builtin_bit_cast(T_, __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS_, 0xF, true));
}
template <typename T_> __device__ __forceinline__ T_ wave_scan(T_ x) {
  x += dpp_or_0<0x111, 0xF>(x);      // row_shr 1, 2, 4, 8
  x += dpp_or_0<0x112, 0xF>(x);
  x += dpp_or_0<0x114, 0xF>(x);
  x += dpp_or_0<0x118, 0xF>(x);
  x += dpp_or_0<0x142, 0xA>(x);      // row 0's and 2's last into rows 1 and 3
  x += dpp_or_0<0x143, 0xC>(x);      // row 1's last into rows 2 and 3
  return x;
}

// Run `id` of the call, found by every wave on its own, 64 sequences a round:
// its sequence, its number within it, the runs of an item and the first
// partial slot of the sequence's runs.  A sequence's items fall into runs of
// at most C pages, C such that the call has about TARGET runs (of several
// tiles, whose first see half the pages of the last on average, only from 2 C
// on).  SPLIT: item `id` of those with several runs.  False past the end, and
// for every id where cu_rows decrease: sequences' rows could then number more
// than T, and runs more than the call has, so that some would never arrive at
// their counter and leave it for later calls.  Every workgroup goes over all
// sequences: not to be seen up to some hundred (1024 of one page and 4 heads:
// 22 us a call), but the square of their number counts later (4096: 184 us,
// 8192: 638).
struct Found {
  int s, local, runs, slot0;
};
template <int RT_, bool SPLIT = false>
__device__ __forceinline__ bool plan_find(const AttnArgs &a, int id, Found &f) {
  const int lane = threadIdx.x & 63, B = a.p.B;
  int tiles = 0, items = 0, pages = 0;          // of sequence lane
  bool falls = false;                           // of any so far
  const auto look = [&](int s) {
    tiles = items = pages = 0;
    if (s < B) {
      const Seq q = seq_of<RT_>(a, s);
      tiles = q.tiles;
      items = tiles * a.p.NKV;
      pages = q.pages;
      falls |= q.falls;
    }
  };
  float total = 0.0f;
  for (int s0 = (B - 1) / 64 * 64; s0 >= 0; s0 -= 64) {     // ends with the first 64
    look(s0 + lane);
    total += (float)items * (float)pages;
  }
  if (__ballot(falls)) [[unlikely]] return false;
  total = __builtin_bit_cast(
      float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, wave_scan(total)), 63));
  // (rounded up past the sum's own rounding: the partial slots are counted on C)
  const float c = fminf(total * (1.001f / TARGET), 1e9f);
  const int C = ((int)c + AW) / AW * AW;             // whole steps
  int base = 0, slots = 0;
  for (int s0 = 0; s0 < B; s0 += 64) {
    if (s0) look(s0 + lane);
    const int runs = pages > (tiles > 1 ? 2 * C : C) ? (pages + C - 1) / C : 1;
    const int ns = runs > 1 ? items * runs : 0;
    const int n = !SPLIT ? items * runs : runs > 1 ? items : 0;
    const int in = wave_scan(n), is = wave_scan(ns);
    const uint64_t hit = __ballot(id >= base + in - n && id < base + in);
    if (hit) {
      const int l = __ffsll((long long)hit) - 1;
      f.s = s0 + l;
      f.local = id - base - __builtin_amdgcn_readlane(in - n, l);
      f.runs = __builtin_amdgcn_readlane(runs, l);
      f.slot0 = slots + __builtin_amdgcn_readlane(is - ns, l);
      return true;
    }
    base += __builtin_amdgcn_readlane(in, 63);
    slots += __builtin_amdgcn_readlane(is, 63);
  }
  return false;
}

// Rows of a tile: row r is head head(r) of the group of the sequence's token
// token(r).  G < 2^16 and r < 64, so the quotient is exact in fp32.
struct RowMap {
  int t0, rem, G;
  float inv;
  __device__ RowMap(const AttnArgs &a, int f0) {
    G = a.G;
    inv = a.inv_G;
    t0 = f0 / G;
    rem = f0 - t0 * G;
  }
  __device__ __forceinline__ int token(int r) const {
    return t0 + (int)(((float)(rem + r) + 0.5f) * inv);
  }
  __device__ __forceinline__ int head(int r, int t) const { return rem + r - (t - t0) * G; }
};

// Maximum and sum over lanes l, l ^ 16, l ^ 32, l ^ 48.  (The results are cast
// as whole vectors: a bit cast of one element folds to element 0.)
__device__ __forceinline__ v2f swap32(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const v2u a = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __builtin_bit_cast(v2f, a);
}
__device__ __forceinline__ v2f swap16(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const v2u a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  return __builtin_bit_cast(v2f, a);
}
__device__ __forceinline__ float max4(float x) {
  const v2f a = swap32(x);
  const v2f b = swap16(fmaxf(a[0], a[1]));
  return fmaxf(b[0], b[1]);
}
__device__ __forceinline__ float sum4(float x) {
  const v2f a = swap32(x);
  const v2f b = swap16(a[0] + a[1]);
  return b[0] + b[1];
}

// x * y, and 0 where either is 0, whatever the other.
__device__ __forceinline__ float mul_zero(float x, float y) {
  float r;
  asm("v_mul_legacy_f32 %0, %1, %2" : "=v"(r) : "v"(x), "v"(y));
  return r;
}

__device__ __forceinline__ float exp2_f(float x) { return __builtin_amdgcn_exp2f(x); }

// p d of four keys.  (0 times anything is 0: a key that the row does not see
// may have any scale.)
__device__ __forceinline__ v4f products(v4f p, const float *d) {
  const v4f dv = *reinterpret_cast<const v4f *>(d);
  v4f w;
#pragma unroll
  for (int e = 0; e < 4; e++) w[e] = mul_zero(p[e], dv[e]);
  return w;
}
// The same, W, as the sum of two fp16 halves.
__device__ __forceinline__ void halves(v4f x, float minus, h4 &hi, h4 &lo) {
#pragma unroll
  for (int e = 0; e < 4; e += 2) {
    v2f w, z;
    w[0] = x[e];
    w[1] = x[e + 1];
    const h2 y = __builtin_convertvector(w, h2);
    z[0] = fmaf((float)y[0], minus, w[0]);
    z[1] = fmaf((float)y[1], minus, w[1]);
    const h2 y2 = __builtin_convertvector(z, h2);
    hi[e] = y[0]; hi[e + 1] = y[1];
    lo[e] = y2[0]; lo[e + 1] = y2[1];
  }
}
__device__ __forceinline__ void make_w(v4f p, const float *d, float minus, h4 &hi, h4 &lo) {
  halves(products(p, d), minus, hi, lo);
}
__device__ __forceinline__ float max_finite(float m, v4f w) {
#pragma unroll
  for (int e = 0; e < 4; e++) {
    const float y = fabsf(w[e]);
    m = fmaxf(m, y < INFINITY ? y : 0.0f);
  }
  return m;
}
// 2^e's bits without the sign, -126 <= e <= 128 (infinity's).
__device__ __forceinline__ uint32_t bits_of_2(int e) { return (uint32_t)(e + 127) << 24; }
__device__ __forceinline__ v4f ldexp4(v4f x, int by) {
#pragma unroll
  for (int e = 0; e < 4; e++) x[e] = ldexpf(x[e], by);
  return x;
}
__device__ __forceinline__ void put(h8 &v, int i, h4 x) {
#pragma unroll
  for (int e = 0; e < 4; e++) v[4 * i + e] = x[e];
}
// A rotation within 16 lanes (every lane valid, so no old value is kept).
template <int CTRL> __device__ __forceinline__ int ror(int x) {
  return __builtin_amdgcn_mov_dpp(x, CTRL, 0xF, 0xF, true);
}
template <int CTRL> __device__ __forceinline__ float ror_f(float x) {
  return __builtin_bit_cast(float, ror<CTRL>(__builtin_bit_cast(int, x)));
}

// Of lane l + (16 / PK) z of the 16.
template <int PK> __device__ __forceinline__ h4 from_col(h4 x, int z) {
  const v2u u = __builtin_bit_cast(v2u, x);
  const int by = 16 / PK * z;
  v2u r;
#pragma unroll
  for (int i = 0; i < 2; i++)
    r[i] = (uint32_t)(by == 0   ? (int)u[i]
                      : by == 4 ? ror<DPP_ROR12>((int)u[i])
                      : by == 8 ? ror<DPP_ROR8>((int)u[i])
                                : ror<DPP_ROR4>((int)u[i]));
  return __builtin_bit_cast(h4, r);
}

template <bool SYM> struct ScaleT { typedef _Float16 type; };
template <> struct ScaleT<true> { typedef float type; };

// NT tiles of 16 product columns, or with PK > 1 one of 16 / PK rows: the
// columns c, c + 16 / PK, .. then hold one row's scores for PK groups of 16
// keys (see the kernel).
template <int NB, bool SYM, int NT, int PK> struct Shape {
  static_assert(NT == 1 || PK == 1, "packed rows are one tile");
  static constexpr int D = 32 * NB;
  static constexpr int ROWS = 16 * NT / PK;
  static constexpr int BW = NB > AW ? NB / AW : 1;   // blocks of columns of a wave
  static constexpr int PS = NB < AW ? AW / NB : 1;   // waves that share a block
  static constexpr int NP = AW / PS;                 // pages of a step whose values a wave takes
  static constexpr int CH = 4 / PK;                  // score products kept apart: 16 PK keys each
  static_assert(NP * BW == NB, "one buffer for keys and values");
};

template <int NB, bool SYM, int NT, int PK> struct __align__(16) Lds {
  typedef Shape<NB, SYM, NT, PK> Sh;
  uint32_t q[NT * NB * PK * 64 * 2];           // Q codes in operand order
  union {
    v4f p[AW][NT * Sh::CH][64];                // a step's probabilities, as the lanes hold them
    v4f sums[Sh::PS > 1 ? AW : 1][2 * NT][64]; // at the end
  };
  float vs[AW][NB * 64];                       // the waves' value scales, times a power of two
  typename ScaleT<SYM>::type ks[AW][NB * 64];
  float qd[NT * NB * 16];
  float mx[16 * NT][AW];                       // the waves' maxima
  float l[AW][16 * NT];
  float2 rl[Sh::ROWS];                         // joins: references and sums
  int flag;
};

// N scales of raw words.
template <bool SYM> __device__ __forceinline__ float scale_of(const uint32_t *w, int i) {
  return SYM ? __builtin_bit_cast(float, w[i]) : f16_bits_to_f32(w[i / 2] >> (16 * (i & 1)));
}

template <int N>
__device__ __forceinline__ void load_words(const uint8_t *p, uint32_t (&w)[N]) {
  if constexpr (N == 1) {
    w[0] = *reinterpret_cast<const uint32_t *>(p);
  } else if constexpr (N == 2) {
    const v2u t = *reinterpret_cast<const v2u *>(p);
    w[0] = t[0]; w[1] = t[1];
  } else {
#pragma unroll
    for (int i = 0; i < N; i += 4) {
      const v4u t = reinterpret_cast<const v4u *>(p)[i / 4];
      w[i] = t[0]; w[i + 1] = t[1]; w[i + 2] = t[2]; w[i + 3] = t[3];
    }
  }
}

// Over the lanes that hold one row's scores: l ^ 16, ^ 32, ^ 48 and with
// packed rows the columns 16 / PK apart.
template <int PK> __device__ __forceinline__ float max_row(float x) {
  if (PK > 1) x = fmaxf(x, ror_f<DPP_ROR8>(x));
  if (PK > 2) x = fmaxf(x, ror_f<DPP_ROR4>(x));
  return max4(x);
}
template <int PK> __device__ __forceinline__ float sum_cols(float x) {
  if (PK > 1) x += ror_f<DPP_ROR8>(x);
  if (PK > 2) x += ror_f<DPP_ROR4>(x);
  return x;
}

// Number i of the 16 / PK keys that a lane holds of a page, less the lane's
// first.
template <int PK> __device__ __forceinline__ constexpr int key_off(int i) {
  return (i >> 2) * 16 * PK + (i & 3);
}

// Joins n partial results, `step` slots apart, of the slots at `part`: a row's
// weights by 16 lanes (w: LDS, n x ROWS), then every thread its columns of all
// of them, in order; the first JB of those are on their way meanwhile.
// fin(row, column, sum, R, l) takes 4 columns at a time; w is free afterwards.
template <int D, int ROWS, typename F>
__device__ __forceinline__ void join(int tid, float *part, int step, int n, float *w, float2 *rl,
                                     F &&fin) {
  constexpr int PB = ROWS * (D + 2), PER = D / 4, IT = (ROWS * PER + AT - 1) / AT;
  constexpr int JB = IT >= 8 ? 1 : 8 / IT;
  const Rsrc rs = shared_at(part);
  const int last = n - 1;
  v4f x[IT][JB];
#pragma unroll
  for (int it = 0; it < IT; it++) {
    const int i = tid + it * AT, row = min(i / PER, ROWS - 1), c = i % PER * 4;
#pragma unroll
    for (int k = 0; k < JB; k++) x[it][k] = shared4(rs, min(k, last) * step * PB + row * D + c);
  }
  for (int r = tid / 16; r < ROWS; r += AT / 16) {
    const int k0 = tid % 16;
    const v2f q0 = shared2(rs, min(k0, last) * step * PB + ROWS * D + 2 * r);
    float R = k0 < n && q0[1] != 0.0f ? q0[0] : -FLT_MAX, l = 0.0f;
    for (int k = k0 + 16; k < n; k += 16) {
      const v2f q = shared2(rs, k * step * PB + ROWS * D + 2 * r);
      if (q[1] != 0.0f) R = fmaxf(R, q[0]);
    }
    R = fmaxf(R, ror_f<DPP_ROR8>(R));
    R = fmaxf(R, ror_f<DPP_ROR4>(R));
    R = fmaxf(R, ror_f<0x122>(R));
    R = fmaxf(R, ror_f<0x121>(R));
    for (int k = k0; k < n; k += 16) {
      const v2f q = k < 16 ? q0 : shared2(rs, k * step * PB + ROWS * D + 2 * r);
      const float f = q[1] != 0.0f ? exp2_f(q[0] - R) : 0.0f;
      w[k * ROWS + r] = f;
      l = fmaf(q[1], f, l);
    }
    l += ror_f<DPP_ROR8>(l);
    l += ror_f<DPP_ROR4>(l);
    l += ror_f<0x122>(l);
    l += ror_f<0x121>(l);
    if (k0 == 0) rl[r] = make_float2(R, l);
  }
  __syncthreads();
#pragma unroll
  for (int it = 0; it < IT; it++) {
    const int i = tid + it * AT, row = min(i / PER, ROWS - 1), c = i % PER * 4;
    v4f s = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < JB; k++)
      if (k < n) s += x[it][k] * w[k * ROWS + row];
#pragma unroll 8
    for (int k = JB; k < n; k++) s += shared4(rs, k * step * PB + row * D + c) * w[k * ROWS + row];
    if (i < ROWS * PER) fin(row, c, s, rl[row].x, rl[row].y);
  }
}

// Packed rows (PK = 2 or 4): a tile of 8 or 4 rows would leave half or three
// quarters of a product's columns, and of every lane's work on scores, empty.
// Instead PK products of 16 keys each accumulate into one result, with Q's
// codes in columns 16 / PK s .. of product s and zeros in the others, so
// column c holds row c % ROWS against key group c / ROWS.  W is formed so
// packed too; for the value products the groups' halves move to the row's
// first column, and what they give in the other columns is not used.
template <int NB, bool SYM, int NT, int PK>
__global__ __launch_bounds__(AT, (NB * NT > 8 ? 2 : NT > 1 || NB > 4 ? 3 : 4)) void attn_kernel(AttnArgs a) {
  typedef Shape<NB, SYM, NT, PK> Sh;
  typedef typename ScaleT<SYM>::type sc_t;
  constexpr int D = Sh::D, ROWS = Sh::ROWS, PS = Sh::PS, NP = Sh::NP, BW = Sh::BW, CH = Sh::CH;
  constexpr int64_t TILE = kv_tile_bytes(D, SYM);
  constexpr int SB = kv_scale_bytes(SYM), SW = NB * SB / 4;   // words of scales a lane stages
  __shared__ Lds<NB, SYM, NT, PK> lds;
  for (int id = blockIdx.x; id < a.ids; id += gridDim.x) {
    // (taken anew each time round: what depends on it alone would otherwise
    // move out of this loop, that few go round twice, and hold registers)
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
    const int g = lane >> 4, col = lane & 15, grp = PK > 1 ? col / ROWS : 0;
    const int blk = NB < AW ? wave % NB : wave * BW, sub = NB < AW ? wave / NB : 0;
    Found f;
    if (!plan_find<ROWS>(a, id, f)) return;
    const Seq sq = seq_of<ROWS>(a, f.s);
    const int it = f.runs == 1 ? f.local : f.local / f.runs, run = f.local - it * f.runs;
    const int tl = it / a.p.NKV, h = it - tl * a.p.NKV, tile = sq.tiles - 1 - tl;  // longest first
    const int f0 = tile * ROWS, fn = min(ROWS, sq.qlen * a.G - f0);  // rows of the tile
    const RowMap rm(a, f0);
    const int pos0 = sq.pos + rm.token(0), pos1 = sq.pos + rm.token(fn - 1);
    // the tile's pages within this run
    const int key0 = a.window > 0 && pos0 >= a.window ? pos0 - a.window + 1 : 0;
    const int behind = a.window > 0 && pos1 >= a.window ? pos1 - a.window : -1;   // a row's window
    const int per = f.runs == 1 ? sq.pages : (sq.pages + f.runs - 1) / f.runs;
    const int plo = max(key0 / KV_PAGE, sq.lo + run * per);
    const int phi = min(sq.lo + min(sq.pages, (run + 1) * per), pos1 < 0 ? 0 : pos1 / KV_PAGE + 1);

    // page ids of a step: lane j < AW has page at0 + j's (-1: none)
    const int32_t *table = a.p.pages + (int64_t)f.s * a.p.max_pages;
    const auto raw_ids = [&](int at0) { return lane < AW && at0 + lane < phi ? table[at0 + lane] : -1; };
    const auto checked = [&](int v) { return v < 0 || v >= a.p.n_pages ? -1 : v; };
    int ids = raw_ids(plo);

    // Q rows (rows past the last repeat it); the first step's loads go out behind them
    constexpr int QI = (ROWS * NB * 8 + AT - 1) / AT;
    v4f x[QI];
#pragma unroll
    for (int k = 0; k < QI; k++) {
      const int i = tid + k * AT, row = min((i >> 3) / NB, fn - 1), b = (i >> 3) % NB;
      const int t = rm.token(row);
      x[k] = *reinterpret_cast<const v4f *>(a.q + (sq.r0 + t) * a.qs +
                                            (int64_t)(h * a.G + rm.head(row, t)) * D + b * 32 + 4 * (i & 7));
    }
    ids = checked(ids);

    // One buffer for both: K block b of the wave's page, and once that is used,
    // the wave's columns of a V page (NP BW = NB pieces), and so on: half a
    // step lies between a load and its use, in half the registers.
    v4u buf[NB];
    uint32_t ksr[SW], vsr[SW];
    // where lane l's NB scales of the wave's value blocks are: piece l / (64 / NB)
    const int spc = lane / (64 / NB), sof = lane % (64 / NB) * NB;
    const int spg = sub * NP + spc / BW, sbk = blk + spc % BW;
    const int64_t head = (int64_t)h * TILE, stride = (int64_t)a.p.NKV * TILE;
    const auto k_tile = [&](int ids) {
      return a.p.k + (int64_t)max(__builtin_amdgcn_readlane(ids, wave), 0) * stride + head;
    };
    const auto load_k = [&](const uint8_t *t, int b) {
      buf[b] = reinterpret_cast<const v4u *>(t + b * 1024)[lane];
    };
    const auto load_ks = [&](const uint8_t *t) {
      load_words(t + NB * 1024 + lane * (SW * 4), ksr);
    };
    const auto load_vs = [&](int ids) {
      const int64_t page = max(__shfl(ids, spg), 0);
      load_words(a.p.v + page * stride + head + NB * 1024 + (sbk * 64 + sof) * SB, vsr);
    };
    const auto load_v = [&](int ids, int c) {
      const int64_t page = max(__builtin_amdgcn_readlane(ids, sub * NP + c / BW), 0);
      buf[c] = reinterpret_cast<const v4u *>(a.p.v + page * stride + head + (blk + c % BW) * 1024)[lane];
    };
    {
      const uint8_t *t = k_tile(ids);
      load_ks(t);
#pragma unroll
      for (int b = 0; b < NB; b++) load_k(t, b);
    }
    load_vs(ids);
#pragma unroll
    for (int k = 0; k < QI; k++) {
      const int i = tid + k * AT, j = i & 7, row = (i >> 3) / NB, b = (i >> 3) % NB;
      const float v[4] = {x[k][0], x[k][1], x[k][2], x[k][3]};
      float d;
      const uint32_t codes = kv_q8_block8<SYM>(v, d);
      const int nt = row >> 4, r = row & 15;
      if (row < ROWS) {
#pragma unroll
        for (int s = 0; s < PK; s++)
#pragma unroll
          for (int z = 0; z < PK; z++)
            lds.q[(((nt * NB + b) * PK + s) * 64 + 16 * (j & 3) + r + ROWS * z) * 2 + (j >> 2)] =
                s == z ? codes : 0u;
        if (j < PK) lds.qd[(nt * NB + b) * 16 + r + (PK > 1 ? ROWS * j : 0)] = d * a.sign;
      }
    }
    __syncthreads();

    // this lane's rows see lo_key < key <= hi_key; both less the lane's first key of a page
    const int kbase = 4 * g + 16 * grp;
    int hi_key[NT], lo_key[NT];
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
      const int pos = sq.pos + rm.token(min(16 * nt + (PK > 1 ? col % ROWS : col), fn - 1));
      hi_key[nt] = pos - kbase;
      lo_key[nt] = (a.window > 0 && a.window <= pos ? pos - a.window : -1) - kbase;
    }
    // first token of the lane's NB value scales within its page, as kv_scale_at has them
    const int vtok = sof / 16 * 4 + sof / 4 % 4 * 16 + sof % 4;

    float m[NT], mk[NT], l[NT];
    v4f acc[NT][BW][2];
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
      m[nt] = -FLT_MAX;
      mk[nt] = -FLT_MAX;
      l[nt] = 0.0f;
#pragma unroll
      for (int b = 0; b < BW; b++) acc[nt][b][0] = acc[nt][b][1] = v4f{0.f, 0.f, 0.f, 0.f};
    }
    // value scales are below 2^vexp, their bits above `limit` (0: none so far),
    // and enter the product times 2^(15 - vexp); once wide, scales and sums
    // stand as they are
    int vexp = -126;
    uint32_t limit = 0;
    bool far = false;                  // some row's maximum is FAR from 0
    sc_t *ks = lds.ks[wave];
    float *vs = lds.vs[wave];
    float minus = -1.0f;               // opaque, so that the halves' difference is one mixed FMA
    asm("" : "+v"(minus));
    // opaque too: as literals they would keep the mask and the bias apart
    uint32_t low4 = 0x000F000Fu, high4 = 0x00F000F0u, bias = 0x64006400u;
    asm("" : "+v"(low4), "+v"(high4), "+v"(bias));
    const v4i c0 = {0x4B400000, 0x4B400000, 0x4B400000, 0x4B400000};
    // the value codes of 32 keys, of words 2 hh and + 1
    const auto value_codes = [&](const v4u &word4, int hh, h8 (&c)[2]) {
#pragma unroll
      for (int i = 0; i < 2; i++) {
        // a nibble n in an fp16 number's low bits: 1024 + n or 1024 + 16 n
        const uint32_t y = word4[2 * hh + i], z = y >> 8;
        const h2 off = {(_Float16)-1032.0f, (_Float16)-1032.0f};
        const h2 six = {(_Float16)0.0625f, (_Float16)0.0625f};
        const h2 off2 = {(_Float16)-72.0f, (_Float16)-72.0f};
        const h2 a0 = __builtin_bit_cast(h2, (y & low4) | bias) + off;
        const h2 a1 = __builtin_bit_cast(h2, (z & low4) | bias) + off;
        const h2 b0 = __builtin_elementwise_fma(__builtin_bit_cast(h2, (y & high4) | bias), six, off2);
        const h2 b1 = __builtin_elementwise_fma(__builtin_bit_cast(h2, (z & high4) | bias), six, off2);
        c[0][4 * i] = a0[0]; c[0][4 * i + 1] = a0[1]; c[0][4 * i + 2] = a1[0]; c[0][4 * i + 3] = a1[1];
        c[1][4 * i] = b0[0]; c[1][4 * i + 1] = b0[1]; c[1][4 * i + 2] = b1[0]; c[1][4 * i + 3] = b1[1];
      }
    };
    for (int at0 = plo; at0 < phi; at0 += AW) {
      const bool more = at0 + AW < phi;
      const int raw_next = raw_ids(at0 + AW);
      const int key = (at0 + wave) * KV_PAGE;
      // ---- scores of page at0 + wave
      const bool here = __builtin_amdgcn_readlane(ids, wave) >= 0;
#pragma unroll
      for (int w = 0; w < SW; w++) reinterpret_cast<word *>(ks)[lane * SW + w] = ksr[w];
      float S[NT][4 * CH];
#pragma unroll
      for (int nt = 0; nt < NT; nt++)
#pragma unroll
        for (int i = 0; i < 4 * CH; i++) S[nt][i] = 0.0f;
#pragma unroll
      for (int b = 0; b < NB; b++) {
        long qb[NT][PK];
        float dq[NT], cq[NT];
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
#pragma unroll
          for (int s = 0; s < PK; s++)
            qb[nt][s] = reinterpret_cast<const long *>(lds.q)[((nt * NB + b) * PK + s) * 64 + lane];
          dq[nt] = lds.qd[(nt * NB + b) * 16 + col];
          cq[nt] = -12582912.0f * dq[nt];
        }
        sc_t dk[4 * CH];
#pragma unroll
        for (int i = 0; i < 4 * CH; i++) dk[i] = ks[b * 64 + g * 16 + 4 * grp + 4 * PK * (i >> 2) + (i & 3)];
#pragma unroll
        for (int c = 0; c < CH; c++) {
          v4i r[NT];
#pragma unroll
          for (int s = 0; s < PK; s++) {
            const uint32_t y = buf[b][c * PK + s];
            const long kb = (long)((uint64_t)(y & 0xF0F0F0F0u) << 32 | (y << 4 & 0xF0F0F0F0u));
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
              r[nt] = __builtin_amdgcn_mfma_i32_16x16x32_i8(kb, qb[nt][s], s ? r[nt] : c0, 0, 0, 0);
          }
#pragma unroll
          for (int nt = 0; nt < NT; nt++) {
            const v4f rf = __builtin_bit_cast(v4f, r[nt]);
#pragma unroll
            for (int e = 0; e < 4; e++) {
              // SYM: an fp32 scale times 1.5 2^23 would round, so s comes first
              const float t = SYM ? (rf[e] - 12582912.0f) * dq[nt] : fmaf(rf[e], dq[nt], cq[nt]);
              S[nt][4 * c + e] = fmaf(t, (float)dk[4 * c + e], S[nt][4 * c + e]);
            }
          }
          // pinned in order: moved together, the products and scales of all
          // blocks would be live at once
          if (c == CH - 1 || c == 1) {
#pragma unroll
            for (int nt = 0; nt < NT; nt++)
#pragma unroll
              for (int i = 0; i < 4 * CH; i++) asm volatile("" : "+v"(S[nt][i]));
          }
        }
        load_v(ids, b);
      }
      // keys that not every row sees; an absent page's are seen by none
      if (!here || key + KV_PAGE - 1 > pos0 || key <= behind) {
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
          const int last = here ? hi_key[nt] - key : -100, before = lo_key[nt] - key;
#pragma unroll
          for (int i = 0; i < 4 * CH; i++)
            if (key_off<PK>(i) > last || key_off<PK>(i) <= before) S[nt][i] = -INFINITY;
        }
      }
#pragma unroll
      for (int nt = 0; nt < NT; nt++) {
        float mx = -FLT_MAX;
#pragma unroll
        for (int i = 0; i < 4 * CH; i++) mx = fmaxf(mx, S[nt][i]);
        mx = max_row<PK>(mx);
        if (lane < 16) lds.mx[16 * nt + lane][wave] = mx;
      }

      // ---- the wave's value scales of the step; keys that no row sees count for nothing
      {
        const int vkey = (at0 + spg) * KV_PAGE + vtok;
        const bool vhere = __shfl(ids, spg) >= 0;
        // (magnitudes by their bits without the sign; a 0 less 1 is above all)
        float dv[NB];
        uint32_t most = 0, least = 0xFFFFFFFFu;
#pragma unroll
        for (int i = 0; i < NB; i++) {
          dv[i] = scale_of<SYM>(vsr, i);
          const int kk = vkey + (i >> 2) * 16 + (i & 3);
          if (!vhere || kk > pos1 || kk < key0) dv[i] = 0.0f;
          const uint32_t y = __builtin_bit_cast(uint32_t, dv[i]) << 1;
          most = max(most, y);
          least = min(least, y - 1);
        }
        if (__ballot(most >= bits_of_2(vexp) || least < limit)) {
          float vmax = 0.0f;
#pragma unroll
          for (int i = 0; i < NB; i++) vmax = fmaxf(vmax, fabsf(dv[i]) < INFINITY ? fabsf(dv[i]) : 0.0f);
#pragma unroll
          for (int o = 32; o > 0; o >>= 1) vmax = fmaxf(vmax, __shfl_xor(vmax, o));
          int to = max(vexp, __builtin_amdgcn_readfirstlane(ilogbf(vmax) + 1));
          if (limit == 0 && vexp != WIDE) limit = bits_of_2(max(to - UNDER, -126)) - 1;
          if (to == WIDE || to > (int)(limit >> 24) - 126 + UNDER + OVER || __ballot(least < limit)) {
            to = WIDE;
            limit = 0;
          }
          const int by = (vexp == WIDE ? 15 : vexp) - (to == WIDE ? 15 : to);
#pragma unroll
          for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int b = 0; b < BW; b++)
#pragma unroll
              for (int s = 0; s < 2; s++) acc[nt][b][s] = ldexp4(acc[nt][b][s], by);
          vexp = to;
        }
        const int up = vexp == WIDE ? 0 : 15 - vexp;
#pragma unroll
        for (int i = 0; i < NB; i++) vs[lane * NB + i] = ldexpf(dv[i], up);
      }
      const int next = checked(raw_next);
      const uint8_t *const kt = k_tile(next);
      if (more) {
        load_vs(next);
        load_ks(kt);
      }
      __syncthreads();

      // ---- running maximum, the same in every wave
      bool grow = false;
      float mn[NT];
#pragma unroll
      for (int nt = 0; nt < NT; nt++) {
        const v4f w = *reinterpret_cast<const v4f *>(lds.mx[16 * nt + col]);
        mn[nt] = fmaxf(m[nt], fmaxf(fmaxf(w[0], w[1]), fmaxf(w[2], w[3])));
        grow |= mn[nt] > m[nt];
      }
      if (__ballot(grow)) {
        bool f = false;
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
          // (a row without keys so far has no product to take: it could overflow)
          const float mkn = mn[nt] == -FLT_MAX ? -FLT_MAX : mn[nt] * a.k;
          const float al = m[nt] == -FLT_MAX ? 0.0f : exp2_f(mk[nt] - mkn);
          m[nt] = mn[nt];
          mk[nt] = mkn;
          f |= fabsf(mkn) >= FAR && mkn != -FLT_MAX;
          l[nt] *= al;
#pragma unroll
          for (int b = 0; b < BW; b++) {
            acc[nt][b][0] *= al;
            acc[nt][b][1] *= al;
          }
        }
        far = __ballot(f) != 0;
      }
      // Below FAR the product's rounding in mk makes the largest probability
      // 2^(1/8) at most, in sums and halves alike; from there on scores are taken
      // less the maximum first, so that it is 1.
      float ref[NT];
#pragma unroll
      for (int nt = 0; nt < NT; nt++) ref[nt] = mk[nt];
      if (far) [[unlikely]] {
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
          ref[nt] = 0.0f;
#pragma unroll
          for (int i = 0; i < 4 * CH; i++) S[nt][i] -= m[nt];
        }
      }
      // ---- probabilities (a masked score's is exp2(-infinity) = 0)
#pragma unroll
      for (int nt = 0; nt < NT; nt++) {
        v4f s = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < CH; c++) {
          v4f p;
#pragma unroll
          for (int e = 0; e < 4; e++) p[e] = exp2_f(fmaf(S[nt][4 * c + e], a.k, -ref[nt]));
          lds.p[wave][CH * nt + c][lane] = p;
          s += p;
        }
        l[nt] += (s[0] + s[1]) + (s[2] + s[3]);
      }
      __syncthreads();

      // ---- values of the wave's columns
      if (vexp == WIDE) [[unlikely]] {
        // each row's products by a power of two of their own, into sums as they
        // are; codes read again, so that this stays a loop (and places found
        // again, so that none holds a register outside).  1.3 to 1.6 times the
        // time (48 rows over 6000 keys 77 us, 2 x 2048 over 8192 1320)
        int ln = lane;
        asm volatile("" : "+v"(ln));
        const auto at = [&] { return (ln >> 4) * 16 + (PK > 1 ? (ln & 15) / ROWS * 4 : 0); };
#pragma unroll 1
        for (int j = 0; j < NP && at0 + sub * NP + j < phi; j++) {
          const int pgj = sub * NP + j;
          const int64_t page = max(__builtin_amdgcn_readlane(ids, pgj), 0);
#pragma unroll
          for (int bb = 0; bb < BW; bb++) {
            const v4u y4 = reinterpret_cast<const v4u *>(a.p.v + page * stride + head + (blk + bb) * 1024)[ln];
            const float *const d = vs + (j * BW + bb) * 64;
#pragma unroll
            for (int hh = 0; hh < 2; hh++) {
              h8 c[2];
              value_codes(y4, hh, c);
#pragma unroll
              for (int nt = 0; nt < NT; nt++) {
                constexpr int N = PK == 1 ? 2 : CH;
                v4f w[N];
                float most = 0.0f;
#pragma unroll
                for (int i = 0; i < N; i++) {
                  w[i] = products(lds.p[pgj][4 * nt + (PK == 1 ? 2 * hh : 0) + i][ln],
                                  d + at() + (PK == 1 ? 8 * hh : 0) + 4 * PK * i);
                  most = max_finite(most, w[i]);
                }
                const int up = 15 - __builtin_amdgcn_frexp_expf(max_row<PK>(most));
                h4 x[N], y[N];
#pragma unroll
                for (int i = 0; i < N; i++) halves(ldexp4(w[i], up), minus, x[i], y[i]);
                h8 hi, lo;
#pragma unroll
                for (int i = 0; i < 2; i++) {
                  if constexpr (PK == 1) {
                    put(hi, i, x[i]);
                    put(lo, i, y[i]);
                  } else {
                    put(hi, i, from_col<PK>(x[(2 * hh + i) / PK], (2 * hh + i) % PK));
                    put(lo, i, from_col<PK>(y[(2 * hh + i) / PK], (2 * hh + i) % PK));
                  }
                }
#pragma unroll
                for (int s = 0; s < 2; s++) {
                  v4f t = __builtin_amdgcn_mfma_f32_16x16x32_f16(c[s], hi, v4f{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
                  t = __builtin_amdgcn_mfma_f32_16x16x32_f16(c[s], lo, t, 0, 0, 0);
                  acc[nt][bb][s] += ldexp4(t, -up);
                }
                asm volatile("" : "+v"(acc[nt][bb][0]), "+v"(acc[nt][bb][1]), "+v"(ln));
              }
            }
          }
        }
#pragma unroll
        for (int b = 0; b < NB; b++) {
          buf[b] = v4u{0, 0, 0, 0};
          if (more) load_k(kt, b);
        }
      } else {
#pragma unroll
        for (int j = 0; j < NP; j++) {
          const int pgj = sub * NP + j;
          if (at0 + pgj < phi) {
#pragma unroll
            for (int bb = 0; bb < BW; bb++) {
              const int pc = j * BW + bb;
              // W of the lane's keys, as two halves
              h4 whi[NT][CH], wlo[NT][CH];
              if (PK > 1) make_w(lds.p[pgj][0][lane], vs + pc * 64 + g * 16 + 4 * grp, minus, whi[0][0], wlo[0][0]);
              if (PK == 2) make_w(lds.p[pgj][CH - 1][lane], vs + pc * 64 + g * 16 + 4 * grp + 8, minus, whi[0][CH - 1], wlo[0][CH - 1]);
#pragma unroll
              for (int hh = 0; hh < 2; hh++) {         // 32 keys at a time
                h8 c[2];                               // elements l % 16 and + 16
                value_codes(buf[pc], hh, c);
#pragma unroll
                for (int nt = 0; nt < NT; nt++) {
                  h8 hi, lo;
                  if constexpr (PK == 1) {
#pragma unroll
                    for (int i = 0; i < 2; i++) {
                      h4 x, y;
                      make_w(lds.p[pgj][4 * nt + 2 * hh + i][lane], vs + pc * 64 + g * 16 + 8 * hh + 4 * i, minus, x, y);
                      put(hi, i, x);
                      put(lo, i, y);
                    }
                  } else {
#pragma unroll
                    for (int i = 0; i < 2; i++) {        // key group 2 hh + i
                      const int ch = (2 * hh + i) / PK, z = (2 * hh + i) % PK;
                      put(hi, i, from_col<PK>(whi[0][ch], z));
                      put(lo, i, from_col<PK>(wlo[0][ch], z));
                    }
                  }
#pragma unroll
                  for (int s = 0; s < 2; s++) {
                    acc[nt][bb][s] = __builtin_amdgcn_mfma_f32_16x16x32_f16(c[s], hi, acc[nt][bb][s], 0, 0, 0);
                    acc[nt][bb][s] = __builtin_amdgcn_mfma_f32_16x16x32_f16(c[s], lo, acc[nt][bb][s], 0, 0, 0);
                  }
                }
#pragma unroll
                for (int nt = 0; nt < NT; nt++) asm volatile("" : "+v"(acc[nt][bb][0]), "+v"(acc[nt][bb][1]));
              }
            }
          }
          if (more) {
#pragma unroll
            for (int bb = 0; bb < BW; bb++) load_k(kt, j * BW + bb);
          }
        }
      }
      ids = next;
    }

    // the waves' sums; where PS waves share columns, their products too
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
      l[nt] = sum_cols<PK>(sum4(l[nt]));
      if (lane < 16) lds.l[wave][16 * nt + lane] = l[nt];
#pragma unroll
      for (int b = 0; b < BW; b++)
#pragma unroll
        for (int s = 0; s < 2; s++)
#pragma unroll
          for (int y = 0; y < 4; y++)
            acc[nt][b][s][y] = ldexpf(acc[nt][b][s][y], vexp == WIDE ? 0 : vexp - 15);
    }
    if constexpr (PS > 1) {
      __syncthreads();                 // the last step's probabilities have been read
      if (sub > 0) {
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
          for (int s = 0; s < 2; s++) lds.sums[wave][2 * nt + s][lane] = acc[nt][0][s];
      }
    }
    __syncthreads();
    const bool whole = f.runs == 1;
    const int first = f.slot0 + it * f.runs;              // slot of the item's run 0
    const Rsrc pr = shared_at(a.part + (int64_t)(whole ? 0 : first + run) * (ROWS * (D + 2)));
    // (every item's do, by slots_bound; no write hangs on it)
    const bool fits = whole || first + f.runs <= a.slots;
    if (sub == 0 && col < ROWS && fits) {
#pragma unroll
      for (int nt = 0; nt < NT; nt++) {
        const int row = 16 * nt + col;
        const float lt = (lds.l[0][row] + lds.l[1][row]) + (lds.l[2][row] + lds.l[3][row]);
        if constexpr (PS > 1) {
#pragma unroll
          for (int q = 1; q < PS; q++)
#pragma unroll
            for (int s = 0; s < 2; s++) acc[nt][0][s] += lds.sums[wave + q * NB][2 * nt + s][lane];
        }
        const int t = rm.token(min(row, fn - 1));
        const int64_t o = (sq.r0 + t) * a.NH + h * a.G + rm.head(min(row, fn - 1), t);
        const float inv = lt != 0.0f ? 1.0f / lt : 0.0f;
#pragma unroll
        for (int b = 0; b < BW; b++) {
          const int at = (blk + b) * 32 + 4 * g;
          if (!whole) {
            share(pr, row * D + at, acc[nt][b][0]);
            share(pr, row * D + at + 16, acc[nt][b][1]);
          } else if (row < fn) {
            *reinterpret_cast<v4f *>(a.out + o * D + at) = acc[nt][b][0] * inv;
            *reinterpret_cast<v4f *>(a.out + o * D + at + 16) = acc[nt][b][1] * inv;
          }
        }
        if (wave == 0 && g == 0) {
          if (!whole) {
            share(pr, ROWS * D + 2 * row, v2f{mk[nt], lt});
          } else if (a.lse && row < fn) {
            a.lse[o] = lt != 0.0f ? (mk[nt] + log2f(lt)) * 0.693147180559945f : -INFINITY;
          }
        }
      }
    }
    // The last of a group of runs to get here joins the group, the last group
    // the item: in the order of the runs, whoever was last.
    if (!whole && fits && a.fused) {
      const auto store = [&](int row, int c, v4f s, float R, float l) {
        if (row >= fn) return;
        const int t = rm.token(row);
        const int64_t o = (sq.r0 + t) * a.NH + h * a.G + rm.head(row, t);
        *reinterpret_cast<v4f *>(a.out + o * D + c) = l != 0.0f ? s * (1.0f / l) : s * 0.0f;
        if (c == 0 && a.lse) a.lse[o] = l != 0.0f ? (R + log2f(l)) * 0.693147180559945f : -INFINITY;
      };
      constexpr int64_t PB = ROWS * (D + 2);
      float *const w = reinterpret_cast<float *>(lds.p);
      const int groups = (f.runs + GROUP - 1) / GROUP, gr = run / GROUP;
      const int n = min(GROUP, f.runs - gr * GROUP);
      float *const gp = a.part + (first + gr * GROUP) * PB;
      if (last_of(a.count + first + gr * GROUP, n, &lds.flag)) {
        if (groups == 1) {
          join<D, ROWS>(tid, gp, 1, n, w, lds.rl, store);
        } else {
          // a thread writes only the columns that it alone has read
          join<D, ROWS>(tid, gp, 1, n, w, lds.rl, [&](int row, int c, v4f s, float R, float l) {
            share(shared_at(gp), row * D + c, s);
            if (c == 0) share(shared_at(gp), ROWS * D + 2 * row, v2f{R, l});
          });
          if (last_of(a.count + SLOTS_MAX + first, groups, &lds.flag)) {
            join<D, ROWS>(tid, a.part + first * PB, GROUP, groups, w, lds.rl, store);
          }
        }
      }
    }
    __syncthreads();
  }
}

// The same as a launch of its own, for few items of many runs: a workgroup a
// row of item blockIdx.x (counted over the items with several runs), D / 4
// lanes by groups that take the runs in turn.
template <int NB, int ROWS> __global__ __launch_bounds__(JT) void join_kernel(AttnArgs a) {
  constexpr int D = 32 * NB, L = D / 4, NG = JT / L;
  constexpr int64_t PB = ROWS * (D + 2);
  __shared__ v4f so[NG][L];
  __shared__ float sw[SLOTS_MAX], sl;
  Found f;
  if (!plan_find<ROWS, true>(a, blockIdx.x, f)) return;
  const Seq sq = seq_of<ROWS>(a, f.s);
  const int tl = f.local / a.p.NKV, h = f.local - tl * a.p.NKV, f0 = (sq.tiles - 1 - tl) * ROWS;
  const int row = blockIdx.y;
  if (row >= min(ROWS, sq.qlen * a.G - f0)) return;
  const int slot = f.slot0 + f.local * f.runs, n = f.runs;
  if (slot + n > a.slots) return;
  const float *part = a.part + slot * PB;
  float R = -FLT_MAX;
  if (threadIdx.x < 64) {
    for (int i = threadIdx.x; i < n; i += 64) {
      const v2f q = *reinterpret_cast<const v2f *>(part + i * PB + ROWS * D + 2 * row);
      if (q[1] != 0.0f) R = fmaxf(R, q[0]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) R = fmaxf(R, __shfl_xor(R, o));
    float l = 0.0f;
    for (int i = threadIdx.x; i < n; i += 64) {
      const v2f q = *reinterpret_cast<const v2f *>(part + i * PB + ROWS * D + 2 * row);
      const float w = q[1] != 0.0f ? exp2_f(q[0] - R) : 0.0f;
      sw[i] = w;
      l = fmaf(q[1], w, l);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) l += __shfl_xor(l, o);
    if (threadIdx.x == 0) sl = l;
  }
  __syncthreads();
  const int grp = threadIdx.x / L, c4 = threadIdx.x % L;
  v4f s = v4f{0.f, 0.f, 0.f, 0.f};
  const float *src = part + row * D + 4 * c4;
#pragma unroll 8
  for (int i = grp; i < n; i += NG) s += *reinterpret_cast<const v4f *>(src + i * PB) * sw[i];
  so[grp][c4] = s;
  __syncthreads();
  if (grp != 0) return;
  s = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int i = 0; i < NG; i++) s += so[i][c4];
  const RowMap rm(a, f0);
  const int t = rm.token(row);
  const int64_t o = (sq.r0 + t) * a.NH + h * a.G + rm.head(row, t);
  const float l = sl;
  *reinterpret_cast<v4f *>(a.out + o * D + 4 * c4) = l != 0.0f ? s * (1.0f / l) : s * 0.0f;
  if (c4 == 0 && a.lse) a.lse[o] = l != 0.0f ? (R + log2f(l)) * 0.693147180559945f : -INFINITY;
}

// The rows of a plan without any page (the kernels above load page 0 in an
// absent one's place): a workgroup a row.
__global__ __launch_bounds__(AT) void no_keys_kernel(AttnArgs a, int D) {
  for (int64_t r = blockIdx.x; r < a.T; r += gridDim.x) {
    int token;
    if (kv_find(a.p, a.T, r, token) < 0) continue;
    for (int i = threadIdx.x; i < a.NH * D / 4; i += AT)
      reinterpret_cast<v4f *>(a.out + r * a.NH * D)[i] = v4f{0.f, 0.f, 0.f, 0.f};
    if (a.lse)
      for (int i = threadIdx.x; i < a.NH; i += AT) a.lse[r * a.NH + i] = -INFINITY;
  }
}

// Rows of a tile: 4 or 8 packed where a sequence has no more of a KV head on
// average (a decode step of few heads a group), the 16 of one product, or 32,
// which share the page's loads and decoded codes.  More rows a tile are less
// work in all but fewer workgroups, and longer ones: 32 only where they number
// 1024 and more (2048 tokens of 32 heads of 128: 108 us against 121 with 16;
// 512 tokens of 16 heads of 256, 256 tiles: 25.6 against 18.4), 8 where
// tiles of 16 would number less than 64, at 256 columns 256 (128 tokens of 16
// heads of 256: 10.1 us against 11.2; one token of 16 heads of 128 over 8000
// keys: 15 against 21; past it 2 % to 10 % slower).
int tile_rows(const w4a8_kv *kv, int64_t T, int64_t NH) {
  const int64_t rows = T * (NH / kv->NKV), B = std::max<int64_t>(1, kv->B);
  if (rows <= 4 * B) return 4;
  if (rows <= 8 * B || T * NH < (kv->D == 256 ? 4096 : 1024)) return 8;
  return T * NH >= 32 * 1024 && rows > 16 * B ? 32 : 16;
}

// Bounds on the call's items, and on the partial results it can need: a
// sequence's rows are a multiple of G, so its last tile holds gcd(G, rows of a
// tile) at least; a sequence is split only into runs of more than half of C >=
// total / TARGET pages, so the runs of split items number at most 2 TARGET.
int64_t items_bound(const w4a8_kv *kv, int64_t T, int64_t NH) {
  const int rt = tile_rows(kv, T, NH);
  const int64_t G = NH / kv->NKV;
  return (T * G + std::min(kv->B, T) * (rt - std::gcd(G, (int64_t)rt))) / rt * kv->NKV;
}
int64_t slots_bound(const w4a8_kv *kv, int64_t T, int64_t NH) {
  if (kv->max_pages <= AW || kv->B == 0) return 0;
  const int64_t runs = (kv->max_pages + AW - 1) / AW;
  return std::min<int64_t>(SLOTS_MAX, items_bound(kv, T, NH) * runs);
}

// Whether the last workgroups join the runs.  They read past the L2 caches,
// some 30 KB a round trip: right for a few runs an item, which they join while
// others still work, in place of a launch (one row of 32 heads of 128 over 2000
// keys, 8 runs: 11 us against 13; 16 runs: 13.5 against 13).  A launch puts
// 1024 threads on a row: better from a group of runs, or 2048 columns of a
// row's, on (16 heads of 256 over 4000 keys, 16 runs: 14.9 us against 20.5; over
// 131072, 256 runs: 30 against 37).  (An average: a long sequence among short
// ones may have more runs, and is joined in two levels.)
bool joins_fused(const w4a8_kv *kv, int64_t T, int64_t NH) {
  const int64_t runs = std::min<int64_t>((kv->max_pages + AW - 1) / AW,
                                         TARGET / std::max<int64_t>(1, items_bound(kv, T, NH)));
  return runs <= GROUP && runs * kv->D < 2048;
}

int attn_sizes(const w4a8_kv *kv, int64_t T, int64_t NH) {
  if (int rc = kv_check_sizes(kv); rc != W4A8_OK) return rc;
  if (NH < 1 || NH % kv->NKV != 0 || T < 0) return W4A8_ESHAPE;
  if (NH / kv->NKV >= (1 << 16) || T >= ((int64_t)1 << 31) || T * NH >= ((int64_t)1 << 31))
    return W4A8_ERANGE;
  return W4A8_OK;
}

template <int NB, bool SYM, int NT, int PK>
int launch(const AttnArgs &a, int64_t items, hipStream_t s) {
  const int64_t grid = std::min<int64_t>(a.ids, 1 << 20);
  attn_kernel<NB, SYM, NT, PK><<<dim3((unsigned)grid), dim3(AT), 0, s>>>(a);
  if (int rc = check_launch(); rc != W4A8_OK || a.slots == 0 || a.fused) return rc;
  constexpr int ROWS = 16 * NT / PK;
  const int64_t joins = std::min<int64_t>(items, TARGET);
  join_kernel<NB, ROWS><<<dim3((unsigned)joins, (unsigned)std::min<int64_t>(ROWS, a.T * a.G)),
                          dim3(JT), 0, s>>>(a);
  return check_launch();
}

template <int NB, bool SYM>
int launch_rows(const AttnArgs &a, int rows, int64_t items, hipStream_t s) {
  switch (rows) {
    case 4: return launch<NB, SYM, 1, 4>(a, items, s);
    case 8: return launch<NB, SYM, 1, 2>(a, items, s);
    case 16: return launch<NB, SYM, 1, 1>(a, items, s);
    default: return launch<NB, SYM, 2, 1>(a, items, s);
  }
}

}  // namespace
}  // namespace w4a8

using namespace w4a8;

extern "C" size_t attn_q4_workspace_size(const w4a8_kv *kv, int64_t T, int64_t NH) {
  if (attn_sizes(kv, T, NH) != W4A8_OK) return 0;
  const int64_t n = slots_bound(kv, T, NH);
  return n == 0 ? 16 : (size_t)(COUNTERS + n * tile_rows(kv, T, NH) * (kv->D + 2) * 4);
}

extern "C" int attn_q4_forward(const w4a8_kv *kv, const float *q, int64_t q_stride, float *out,
                               float *lse, int64_t T, int64_t NH, float scale, int64_t window,
                               void *workspace, size_t ws_bytes, void *stream) {
  if (int rc = kv_check(kv); rc != W4A8_OK) return rc;
  if (!q || !out || !workspace) return W4A8_ENULL;
  if (int rc = attn_sizes(kv, T, NH); rc != W4A8_OK) return rc;
  if (window < 0 || !std::isfinite(scale) || q_stride < NH * kv->D || q_stride % 4 != 0)
    return W4A8_ESHAPE;
  const int64_t lim = (int64_t)1 << 31;
  if (q_stride >= lim) return W4A8_ERANGE;
  if (!aligned16(q) || !aligned16(out) || !aligned16(workspace) ||
      (reinterpret_cast<uintptr_t>(lse) & 3u))
    return W4A8_EALIGN;
  if (out == q) return W4A8_EALIAS;
  if (ws_bytes < attn_q4_workspace_size(kv, T, NH)) return W4A8_EWORKSPACE;
  if (T == 0 || kv->B == 0) return W4A8_OK;
  if (int rc = check_device(); rc != W4A8_OK) return rc;
  const int64_t items = items_bound(kv, T, NH);
  AttnArgs a = {kv_plan(kv), q, q_stride, out, lse, T, (int)NH, (int)(NH / kv->NKV),
                // a factor of 0 goes to Q, so that a masked score's -infinity stays one
                scale != 0.0f ? std::fabs(scale) * 1.44269504f / 16.0f : 1.0f,
                scale < 0.0f ? -1.0f : scale == 0.0f ? 0.0f : 1.0f,
                window < lim ? (int)window : 0,  // wider than any sequence
                reinterpret_cast<int *>(workspace),
                reinterpret_cast<float *>(reinterpret_cast<uint8_t *>(workspace) + COUNTERS), (int)slots_bound(kv, T, NH),
                // a split item's runs beyond the first are C pages each
                items + std::min<int64_t>(slots_bound(kv, T, NH), TARGET), joins_fused(kv, T, NH),
                1.0f / (float)(NH / kv->NKV)};
  const bool sym = kv->format == W4A8_KV_Q4_SYM;
  const int rows = tile_rows(kv, T, NH);
  const hipStream_t s = as_stream(stream);
  if (kv->n_pages == 0) {
    no_keys_kernel<<<dim3((unsigned)std::min<int64_t>(T, 1 << 16)), dim3(AT), 0, s>>>(a, (int)kv->D);
    return check_launch();
  }
  if (kv->D == 64) return sym ? launch_rows<2, true>(a, rows, items, s) : launch_rows<2, false>(a, rows, items, s);
  if (kv->D == 128) return sym ? launch_rows<4, true>(a, rows, items, s) : launch_rows<4, false>(a, rows, items, s);
  return sym ? launch_rows<8, true>(a, rows, items, s) : launch_rows<8, false>(a, rows, items, s);
}
