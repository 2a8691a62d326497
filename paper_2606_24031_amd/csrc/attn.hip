// Softmax attention over the paged 4-bit cache (Sec. 2.2: 10 of the 40 blocks
// are softmax attention with grouped query heads; Sec. 3.2 runs it in one
// pass with a running maximum and sum).
//
// A work item is a tile of 16 or 32 query rows of one KV head of a sequence
// (row f of a sequence: token f / G, head f % G of the group), times a run of
// pages when the rows alone would leave compute units idle; a second launch
// then joins the runs' partial results in a fixed order.  The four waves of a
// workgroup take the item's pages in turn, each on its own: no barrier until
// they join.  A wave takes a page of 64 keys at a time, everything in
// registers but the block scales:
//   scores   S^T = K Q^T: one v_mfma_i32_16x16x32_i8 per 16 keys, 16 rows and
//            block of 32, K codes straight from the page (a 16-byte load a
//            lane and block), Q codes from LDS.  The accumulator starts at
//            0x4B400000, so the int32 result read as a float is 1.5 2^23 +
//            16 s; with the row's fp16 scale d_q one FMA gives 16 s d_q
//            rounded once, the second adds it times d_k.
//   softmax  base 2 with a running maximum m per row: rescaled only on pages
//            where some row's maximum grows.  fp32.
//   values   O^T += V^T W^T with W = p d_v per block of 32 columns: V codes
//            are small integers, exact in fp16, and W goes in as hi + lo, two
//            fp16 halves (22 bits; one fp16 or bf16 would be off by 2^-12 or
//            2^-9, more than everything else here together).  d_v is scaled
//            by a power of two, kept per wave, to put the largest value scale
//            met so far just below 2^15: halves neither overflow nor lose
//            bits unless a block's scale lies 2^17 and more below it.
// The lane layout of the score product's result (row l % 16, keys 4 (l / 16)
// + e) is the one the value product wants for W, so probabilities never leave
// the lane, and both products keep a query row in one lane column, so the
// running maximum and sum need only exchanges between lanes l, l+16, l+32,
// l+48.
// Bound: long decodes by HBM (36 bytes a key and 32 columns of K and V, read
// once for all G heads of a group) and by VALU issue, which is close behind;
// prompts by VALU issue: the two scaling operations a score and block and the
// three that make W's halves.
#include <algorithm>
#include <cfloat>
#include <cmath>

#include "kv_dev.h"
#include "w4a8_dev.h"
#include "w4a8_host.h"

namespace w4a8 {

namespace {

constexpr int JT = 512;               // threads of the joining kernel

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
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
  int64_t window;
  float *part;      // partial results, `slots` of them
  int slots;
  int cmin, target; // fewest pages of a run; runs wanted
};

// What a sequence asks for.
struct Seq {
  int64_t r0;       // its first row
  int qlen, len;    // rows, tokens (as given)
  int lo, pages;    // first page any row sees, pages from there on
  int tiles;
};

template <int RT_>
__device__ __forceinline__ Seq seq_of(const AttnArgs &a, int s) {
  Seq r;
  const int64_t r0 = kv_clamp_row(a.p.cu[s], a.T), r1 = kv_clamp_row(a.p.cu[s + 1], a.T);
  r.r0 = r0;
  r.qlen = r1 > r0 ? (int)(r1 - r0) : 0;
  r.len = a.p.len[s];
  const int64_t hi = min((int64_t)r.len, (int64_t)a.p.max_pages * KV_PAGE);
  int64_t lo = 0;
  if (a.window > 0) lo = max((int64_t)0, (int64_t)r.len - r.qlen - a.window + 1);
  r.lo = (int)(lo / KV_PAGE);
  const int64_t end = (hi + KV_PAGE - 1) / KV_PAGE;
  r.pages = r.qlen > 0 && hi > 0 && end > r.lo ? (int)(end - r.lo) : 0;
  r.tiles = (int)(((int64_t)r.qlen * a.G + RT_ - 1) / RT_);
  return r;
}

// Item or run `id` of the call, found by every wave on its own: 64 sequences
// a round.  Runs (split = false): the sequence, the number within it and the
// first partial slot of its runs; joins (split = true): counted over items
// with several runs only.  Returns false past the end.
struct Found {
  int s, local, runs, slot0;
};
template <int RT_>
__device__ __forceinline__ bool plan_find(const AttnArgs &a, int id, bool split, Found &f) {
  const int lane = threadIdx.x & 63, B = a.p.B;
  int items = 0, pages = 0;          // of sequence lane
  const auto look = [&](int s) {
    items = pages = 0;
    if (s < B) {
      const Seq q = seq_of<RT_>(a, s);
      items = q.tiles * a.p.NKV;
      pages = q.pages;
    }
  };
  int64_t total = 0;
  for (int s0 = (B - 1) / 64 * 64; s0 >= 0; s0 -= 64) {     // ends with the first 64
    look(s0 + lane);
    total += (int64_t)items * pages;
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) total += __shfl_xor(total, o);
  const int C = (int)max((int64_t)a.cmin, (total + a.target - 1) / a.target);
  int base = 0, slots = 0;
  for (int s0 = 0; s0 < B; s0 += 64) {
    if (s0) look(s0 + lane);
    const int runs = pages > C ? (pages + C - 1) / C : 1;
    const int ns = runs > 1 ? items * runs : 0;
    const int n = split ? (runs > 1 ? items : 0) : items * runs;
    int in = n, is = ns;              // inclusive scans
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(in, o), y = __shfl_up(is, o);
      if (lane >= o) { in += x; is += y; }
    }
    const uint64_t hit = __ballot(id >= base + in - n && id < base + in);
    if (hit) {
      const int l = __ffsll((long long)hit) - 1;
      f.s = __builtin_amdgcn_readfirstlane(s0 + l);
      f.local = __builtin_amdgcn_readfirstlane(id - base - __builtin_amdgcn_readlane(in - n, l));
      f.runs = __builtin_amdgcn_readlane(runs, l);
      f.slot0 = slots + __builtin_amdgcn_readlane(is - ns, l);
      return true;
    }
    base += __builtin_amdgcn_readlane(in, 63);
    slots += __builtin_amdgcn_readlane(is, 63);
  }
  return false;
}

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

template <bool SYM> struct ScaleT { typedef _Float16 type; };
template <> struct ScaleT<true> { typedef float type; };

// Floats between the rows of the waves' partial results in LDS: four more
// than the columns, so rows start in different banks.
template <int NB, int NT, int AW> struct Shape {
  static constexpr int D = 32 * NB;
  static constexpr int ROWS = 16 * NT;
  static constexpr int CB = NB < 16 / (NT * AW) ? NB : 16 / (NT * AW);   // blocks joined at a time (35 KB)
  static constexpr int LD = 32 * CB + 4;
};

template <int NB, bool SYM, int NT, int AW>
struct __align__(16) Lds {
  typedef Shape<NB, NT, AW> Sh;
  union {
    struct {
      uint32_t q[NT * NB * 64 * 2];            // Q codes in operand order
      float qd[NT * NB * 16];
      float vs[AW][NB * 64];
      typename ScaleT<SYM>::type ks[AW][NB * 64];
    } in;
    float o[AW][Sh::ROWS * Sh::LD];
  };
  float R[AW][Sh::ROWS], l[AW][Sh::ROWS];      // the waves' references and sums
  float whole[Sh::ROWS];                       // the joined sum
};

// A lane's share of a page.
template <int NB, bool SYM> struct Page {
  v4u k[NB], v[NB];
  // NB scales each of K and V: numbers lane * NB .. + NB - 1 of the tile
  static constexpr int SW = NB * (SYM ? 4 : 2) / 4;
  uint32_t ks[SW], vs[SW];
};

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

// Tokens of the scales that lane `lane` stages, number i of its NB: tbase +
// toff(i) (the inverse of kv_scale_at within a block).
template <int NB> __device__ __forceinline__ int scale_token(int lane) {
  const int n = lane * NB & 63;
  return n >> 4 << 2 | (n >> 2 & 3) << 4 | (n & 3);
}
constexpr int scale_token_off(int i) { return (i >> 2) * 16 + (i & 3); }

template <int NB, bool SYM, int NT, int AW>
__global__ __launch_bounds__(64 * AW, 2) void attn_kernel(AttnArgs a) {
  typedef Shape<NB, NT, AW> Sh;
  typedef typename ScaleT<SYM>::type sc_t;
  constexpr int D = Sh::D, ROWS = Sh::ROWS, SW = Page<NB, SYM>::SW, AT = 64 * AW;
  constexpr int64_t TILE = kv_tile_bytes(D, SYM);
  __shared__ Lds<NB, SYM, NT, AW> lds;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int g = lane >> 4;

  for (int id = blockIdx.x;; id += gridDim.x) {
    Found f;
    if (!plan_find<ROWS>(a, id, false, f)) return;
    const Seq sq = seq_of<ROWS>(a, f.s);
    const int run = f.local % f.runs, it = f.local / f.runs;
    const int h = it % a.p.NKV, tile = sq.tiles - 1 - it / a.p.NKV;   // longest first
    const int f0 = tile * ROWS, fn = min(ROWS, sq.qlen * a.G - f0);  // rows of the tile
    const int base_pos = sq.len - sq.qlen;
    const int pos0 = base_pos + f0 / a.G, pos1 = base_pos + (f0 + fn - 1) / a.G;
    // the tile's pages within this run
    int64_t key0 = 0;
    if (a.window > 0) key0 = max((int64_t)0, (int64_t)pos0 - a.window + 1);
    const int per = (sq.pages + f.runs - 1) / f.runs;
    const int plo = max((int)(key0 / KV_PAGE), sq.lo + run * per);
    int phi = min(sq.lo + min(sq.pages, (run + 1) * per), pos1 < 0 ? 0 : pos1 / KV_PAGE + 1);
    if (a.p.n_pages == 0) phi = plo;

    const int32_t *table = a.p.pages + (int64_t)f.s * a.p.max_pages;
    const int64_t head = (int64_t)h * TILE;
    const auto present = [&](int page) { return page >= 0 && page < a.p.n_pages; };
    const auto tile_at = [&](int page) {
      return (int64_t)(present(page) ? page : 0) * a.p.NKV * TILE + head;
    };
    Page<NB, SYM> pg;
    const auto load_k = [&](int page) {
      const uint8_t *t = a.p.k + tile_at(page);
#pragma unroll
      for (int b = 0; b < NB; b++) pg.k[b] = reinterpret_cast<const v4u *>(t + b * 1024)[lane];
      load_words(t + NB * 1024 + lane * (SW * 4), pg.ks);
    };
    const auto load_v = [&](int page) {
      const uint8_t *t = a.p.v + tile_at(page);
      load_words(t + NB * 1024 + lane * (SW * 4), pg.vs);
#pragma unroll
      for (int b = 0; b < NB; b++) pg.v[b] = reinterpret_cast<const v4u *>(t + b * 1024)[lane];
    };
    int at = plo + wave;
    int page = at < phi ? table[at] : -1;

    // Q codes and scales of the tile's rows (rows past the last repeat it);
    // the first page's loads go out behind Q's
    constexpr int QI = ROWS * NB * 8 / AT > 0 ? ROWS * NB * 8 / AT : 1;
    v4f x[QI];
#pragma unroll
    for (int k = 0; k < QI; k++) {
      const int i = threadIdx.x + k * AT, j = i & 7, blk = i >> 3;
      const int row = min(blk / NB, ROWS - 1), b = blk % NB, fr = f0 + min(row, fn - 1);
      x[k] = *reinterpret_cast<const v4f *>(
          a.q + (sq.r0 + fr / a.G) * a.qs + (int64_t)(h * a.G + fr % a.G) * D + b * 32 + 4 * j);
    }
    if (at < phi) {
      load_k(page);
      load_v(page);
    }
#pragma unroll
    for (int k = 0; k < QI; k++) {
      const int i = threadIdx.x + k * AT, j = i & 7, blk = i >> 3, row = blk / NB, b = blk % NB;
      const float v[4] = {x[k][0], x[k][1], x[k][2], x[k][3]};
      float d;
      const uint32_t codes = kv_q8_block8<SYM>(v, d);
      const int nt = row >> 4, r = row & 15;
      if (row < ROWS) {
        lds.in.q[((nt * NB + b) * 64 + 16 * (j & 3) + r) * 2 + (j >> 2)] = codes;
        if (j == 0) lds.in.qd[(nt * NB + b) * 16 + r] = d * a.sign;
      }
    }
    __syncthreads();

    // this lane's rows see lo_key < key <= hi_key; both less 4 g, the lane's first key of a page
    int hi_key[NT], lo_key[NT];
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
      const int pos = base_pos + (f0 + min(16 * nt + (lane & 15), fn - 1)) / a.G;
      hi_key[nt] = pos - 4 * g;
      lo_key[nt] = (a.window > 0 && a.window <= pos ? (int)(pos - a.window) : -1) - 4 * g;
    }
    const int tbase = scale_token<NB>(lane);

    float m[NT], mk[NT], l[NT];
    v4f acc[NT][NB][2];
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
      m[nt] = -FLT_MAX;
      mk[nt] = -FLT_MAX;
      l[nt] = 0.0f;
#pragma unroll
      for (int b = 0; b < NB; b++) acc[nt][b][0] = acc[nt][b][1] = v4f{0.f, 0.f, 0.f, 0.f};
    }
    // value scales are below 2^vexp and enter the product times 2^(15 - vexp)
    int vexp = -126;
    sc_t *ks = lds.in.ks[wave];
    float *vs = lds.in.vs[wave];
    float minus = -1.0f;               // opaque, so that the halves' difference is one mixed FMA
    asm("" : "+v"(minus));
    for (; at < phi; at += AW) {
      const int next_page = at + AW < phi ? table[at + AW] : -1;
      const int key = at * KV_PAGE;
      // pages that some row does not see whole; an absent page is seen by none
      const bool here = present(page);
      const bool masked = !here || key + KV_PAGE - 1 > pos0 ||
                          (a.window > 0 && key <= pos1 - a.window);
      // stage the scales; keys that no row sees count for nothing
#pragma unroll
      for (int w = 0; w < SW; w++) reinterpret_cast<word *>(ks)[lane * SW + w] = pg.ks[w];
      {
        float dv[NB], vmax = 0.0f;
#pragma unroll
        for (int i = 0; i < NB; i++)
          dv[i] = SYM ? __builtin_bit_cast(float, pg.vs[i % SW])
                      : f16_bits_to_f32(pg.vs[(i / 2) % SW] >> (16 * (i & 1)));
        if (masked) {
          const int last = here ? pos1 - key - tbase : -1;
          const int before = (int)max((int64_t)0, key0 - key) - tbase;
#pragma unroll
          for (int i = 0; i < NB; i++)
            if (scale_token_off(i) > last || scale_token_off(i) < before) dv[i] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < NB; i++) {
          const float y = fabsf(dv[i]);
          vmax = fmaxf(vmax, y < INFINITY ? y : 0.0f);
        }
        if (__ballot(vmax >= ldexpf(1.0f, vexp))) {
#pragma unroll
          for (int o = 32; o > 0; o >>= 1) vmax = fmaxf(vmax, __shfl_xor(vmax, o));
          const int e = __builtin_amdgcn_readfirstlane(ilogbf(vmax) + 1);
#pragma unroll
          for (int nt = 0; nt < NT; nt++)
#pragma unroll
            for (int b = 0; b < NB; b++)
#pragma unroll
              for (int s = 0; s < 2; s++)
#pragma unroll
                for (int y = 0; y < 4; y++) acc[nt][b][s][y] = ldexpf(acc[nt][b][s][y], vexp - e);
          vexp = e;
        }
#pragma unroll
        for (int i = 0; i < NB; i++) vs[lane * NB + i] = ldexpf(dv[i], 15 - vexp);
      }

      // scores
      float S[NT][16];
#pragma unroll
      for (int nt = 0; nt < NT; nt++)
#pragma unroll
        for (int i = 0; i < 16; i++) S[nt][i] = 0.0f;
#pragma unroll
      for (int b = 0; b < NB; b++) {
        long qb[NT];
        float dq[NT], cq[NT];
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
          qb[nt] = reinterpret_cast<const long *>(lds.in.q)[(nt * NB + b) * 64 + lane];
          dq[nt] = lds.in.qd[(nt * NB + b) * 16 + (lane & 15)];
          cq[nt] = -12582912.0f * dq[nt];
        }
        sc_t dk[16];
#pragma unroll
        for (int i = 0; i < 16; i++) dk[i] = ks[b * 64 + g * 16 + i];
#pragma unroll
        for (int i = 0; i < 4; i++) {
          const uint32_t y = pg.k[b][i];
          const long kb = (long)((uint64_t)(y & 0xF0F0F0F0u) << 32 | (y << 4 & 0xF0F0F0F0u));
#pragma unroll
          for (int nt = 0; nt < NT; nt++) {
            const v4i c = {0x4B400000, 0x4B400000, 0x4B400000, 0x4B400000};
            const v4f r = __builtin_bit_cast(
                v4f, __builtin_amdgcn_mfma_i32_16x16x32_i8(kb, qb[nt], c, 0, 0, 0));
#pragma unroll
            for (int e = 0; e < 4; e++) {
              // SYM: an fp32 scale times 1.5 2^23 would round, so s comes first
              const float t = SYM ? (r[e] - 12582912.0f) * dq[nt] : fmaf(r[e], dq[nt], cq[nt]);
              S[nt][4 * i + e] = fmaf(t, (float)dk[4 * i + e], S[nt][4 * i + e]);
            }
          }
        }
        // one block at a time: moved together, the blocks' products and scales
        // would all be live at once
#pragma unroll
        for (int nt = 0; nt < NT; nt++)
#pragma unroll
          for (int i = 0; i < 16; i++) asm volatile("" : "+v"(S[nt][i]));
      }
      if (at + AW < phi) load_k(next_page);

      // running maximum
      float mx[NT];
      bool grow = false;
#pragma unroll
      for (int nt = 0; nt < NT; nt++) {
        if (masked) {
          const int last = here ? hi_key[nt] - key : -1, before = lo_key[nt] - key;
#pragma unroll
          for (int i = 0; i < 16; i++)
            if (scale_token_off(i) > last || scale_token_off(i) <= before) S[nt][i] = -INFINITY;
        }
        mx[nt] = -FLT_MAX;
#pragma unroll
        for (int i = 0; i < 16; i++) mx[nt] = fmaxf(mx[nt], S[nt][i]);
        mx[nt] = max4(mx[nt]);
        grow |= mx[nt] > m[nt];
      }
      if (__ballot(grow)) {
#pragma unroll
        for (int nt = 0; nt < NT; nt++) {
          const float mn = fmaxf(m[nt], mx[nt]), mkn = mn * a.k;
          const float al = m[nt] == -FLT_MAX ? 0.0f : exp2_f(mk[nt] - mkn);
          m[nt] = mn;
          mk[nt] = mkn;
          l[nt] *= al;
#pragma unroll
          for (int b = 0; b < NB; b++) {
            acc[nt][b][0] *= al;
            acc[nt][b][1] *= al;
          }
        }
      }
      // probabilities (a masked score's is exp2(-infinity) = 0)
#pragma unroll
      for (int nt = 0; nt < NT; nt++) {
#pragma unroll
        for (int i = 0; i < 16; i++) S[nt][i] = exp2_f(fmaf(S[nt][i], a.k, -mk[nt]));
        float s[8];
#pragma unroll
        for (int i = 0; i < 8; i++) s[i] = S[nt][i] + S[nt][i + 8];
#pragma unroll
        for (int o = 4; o > 0; o >>= 1)
#pragma unroll
          for (int i = 0; i < o; i++) s[i] += s[i + o];
        l[nt] += s[0];
      }
      __builtin_amdgcn_sched_barrier(0);
      // values, 32 keys at a time
#pragma unroll
      for (int b = 0; b < NB; b++) {
#pragma unroll
        for (int hh = 0; hh < 2; hh++) {
          float d[8];
#pragma unroll
          for (int i = 0; i < 8; i++) d[i] = vs[b * 64 + g * 16 + 8 * hh + i];
          h8 c[2];                       // elements l % 16 and + 16
#pragma unroll
          for (int i = 0; i < 2; i++) {
            const uint32_t y = pg.v[b][2 * hh + i], z = y >> 8;
            const h2 off = {(_Float16)-1032.0f, (_Float16)-1032.0f};
            const h2 six = {(_Float16)0.0625f, (_Float16)0.0625f};
            const h2 off2 = {(_Float16)-72.0f, (_Float16)-72.0f};
            const h2 a0 = __builtin_bit_cast(h2, (y & 0x000F000Fu) | 0x64006400u) + off;
            const h2 a1 = __builtin_bit_cast(h2, (z & 0x000F000Fu) | 0x64006400u) + off;
            const h2 b0 = __builtin_elementwise_fma(
                __builtin_bit_cast(h2, (y & 0x00F000F0u) | 0x64006400u), six, off2);
            const h2 b1 = __builtin_elementwise_fma(
                __builtin_bit_cast(h2, (z & 0x00F000F0u) | 0x64006400u), six, off2);
            c[0][4 * i] = a0[0]; c[0][4 * i + 1] = a0[1]; c[0][4 * i + 2] = a1[0]; c[0][4 * i + 3] = a1[1];
            c[1][4 * i] = b0[0]; c[1][4 * i + 1] = b0[1]; c[1][4 * i + 2] = b1[0]; c[1][4 * i + 3] = b1[1];
          }
#pragma unroll
          for (int nt = 0; nt < NT; nt++) {
            h8 hi, lo;
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
              v2f w;
              // 0 times anything is 0: a key that the row does not see may have any scale
              w[0] = mul_zero(S[nt][8 * hh + i], d[i]);
              w[1] = mul_zero(S[nt][8 * hh + i + 1], d[i + 1]);
              const h2 y = __builtin_convertvector(w, h2);
              v2f z;
              z[0] = fmaf((float)y[0], minus, w[0]);
              z[1] = fmaf((float)y[1], minus, w[1]);
              const h2 y2 = __builtin_convertvector(z, h2);
              hi[i] = y[0]; hi[i + 1] = y[1];
              lo[i] = y2[0]; lo[i + 1] = y2[1];
            }
#pragma unroll
            for (int s = 0; s < 2; s++) {
              acc[nt][b][s] = __builtin_amdgcn_mfma_f32_16x16x32_f16(c[s], hi, acc[nt][b][s], 0, 0, 0);
              acc[nt][b][s] = __builtin_amdgcn_mfma_f32_16x16x32_f16(c[s], lo, acc[nt][b][s], 0, 0, 0);
            }
          }
        }
        #pragma unroll
          for (int nt = 0; nt < NT; nt++) asm volatile("" : "+v"(acc[nt][b][0]), "+v"(acc[nt][b][1]));
      }
      if (at + AW < phi) load_v(next_page);
      page = next_page;
    }

    // join the waves: reference R (base-2 exponent taken out of l and acc)
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
      l[nt] = sum4(l[nt]);
      if (lane < 16) {
        lds.R[wave][16 * nt + lane] = mk[nt];
        lds.l[wave][16 * nt + lane] = l[nt];
      }
    }
    __syncthreads();               // also: nobody reads lds.in any more
    float Rj[NT], lj[NT];
#pragma unroll
    for (int nt = 0; nt < NT; nt++) {
      const int row = 16 * nt + (lane & 15);
      float R = -FLT_MAX, s = 0.0f;
#pragma unroll
      for (int w = 0; w < AW; w++)
        if (lds.l[w][row] != 0.0f) R = fmaxf(R, lds.R[w][row]);
#pragma unroll
      for (int w = 0; w < AW; w++)
        if (lds.l[w][row] != 0.0f) s = fmaf(lds.l[w][row], exp2_f(lds.R[w][row] - R), s);
      Rj[nt] = R;
      lj[nt] = s;
      const float fac = l[nt] != 0.0f ? exp2_f(mk[nt] - R) : 0.0f;
#pragma unroll
      for (int b = 0; b < NB; b++)
#pragma unroll
        for (int s2 = 0; s2 < 2; s2++)
#pragma unroll
          for (int x = 0; x < 4; x++)
            acc[nt][b][s2][x] = l[nt] != 0.0f ? ldexpf(acc[nt][b][s2][x], vexp - 15) * fac : 0.0f;
    }
    const bool whole = f.runs == 1;
    const int slot = whole ? 0 : f.slot0 + f.local;
    float *part = a.part + (int64_t)slot * (ROWS * (D + 2));
    const bool fits = whole || slot < a.slots;
    if (wave == 0 && lane < 16) {
#pragma unroll
      for (int nt = 0; nt < NT; nt++) {
        const int row = 16 * nt + lane;
        lds.whole[row] = lj[nt];
        if (!whole && fits) {
          part[ROWS * D + 2 * row] = Rj[nt];
          part[ROWS * D + 2 * row + 1] = lj[nt];
        } else if (whole && a.lse && row < fn) {
          const int fr = f0 + row;
          a.lse[(sq.r0 + fr / a.G) * a.NH + h * a.G + fr % a.G] =
              lj[nt] != 0.0f ? (Rj[nt] + log2f(lj[nt])) * 0.693147180559945f : -INFINITY;
        }
      }
    }
#pragma unroll
    for (int b0 = 0; b0 < NB; b0 += Sh::CB) {
      __syncthreads();
#pragma unroll
      for (int nt = 0; nt < NT; nt++)
#pragma unroll
        for (int b = 0; b < Sh::CB; b++)
#pragma unroll
          for (int s = 0; s < 2; s++)
            *reinterpret_cast<v4f *>(&lds.o[wave][(16 * nt + (lane & 15)) * Sh::LD + b * 32 +
                                                  s * 16 + 4 * g]) = acc[nt][b0 + b][s];
      __syncthreads();
      constexpr int C4 = Sh::CB * 8;           // 16-byte pieces of a row
      for (int i = threadIdx.x; i < ROWS * C4; i += AT) {
        const int row = i / C4, c4 = i % C4;
        v4f s = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < AW; w++) s += *reinterpret_cast<const v4f *>(&lds.o[w][row * Sh::LD + 4 * c4]);
        if (whole) {
          if (row < fn) {
            const int fr = f0 + row;
            const float lr = lds.whole[row];
            const float inv = lr != 0.0f ? 1.0f / lr : 0.0f;
            *reinterpret_cast<v4f *>(a.out + ((sq.r0 + fr / a.G) * a.NH + h * a.G + fr % a.G) * D +
                                     b0 * 32 + 4 * c4) = s * inv;
          }
        } else if (fits) {
          *reinterpret_cast<v4f *>(part + row * D + b0 * 32 + 4 * c4) = s;
        }
      }
    }
    __syncthreads();
  }
}

// Joins the runs of item blockIdx.x (counted over the items with several
// runs), row blockIdx.y of its tile: D / 4 lanes by groups that take the runs
// in turn, summed in a fixed order.
template <int NB, int NT>
__global__ __launch_bounds__(JT) void join_kernel(AttnArgs a) {
  constexpr int D = 32 * NB, ROWS = 16 * NT, L = D / 4, NG = JT / L;
  __shared__ v4f so[NG][L];
  __shared__ float sr[NG], sl[NG];
  Found f;
  if (!plan_find<ROWS>(a, blockIdx.x, true, f)) return;
  const Seq sq = seq_of<ROWS>(a, f.s);
  const int h = f.local % a.p.NKV, tile = sq.tiles - 1 - f.local / a.p.NKV;
  const int row = blockIdx.y, fr = tile * ROWS + row;
  if (fr >= sq.qlen * a.G) return;
  const int grp = threadIdx.x / L, c4 = threadIdx.x % L;
  const int slot = f.slot0 + f.local * f.runs;
  const int n = min(f.runs, a.slots - slot);
  const float *part = a.part + (int64_t)slot * (ROWS * (D + 2));
  // the reference first: every thread's runs, then all groups'
  float R = -FLT_MAX;
  for (int i = threadIdx.x; i < n; i += JT) {
    const float *p = part + (int64_t)i * (ROWS * (D + 2)) + ROWS * D + 2 * row;
    if (p[1] != 0.0f) R = fmaxf(R, p[0]);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) R = fmaxf(R, __shfl_xor(R, o));
  if ((threadIdx.x & 63) == 0) sr[threadIdx.x >> 6] = R;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < JT / 64; w++) R = fmaxf(R, sr[w]);
  v4f s = v4f{0.f, 0.f, 0.f, 0.f};
  float l = 0.0f;
#pragma unroll 4
  for (int i = grp; i < n; i += NG) {
    const float *p = part + (int64_t)i * (ROWS * (D + 2));
    const float lr = p[ROWS * D + 2 * row + 1];
    const float w = lr != 0.0f ? exp2_f(p[ROWS * D + 2 * row] - R) : 0.0f;
    const v4f x = *reinterpret_cast<const v4f *>(p + row * D + 4 * c4);
    s += x * w;
    l = fmaf(lr, w, l);
  }
  so[grp][c4] = s;
  if (c4 == 0) sl[grp] = l;
  __syncthreads();
  if (grp != 0) return;
  l = 0.0f;
  s = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < NG; i++) {
    s += so[i][c4];
    l += sl[i];
  }
  const int64_t at = (sq.r0 + fr / a.G) * a.NH + h * a.G + fr % a.G;
  *reinterpret_cast<v4f *>(a.out + at * D + 4 * c4) = l != 0.0f ? s * (1.0f / l) : s * 0.0f;
  if (c4 == 0 && a.lse)
    a.lse[at] = l != 0.0f ? (R + log2f(l)) * 0.693147180559945f : -INFINITY;
}

// Rows of a tile: 32 once sequences have more than 16 on average (a tile's
// rows share the page's loads and decoded codes), 16 for the few rows of a
// decode step, and for D = 256, whose 32-row sums would not fit in registers.
// Waves of a workgroup: 8 on 16-row tiles, so that a short context needs no
// second launch, 4 on 32-row ones.
int tile_rows(const w4a8_kv *kv, int64_t T, int64_t NH) {
  const int64_t rows = T * (NH / kv->NKV);
  return kv->D <= 128 && kv->B > 0 && rows > 16 * kv->B ? 32 : 16;
}
constexpr int CMIN = 16;              // fewest pages of a run
constexpr int TARGET = 512;           // runs wanted

// Bounds on the call's items, and on the partial results it can need: a
// sequence is split only into runs of more than half of C = total / TARGET
// pages, so the runs of split items number at most 2 TARGET.
int64_t items_bound(const w4a8_kv *kv, int64_t T, int64_t NH) {
  const int rt = tile_rows(kv, T, NH);
  const int64_t G = NH / kv->NKV;
  return ((T * G) / rt + std::min(kv->B, T)) * kv->NKV;
}
int64_t slots_bound(const w4a8_kv *kv, int64_t T, int64_t NH) {
  if (kv->max_pages <= CMIN) return 0;
  const int64_t runs = (kv->max_pages + CMIN - 1) / CMIN;
  return std::min<int64_t>(2 * TARGET, items_bound(kv, T, NH) * runs);
}

int attn_sizes(const w4a8_kv *kv, int64_t T, int64_t NH) {
  if (int rc = kv_check_sizes(kv); rc != W4A8_OK) return rc;
  if (NH < 1 || NH % kv->NKV != 0 || T < 0) return W4A8_ESHAPE;
  if (NH >= ((int64_t)1 << 31) || T >= ((int64_t)1 << 31) || T * NH >= ((int64_t)1 << 31))
    return W4A8_ERANGE;
  return W4A8_OK;
}

template <int NB, bool SYM, int NT, int AW>
int launch(const AttnArgs &a, int64_t items, hipStream_t s) {
  const int64_t grid = std::min<int64_t>(items + a.slots, 1 << 20);
  attn_kernel<NB, SYM, NT, AW><<<dim3((unsigned)grid), dim3(64 * AW), 0, s>>>(a);
  if (int rc = check_launch(); rc != W4A8_OK || a.slots == 0) return rc;
  const int64_t joins = std::min<int64_t>(items, TARGET);
  join_kernel<NB, NT><<<dim3((unsigned)joins, 16 * NT), dim3(JT), 0, s>>>(a);
  return check_launch();
}

template <int NB, bool SYM>
int launch_rows(const AttnArgs &a, bool wide, int64_t items, hipStream_t s) {
  if constexpr (NB <= 4)
    if (wide) return launch<NB, SYM, 2, 4>(a, items, s);
  return launch<NB, SYM, 1, 8>(a, items, s);
}

}  // namespace
}  // namespace w4a8

using namespace w4a8;

extern "C" size_t attn_q4_workspace_size(const w4a8_kv *kv, int64_t T, int64_t NH) {
  if (attn_sizes(kv, T, NH) != W4A8_OK) return 0;
  const int64_t n = slots_bound(kv, T, NH) * tile_rows(kv, T, NH) * (kv->D + 2) * 4;
  return (size_t)std::max<int64_t>(16, n);
}

extern "C" int attn_q4_forward(const w4a8_kv *kv, const float *q, int64_t q_stride, float *out,
                               float *lse, int64_t T, int64_t NH, float scale, int64_t window,
                               void *workspace, size_t ws_bytes, void *stream) {
  if (int rc = kv_check(kv); rc != W4A8_OK) return rc;
  if (!q || !out || !workspace) return W4A8_ENULL;
  if (int rc = attn_sizes(kv, T, NH); rc != W4A8_OK) return rc;
  if (window < 0 || !std::isfinite(scale) || q_stride < NH * kv->D || q_stride % 4 != 0)
    return W4A8_ESHAPE;
  if (q_stride >= ((int64_t)1 << 31)) return W4A8_ERANGE;
  if (!aligned16(q) || !aligned16(out) || !aligned16(workspace) ||
      (reinterpret_cast<uintptr_t>(lse) & 3u))
    return W4A8_EALIGN;
  if (out == q) return W4A8_EALIAS;
  if (ws_bytes < attn_q4_workspace_size(kv, T, NH)) return W4A8_EWORKSPACE;
  if (T == 0 || kv->B == 0) return W4A8_OK;
  if (int rc = check_device(); rc != W4A8_OK) return rc;
  AttnArgs a = {kv_plan(kv), q, q_stride, out, lse, T, (int)NH, (int)(NH / kv->NKV),
                // a factor of 0 goes to Q, so that a masked score's -infinity stays one
                scale != 0.0f ? std::fabs(scale) * 1.44269504f / 16.0f : 1.0f,
                scale < 0.0f ? -1.0f : scale == 0.0f ? 0.0f : 1.0f, window,
                reinterpret_cast<float *>(workspace), (int)slots_bound(kv, T, NH), CMIN, TARGET};
  const int64_t items = items_bound(kv, T, NH);
  const bool sym = kv->format == W4A8_KV_Q4_SYM, wide = tile_rows(kv, T, NH) == 32;
  const hipStream_t s = as_stream(stream);
  if (kv->D == 64) return sym ? launch_rows<2, true>(a, wide, items, s) : launch_rows<2, false>(a, wide, items, s);
  if (kv->D == 128) return sym ? launch_rows<4, true>(a, wide, items, s) : launch_rows<4, false>(a, wide, items, s);
  return sym ? launch_rows<8, true>(a, wide, items, s) : launch_rows<8, false>(a, wide, items, s);
}
