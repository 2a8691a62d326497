// 8-bit rows: int8 codes with one fp32 scale a row (the quantizer), and the
// product of activation rows with weight rows in exact int32 sums, scaled once:
//   y[m][n] = (float)(sum_k xq[m][k] wq[n][k]) * (xd[m] wd[n]) + bias[n].
//
// The quantizer reads 4 bytes and writes one per value, in one pass where a row
// fits a workgroup's registers: 5120 x 4096 24 us (4.4 TB/s; a large copy reaches
// 5.05), one row 2.1 us.
//
// The product: sums are whole numbers, so any split of a row's length and any
// order give the same bits.  Up to 16 rows, and up to 64 where one workgroup a
// compute unit covers the channels, stream the weights once (1 x 151936 x 2048: 59
// us, 5.3 TB/s; 1 x 12288 x 2048 6.2); more rows take tiles.  Large tiles are
// bound by what the card draws: 5120 x 12288 x 4096 takes 253 us (2.03 POP/s) and 217
// with operands of zero; the matrix cores work in 61 % of the cycles, at clocks that
// fall to 1.6 GHz.  8192^3: 2.23 POP/s (the library's int8 product 2.51), 4096^3
// 1.87 (2.04).  Tiles that fill the card once (947 x 12288 x 2048: 33 us) are bound
// by the stages: a 256 x 256 tile's stage of 64 codes takes 0.73 us, of which its
// products are 0.43, so 23 us for the 32 stages; the rest is the launch, the first
// loads and the output (46.5 MB, 9 us at a copy's rate), which all tiles store after
// their last stage, at one time.  64 compute units have no tile.  Measured slower: 128 x 128 waves (four a tile; 549 us at 8192^3
// where eight of 128 x 64 took 523), wave priorities, tiles of 192 (5120 x 12288 x
// 4096 289 to 312 us).
#include "choice.h"
#include "dma_dev.h"
#include "w4a8_dev.h"
#include "w4a8_host.h"

namespace w4a8 {

namespace {

constexpr int QNT = 256;            // threads of a quantizing workgroup: one row
constexpr int KNT = 512;            // ... of a product of few rows: eight waves
constexpr int PAD = W4A8_Q8_ROW_PAD;

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v16i __attribute__((ext_vector_type(16)));
typedef float v4f __attribute__((ext_vector_type(4)));

// ------------------------------------------------------------------ quantizer
__device__ __forceinline__ int odd_value(float v) { return !(fabsf(v) < __builtin_inff()); }
__device__ __forceinline__ uint32_t code(float v, float id) { return (uint32_t)round_clamp(v * id, 127) & 0xFFu; }

// The row's scale and its inverse from each thread's largest magnitude and
// whether it saw a NaN or an infinity.
__device__ __forceinline__ float row_scale(float amax, int odd, float &id) {
  __shared__ float top[QNT / 64];
  __shared__ int bad[QNT / 64];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) amax = fmaxf(amax, __shfl_xor(amax, o));
  odd = __any(odd);
  if ((threadIdx.x & 63) == 0) { top[threadIdx.x >> 6] = amax; bad[threadIdx.x >> 6] = odd; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < QNT / 64; w++) { amax = fmaxf(amax, top[w]); odd |= bad[w]; }
  const float d = odd ? __builtin_nanf("") : amax * (1.0f / 127.0f);
  id = odd ? 0.0f : sym_inverse(d);
  return d;
}

// One row a workgroup, in registers: V times four values a thread, K a multiple
// of 4 and rows 16-byte aligned.
template <int V>
__global__ __launch_bounds__(QNT) void q8_row_kernel(const float *__restrict__ x, int64_t xs,
                                                     int8_t *__restrict__ q, float *__restrict__ d,
                                                     int K, int KP) {
  const int64_t r = blockIdx.x;
  const float *xr = x + r * xs;
  v4f v[V];
  float amax = 0.0f;
  int odd = 0;
#pragma unroll
  for (int i = 0; i < V; i++) {
    const int k = 4 * (threadIdx.x + QNT * i);
    v[i] = k < K ? *reinterpret_cast<const v4f *>(xr + k) : v4f{0.f, 0.f, 0.f, 0.f};
  }
#pragma unroll
  for (int i = 0; i < V; i++)
#pragma unroll
    for (int e = 0; e < 4; e++) {
      odd |= odd_value(v[i][e]);
      amax = fmaxf(amax, fabsf(v[i][e]));
    }
  float id;
  const float dr = row_scale(amax, odd, id);
  if (threadIdx.x == 0) d[r] = dr;
#pragma unroll
  for (int i = 0; i < V; i++) {
    const int k = 4 * (threadIdx.x + QNT * i);
    if (k < KP)
      *reinterpret_cast<uint32_t *>(q + r * KP + k) =
          dr == dr ? code(v[i][0], id) | code(v[i][1], id) << 8 | code(v[i][2], id) << 16 | code(v[i][3], id) << 24
                   : 0u;
  }
}

// Rows of any length and alignment, read twice.
__global__ __launch_bounds__(QNT) void q8_any_row_kernel(const float *__restrict__ x, int64_t xs,
                                                         int8_t *__restrict__ q, float *__restrict__ d,
                                                         int K, int KP) {
  const int64_t r = blockIdx.x;
  const float *xr = x + r * xs;
  float amax = 0.0f;
  int odd = 0;
  for (int k = threadIdx.x; k < K; k += QNT) {
    odd |= odd_value(xr[k]);
    amax = fmaxf(amax, fabsf(xr[k]));
  }
  float id;
  const float dr = row_scale(amax, odd, id);
  if (threadIdx.x == 0) d[r] = dr;
  for (int k = 4 * threadIdx.x; k < KP; k += 4 * QNT) {
    uint32_t packed = 0;
#pragma unroll
    for (int i = 0; i < 4; i++)
      if (k + i < K && dr == dr) packed |= code(xr[k + i], id) << (8 * i);
    *reinterpret_cast<uint32_t *>(q + r * KP + k) = packed;
  }
}

// ------------------------------------------------------------------ product
struct QArgs {
  const int8_t *xq, *wq;
  const float *xd, *wd, *bias;
  float *y;
  int64_t ys;
  int M, N, KP;
  int mt, nt;                       // tiles of rows and of channels
  int vec;                          // rows of y start 16-byte aligned
};

// Four neighbouring channels of a row: scaled, plus bias, stored.
__device__ __forceinline__ void put4(const QArgs &a, int m, int n, v4i s, float xd, v4f wd, v4f bias) {
  v4f y;
#pragma unroll
  for (int e = 0; e < 4; e++) {
    y[e] = (float)s[e] * (xd * wd[e]);
    if (a.bias) y[e] += bias[e];
  }
  float *p = a.y + (int64_t)m * a.ys + n;
  if (a.vec && n + 4 <= a.N) {
    *reinterpret_cast<v4f *>(p) = y;
  } else {
#pragma unroll
    for (int e = 0; e < 4; e++)
      if (n + e < a.N) p[e] = y[e];
  }
}
__device__ __forceinline__ v4f load_channels(const QArgs &a, const float *p, int n) {
  v4f v;
#pragma unroll
  for (int e = 0; e < 4; e++) v[e] = p[min(n + e, a.N - 1)];
  return v;
}

// Tiles of TN channels by TM rows, waves of RN by RM on 32 x 32 x 32
// products; the weights are the A operand, so that element e of a sum in lane l
// is channel 8 (e / 4) + 4 (l / 32) + e % 4 and row l % 32.  64 codes of every row
// a stage, by direct loads into a ring of NS slots; the 16-byte pieces of a row
// stand XOR-swizzled by the row, so that 16 lanes that read one piece of 16
// rows meet distinct banks.
template <int TN, int TM, int WN, int WM, int NS>
struct Tile {
  static constexpr int RN = TN / WN, RM = TM / WM, BN = RN / 32, BM = RM / 32;
  static constexpr int NW = WN * WM, NT = 64 * NW;
  static constexpr int SLOT = (TN + TM) * 64, PER = (TN + TM) / 16 / NW;
  static constexpr int OS = RN + 4;                // row stride of a wave's output in LDS
  static constexpr int LDS = NS * SLOT > NW * 32 * OS * 4 ? NS * SLOT : NW * 32 * OS * 4;
  static_assert(BN * 32 == RN && BM * 32 == RM && PER * 16 * NW == TN + TM && NS >= 3, "tile");
};

template <int TN, int TM, int WN, int WM, int NS>
__global__ __launch_bounds__(64 * WN * WM, 2) void q8_tile_kernel(QArgs a) {
  using T = Tile<TN, TM, WN, WM, NS>;
  __shared__ __align__(16) uint8_t lds[T::LDS];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  // Each XCD (workgroup b runs on XCD b mod 8) takes an even contiguous share of
  // the tiles, in the order of groups of 8 row tiles, within a group channels by
  // channels: what runs on it at once shares rows and channels in its L2.
  const int total = a.mt * a.nt, x = blockIdx.x & 7;
  int w = x * (total >> 3) + min(x, total & 7) + (blockIdx.x >> 3);
  const int g = w / (8 * a.nt), gm = min(8, a.mt - 8 * g);
  w -= g * 8 * a.nt;
  const int m0 = (8 * g + w % gm) * TM, n0 = (w / gm) * TN;

  // direct loads: 16 rows of 64 bytes an instruction, rows past the last repeat it
  const uint8_t *src[T::PER];
  uint32_t off[T::PER];
  const uint32_t piece = 16 * ((lane & 3) ^ ((lane >> 4) & 3));
#pragma unroll
  for (int u = 0; u < T::PER; u++) {
    const int r = 16 * (wave + T::NW * u);         // of the tile's TN + TM
    const bool is_w = r < TN;
    const int first = is_w ? n0 : m0, last = (is_w ? a.N : a.M) - 1;
    src[u] = reinterpret_cast<const uint8_t *>(is_w ? a.wq : a.xq) + (int64_t)first * a.KP;
    off[u] = (uint32_t)(min(first + r - (is_w ? 0 : TN) + (lane >> 2), last) - first) * (uint32_t)a.KP + piece;
  }
  const int S = a.KP / 64;
  const auto load_stage = [&](int t) {
    uint8_t *const slot = lds + (t % NS) * T::SLOT;
#pragma unroll
    for (int u = 0; u < T::PER; u++) lds_dma16(src[u] + t * 64, off[u], slot + 1024 * (wave + T::NW * u));
  };
  const int wn = wave % WN, wm = wave / WN, l32 = lane & 31, lh = lane >> 5;
  const int nl = n0 + wn * T::RN + 4 * l32;        // this lane's channels when rows are stored
  v4f wd, bias = {0.f, 0.f, 0.f, 0.f};
  float xd[T::BM];
  wd = load_channels(a, a.wd, nl);
  if (a.bias) bias = load_channels(a, a.bias, nl);
#pragma unroll
  for (int j = 0; j < T::BM; j++) xd[j] = a.xd[min(m0 + wm * T::RM + 32 * j + l32, a.M - 1)];
#pragma unroll
  for (int t = 0; t < NS; t++)
    if (t < S) load_stage(t);

  // Half a stage's operands are read between the products of the half before: a
  // stage's second half among its first's, the next stage's first half, and the
  // loads of the stage NS on, among its second's, behind the barrier that says the
  // next stage has landed (the younger NS - 2 may be under way) and that every
  // wave has read this one, whose slot the loads fill.  A product takes 32
  // cycles and the two or three other instructions behind it are issued meanwhile.
  const uint32_t at = l32 * 64 + 16 * (lh ^ ((l32 >> 2) & 3));
  v16i acc[T::BN][T::BM] = {};
  v4i w0[T::BN], x0[T::BM], w1[T::BN], x1[T::BM];
  constexpr int NP = T::BN * T::BM, NR = T::BN + T::BM;
  const auto read = [&](const uint8_t *slot, int k, int u, v4i (&wv)[T::BN], v4i (&xv)[T::BM]) {
    if (u < T::BM)
      xv[u] = *reinterpret_cast<const v4i *>(slot + (TN + wm * T::RM + 32 * u) * 64 + (at ^ (32 * k)));
    else
      wv[u - T::BM] = *reinterpret_cast<const v4i *>(slot + (wn * T::RN + 32 * (u - T::BM)) * 64 + (at ^ (32 * k)));
  };
  // the products of (wv, xv) with the reads of half k of `next` into (wn, xn) and, if
  // `dma`, the loads of stage t
  const auto half = [&](const v4i (&wv)[T::BN], const v4i (&xv)[T::BM], const uint8_t *next, int k,
                        v4i (&wnext)[T::BN], v4i (&xnext)[T::BM], bool dma, int t, uint8_t *slot) {
#pragma unroll
    for (int p = 0; p < NP; p++) {
      const int i = p / T::BM, j = p % T::BM;
      acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(wv[i], xv[j], acc[i][j], 0, 0, 0);
#pragma unroll
      for (int u = p * NR / NP; u < (p + 1) * NR / NP; u++) read(next, k, u, wnext, xnext);
      if (dma)
#pragma unroll
        for (int u = p * T::PER / NP; u < (p + 1) * T::PER / NP; u++)
          lds_dma16(src[u] + t * 64, off[u], slot + 1024 * (wave + T::NW * u));
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  if (S >= NS)
    wait_barrier<(NS - 1) * T::PER>();
  else
    wait_barrier<0>();
#pragma unroll
  for (int u = 0; u < NR; u++) read(lds, 0, u, w0, x0);
  for (int t = 0, sl = 0; t < S; t++) {            // the stage, its slot
    const int sn = sl + 1 == NS ? 0 : sl + 1;
    uint8_t *const slot = lds + sl * T::SLOT;
    half(w0, x0, slot, 1, w1, x1, false, 0, nullptr);
    if (t + NS - 1 < S)
      wait_barrier<(NS - 2) * T::PER>();
    else
      wait_barrier<0>();
    // (past the last stage what is read is not used)
    half(w1, x1, lds + sn * T::SLOT, 0, w0, x0, t + NS < S, t + NS, slot);
    sl = sn;
  }
  // the sums through LDS, a wave's 32 rows at a time, so that whole rows of its
  // channels are stored
  wait_barrier<0>();
  int *const o = reinterpret_cast<int *>(lds) + wave * 32 * T::OS;
#pragma unroll
  for (int j = 0; j < T::BM; j++) {
#pragma unroll
    for (int i = 0; i < T::BN; i++)
#pragma unroll
      for (int q = 0; q < 4; q++)
        *reinterpret_cast<v4i *>(o + l32 * T::OS + 32 * i + 8 * q + 4 * lh) =
            v4i{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
    constexpr int LR = T::RN / 4, PR = 64 / LR;    // lanes of a row, rows an instruction
    const int c = lane % LR, m = m0 + wm * T::RM + 32 * j;
    const v4f wc = LR == 32 ? wd : load_channels(a, a.wd, n0 + wn * T::RN + 4 * c);
    const v4f bc = LR == 32 || !a.bias ? bias : load_channels(a, a.bias, n0 + wn * T::RN + 4 * c);
#pragma unroll 4
    for (int u = 0; u < 32 / PR; u++) {
      const int r = PR * u + lane / LR;
      const v4i s = *reinterpret_cast<const v4i *>(o + r * T::OS + 4 * c);
      const float d = __shfl(xd[j], r);
      const int n = n0 + wn * T::RN + 4 * c;
      if (m + r < a.M && n < a.N) put4(a, m + r, n, s, d, wc, bc);
    }
  }
}

// Few rows: 16 RN channels by 16 MT rows a workgroup, eight waves that split the
// row length, operands straight from memory: the weights stream once, the rows'
// codes come from the L2 cache.  The waves' sums (whole numbers: any order
// gives the same) are added up in LDS.  Small calls are a chain of launch, one
// or two trips to memory, the join and the store: 1 x 2048 x 4096 5.8 us, 48 x 2048 x
// 4096 10.8; four or sixteen waves 7.0 and 5.7, 12.0 and 10.6.  At 48 rows three of
// four operand loads are activation codes, all 196 KB of them read by each of the 128
// workgroups, and the join's atomics meet 16 of the LDS's banks.
template <int MT, int RN>
__global__ __launch_bounds__(KNT) void q8_few_kernel(QArgs a) {
  constexpr int OS = 16 * RN + 4, U = RN * MT >= 8 ? 2 : 4;
  __shared__ __align__(16) int o[16 * MT * OS];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int l16 = lane & 15, lq = lane >> 4;
  const int n0 = blockIdx.x * 16 * RN;
  for (int i = threadIdx.x; i < 16 * MT * OS; i += KNT) o[i] = 0;
  const int8_t *wp[RN], *xp[MT];
#pragma unroll
  for (int i = 0; i < RN; i++) wp[i] = a.wq + (int64_t)min(n0 + 16 * i + l16, a.N - 1) * a.KP + 16 * lq;
#pragma unroll
  for (int j = 0; j < MT; j++) xp[j] = a.xq + (int64_t)min(16 * j + l16, a.M - 1) * a.KP + 16 * lq;
  // the wave's steps of 64 codes, two at least
  const int steps = a.KP / 64, per = ((steps / 2 + KNT / 64 - 1) / (KNT / 64)) * 2;
  const int s0 = wave * per, s1 = min(s0 + per, steps);
  v4i acc[RN][MT] = {};
  for (int s = s0; s < s1; s += U) {
    v4i wv[U][RN], xv[U][MT];
#pragma unroll
    for (int u = 0; u < U; u++) {
      const int k = 64 * min(s + u, s1 - 1);
#pragma unroll
      for (int i = 0; i < RN; i++) wv[u][i] = *reinterpret_cast<const v4i *>(wp[i] + k);
#pragma unroll
      for (int j = 0; j < MT; j++) xv[u][j] = *reinterpret_cast<const v4i *>(xp[j] + k);
    }
#pragma unroll
    for (int u = 0; u < U; u++) {
      if (u > 0 && s + u >= s1) break;
#pragma unroll
      for (int i = 0; i < RN; i++)
#pragma unroll
        for (int j = 0; j < MT; j++)
          acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[u][i], xv[u][j], acc[i][j], 0, 0, 0);
    }
  }
  __syncthreads();
  if (s0 < s1)
#pragma unroll
    for (int i = 0; i < RN; i++)
#pragma unroll
      for (int j = 0; j < MT; j++)
#pragma unroll
        for (int e = 0; e < 4; e++) atomicAdd(&o[(16 * j + l16) * OS + 16 * i + 4 * lq + e], acc[i][j][e]);
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * MT * 4 * RN; i += KNT) {
    const int m = i / (4 * RN), c = 4 * (i % (4 * RN)), n = n0 + c;
    if (m < a.M && n < a.N)
      put4(a, m, n, *reinterpret_cast<const v4i *>(&o[m * OS + c]), a.xd[m], load_channels(a, a.wd, n),
           a.bias ? load_channels(a, a.bias, n) : v4f{0.f, 0.f, 0.f, 0.f});
  }
}

template <int TN, int TM, int WN, int WM, int NS>
int launch_tiles(QArgs a, hipStream_t s) {
  a.nt = (a.N + TN - 1) / TN;
  a.mt = (a.M + TM - 1) / TM;
  q8_tile_kernel<TN, TM, WN, WM, NS><<<dim3((unsigned)(a.nt * a.mt)), dim3(64 * WN * WM), 0, s>>>(a);
  return check_launch();
}

template <int MT, int RN>
int launch_few(const QArgs &a, hipStream_t s) {
  q8_few_kernel<MT, RN><<<dim3((a.N + 16 * RN - 1) / (16 * RN)), dim3(KNT), 0, s>>>(a);
  return check_launch();
}

inline bool aligned4(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
constexpr int64_t KTOP = (int64_t)1 << 17, TOP = (int64_t)1 << 31;

}  // namespace

}  // namespace w4a8

using namespace w4a8;

extern "C" size_t q8_row_bytes(int64_t K) {
  return K < 1 || K >= KTOP ? 0 : (size_t)((K + PAD - 1) / PAD * PAD);
}

extern "C" int q8_row_quantize(const float *x, int64_t x_stride, int8_t *q, float *d, int64_t rows,
                               int64_t K, void *stream) {
  if (rows < 0 || K < 1 || x_stride < K) return W4A8_ESHAPE;
  if (K >= KTOP || rows >= (1 << 24) || x_stride >= TOP) return W4A8_ERANGE;
  if (!x || !q || !d) return W4A8_ENULL;
  if (!aligned4(x) || !aligned16(q) || !aligned4(d)) return W4A8_EALIGN;
  if (rows == 0) return W4A8_OK;
  if (int rc = check_device(); rc != W4A8_OK) return rc;
  const int KP = (int)q8_row_bytes(K);
  const dim3 grid((unsigned)rows), nt(QNT);
  hipStream_t s = as_stream(stream);
  const bool vec = K % 4 == 0 && x_stride % 4 == 0 && aligned16(x);
  if (vec && K <= 4 * QNT)
    q8_row_kernel<1><<<grid, nt, 0, s>>>(x, x_stride, q, d, (int)K, KP);
  else if (vec && K <= 8 * QNT)
    q8_row_kernel<2><<<grid, nt, 0, s>>>(x, x_stride, q, d, (int)K, KP);
  else if (vec && K <= 16 * QNT)
    q8_row_kernel<4><<<grid, nt, 0, s>>>(x, x_stride, q, d, (int)K, KP);
  else if (vec && K <= 32 * QNT)
    q8_row_kernel<8><<<grid, nt, 0, s>>>(x, x_stride, q, d, (int)K, KP);
  else
    q8_any_row_kernel<<<grid, nt, 0, s>>>(x, x_stride, q, d, (int)K, KP);
  return check_launch();
}

extern "C" int q8q8_gemm(const int8_t *xq, const float *xd, const int8_t *wq, const float *wd,
                         const float *bias, float *y, int64_t y_stride, int64_t M, int64_t N,
                         int64_t K, void *stream) {
  if (M < 0 || N < 1 || K < 1 || y_stride < N) return W4A8_ESHAPE;
  // (a grid's threads are counted in 32 bits)
  if (K >= KTOP || M >= (1 << 26) || N >= (1 << 26) || y_stride >= TOP || ((M + 63) / 64) * ((N + 63) / 64) >= (1 << 23))
    return W4A8_ERANGE;
  if (!xq || !xd || !wq || !wd || !y) return W4A8_ENULL;
  if (!aligned16(xq) || !aligned16(wq) || !aligned4(xd) || !aligned4(wd) || !aligned4(bias) || !aligned4(y))
    return W4A8_EALIGN;
  for (const void *p : {(const void *)xq, (const void *)xd, (const void *)wq, (const void *)wd, (const void *)bias})
    if (p == y) return W4A8_EALIAS;
  if (M == 0) return W4A8_OK;
  if (int rc = check_device(); rc != W4A8_OK) return rc;
  QArgs a{xq, wq, xd, wd, bias, y, y_stride, (int)M, (int)N, (int)q8_row_bytes(K), 0, 0,
          y_stride % 4 == 0 && aligned16(y)};
  hipStream_t s = as_stream(stream);
  switch (q8_way(M, N, device_cus())) {
    case Q8_FEW_1x1: return launch_few<1, 1>(a, s);
    case Q8_FEW_1x2: return launch_few<1, 2>(a, s);
    case Q8_FEW_2x1: return launch_few<2, 1>(a, s);
    case Q8_FEW_3x1: return launch_few<3, 1>(a, s);
    case Q8_FEW_4x1: return launch_few<4, 1>(a, s);
    case Q8_256x256: return launch_tiles<256, 256, 2, 4, 4>(a, s);
    case Q8_256x128: return launch_tiles<256, 128, 2, 2, 3>(a, s);
    case Q8_128x128: return launch_tiles<128, 128, 2, 2, 4>(a, s);
    case Q8_128x64: return launch_tiles<128, 64, 2, 2, 4>(a, s);
    default: return launch_tiles<64, 64, 2, 2, 4>(a, s);
  }
}
