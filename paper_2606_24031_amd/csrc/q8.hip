// 8-bit rows: int8 codes with one fp32 scale a row (the quantizer), and the
// product of activation rows with weight rows in exact int32 sums.
#include "w4a8_dev.h"
#include "w4a8_host.h"

namespace w4a8 {

namespace {

constexpr int QNT = 256;            // threads of a quantizing workgroup: one row
constexpr int TNT = 256;            // ... of a product tile: four waves
constexpr int PAD = W4A8_Q8_ROW_PAD;

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));

// One row a workgroup: its largest magnitude, then the codes, four a thread.
__global__ __launch_bounds__(QNT) void q8_row_kernel(const float *__restrict__ x, int64_t xs,
                                                     int8_t *__restrict__ q, float *__restrict__ d,
                                                     int K, int KP) {
  __shared__ float top[QNT / 64];
  __shared__ int bad[QNT / 64];
  const int64_t r = blockIdx.x;
  const float *xr = x + r * xs;
  float amax = 0.0f;
  int odd = 0;                      // a NaN or an infinity
  for (int k = threadIdx.x; k < K; k += QNT) {
    const float v = fabsf(xr[k]);
    odd |= !(v < __builtin_inff());
    amax = fmaxf(amax, v);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    amax = fmaxf(amax, __shfl_xor(amax, o));
    odd |= __shfl_xor(odd, o);
  }
  if ((threadIdx.x & 63) == 0) { top[threadIdx.x >> 6] = amax; bad[threadIdx.x >> 6] = odd; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < QNT / 64; w++) { amax = fmaxf(amax, top[w]); odd |= bad[w]; }
  const float dr = odd ? __builtin_nanf("") : amax * (1.0f / 127.0f);
  const float id = odd ? 0.0f : sym_inverse(dr);
  if (threadIdx.x == 0) d[r] = dr;
  for (int k = 4 * threadIdx.x; k < KP; k += 4 * QNT) {
    uint32_t packed = 0;
#pragma unroll
    for (int i = 0; i < 4; i++)
      if (k + i < K && !odd) packed |= ((uint32_t)round_clamp(xr[k + i] * id, 127) & 0xFFu) << (8 * i);
    *reinterpret_cast<uint32_t *>(q + r * KP + k) = packed;
  }
}

struct QArgs {
  const int8_t *xq, *wq;
  const float *xd, *wd, *bias;
  float *y;
  int64_t ys, M, N;
  int KP, nt;                       // bytes of a row; tiles of 64 channels
};

// 64 rows by 64 channels a workgroup, 32 x 32 a wave, operands straight from
// memory: the weights are the A operand, so a lane holds four neighbouring
// channels of one row.
__global__ __launch_bounds__(TNT) void q8_tile_kernel(QArgs a) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, l16 = lane & 15, lq = lane >> 4;
  const int64_t n0 = (int64_t)(blockIdx.x % a.nt) * 64 + 32 * (wave & 1);
  const int64_t m0 = (int64_t)(blockIdx.x / a.nt) * 64 + 32 * (wave >> 1);
  const int8_t *wp[2], *xp[2];
#pragma unroll
  for (int i = 0; i < 2; i++) {
    wp[i] = a.wq + min(n0 + 16 * i + l16, a.N - 1) * a.KP + 16 * lq;
    xp[i] = a.xq + min(m0 + 16 * i + l16, a.M - 1) * a.KP + 16 * lq;
  }
  v4i acc[2][2] = {};
  for (int k = 0; k < a.KP; k += 64) {
    v4i wv[2], xv[2];
#pragma unroll
    for (int i = 0; i < 2; i++) {
      wv[i] = *reinterpret_cast<const v4i *>(wp[i] + k);
      xv[i] = *reinterpret_cast<const v4i *>(xp[i] + k);
    }
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
      for (int j = 0; j < 2; j++)
        acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(wv[i], xv[j], acc[i][j], 0, 0, 0);
  }
#pragma unroll
  for (int j = 0; j < 2; j++) {
    const int64_t m = m0 + 16 * j + l16;
    if (m >= a.M) continue;
    const float xd = a.xd[m];
#pragma unroll
    for (int i = 0; i < 2; i++)
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int64_t n = n0 + 16 * i + 4 * lq + e;
        if (n >= a.N) continue;
        float y = (float)acc[i][j][e] * (xd * a.wd[n]);
        if (a.bias) y += a.bias[n];
        a.y[m * a.ys + n] = y;
      }
  }
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
  if (K >= KTOP || rows >= TOP || x_stride >= TOP) return W4A8_ERANGE;
  if (!x || !q || !d) return W4A8_ENULL;
  if (!aligned4(x) || !aligned16(q) || !aligned4(d)) return W4A8_EALIGN;
  if (rows == 0) return W4A8_OK;
  if (int rc = check_device(); rc != W4A8_OK) return rc;
  q8_row_kernel<<<dim3((unsigned)rows), dim3(QNT), 0, as_stream(stream)>>>(x, x_stride, q, d, (int)K,
                                                                         (int)q8_row_bytes(K));
  return check_launch();
}

extern "C" int q8q8_gemm(const int8_t *xq, const float *xd, const int8_t *wq, const float *wd,
                         const float *bias, float *y, int64_t y_stride, int64_t M, int64_t N,
                         int64_t K, void *stream) {
  if (M < 0 || N < 1 || K < 1 || y_stride < N) return W4A8_ESHAPE;
  if (K >= KTOP || M >= TOP || N >= TOP || y_stride >= TOP) return W4A8_ERANGE;
  const int64_t nt = (N + 63) / 64, mt = (M + 63) / 64;
  if (nt * mt >= (1 << 23)) return W4A8_ERANGE;
  if (!xq || !xd || !wq || !wd || !y) return W4A8_ENULL;
  if (!aligned16(xq) || !aligned16(wq) || !aligned4(xd) || !aligned4(wd) || !aligned4(bias) || !aligned4(y))
    return W4A8_EALIGN;
  for (const void *p : {(const void *)xq, (const void *)xd, (const void *)wq, (const void *)wd, (const void *)bias})
    if (p == y) return W4A8_EALIAS;
  if (M == 0) return W4A8_OK;
  if (int rc = check_device(); rc != W4A8_OK) return rc;
  QArgs a{xq, wq, xd, wd, bias, y, y_stride, M, N, (int)q8_row_bytes(K), (int)nt};
  q8_tile_kernel<<<dim3((unsigned)(nt * mt)), dim3(TNT), 0, as_stream(stream)>>>(a);
  return check_launch();
}
