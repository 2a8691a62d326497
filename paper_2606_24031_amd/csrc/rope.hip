// Rotary positions (the softmax-attention blocks of Sec. 2.2; the paper does
// not spell its positions out, so this is the standard rotary embedding):
// the frequency table and the rotation of rows of heads.
#include <algorithm>
#include <cmath>

#include "rope_dev.h"
#include "w4a8_host.h"

namespace w4a8 {

namespace {

constexpr int RT = 256;

// inv_freq[i] = base^(-2i / n), scaled (see w4a8.h).
__global__ void frequencies_kernel(double *__restrict__ f, int half, double base, int kind,
                                   double factor, double lo, double hi) {
  const int i = blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= half) return;
  const double v = pow(base, -2.0 * (double)i / (double)(2 * half));
  double w = v;
  if (kind == W4A8_ROPE_LINEAR) w = v / factor;
  if (kind == W4A8_ROPE_PARTS) {
    double m = ((double)i - lo) / fmax(hi - lo, 0.001);
    m = fmin(fmax(m, 0.0), 1.0);
    w = v * (1.0 - m) + v / factor * m;
  }
  f[i] = w;
}

// Workgroup (x, y): rows x * rows .. + rows - 1, heads y * heads .. + heads - 1.
// Bound by HBM for a prompt (8 bytes an element; the fp64 work of a row's
// cosines is shared by its heads): 5120 rows of 32 heads of 128 in 35 us, 4.8
// TB/s, as a copy.  One row takes 3 us, the launch and the loads of the position
// and the frequencies.
__global__ __launch_bounds__(RT) void rope_kernel(RopeArgs r, const float *x, int64_t xs, float *y,
                                                  int64_t ys, int64_t T, int NH, int D, int rows,
                                                  int heads) {
  __shared__ double2 cs[ROPE_PAIRS];
  const int h0 = blockIdx.y * heads, nh = min(heads, NH - h0);
  const RopeUnits ru(r.half, r.interleaved, D);
  const int per = nh * ru.units;
  for (int64_t t0 = (int64_t)blockIdx.x * rows; t0 < T; t0 += (int64_t)gridDim.x * rows) {
    const int n = (int)min((int64_t)rows, T - t0);
    rope_table(r, cs, t0, n);
    __syncthreads();
    for (int i = threadIdx.x; i < n * per; i += RT) {
      const int row = i / per, k = i - row * per;
      const int h = k / ru.units, u = k - h * ru.units;
      const int64_t t = t0 + row;
      rope_unit(r, ru, x + t * xs + (int64_t)(h0 + h) * D, y + t * ys + (int64_t)(h0 + h) * D,
                cs + row * r.half, u);
    }
    __syncthreads();
  }
}

}  // namespace

int rope_check(const w4a8_rope *rope, int64_t D) {
  if (!rope->inv_freq || !rope->pos) return W4A8_ENULL;
  if (rope->n_rot < 2 || rope->n_rot % 2 != 0 || rope->n_rot > D ||
      (rope->layout != W4A8_ROPE_HALF && rope->layout != W4A8_ROPE_INTERLEAVED) ||
      !std::isfinite(rope->mscale))
    return W4A8_ESHAPE;
  if ((reinterpret_cast<uintptr_t>(rope->inv_freq) & 7u) ||
      (reinterpret_cast<uintptr_t>(rope->pos) & 3u))
    return W4A8_EALIGN;
  return W4A8_OK;
}

}  // namespace w4a8

using namespace w4a8;

extern "C" int rope_frequencies(double *inv_freq, int64_t n_rot, double base, int kind,
                                double factor, double orig_len, double beta_fast,
                                double beta_slow, void *stream) {
  if (!inv_freq) return W4A8_ENULL;
  if (n_rot < 2 || n_rot % 2 != 0 || !std::isfinite(base) || !(base > 1.0)) return W4A8_ESHAPE;
  if (kind != W4A8_ROPE_PLAIN && kind != W4A8_ROPE_LINEAR && kind != W4A8_ROPE_PARTS)
    return W4A8_ESHAPE;
  if (kind != W4A8_ROPE_PLAIN && (!std::isfinite(factor) || !(factor > 0.0))) return W4A8_ESHAPE;
  double lo = 0.0, hi = 0.0;
  if (kind == W4A8_ROPE_PARTS) {
    if (!std::isfinite(orig_len) || !std::isfinite(beta_fast) || !(orig_len > 0.0) ||
        !(beta_slow > 0.0) || !(beta_fast >= beta_slow))
      return W4A8_ESHAPE;
    const double n = (double)n_rot;
    const auto pair = [&](double turns) {
      return n * std::log(orig_len / (turns * 2.0 * M_PI)) / (2.0 * std::log(base));
    };
    lo = std::fmax(0.0, std::floor(pair(beta_fast)));
    hi = std::fmin(n - 1.0, std::ceil(pair(beta_slow)));
  }
  if (n_rot > 1024) return W4A8_ERANGE;
  if (reinterpret_cast<uintptr_t>(inv_freq) & 7u) return W4A8_EALIGN;
  if (int rc = check_device(); rc != W4A8_OK) return rc;
  const int half = (int)(n_rot / 2);
  frequencies_kernel<<<dim3((half + 63) / 64), dim3(64), 0, as_stream(stream)>>>(
      inv_freq, half, base, kind, factor, lo, hi);
  return check_launch();
}

extern "C" int rope_rotate(const w4a8_rope *rope, const float *x, int64_t x_stride, float *out,
                           int64_t out_stride, int64_t T, int64_t NH, int64_t D, void *stream) {
  if (!rope || !x || !out) return W4A8_ENULL;
  if (D < 4 || D % 4 != 0 || NH < 1 || T < 0) return W4A8_ESHAPE;
  if (D > 1024 || NH >= (1 << 16) || T >= ((int64_t)1 << 31)) return W4A8_ERANGE;
  if (int rc = rope_check(rope, D); rc != W4A8_OK) return rc;
  if (x_stride < NH * D || out_stride < NH * D || x_stride % 4 != 0 || out_stride % 4 != 0)
    return W4A8_ESHAPE;
  if (x_stride >= ((int64_t)1 << 31) || out_stride >= ((int64_t)1 << 31)) return W4A8_ERANGE;
  if (!aligned16(x) || !aligned16(out)) return W4A8_EALIGN;
  if (x == out && x_stride != out_stride) return W4A8_EALIAS;
  if (T == 0) return W4A8_OK;
  int cus = 0;
  if (int rc = check_device(&cus); rc != W4A8_OK) return rc;
  const RopeArgs r = rope_args(rope);
  const RopeUnits ru(r.half, r.interleaved, (int)D);
  // A row's units on one workgroup, so its cosines are taken once; a few rows
  // to a workgroup where a row is short, and while rows are fewer than compute
  // units a row's heads over several workgroups.
  int rows = 1, heads = (int)NH;
  while (rows * 2 * (int64_t)NH * ru.units <= 4 * RT && rows * 2 * r.half <= ROPE_PAIRS &&
         T / (rows * 2) >= 2 * cus)
    rows *= 2;
  while (heads > 1 && (int64_t)heads * ru.units > RT && T * ((NH + heads - 1) / heads) < cus)
    heads = (heads + 1) / 2;
  const int64_t gx = std::min<int64_t>((T + rows - 1) / rows, 1 << 22);
  rope_kernel<<<dim3((unsigned)gx, (unsigned)((NH + heads - 1) / heads)), dim3(RT), 0,
                as_stream(stream)>>>(r, x, x_stride, out, out_stride, T, (int)NH, (int)D, rows,
                                     heads);
  return check_launch();
}
