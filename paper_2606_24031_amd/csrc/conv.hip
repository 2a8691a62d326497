// The short causal convolution in front of a recurrence: per channel the W
// last rows' products with W weights, a bias, SiLU; rows before a sequence's
// first come from its state, which is left as the last W - 1 inputs.
//
// A wave takes 256 neighbouring channels (16 bytes a lane) of a run of rows,
// the W - 1 rows before in registers.  A row belongs to its own run, but a
// sequence's first W - 1 rows to the run of its first: so one wave reads a
// sequence's state, and that wave writes the new one, which may stand in the
// same slot.
//
// Bound by memory: 5393 rows of 12288 channels (530 MB read and written) 103 to 108
// us, 5.0 TB/s, what a large copy reaches; the rows before a run are read again,
// from the L2 cache.  A decode batch is a chain of launch, the plan, state and row:
// 32 requests of 4352 channels 4.1 us (20 with 16 rows a run).
#include "seq_dev.h"
#include "w4a8_dev.h"

namespace w4a8 {

namespace {

constexpr int CNT = 256;            // threads: four waves, a run of rows each

typedef float v4f __attribute__((ext_vector_type(4)));

struct ConvArgs {
  Seqs q;
  const float *x, *w, *bias;
  float *state, *out;
  int64_t xs, os;
  int CH, R, nx;                    // channels, rows of a run, groups of 256 channels
};

__device__ __forceinline__ v4f fma4(v4f a, v4f b, v4f c) {
  return v4f{fmaf(a.x, b.x, c.x), fmaf(a.y, b.y, c.y), fmaf(a.z, b.z, c.z), fmaf(a.w, b.w, c.w)};
}

template <int W, bool SILU>
__global__ __launch_bounds__(CNT) void conv_kernel(ConvArgs a) {
  constexpr int H = W - 1;          // rows of history
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const int64_t run = (int64_t)(blockIdx.x / a.nx) * (CNT / 64) + wave;
  const int c = (int)(blockIdx.x % a.nx) * 256 + 4 * lane;
  if (run * a.R >= a.q.T || c >= a.CH) return;
  const int r0 = (int)(run * a.R), r1 = (int)min(run * a.R + a.R, (int64_t)a.q.T);
  v4f w[W];
#pragma unroll
  for (int i = 0; i < W; i++) w[i] = *reinterpret_cast<const v4f *>(a.w + (int64_t)i * a.CH + c);
  const v4f bias = a.bias ? *reinterpret_cast<const v4f *>(a.bias + c) : v4f{0.f, 0.f, 0.f, 0.f};
  const auto row = [&](int t) { return *reinterpret_cast<const v4f *>(a.x + t * a.xs + c); };

  for (int b = max(seq_of(a.q, r0), 0); b < a.q.B; b++) {
    const int begin = seq_begin(a.q, b), end = seq_begin(a.q, b + 1);
    if (begin >= r1) break;
    // the rows of b that are this run's
    const bool mine = begin >= r0;
    int t = mine ? begin : max(r0, begin + H);
    const int stop = min(end, mine ? max(r1, begin + H) : r1);
    if (t >= stop) continue;
    v4f h[H];
    if (mine) {
      const int64_t src = seq_src(a.q, b), dst = seq_dst(a.q, b);
#pragma unroll
      for (int k = 0; k < H; k++)
        h[k] = src < 0 ? v4f{0.f, 0.f, 0.f, 0.f}
                       : *reinterpret_cast<const v4f *>(a.state + (src * H + k) * a.CH + c);
      if (dst >= 0) {
        // the last H of the old state and the rows
        const int n = end - begin;
#pragma unroll
        for (int k = 0; k < H; k++) {
          v4f s = row(max(end - H + k, begin));
#pragma unroll
          for (int m = k + 1; m < H; m++)
            if (k + n == m) s = h[m];
          *reinterpret_cast<v4f *>(a.state + (dst * H + k) * a.CH + c) = s;
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < H; k++) h[k] = row(t - H + k);
    }
    for (; t < stop; t++) {
      const v4f x = row(t);
      v4f y = w[0] * h[0];
#pragma unroll
      for (int k = 1; k < H; k++) y = fma4(w[k], h[k], y);
      y = fma4(w[H], x, y) + bias;
      if (SILU) y = v4f{silu_f32(y.x), silu_f32(y.y), silu_f32(y.z), silu_f32(y.w)};
      *reinterpret_cast<v4f *>(a.out + t * a.os + c) = y;
#pragma unroll
      for (int k = 0; k + 1 < H; k++) h[k] = h[k + 1];
      h[H - 1] = x;
    }
  }
}

template <int W>
int launch_conv(const ConvArgs &a, bool silu, unsigned grid, hipStream_t s) {
  if (silu)
    conv_kernel<W, true><<<dim3(grid), dim3(CNT), 0, s>>>(a);
  else
    conv_kernel<W, false><<<dim3(grid), dim3(CNT), 0, s>>>(a);
  return check_launch();
}

}  // namespace

}  // namespace w4a8

extern "C" int short_conv(const w4a8_seqs *seqs, const float *x, int64_t x_stride, const float *w,
                          const float *bias, float *state, float *out, int64_t out_stride, int64_t T,
                          int64_t CH, int64_t W, int32_t act, void *stream) {
  using namespace w4a8;
  int rc = seqs_sizes(seqs, T);
  if (rc != W4A8_OK) return rc;
  if (CH < 4 || CH % 4 != 0 || W < 2 || W > 4 || (act != W4A8_CONV_NONE && act != W4A8_CONV_SILU) ||
      x_stride < CH || x_stride % 4 != 0 || out_stride < CH || out_stride % 4 != 0)
    return W4A8_ESHAPE;
  if (CH >= (1 << 24) || x_stride >= ((int64_t)1 << 31) || out_stride >= ((int64_t)1 << 31) ||
      T * CH >= ((int64_t)1 << 40))
    return W4A8_ERANGE;
  if (!x || !w || !out || (seqs->n_slots > 0 && !state)) return W4A8_ENULL;
  if ((rc = seqs_pointers(seqs)) != W4A8_OK) return rc;
  if (!aligned16(x) || !aligned16(w) || !aligned16(bias) || !aligned16(state) || !aligned16(out))
    return W4A8_EALIGN;
  if (out == x || state == x || state == out) return W4A8_EALIAS;
  if (T == 0 || seqs->B == 0) return W4A8_OK;
  if ((rc = check_device()) != W4A8_OK) return rc;
  ConvArgs a{};
  a.q = seqs_args(seqs, T);
  a.x = x; a.w = w; a.bias = bias; a.state = state; a.out = out;
  a.xs = x_stride; a.os = out_stride; a.CH = (int)CH;
  a.nx = (int)((CH + 255) / 256);
  // Runs of 16 rows, fewer while the call would leave a compute unit fewer than 32
  // waves, so that a decode batch's sequences are not taken one behind the other;
  // more where the grid would be too large (its threads are counted in 32 bits).
  int64_t grid, R = 16;
  while (R > 1 && a.nx * T < 32 * R * device_cus()) R /= 2;
  for (;; R *= 2) {
    grid = a.nx * ((T + R * (CNT / 64) - 1) / (R * (CNT / 64)));
    if (grid < (1 << 23)) break;
  }
  a.R = (int)R;
  const bool silu = act == W4A8_CONV_SILU;
  hipStream_t s = as_stream(stream);
  return W == 2   ? launch_conv<2>(a, silu, (unsigned)grid, s)
         : W == 3 ? launch_conv<3>(a, silu, (unsigned)grid, s)
                  : launch_conv<4>(a, silu, (unsigned)grid, s);
}
