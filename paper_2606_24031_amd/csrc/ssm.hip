// The selective state space scan: per head h and row t of a sequence
//   S_t = exp(d_t A) S_{t-1} + d_t B_t x_t^T,   y_t = C_t^T S_t + D x_t
// with S in R^{N x P}, d_t the row's step (softplus of a projection), B and C
// shared by the heads of a group, y gated by SiLU(z).
#include "seq_dev.h"
#include "w4a8_dev.h"

namespace w4a8 {

namespace {

constexpr int SC = 64;              // rows of a chunk
constexpr int STEP_NT = 256;        // threads of a step workgroup

typedef float v4f __attribute__((ext_vector_type(4)));

struct ScanArgs {
  Seqs q;
  const float *x, *dt, *b, *c, *z, *A, *D, *bias;
  float *state, *y;
  int64_t xs, ds, bs, cs, zs, ys;
  int NH, G, NG, P, nsl;            // heads, heads of a group, groups, columns, slices of columns
  int softplus;
};

// The step of a row: dt + bias, and log(1 + exp(.)) of it.
__device__ __forceinline__ float step_of(float dt, float bias, int softplus) {
  const float v = dt + bias;
  return softplus ? fmaxf(v, 0.0f) + log1pf(expf(-fabsf(v))) : v;
}

// One sequence's rows for COLS columns of a head, the recurrence as written.
// A lane holds four columns of every RG-th row of S, in registers from the
// first row of the sequence to its last.
template <int N, int COLS, int NT>
__device__ __forceinline__ void step_rows(const ScanArgs &a, int b, int h, int c0, int begin, int end,
                                          float (*red)[COLS]) {
  constexpr int CL = COLS / 4, RG = NT / CL, RPT = N / RG;
  static_assert(RPT >= 1 && RPT * RG == N && CL <= 64, "rows of S over the threads");
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int c = c0 + 4 * (tid % CL), r0 = tid / CL;
  const bool live = c < a.P;
  const int64_t src = seq_src(a.q, b), dst = seq_dst(a.q, b);
  const float A = a.A[h], bias = a.bias ? a.bias[h] : 0.0f, D = a.D ? a.D[h] : 0.0f;
  const int g = h / a.G;
  v4f S[RPT];
#pragma unroll
  for (int m = 0; m < RPT; m++)
    S[m] = src >= 0 && live
               ? *reinterpret_cast<const v4f *>(a.state + ((src * a.NH + h) * N + r0 + RG * m) * a.P + c)
               : v4f{0.f, 0.f, 0.f, 0.f};
  for (int t = begin; t < end; t++) {
    const float *bt = a.b + t * a.bs + (int64_t)g * N, *ct = a.c + t * a.cs + (int64_t)g * N;
    const v4f x = live ? *reinterpret_cast<const v4f *>(a.x + t * a.xs + (int64_t)h * a.P + c)
                       : v4f{0.f, 0.f, 0.f, 0.f};
    const float d = step_of(a.dt[t * a.ds + h], bias, a.softplus);
    const float keep = expf(d * A);
    const v4f dx = d * x;
    v4f y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int m = 0; m < RPT; m++) {
      const float bn = bt[r0 + RG * m], cn = ct[r0 + RG * m];
#pragma unroll
      for (int e = 0; e < 4; e++) {
        S[m][e] = fmaf(keep, S[m][e], bn * dx[e]);
        y[e] = fmaf(cn, S[m][e], y[e]);
      }
    }
#pragma unroll
    for (int o = CL; o < 64; o <<= 1)
#pragma unroll
      for (int e = 0; e < 4; e++) y[e] += __shfl_xor(y[e], o);
    if (lane < CL) *reinterpret_cast<v4f *>(&red[wave][4 * lane]) = y;
    __syncthreads();
    if (tid < CL && live) {
      v4f s = D * x;
#pragma unroll
      for (int w = 0; w < NT / 64; w++) s += *reinterpret_cast<const v4f *>(&red[w][4 * tid]);
      if (a.z) {
        const v4f z = *reinterpret_cast<const v4f *>(a.z + t * a.zs + (int64_t)h * a.P + c);
        s *= v4f{silu_f32(z.x), silu_f32(z.y), silu_f32(z.z), silu_f32(z.w)};
      }
      *reinterpret_cast<v4f *>(a.y + t * a.ys + (int64_t)h * a.P + c) = s;
    }
    __syncthreads();                // red is rewritten for the next row
  }
  if (dst >= 0 && live)
#pragma unroll
    for (int m = 0; m < RPT; m++)
      *reinterpret_cast<v4f *>(a.state + ((dst * a.NH + h) * N + r0 + RG * m) * a.P + c) = S[m];
}

template <int N, int COLS>
__global__ __launch_bounds__(STEP_NT) void step_kernel(ScanArgs a) {
  __shared__ __align__(16) float red[STEP_NT / 64][COLS];
  const int sl = blockIdx.x % a.nsl, bh = blockIdx.x / a.nsl, h = bh % a.NH, b = bh / a.NH;
  const int begin = seq_begin(a.q, b), end = seq_begin(a.q, b + 1);
  if (begin >= end) return;
  step_rows<N, COLS, STEP_NT>(a, b, h, sl * COLS, begin, end, red);
}

int ssm_sizes(const w4a8_seqs *q, const w4a8_ssm *m, int64_t T) {
  if (!m) return W4A8_ENULL;
  int rc = seqs_sizes(q, T);
  if (rc != W4A8_OK) return rc;
  if (m->NH < 1 || m->NG < 1 || m->NH % m->NG != 0 || (m->N != 64 && m->N != 128 && m->N != 256) ||
      m->P < 16 || m->P % 16 != 0)
    return W4A8_ESHAPE;
  // (a grid's threads are counted in 32 bits)
  if (m->NH >= (1 << 16) || m->P > 4096 || q->B * m->NH * m->P >= ((int64_t)1 << 27) ||
      (T / SC + q->B + 1) * m->NG >= ((int64_t)1 << 23))
    return W4A8_ERANGE;
  return W4A8_OK;
}

template <int N>
int launch_ssm(ScanArgs a, hipStream_t s) {
  a.nsl = (a.P + 63) / 64;
  step_kernel<N, 64><<<dim3((unsigned)(a.q.B * a.NH * a.nsl)), dim3(STEP_NT), 0, s>>>(a);
  return check_launch();
}

}  // namespace

}  // namespace w4a8

using namespace w4a8;

extern "C" size_t ssm_workspace_size(const w4a8_seqs *seqs, const w4a8_ssm *ssm, int64_t T) {
  if (ssm_sizes(seqs, ssm, T) != W4A8_OK) return 0;
  return 256;
}

extern "C" int ssm_scan(const w4a8_seqs *seqs, const w4a8_ssm *m, float *state, float *y,
                        int64_t y_stride, int64_t T, void *workspace, size_t ws_bytes, void *stream) {
  int rc = ssm_sizes(seqs, m, T);
  if (rc != W4A8_OK) return rc;
  const int64_t xrow = m->NH * m->P, brow = m->NG * m->N, top = (int64_t)1 << 31;
  if (m->x_stride < xrow || m->x_stride % 4 != 0 || m->b_stride < brow || m->b_stride % 4 != 0 ||
      m->c_stride < brow || m->c_stride % 4 != 0 || m->dt_stride < m->NH || y_stride < xrow ||
      y_stride % 4 != 0 || (m->z && (m->z_stride < xrow || m->z_stride % 4 != 0)))
    return W4A8_ESHAPE;
  if (m->x_stride >= top || m->b_stride >= top || m->c_stride >= top || m->dt_stride >= top ||
      y_stride >= top || (m->z && m->z_stride >= top))
    return W4A8_ERANGE;
  if (!m->x || !m->dt || !m->b || !m->c || !m->A || !y || !workspace || (seqs->n_slots > 0 && !state))
    return W4A8_ENULL;
  if ((rc = seqs_pointers(seqs)) != W4A8_OK) return rc;
  if (!aligned16(m->x) || !aligned16(m->b) || !aligned16(m->c) || !aligned16(m->z) || !aligned16(y) ||
      !aligned16(state) || !aligned16(workspace) || !aligned4(m->dt) || !aligned4(m->A) ||
      !aligned4(m->D) || !aligned4(m->dt_bias))
    return W4A8_EALIGN;
  for (const float *p : {m->x, m->dt, m->b, m->c, m->z, m->A, m->D, m->dt_bias})
    if (p && (p == y || p == state)) return W4A8_EALIAS;
  if (y == state) return W4A8_EALIAS;
  if (ws_bytes < ssm_workspace_size(seqs, m, T)) return W4A8_EWORKSPACE;
  if (T == 0 || seqs->B == 0) return W4A8_OK;
  if ((rc = check_device()) != W4A8_OK) return rc;
  ScanArgs a{};
  a.q = seqs_args(seqs, T);
  a.x = m->x; a.dt = m->dt; a.b = m->b; a.c = m->c; a.z = m->z;
  a.A = m->A; a.D = m->D; a.bias = m->dt_bias;
  a.state = state; a.y = y;
  a.xs = m->x_stride; a.ds = m->dt_stride; a.bs = m->b_stride; a.cs = m->c_stride;
  a.zs = m->z_stride; a.ys = y_stride;
  a.NH = (int)m->NH; a.NG = (int)m->NG; a.G = (int)(m->NH / m->NG); a.P = (int)m->P;
  a.softplus = m->softplus;
  hipStream_t s = as_stream(stream);
  return m->N == 64 ? launch_ssm<64>(a, s) : m->N == 128 ? launch_ssm<128>(a, s) : launch_ssm<256>(a, s);
}
