// The selective state space scan: per head h and row t of a sequence
//   S_t = exp(d_t A) S_{t-1} + d_t B_t x_t^T,   y_t = C_t^T S_t + D x_t
// with S in R^{N x P}, d_t the row's step (softplus of a projection), B and C
// shared by the heads of a group, y gated by SiLU(z).
//
// Short sequences go row by row (step): the state is read and written once, 48
// sequences of one row, 64 heads of 128 x 64: 32 to 42 us, 4.8 to 6.3 TB/s; one
// sequence 4.6 us, a chain of launch, plan, state and the join.
// Others go by chunks of 64 rows, two launches: what does not wait for the chunk
// before (prep: C B^T, decays, operands in the products' order), then a workgroup
// per head and slice of columns with the chunks in order (scan), the state in the
// accumulators of fp32 matrix products.  All arithmetic is fp32 (products of rounded
// halves would be off by more than the rest together), so the products' rate, a
// 16th of bf16's, is a bound: a chunk's products of a 16-column
// slice take 2370 cycles of each SIMD; a step takes 4500: the products do not overlap
// with the SIMD's other work (1350 cycles: decays, addresses, the gate), and about 90
// KB a step come from the L2 caches (14 TB/s in all).  16384 rows, 64 heads of 64:
// 525 us and 21 for prep (256 at the products' rate, 164 for the bytes); the
// 947-token prompt of 32 heads of 128: 35 and 8.
#include "choice.h"
#include "seq_dev.h"
#include "w4a8_dev.h"

namespace w4a8 {

namespace {

constexpr int SC = SSM_CHUNK;
constexpr int SNT = 512;            // threads of a scan workgroup: eight waves
constexpr int STEP_NT = 256;        // ... of a step workgroup

typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));

struct ScanArgs {
  Seqs q;
  const float *x, *dt, *b, *c, *z, *A, *D, *bias;
  float *state, *y, *gram, *dec;    // gram, dec and
  int4 *order;                      // order: the workspace
  int xs, ds, bs, cs, zs, ys;       // strides
  int NH, G, NG, P, nsl;            // heads, heads of a group, groups, columns, slices of columns
  int softplus;
  int done, n;                      // chunks: sequences of up to so many rows are another launch's; sequences taken
};

// The step of a row: dt + bias, and log(1 + exp(.)) of it.
__device__ __forceinline__ float step_of(float dt, float bias, int softplus) {
  const float v = dt + bias;
  return softplus ? fmaxf(v, 0.0f) + log1pf(expf(-fabsf(v))) : v;
}

// One sequence's rows for COLS columns of a head, the recurrence as written.
// A lane holds four columns of every RG-th row of S, in registers from the
// first row of the sequence to its last.  TB rows at a time: their inputs are
// loaded together, and their outputs, sums over the lanes and waves, joined
// behind one barrier.
template <int COLS, int NT, int TB>
struct StepLds {
  float part[TB][NT / 64][COLS];
};
template <int N, int COLS, int NT, int TB>
__device__ __forceinline__ void step_rows(const ScanArgs &a, int b, int h, int c0, int begin, int end,
                                          StepLds<COLS, NT, TB> &L) {
  constexpr int CL = COLS / 4, RG = NT / CL, RPT = N / RG;
  static_assert(RPT >= 1 && RPT * RG == N && CL <= 64 && TB * CL <= NT, "rows of S over the threads");
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int c = c0 + 4 * (tid % CL), r0 = tid / CL;
  const bool live = c < a.P;
  const int cc = min(c, a.P - 4);
  const int64_t src = seq_src(a.q, b), dst = seq_dst(a.q, b), hp = (int64_t)h * a.P;
  const float A = a.A[h], bias = a.bias ? a.bias[h] : 0.0f, D = a.D ? a.D[h] : 0.0f;
  const int64_t gn = (int64_t)(h / a.G) * N + r0;
  v4f S[RPT];
#pragma unroll
  for (int m = 0; m < RPT; m++)
    S[m] = src >= 0 && live
               ? *reinterpret_cast<const v4f *>(a.state + ((src * a.NH + h) * N + r0 + RG * m) * a.P + c)
               : v4f{0.f, 0.f, 0.f, 0.f};
  for (int t0 = begin; t0 < end; t0 += TB) {
    v4f x[TB], xo, zo;                           // (xo, zo: of the output that this thread joins)
    float bn[TB][RPT], cn[TB][RPT], dt[TB];
#pragma unroll
    for (int u = 0; u < TB; u++) {
      const int64_t t = min(t0 + u, end - 1);
      x[u] = *reinterpret_cast<const v4f *>(a.x + t * a.xs + hp + cc);
      dt[u] = a.dt[t * a.ds + h];
#pragma unroll
      for (int m = 0; m < RPT; m++) {
        bn[u][m] = a.b[t * a.bs + gn + RG * m];
        cn[u][m] = a.c[t * a.cs + gn + RG * m];
      }
    }
    const int64_t to = min(t0 + tid / CL, end - 1);
    const bool joins = tid < TB * CL && t0 + tid / CL < end && live;
    if (joins) {
      xo = *reinterpret_cast<const v4f *>(a.x + to * a.xs + hp + cc);
      if (a.z) zo = *reinterpret_cast<const v4f *>(a.z + to * a.zs + hp + cc);
    }
#pragma unroll
    for (int u = 0; u < TB; u++) {
      if (u > 0 && t0 + u >= end) break;
      const float d = step_of(dt[u], bias, a.softplus);
      const float keep = expf(d * A);
      const v4f dx = d * x[u];
      v4f y = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int m = 0; m < RPT; m++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
          S[m][e] = fmaf(keep, S[m][e], bn[u][m] * dx[e]);
          y[e] = fmaf(cn[u][m], S[m][e], y[e]);
        }
#pragma unroll
      for (int o = CL; o < 64; o <<= 1)
#pragma unroll
        for (int e = 0; e < 4; e++) y[e] += __shfl_xor(y[e], o);
      if (lane < CL) *reinterpret_cast<v4f *>(&L.part[u][wave][4 * lane]) = y;
    }
    __syncthreads();
    if (joins) {
      v4f s = D * xo;
#pragma unroll
      for (int w = 0; w < NT / 64; w++)
        s += *reinterpret_cast<const v4f *>(&L.part[tid / CL][w][4 * (tid % CL)]);
      if (a.z) s *= v4f{silu_f32(zo.x), silu_f32(zo.y), silu_f32(zo.z), silu_f32(zo.w)};
      *reinterpret_cast<v4f *>(a.y + to * a.ys + hp + c) = s;
    }
    if (t0 + TB < end) __syncthreads();          // the partial sums are rewritten
  }
  if (dst >= 0 && live)
#pragma unroll
    for (int m = 0; m < RPT; m++)
      *reinterpret_cast<v4f *>(a.state + ((dst * a.NH + h) * N + r0 + RG * m) * a.P + c) = S[m];
}

// Sequences of up to `most` rows row by row, 64 columns of a head a workgroup.
template <int N, int TB>
__global__ __launch_bounds__(STEP_NT) void step_kernel(ScanArgs a, int most) {
  __shared__ __align__(16) StepLds<64, STEP_NT, TB> L;
  const int sl = blockIdx.x % a.nsl, bh = blockIdx.x / a.nsl, h = bh % a.NH, b = bh / a.NH;
  const int begin = seq_begin(a.q, b), end = seq_begin(a.q, b + 1);
  if (begin >= end || end - begin > most) return;
  step_rows<N, 64, STEP_NT, TB>(a, b, h, sl * 64, begin, end, L);
}

// ---------------------------------------------------------------- chunked scan
// Chunk c of sequence b has its products C B^T in the workspace at record
// cu[b] / 64 + b + c: a sequence of n rows has ceil(n / 64) of them, which never
// reach the next sequence's first.
__device__ __forceinline__ int record_of(int begin, int b) { return begin / SC + b; }

// A record holds the ten 16 x 16 tiles (r, j <= r) of a chunk's C B^T, then the
// tiles (n, j) of B^T (16 entries by 16 rows of the chunk) and (r, n) of C, each as
// a lane of a product takes it: four neighbouring columns 4 (l / 16) .. + 3 of
// row l % 16.
constexpr int GRAM = 10 * 256;      // floats
constexpr int rec_floats(int N) { return GRAM + 2 * N * SC; }
__device__ __forceinline__ int tile_at(int r, int j) { return (r * (r + 1) / 2 + j) * 256; }

// Four products of 16 x 16 x 4 of a 16-byte piece of either operand, in two
// sums: lane l's pieces are k = 4 (l / 16) .. + 3 of row (A) and column (B) l % 16
// of 16 k in all; element e of a sum is row 4 (l / 16) + e, column l % 16.
__device__ __forceinline__ void mm4(v4f x, v4f y, v4f &c0, v4f &c1) {
  c0 = __builtin_amdgcn_mfma_f32_16x16x4f32(x.x, y.x, c0, 0, 0, 0);
  c1 = __builtin_amdgcn_mfma_f32_16x16x4f32(x.y, y.y, c1, 0, 0, 0);
  c0 = __builtin_amdgcn_mfma_f32_16x16x4f32(x.z, y.z, c0, 0, 0, 0);
  c1 = __builtin_amdgcn_mfma_f32_16x16x4f32(x.w, y.w, c1, 0, 0, 0);
}
// A value is computed by here.
__device__ __forceinline__ void pin(v4f &v) { asm volatile("" : "+v"(v)); }
__device__ __forceinline__ v4f quad(const float *p) { return *reinterpret_cast<const v4f *>(p); }

// Inclusive sum over the wave's lanes.
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp_add(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint32_t l = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, ROWS, 0xF, false);
  const uint32_t h = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)(u >> 32), CTRL, ROWS, 0xF, false);
  return v + __builtin_bit_cast(double, (uint64_t)h << 32 | l);
}
__device__ __forceinline__ double scan64(double v) {
  v = dpp_add<0x111, 0xF>(v);       // from 1, 2, 4 and 8 lanes before in a row of 16
  v = dpp_add<0x112, 0xF>(v);
  v = dpp_add<0x114, 0xF>(v);
  v = dpp_add<0x118, 0xF>(v);
  v = dpp_add<0x142, 0xA>(v);       // the row before's last lane, into rows 1 and 3
  return dpp_add<0x143, 0xC>(v);    // lane 31, into rows 2 and 3
}

// What the scan takes of a chunk's steps, per head DEC arrays of 64 rows: the
// logarithms (base 2) of the decay up to a row, in two halves, the steps, the
// steps times the decay from a row to the chunk's end, and the decay up to a row.
// Logarithms are summed in fp64 and kept in two halves so that differences of
// long sums keep their precision: rows of strong decay (hundreds) may stand
// beside rows of next to none.
constexpr int DEC = 5, DEC_LH = 0, DEC_LL = 1, DEC_EL = 2, DEC_DL = 3, DEC_WJ = 4;
constexpr int DEC_LDS = 3;          // the first ones go to LDS, the others into x

// The sequences as the scan takes them, longest first (ties by number), so that no
// long one starts when the others end: number, first row, end.  6 sequences of 633 to
// 2000 rows, 64 heads of 64: 236 us, as they come 278.  Places are counted, which
// for up to ORDER_B sequences ends before the records do; more go as they come.
constexpr int ORDER_B = SSM_ORDER_B, ORDER_NT = 256;
__device__ __forceinline__ void order_rows(const ScanArgs &a, int block) {
  __shared__ __align__(16) int rows[ORDER_B];
  const int B = a.q.B, b = block * ORDER_NT + threadIdx.x;
  const int begin = seq_begin(a.q, min(b, B - 1)), end = seq_begin(a.q, min(b, B - 1) + 1);
  int place = b;
  if (B <= ORDER_B) {
    for (int j = threadIdx.x; j < (B + 3) / 4 * 4; j += ORDER_NT)
      rows[j] = j < B ? max(seq_begin(a.q, j + 1) - seq_begin(a.q, j), 0) : -1;
    __syncthreads();
    const int n = max(end - begin, 0);
    place = 0;
    for (int j = 0; j < B; j += 4) {
      const int4 m = *reinterpret_cast<const int4 *>(rows + j);
      place += (m.x > n || (m.x == n && j < b)) + (m.y > n || (m.y == n && j + 1 < b)) +
               (m.z > n || (m.z == n && j + 2 < b)) + (m.w > n || (m.w == n && j + 3 < b));
    }
  }
  if (b < B) a.order[place] = make_int4(b, begin, end, 0);
}

// What the chunks need that does not wait for the one before: a record's pieces,
// a wave each (one trip to memory; a workgroup of four waves for all of a record
// took 12 us for a 947-token prompt), then the steps and decays, a wave per chunk and
// head, a row a lane.
//   C B^T: the rows of B are the A operand, so that a lane's sums are neighbouring
//   columns of one row.  Rows past the sequence's last repeat it (their steps are 0
//   where they are used).
//   B^T and C: a lane's four numbers of a product together and 1 KB an instruction
//   (gathered by the scan 16384 rows of 64 heads of 64 took 718 us, B^T here 631).
constexpr int prep_parts(int N) { return (10 + N / 16 + 4 + 3) / 4; }
template <int N>
__global__ __launch_bounds__(ORDER_NT) void prep_kernel(ScanArgs a, unsigned norder, unsigned ngram) {
  if (blockIdx.x < norder) return order_rows(a, blockIdx.x);
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const unsigned block = blockIdx.x - norder;
  const bool gram = block < ngram;
  const unsigned w = gram ? block : block - ngram, per = gram ? a.NG * prep_parts(N) : (a.NH + 3) / 4;
  const int rec = w / per, part = w % per;
  // the last sequence whose first record is not past rec: its number plus up to T / 64
  int lo = min(max(rec - a.q.T / SC, 0), a.q.B - 1), hi = min(rec + 1, a.q.B);
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (record_of(seq_begin(a.q, m), m) <= rec) lo = m; else hi = m;
  }
  const int begin = seq_begin(a.q, lo), end = seq_begin(a.q, lo + 1);
  const int t0 = begin + (rec - record_of(begin, lo)) * SC;
  if (t0 < begin || t0 >= end || end - begin <= a.done) return;
  if (!gram) {
    const int h = 4 * part + wave;
    if (h >= a.NH) return;
    const double A = (double)a.A[h] * 1.4426950408889634;
    const int t = t0 + lane;
    const float d = t < end ? step_of(a.dt[(int64_t)min(t, end - 1) * a.ds + h], a.bias ? a.bias[h] : 0.0f, a.softplus)
                            : 0.0f;
    // (past 2^20 either way a row's decay is 0 or infinite; kept there, sums stay finite. A
    // NaN stays one)
    const double v = (double)d * A, top = 1048576.0;
    const double s = scan64(t < end ? (v < -top ? -top : v > top ? top : v) : 0.0);
    const uint64_t u = __builtin_bit_cast(uint64_t, s);
    const double all = __builtin_bit_cast(
        double, (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), 63) << 32 |
                    (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)u, 63));
    const float lh = (float)s;
    float *o = a.dec + ((int64_t)rec * a.NH + h) * (DEC * SC) + lane;
    o[DEC_LH * SC] = lh;
    o[DEC_LL * SC] = (float)(s - (double)lh);
    o[DEC_DL * SC] = d;
    o[DEC_WJ * SC] = d * __builtin_amdgcn_exp2f((float)(all - s));
    o[DEC_EL * SC] = __builtin_amdgcn_exp2f(lh);
    return;
  }
  const int g = part / prep_parts(N), job = 4 * (part % prep_parts(N)) + wave;
  const int l16 = lane & 15, lq = lane >> 4;
  float *const out = a.gram + ((int64_t)rec * a.NG + g) * rec_floats(N) + 4 * lane;
  const auto row = [&](const float *p, int stride, int i) {    // row i of the chunk
    return p + (int64_t)min(t0 + i, end - 1) * stride + (int64_t)g * N;
  };
  if (job < 10) {
    const int r = job >= 6 ? 3 : job >= 3 ? 2 : job >= 1 ? 1 : 0, j = job - r * (r + 1) / 2;
    const float *const cp = row(a.c, a.cs, 16 * r + l16) + 4 * lq, *const bp = row(a.b, a.bs, 16 * j + l16) + 4 * lq;
    v4f s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0, cv[N / 16], bv[N / 16];
#pragma unroll
    for (int s = 0; s < N / 16; s++) { bv[s] = quad(bp + 16 * s); cv[s] = quad(cp + 16 * s); }
    __builtin_amdgcn_sched_barrier(0);           // (all loads under way)
#pragma unroll
    for (int s = 0; s < N / 16; s++) mm4(bv[s], cv[s], s0, s1);
    *reinterpret_cast<v4f *>(out + tile_at(r, j)) = s0 + s1;
  } else if (job < 10 + N / 16) {
    const int n = job - 10;
    v4f v[4];
#pragma unroll
    for (int j = 0; j < 4; j++)
#pragma unroll
      for (int e = 0; e < 4; e++) v[j][e] = row(a.b, a.bs, 16 * j + 4 * lq + e)[16 * n + l16];
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int j = 0; j < 4; j++) *reinterpret_cast<v4f *>(out + GRAM + (4 * n + j) * 256) = v[j];
  } else if (job < 14 + N / 16) {
    const int r = job - 10 - N / 16;
    const float *const cp = row(a.c, a.cs, 16 * r + l16) + 4 * lq;
#pragma unroll
    for (int s = 0; s < N / 16; s++)
      *reinterpret_cast<v4f *>(out + GRAM + N * SC + (r * (N / 16) + s) * 256) = quad(cp + 16 * s);
  }
}

// Matrices by column: 16-byte pieces of a column stand XOR-swizzled by the column,
// so that lanes that read a piece of 16 columns, or different pieces of some, meet
// distinct banks (with columns padded by 16 bytes half of the LDS cycles were
// conflicts).
template <int LEN>
__device__ __forceinline__ int piece_at(int col, int piece) { return col * LEN + 4 * (piece ^ (col & 15)); }

// Two workgroups of the slices of 32 columns of 128 rows share a compute unit: with
// one buffer each for the state's columns and the sums of y, for a second barrier a
// step (64 sequences of 128 rows, 64 heads of 64: 313 us; alone 368), and 128 registers.
template <int N, int PS>
struct ScanLds {
  static constexpr int SB = N == 128 && PS == 32 ? 1 : 2;
  float xd[2][PS * SC];             // x by column, times the steps
  float xw[2][PS * SC];             // ... and the decays to the chunk's end
  float st[SB][PS * N];             // the state before the chunk by column
  float yl[SB][N == 64 ? 1 : 2][SC][PS + 4]; // sums of y (N > 64: of either half of the state's rows)
  float dec[2][DEC_LDS][SC];
};

// The chunks of a sequence in order, for one head and PS columns; the state's
// tiles of 16 x 16 in the accumulators of eight waves.  With L the sums of the
// logarithms of the decays, within a chunk
//   y = diag(e^L) C S + (C B^T o e^{L_i - L_j} o d_j) x   (j <= i)
//   S <- e^{L_C} S + B^T diag(d e^{L_C - L}) x.
template <int N, int PS>
__global__ __launch_bounds__(SNT, (ScanLds<N, PS>::SB == 1 ? 4 : 2)) void scan_kernel(ScanArgs a) {
  // tiles of S a wave: TN of its rows by TC of its columns; of y: CT of its columns, over
  // one of KH parts of S's rows
  constexpr int NT = N / 16, PT = PS / 16, KH = NT < 8 ? 1 : 2, CT = PT * KH / 2;
  constexpr int TN = NT < 8 ? 1 : NT / 8, TC = NT < 8 ? PT * NT / 8 : PT;
  constexpr int CF = N / KH / 16, GF = KH == 2 ? 2 : 4, SB = ScanLds<N, PS>::SB;
  static_assert(8 * CT == 4 * KH * PT && 8 * TN * TC == NT * PT, "tiles over the waves");
  __shared__ __align__(16) ScanLds<N, PS> L;
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63;
  const int l16 = lane & 15, lq = lane >> 4;
  // all slices of a head on one XCD (workgroup w runs on XCD w mod 8)
  const int k = blockIdx.x >> 3, bh = (k / a.nsl) * 8 + (blockIdx.x & 7);
  if (bh >= a.n * a.NH) return;
  const int4 place = a.order[bh / a.NH];
  const int b = __builtin_amdgcn_readfirstlane(place.x), begin = __builtin_amdgcn_readfirstlane(place.y),
            end = __builtin_amdgcn_readfirstlane(place.z);
  const int h = bh % a.NH, g = h / a.G, c0 = (k % a.nsl) * PS;
  if (begin >= end || end - begin <= a.done) return;
  const int nch = (end - begin + SC - 1) / SC;
  const float D = a.D ? a.D[h] : 0.0f;

  // roles: sums of y of rows 16 r .. + 15, column tiles from yct on, part kh of the
  // state's rows (waves w and w + 4, of one SIMD, take r and 3 - r); rows of tiles
  // nt[] and column tiles from sct on of S; row xr and columns xc .. + 3 of x, z
  // and y
  const int hi = wave >> 2, r = hi ? 3 - (wave & 3) : wave & 3;
  const int kh = KH == 2 ? hi : 0, yct = KH == 2 ? 0 : hi * CT, sct = NT < 8 ? wave / NT * TC : 0;
  int nt[TN];
#pragma unroll
  for (int i = 0; i < TN; i++) nt[i] = (wave + 8 * i) % NT;
  constexpr int XW = PS / 4;                     // waves that have a row of x
  const int xr = tid / (PS / 4), xc = 4 * (tid % (PS / 4));

  // Everything of a chunk is read as buffers, by offsets that stay, from bases that
  // move on a chunk with each load: no address is computed by the lanes.  The rows'
  // buffers end at the sequence's last row: past it loads give zeros and stores
  // do nothing, so none needs a condition.
  typedef __amdgpu_buffer_rsrc_t Rsrc;
  const auto buffer = [](const float *p, uint32_t bytes) {
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<float *>(p), 0, (int)bytes, 0x00027000);
  };
  const auto load4 = [](Rsrc q, uint32_t at, uint32_t more) {
    return __builtin_bit_cast(v4f, __builtin_amdgcn_raw_buffer_load_b128(q, at, more, 0));
  };
  const auto load1 = [](Rsrc q, uint32_t at, uint32_t more) {
    return __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(q, at, more, 0));
  };
  struct Rows {                                  // a tensor's rows from the next chunk on
    const float *p;
    int stride, left;
  };
  const auto rows = [&](const float *p, int stride) {
    return Rows{p + (int64_t)begin * stride, stride, end - begin};
  };
  const auto next = [&](Rows &q) {
    const Rsrc b = buffer(q.p, (uint32_t)min(q.left, SC) * (uint32_t)q.stride * 4u);
    q.p += (int64_t)SC * q.stride;
    q.left = max(q.left - SC, 0);
    return b;
  };
  const int xrow = min(xr, SC - 1), cx = min(xc, a.P - 4 - c0);
  const uint32_t xat = 4u * (xrow * (uint32_t)a.xs + cx), zat = 4u * (xrow * (uint32_t)a.zs + cx);
  const uint32_t yat = c0 + xc < a.P ? 4u * (xrow * (uint32_t)a.ys + xc) : 0xFFFFFFF0u;
  const uint32_t lane16 = 16 * lane, row4 = 4 * xrow;
  const int64_t hp = (int64_t)h * a.P + c0, rec0 = record_of(begin, b);
  Rows xrows = rows(a.x + hp, a.xs), erows = xrows, yrows = rows(a.y + hp, a.ys),
       zrows = rows((a.z ? a.z : a.x) + hp, a.zs);
  constexpr int RF = rec_floats(N);
  const float *recp = a.gram + (rec0 * a.NG + g) * RF, *decp = a.dec + (rec0 * a.NH + h) * (DEC * SC);
  // A chunk's operands have one set of registers each: the next chunk's are
  // loaded into them behind their last use, a step ahead of their own.  (A
  // scheduling barrier before each load: moved up, it would need other registers,
  // and copies at the loop's end that wait for it: 616 us.)
  v4f cf[CF], gf[GF], bf[TN][4], x, xe, z;      // (xe: x for the outputs)
  float dec1, dl, wj;                            // of one of the decay arrays; of x's row
  Rsrc rec;
  const auto load_c = [&]() {
    rec = buffer(recp, 4 * RF);
    recp += (int64_t)a.NG * RF;
#pragma unroll
    for (int s = 0; s < CF; s++) cf[s] = load4(rec, lane16, 4 * (GRAM + N * SC + (r * NT + kh * CF + s) * 256));
  };
  const auto load_b = [&]() {
#pragma unroll
    for (int i = 0; i < TN; i++)
#pragma unroll
      for (int s = 0; s < 4; s++) bf[i][s] = load4(rec, lane16, 4 * (GRAM + (4 * nt[i] + s) * 256));
  };
  const auto load_g = [&]() {
#pragma unroll
    for (int s = 0; s < GF; s++) gf[s] = load4(rec, lane16, 4 * tile_at(r, min(KH == 2 ? kh + 2 * s : s, r)));
  };
  const auto load_x = [&]() {
    x = load4(next(xrows), xat, 0);
    const Rsrc q = buffer(decp, 4 * DEC * SC);
    decp += (int64_t)a.NH * (DEC * SC);
    dec1 = load1(q, 4 * lane, 4 * min(wave, DEC_LDS - 1) * SC);
    dl = load1(q, row4, 4 * DEC_DL * SC);
    wj = load1(q, row4, 4 * DEC_WJ * SC);
  };
  const auto load_xe = [&]() { xe = load4(next(erows), xat, 0); };
  const auto load_z = [&]() { z = load4(next(zrows), zat, 0); };
  // x by column, and the decays of a chunk
  const auto stage = [&](int p) {
    if (wave < XW)
#pragma unroll
      for (int e = 0; e < 4; e++) {
        const int at = piece_at<SC>(xc + e, xr >> 2) + (xr & 3);
        L.xd[p][at] = dl * x[e];
        L.xw[p][at] = wj * x[e];
      }
    if (wave < DEC_LDS) L.dec[p][wave][lane] = dec1;
  };

  const int64_t src = seq_src(a.q, b), dst = seq_dst(a.q, b);
  v4f S[TN][TC];
#pragma unroll
  for (int i = 0; i < TN; i++)
#pragma unroll
    for (int k = 0; k < TC; k++) {
      const int col = c0 + 16 * (sct + k) + l16;
#pragma unroll
      for (int e = 0; e < 4; e++)
        S[i][k][e] = src >= 0 && col < a.P
                         ? a.state[((src * a.NH + h) * N + 16 * nt[i] + 4 * lq + e) * a.P + col]
                         : 0.0f;
    }
  const auto put_state = [&](int p) {
#pragma unroll
    for (int i = 0; i < TN; i++)
#pragma unroll
      for (int k = 0; k < TC; k++)
        *reinterpret_cast<v4f *>(&L.st[p][piece_at<N>(16 * (sct + k) + l16, 4 * nt[i] + lq)]) = S[i][k];
  };

  load_x();
  load_c();
  load_b();
  load_g();
  if (SB == 2) load_xe();
  load_z();
  put_state(0);
  stage(0);
  load_x();
  __syncthreads();
  for (int c = 0; c < nch; c++) {
    const int p = c & 1, ps = p & (SB - 1);
    const auto &dec = L.dec[p];
    // C S
    v4f y0[CT], y1[CT];
#pragma unroll
    for (int k = 0; k < CT; k++) y0[k] = y1[k] = v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int s = 0; s < CF; s++)
#pragma unroll
      for (int k = 0; k < CT; k++)
        mm4(cf[s], quad(&L.st[ps][piece_at<N>(16 * (yct + k) + l16, 4 * (kh * CF + s) + lq)]), y0[k], y1[k]);
#pragma unroll
    for (int k = 0; k < CT; k++) { pin(y0[k]); pin(y1[k]); }
    __builtin_amdgcn_sched_barrier(0);
    load_c();
    if (SB == 1) __syncthreads();                // the state before the chunk and the last sums of y are read
    // S
    const float eC = dec[DEC_EL][SC - 1];
#pragma unroll
    for (int i = 0; i < TN; i++)
#pragma unroll
      for (int k = 0; k < TC; k++) {
        v4f s1 = {0.f, 0.f, 0.f, 0.f};
        S[i][k] *= eC;
#pragma unroll
        for (int s = 0; s < 4; s++)
          mm4(bf[i][s], quad(&L.xw[p][piece_at<SC>(16 * (sct + k) + l16, 4 * s + lq)]), S[i][k], s1);
        S[i][k] += s1;
        pin(S[i][k]);
      }
    __builtin_amdgcn_sched_barrier(0);
    load_b();
    const v4f el = quad(&dec[DEC_EL][16 * r + 4 * lq]);
#pragma unroll
    for (int k = 0; k < CT; k++) {
      y0[k] = (y0[k] + y1[k]) * el;
      y1[k] = v4f{0.f, 0.f, 0.f, 0.f};
    }
    // (C B^T o decays) x
    const float lhi = dec[DEC_LH][16 * r + l16], lli = dec[DEC_LL][16 * r + l16];
#pragma unroll
    for (int s = 0; s < GF; s++) {
      const int j = KH == 2 ? kh + 2 * s : s;
      if (j > r) continue;
      const v4f lh = quad(&dec[DEC_LH][16 * j + 4 * lq]), ll = quad(&dec[DEC_LL][16 * j + 4 * lq]);
      v4f w;
#pragma unroll
      for (int e = 0; e < 4; e++) {
        w[e] = gf[s][e] * __builtin_amdgcn_exp2f((lhi - lh[e]) + (lli - ll[e]));
        if (16 * j + 4 * lq + e > 16 * r + l16) w[e] = 0.0f;
      }
#pragma unroll
      for (int k = 0; k < CT; k++)
        mm4(w, quad(&L.xd[p][piece_at<SC>(16 * (yct + k) + l16, 4 * j + lq)]), y0[k], y1[k]);
    }
#pragma unroll
    for (int k = 0; k < CT; k++) {
      y0[k] += y1[k];
      pin(y0[k]);
    }
    __builtin_amdgcn_sched_barrier(0);
    load_g();
    if (SB == 1) load_xe();                      // (no registers to spare before)
#pragma unroll
    for (int k = 0; k < CT; k++)
#pragma unroll
      for (int e = 0; e < 4; e++) L.yl[ps][kh][16 * r + 4 * lq + e][16 * (yct + k) + l16] = y0[k][e];
    put_state((p ^ 1) & (SB - 1));
    stage(p ^ 1);                                // (past the last chunk unused)
    __builtin_amdgcn_sched_barrier(0);
    load_x();
    __syncthreads();
    if (wave < XW) {
      v4f o = quad(&L.yl[ps][0][xr][xc]);
      if (KH == 2) o += quad(&L.yl[ps][1][xr][xc]);
      o += D * xe;
      if (a.z) o *= v4f{silu_f32(z.x), silu_f32(z.y), silu_f32(z.z), silu_f32(z.w)};
      __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(v4u, o), next(yrows), yat, 0, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
    if (SB == 2) load_xe();
    load_z();
    __builtin_amdgcn_sched_barrier(0);
  }
  if (dst >= 0)
#pragma unroll
    for (int i = 0; i < TN; i++)
#pragma unroll
      for (int k = 0; k < TC; k++) {
        const int col = c0 + 16 * (sct + k) + l16;
        if (col < a.P)
#pragma unroll
          for (int e = 0; e < 4; e++)
            a.state[((dst * a.NH + h) * N + 16 * nt[i] + 4 * lq + e) * a.P + col] = S[i][k][e];
      }
}

// Records of a call; the scan's loads run two past a sequence's last.
int64_t records(int64_t T, int64_t B) { return T / SC + B + 3; }

int ssm_sizes(const w4a8_seqs *q, const w4a8_ssm *m, int64_t T) {
  if (!m) return W4A8_ENULL;
  int rc = seqs_sizes(q, T);
  if (rc != W4A8_OK) return rc;
  if (m->NH < 1 || m->NG < 1 || m->NH % m->NG != 0 || (m->N != 64 && m->N != 128 && m->N != 256) ||
      m->P < 16 || m->P % 16 != 0)
    return W4A8_ESHAPE;
  // (a grid's threads are counted in 32 bits)
  if (m->NH >= (1 << 16) || m->P > 4096 || q->B * m->NH * m->P >= ((int64_t)1 << 26) ||
      (T / SC + q->B + 3) * (m->NG + m->NH) >= ((int64_t)1 << 21))
    return W4A8_ERANGE;
  return W4A8_OK;
}

template <int N, int PS>
int launch_scan(ScanArgs a, hipStream_t s) {
  a.nsl = (a.P + PS - 1) / PS;
  const unsigned pairs = (unsigned)((a.n * a.NH + 7) / 8 * 8);
  scan_kernel<N, PS><<<dim3(pairs * a.nsl), dim3(SNT), 0, s>>>(a);
  return check_launch();
}

template <int N>
int launch_ssm(ScanArgs a, hipStream_t s) {
  const SsmWay way = ssm_way(a.q.B, a.q.T, a.NH, a.P, N, device_cus());
  constexpr int TB = N == 256 ? 2 : 4;
  a.nsl = (a.P + 63) / 64;
  if (way.rows) {
    const dim3 grid((unsigned)(a.q.B * a.NH * a.nsl));
    if (way.single)
      step_kernel<N, 1><<<grid, dim3(STEP_NT), 0, s>>>(a, way.rows);
    else
      step_kernel<N, TB><<<grid, dim3(STEP_NT), 0, s>>>(a, way.rows);
    if (int rc = check_launch(); rc != W4A8_OK || !way.chunked) return rc;
  }
  a.done = way.rows;
  a.n = way.chunked;
  const unsigned norder = (unsigned)((a.q.B + ORDER_NT - 1) / ORDER_NT);
  const unsigned ngram = (unsigned)(records(a.q.T, a.q.B) * a.NG * prep_parts(N)),
                 ndec = (unsigned)(records(a.q.T, a.q.B) * ((a.NH + 3) / 4));
  prep_kernel<N><<<dim3(norder + ngram + ndec), dim3(ORDER_NT), 0, s>>>(a, norder, ngram);
  if (int rc = check_launch(); rc != W4A8_OK) return rc;
  if constexpr (N == 128)
    if (way.slice == 32) return launch_scan<N, 32>(a, s);
  return launch_scan<N, N == 64 ? 32 : 16>(a, s);
}

}  // namespace

}  // namespace w4a8

using namespace w4a8;

extern "C" size_t ssm_workspace_size(const w4a8_seqs *seqs, const w4a8_ssm *ssm, int64_t T) {
  if (ssm_sizes(seqs, ssm, T) != W4A8_OK) return 0;
  return (size_t)records(T, seqs->B) * (ssm->NG * rec_floats((int)ssm->N) + ssm->NH * DEC * SC) *
             sizeof(float) +
         (size_t)seqs->B * sizeof(int4);
}

extern "C" int ssm_scan(const w4a8_seqs *seqs, const w4a8_ssm *m, float *state, float *y,
                        int64_t y_stride, int64_t T, void *workspace, size_t ws_bytes, void *stream) {
  int rc = ssm_sizes(seqs, m, T);
  if (rc != W4A8_OK) return rc;
  const int64_t xrow = m->NH * m->P, brow = m->NG * m->N, top = (int64_t)1 << 24;
  if (m->x_stride < xrow || m->x_stride % 4 != 0 || m->b_stride < brow || m->b_stride % 4 != 0 ||
      m->c_stride < brow || m->c_stride % 4 != 0 || m->dt_stride < m->NH || y_stride < xrow ||
      y_stride % 4 != 0 || (m->z && (m->z_stride < xrow || m->z_stride % 4 != 0)))
    return W4A8_ESHAPE;
  // (a chunk's rows are addressed in 32 bits)
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
  a.state = state; a.y = y; a.gram = reinterpret_cast<float *>(workspace);
  a.dec = a.gram + records(a.q.T, a.q.B) * m->NG * rec_floats((int)m->N);
  a.order = reinterpret_cast<int4 *>(a.dec + records(a.q.T, a.q.B) * m->NH * DEC * SC);
  a.xs = (int)m->x_stride; a.ds = (int)m->dt_stride; a.bs = (int)m->b_stride; a.cs = (int)m->c_stride;
  a.zs = m->z ? (int)m->z_stride : 0; a.ys = (int)y_stride;
  a.NH = (int)m->NH; a.NG = (int)m->NG; a.G = (int)(m->NH / m->NG); a.P = (int)m->P;
  a.softplus = m->softplus;
  hipStream_t s = as_stream(stream);
  return m->N == 64 ? launch_ssm<64>(a, s) : m->N == 128 ? launch_ssm<128>(a, s) : launch_ssm<256>(a, s);
}
