// The paged 4-bit key/value cache of the softmax-attention layers: storing
// new rows (keys rotated by their positions, both quantized to the block
// formats of Sec. 2.3) and reading rows back.
//
// Storing: a workgroup takes a few rows with all their heads, so a row's
// cosines are computed once; eight lanes own a block, as in the quantizers,
// and store it in the tile order of kv_dev.h.  Bound by reading the fp32 rows
// for a prompt, by the launch and one chain of loads for a decode batch.
#include "kv_dev.h"
#include "rope_dev.h"
#include "w4a8_dev.h"
#include "w4a8_host.h"

namespace w4a8 {

namespace {

constexpr int KT = 256;
constexpr int KROWS = 16;      // most rows of a workgroup

template <bool SYM>
__global__ __launch_bounds__(KT) void append_kernel(KvPlan p, RopeArgs r,
                                                    const float *__restrict__ k, int64_t ks,
                                                    const float *__restrict__ v, int64_t vs,
                                                    const float *q, int64_t qs, float *qo, int NH,
                                                    int D, int64_t T, int rows) {
  __shared__ double2 cs[ROPE_PAIRS];
  __shared__ int64_t tile0[KROWS];   // the row's page's first tile, -1: nothing to store
  __shared__ int slot[KROWS];
  const int wave = threadIdx.x >> 6;
  const int nb = D / QK, lanes = D / 4;
  const RopeUnits ru(r.half, r.interleaved, D);
  for (int64_t t0 = (int64_t)blockIdx.x * rows; t0 < T; t0 += (int64_t)gridDim.x * rows) {
    const int n = (int)min((int64_t)rows, T - t0);
    for (int i = wave; i < n; i += KT / 64) {
      int token;
      const int s = p.B > 0 ? kv_find(p, T, t0 + i, token) : -1;
      if ((threadIdx.x & 63) == 0) {
        int64_t at = -1;
        if (s >= 0 && token >= 0) {
          const int page = p.pages[(int64_t)s * p.max_pages + token / KV_PAGE];
          if (page >= 0 && page < p.n_pages) at = (int64_t)page * p.NKV;
        }
        tile0[i] = at;
        slot[i] = s >= 0 && token >= 0 ? token % KV_PAGE : 0;
      }
    }
    rope_table(r, cs, t0, n);
    __syncthreads();
    if (q) {
      const int per = NH * ru.units;
      for (int i = threadIdx.x; i < n * per; i += KT) {
        const int row = i / per, u = i - row * per, h = u / ru.units;
        rope_unit(r, ru, q + (t0 + row) * qs + (int64_t)h * D,
                  qo + ((t0 + row) * NH + h) * (int64_t)D, cs + row * r.half, u - h * ru.units);
      }
    }
    // keys, then values; D / 4 lanes a head, whole groups of eight
    const int per = 2 * p.NKV * lanes;
    for (int i = threadIdx.x; i < n * per; i += KT) {
      const int row = i / per, u = i - row * per, hk = u / lanes, e4 = u - hk * lanes;
      if (tile0[row] < 0) continue;
      const bool isv = hk >= p.NKV;
      const int h = isv ? hk - p.NKV : hk;
      float x[4];
      if (isv) {
        const float4 t = reinterpret_cast<const float4 *>(v + (t0 + row) * vs + (int64_t)h * D)[e4];
        x[0] = t.x; x[1] = t.y; x[2] = t.z; x[3] = t.w;
      } else {
        rope_four(r, k + (t0 + row) * ks + (int64_t)h * D, cs + row * r.half, e4, x);
      }
      const int b = e4 / 8, j = e4 % 8, t = slot[row];
      uint32_t d16 = 0;
      float d32 = 0.0f;
      const uint32_t codes = SYM ? kv_q4_sym_block8(x, d32) : q4_0_block8(x, j, d16);
      const uint32_t pay = codes | (uint32_t)__shfl_xor((int)codes, 4, 8) << 4;
      if (j >= 4) continue;
      uint8_t *tile = (isv ? p.v : p.k) + (tile0[row] + h) * kv_tile_bytes(D, SYM);
      if (isv) {
#pragma unroll
        for (int y = 0; y < 4; y++)
          tile[kv_v_byte(b, 4 * j + y, t)] = (uint8_t)(pay >> (8 * y));
      } else {
        reinterpret_cast<uint32_t *>(tile)[kv_k_dword(b, j, t)] = pay ^ 0x88888888u;
      }
      if (j == 0) {
        uint8_t *sc = tile + nb * 1024;
        if (SYM) reinterpret_cast<float *>(sc)[kv_scale_at(b, t)] = d32;
        else reinterpret_cast<uint16_t *>(sc)[kv_scale_at(b, t)] = (uint16_t)d16;
      }
    }
    __syncthreads();
  }
}

// One wave a row: its heads' values, four elements a lane.
template <bool SYM>
__global__ __launch_bounds__(KT) void read_kernel(KvPlan p, float *__restrict__ ko,
                                                  float *__restrict__ vo, int D, int64_t T) {
  const int lane = threadIdx.x & 63;
  const int nb = D / QK, lanes = D / 4, per = p.NKV * lanes;
  for (int64_t r = (int64_t)blockIdx.x * (KT / 64) + (threadIdx.x >> 6); r < T;
       r += (int64_t)gridDim.x * (KT / 64)) {
    int token;
    const int s = kv_find(p, T, r, token);
    if (s < 0) continue;                       // a row of no sequence
    int page = -1;
    if (token >= 0) page = p.pages[(int64_t)s * p.max_pages + token / KV_PAGE];
    const bool here = page >= 0 && page < p.n_pages;
    const int t = here ? token % KV_PAGE : 0;
    for (int i = lane; i < 2 * per; i += 64) {
      const bool isv = i >= per;
      float *o = isv ? vo : ko;
      if (!o) continue;
      const int u = isv ? i - per : i, h = u / lanes, e4 = u - h * lanes, b = e4 / 8, j = e4 % 8;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (here) {
        const uint8_t *tile = (isv ? p.v : p.k) + ((int64_t)page * p.NKV + h) * kv_tile_bytes(D, SYM);
        uint32_t w = 0;
        if (isv) {
#pragma unroll
          for (int y = 0; y < 4; y++) w |= (uint32_t)tile[kv_v_byte(b, 4 * (j & 3) + y, t)] << (8 * y);
        } else {
          w = reinterpret_cast<const uint32_t *>(tile)[kv_k_dword(b, j & 3, t)] ^ 0x88888888u;
        }
        w = (j < 4 ? w : w >> 4) & 0x0F0F0F0Fu;
        const uint8_t *sc = tile + nb * 1024;
        const float d = SYM ? reinterpret_cast<const float *>(sc)[kv_scale_at(b, t)]
                            : f16_bits_to_f32(reinterpret_cast<const uint16_t *>(sc)[kv_scale_at(b, t)]);
        x = make_float4(((float)(w & 255u) - 8.0f) * d, ((float)(w >> 8 & 255u) - 8.0f) * d,
                        ((float)(w >> 16 & 255u) - 8.0f) * d, ((float)(w >> 24) - 8.0f) * d);
      }
      reinterpret_cast<float4 *>(o + (r * p.NKV + h) * (int64_t)D)[e4] = x;
    }
  }
}

}  // namespace

int kv_check_sizes(const w4a8_kv *kv) {
  if (!kv) return W4A8_ENULL;
  if ((kv->D != 64 && kv->D != 128 && kv->D != 256) || kv->NKV < 1 || kv->B < 0 ||
      kv->n_pages < 0 || kv->max_pages < 0 ||
      (kv->format != W4A8_KV_Q4_0 && kv->format != W4A8_KV_Q4_SYM))
    return W4A8_ESHAPE;
  if (kv->NKV >= (1 << 16) || kv->B >= (1 << 20) || kv->n_pages >= ((int64_t)1 << 31) ||
      kv->max_pages >= (1 << 24))
    return W4A8_ERANGE;
  return W4A8_OK;
}

int kv_check(const w4a8_kv *kv) {
  if (int rc = kv_check_sizes(kv); rc != W4A8_OK) return rc;
  if (kv->n_pages > 0 && (!kv->k_pages || !kv->v_pages)) return W4A8_ENULL;
  if (kv->B > 0 && (!kv->kv_len || !kv->cu_rows || (kv->max_pages > 0 && !kv->page_table)))
    return W4A8_ENULL;
  if (!aligned16(kv->k_pages) || !aligned16(kv->v_pages)) return W4A8_EALIGN;
  const uintptr_t m = reinterpret_cast<uintptr_t>(kv->page_table) |
                      reinterpret_cast<uintptr_t>(kv->kv_len) |
                      reinterpret_cast<uintptr_t>(kv->cu_rows);
  return (m & 3u) ? W4A8_EALIGN : W4A8_OK;
}

}  // namespace w4a8

using namespace w4a8;

extern "C" size_t kv_q4_tile_bytes(int64_t D, int32_t format) {
  if ((D != 64 && D != 128 && D != 256) ||
      (format != W4A8_KV_Q4_0 && format != W4A8_KV_Q4_SYM))
    return 0;
  return (size_t)kv_tile_bytes((int)D, format == W4A8_KV_Q4_SYM);
}

extern "C" int kv_q4_append(const w4a8_kv *kv, const w4a8_rope *rope, const float *k,
                            int64_t k_stride, const float *v, int64_t v_stride, const float *q,
                            int64_t q_stride, float *q_out, int64_t NH, int64_t T, void *stream) {
  if (int rc = kv_check(kv); rc != W4A8_OK) return rc;
  if (!k || !v || (q && !q_out)) return W4A8_ENULL;
  const int64_t w = kv->NKV * kv->D;
  if (T < 0 || k_stride < w || v_stride < w || k_stride % 4 != 0 || v_stride % 4 != 0)
    return W4A8_ESHAPE;
  if (q && (!rope || NH < 1 || q_stride < NH * kv->D || q_stride % 4 != 0)) return W4A8_ESHAPE;
  const int64_t most = (int64_t)1 << 31;
  if (T >= most || k_stride >= most || v_stride >= most || (q && (NH >= (1 << 16) || q_stride >= most)))
    return W4A8_ERANGE;
  if (rope)
    if (int rc = rope_check(rope, kv->D); rc != W4A8_OK) return rc;
  if (!aligned16(k) || !aligned16(v) || (q && (!aligned16(q) || !aligned16(q_out))))
    return W4A8_EALIGN;
  if (q && (q_out == k || q_out == v || (q_out == q && q_stride != NH * kv->D)))
    return W4A8_EALIAS;
  if (T == 0 || (kv->B == 0 && !q)) return W4A8_OK;
  int cus = 0;
  if (int rc = check_device(&cus); rc != W4A8_OK) return rc;
  const RopeArgs r = rope_args(rope);
  // rows of a workgroup: one, or more once every compute unit has two
  // workgroups and while the rows' pairs fit the table
  int rows = 1;
  while (rows * 2 <= KROWS && rows * 2 * r.half <= ROPE_PAIRS && T / (rows * 2) >= 2 * cus)
    rows *= 2;
  const int64_t gx = (T + rows - 1) / rows;
  const dim3 grid((unsigned)(gx < (1 << 22) ? gx : (1 << 22)));
  const KvPlan p = kv_plan(kv);
  if (kv->format == W4A8_KV_Q4_SYM)
    append_kernel<true><<<grid, dim3(KT), 0, as_stream(stream)>>>(
        p, r, k, k_stride, v, v_stride, q, q_stride, q_out, (int)NH, (int)kv->D, T, rows);
  else
    append_kernel<false><<<grid, dim3(KT), 0, as_stream(stream)>>>(
        p, r, k, k_stride, v, v_stride, q, q_stride, q_out, (int)NH, (int)kv->D, T, rows);
  return check_launch();
}

extern "C" int kv_q4_read(const w4a8_kv *kv, float *k_out, float *v_out, int64_t T, void *stream) {
  if (int rc = kv_check(kv); rc != W4A8_OK) return rc;
  if (T < 0) return W4A8_ESHAPE;
  if (T >= ((int64_t)1 << 31)) return W4A8_ERANGE;
  if (!aligned16(k_out) || !aligned16(v_out)) return W4A8_EALIGN;
  if (k_out && k_out == v_out) return W4A8_EALIAS;
  if (T == 0 || kv->B == 0 || (!k_out && !v_out)) return W4A8_OK;
  if (int rc = check_device(); rc != W4A8_OK) return rc;
  const int64_t gx = (T + KT / 64 - 1) / (KT / 64);
  const dim3 grid((unsigned)(gx < (1 << 22) ? gx : (1 << 22)));
  const KvPlan p = kv_plan(kv);
  if (kv->format == W4A8_KV_Q4_SYM)
    read_kernel<true><<<grid, dim3(KT), 0, as_stream(stream)>>>(p, k_out, v_out, (int)kv->D, T);
  else
    read_kernel<false><<<grid, dim3(KT), 0, as_stream(stream)>>>(p, k_out, v_out, (int)kv->D, T);
  return check_launch();
}
