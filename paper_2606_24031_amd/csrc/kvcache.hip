// The paged 4-bit key/value cache of the softmax-attention layers: storing
// new rows (keys rotated by their positions, both quantized to the block
// formats of Sec. 2.3) and reading rows back.
//
// Storing: a workgroup takes one row with all its heads, or some of them while
// rows are few, so a row's cosines are computed once or a few times; eight
// lanes own a block, as in the quantizers, and store it in the tile order of
// kv_dev.h.  3083 rows of 32 query and 8 key and value heads of 128 take 40 us,
// 3.2 TB/s: the loads and stores alone 28, the blocks' quantization and the
// scattered bytes of values 7, each row's place and cosines 5.  32 rows of 16
// and 2 heads of 256 take 5 us: the launch and one chain of loads (the row's
// sequence, its page).  Several rows to a workgroup leave the last round of
// workgroups emptier than they save (57 -> 64 us with both kernels), and rows
// of a page gathered on one XCD, whose L2 could then fill its lines, change
// nothing.
//
// Reading: a wave a row, 11 us for the 3083 rows (2.6 TB/s), mostly writing.
#include <algorithm>
#include <type_traits>

#include "kv_dev.h"
#include "rope_dev.h"
#include "w4a8_dev.h"
#include "w4a8_host.h"

namespace w4a8 {

namespace {

constexpr int KT = 256;
// Items of a thread under way: 2 take 40 us on those rows, 1 takes 42 and 4,
// whose registers leave fewer waves, 46.
constexpr int KB = 2;

// Elements 4 u .. + 3 of head h as a lane's share of a block's codes, and the
// block's scale, into token s of the page at tile0.
template <bool SYM>
__device__ __forceinline__ void store_four(const KvPlan &p, const float e[4], int64_t tile0, int s,
                                           bool isv, int h, int u, int D) {
  const int b = u / 8, l = u % 8;
  uint32_t d16 = 0;
  float d32 = 0.0f;
  const uint32_t codes = SYM ? kv_q4_sym_block8(e, d32) : q4_0_block8(e, l, d16);
  const uint32_t pay = codes | (uint32_t)__shfl_xor((int)codes, 4, 8) << 4;
  if (l >= 4) return;
  uint8_t *tile = (isv ? p.v : p.k) + (tile0 + h) * kv_tile_bytes(D, SYM);
  if (isv) {
#pragma unroll
    for (int y = 0; y < 4; y++) tile[kv_v_byte(b, 4 * l + y, s)] = (uint8_t)(pay >> (8 * y));
  } else {
    reinterpret_cast<uint32_t *>(tile)[kv_k_dword(b, l, s)] = pay ^ 0x88888888u;
  }
  if (l == 0) {
    uint8_t *sc = tile + D / QK * 1024;
    if (SYM) reinterpret_cast<float *>(sc)[kv_scale_at(b, s)] = d32;
    else reinterpret_cast<uint16_t *>(sc)[kv_scale_at(b, s)] = (uint16_t)d16;
  }
}

// Workgroup (x, y): part y of row x's items.  First the lanes of its key and
// value heads (D / 4 a head, whole groups of eight), then the units of its
// query heads.  VEC: a pair's other half is loaded 16 bytes wide too, so KB
// items' loads are under way at once, with the row's place and cosines behind
// them; else one item after the other.  by_units = ceil(2^32 / units): the high
// half of its product with i < 2^24 is i / units, units being 256 at most.
template <bool SYM, bool VEC>
__global__ __launch_bounds__(KT) void append_kernel(KvPlan p, RopeArgs r,
                                                    const float *__restrict__ k, int64_t ks,
                                                    const float *__restrict__ v, int64_t vs,
                                                    const float *q, int64_t qs, float *qo, int NH,
                                                    int D, int64_t T, int part, uint32_t by_units) {
  constexpr int N = VEC ? KB : 1;
  __shared__ double2 cs[128];          // D / 2 pairs at most
  __shared__ int64_t s_tile0;          // the row's page's first tile, -1: nothing to store
  __shared__ int s_slot;
  const int lanes = D / 4, lane_bits = 31 - __builtin_clz(lanes);
  const RopeUnits ru(r.half, r.interleaved, D);
  const int kv = 2 * p.NKV * lanes, end = kv + (q ? NH * ru.units : 0);
  const int i0 = blockIdx.y * part, last = min(end, i0 + part);
  for (int64_t t = blockIdx.x; t < T; t += gridDim.x) {
    int tid = threadIdx.x;
    asm volatile("" : "+v"(tid));    // the items' places stay out of this loop's registers
    bool first = true;
    for (int x = i0; x < last; x += N * KT) {
      float4 a[N], b[N];
      int head[N], u[N];             // u: the lane of a key or value head, the unit of a query head
#pragma unroll
      for (int j = 0; j < N; j++) {
        const int i = min(x + tid + j * KT, last - 1), iq = i - kv;
        const bool isv = i >= kv / 2;
        head[j] = iq < 0 ? (i >> lane_bits) - (isv ? p.NKV : 0) : (int)__umulhi((uint32_t)iq, by_units);
        u[j] = iq < 0 ? i & (lanes - 1) : iq - head[j] * ru.units;
        if (!VEC) continue;
        const int2 uq = rope_unit_at(r, u[j]);
        const float *f = (iq >= 0 ? q + t * qs : isv ? v + t * vs : k + t * ks) + head[j] * D +
                         (iq >= 0 ? uq.x : 4 * u[j]);
        const int other = iq >= 0 ? uq.y - uq.x : isv ? 0 : rope_other(r, 4 * u[j]);
        a[j] = *reinterpret_cast<const float4 *>(f);
        b[j] = *reinterpret_cast<const float4 *>(f + other);
      }
      if (first) {
        if (threadIdx.x < 64) {
          int token;
          const int s = p.B > 0 ? kv_find(p, T, t, token) : -1;
          if (threadIdx.x == 0) {
            int64_t at = -1;
            if (s >= 0 && token >= 0) {
              const int page = p.pages[(int64_t)s * p.max_pages + token / KV_PAGE];
              if (page >= 0 && page < p.n_pages) at = (int64_t)page * p.NKV;
            }
            s_tile0 = at;
            s_slot = s >= 0 && token >= 0 ? token % KV_PAGE : 0;
          }
        }
        rope_table(r, cs, t, 1);
        __syncthreads();
        first = false;
      }
      const int64_t tile0 = s_tile0;
      const int slot = s_slot;
#pragma unroll
      for (int j = 0; j < N; j++) {
        const int i = x + tid + j * KT;
        if (i >= last) continue;
        if (i >= kv) {
          float *y = qo + t * NH * (int64_t)D + head[j] * D;
          if (VEC) rope_unit_turn(r, a[j], b[j], y, cs, u[j]);
          else rope_unit(r, ru, q + t * qs + head[j] * D, y, cs, u[j]);
          continue;
        }
        if (tile0 < 0) continue;
        const bool isv = i >= kv / 2;
        float e[4];
        if (isv) {
          if (!VEC) a[j] = reinterpret_cast<const float4 *>(v + t * vs + head[j] * D)[u[j]];
          e[0] = a[j].x; e[1] = a[j].y; e[2] = a[j].z; e[3] = a[j].w;
        } else if (VEC) {
          rope_four_turn(r, a[j], b[j], cs, u[j], e);
        } else {
          rope_four(r, k + t * ks + head[j] * D, cs, u[j], e);
        }
        store_four<SYM>(p, e, tile0, slot, isv, head[j], u[j], D);
      }
    }
    __syncthreads();
  }
}

// A wave: one row's heads, from lane blockIdx.y on; four elements a lane.
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
    const int64_t base = here ? (int64_t)page * p.NKV : 0;
#pragma unroll 2
    for (int i = blockIdx.y * 64 + lane; i < 2 * per; i += gridDim.y * 64) {
      const bool isv = i >= per;
      float *o = isv ? vo : ko;
      if (!o) continue;
      const int u = isv ? i - per : i, h = u / lanes, e4 = u - h * lanes, b = e4 / 8, j = e4 % 8;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      if (here) {
        const uint8_t *tile = (isv ? p.v : p.k) + (base + h) * kv_tile_bytes(D, SYM);
        const uint8_t *sc = tile + nb * 1024;
        const float d = SYM ? reinterpret_cast<const float *>(sc)[kv_scale_at(b, t)]
                            : f16_bits_to_f32(reinterpret_cast<const uint16_t *>(sc)[kv_scale_at(b, t)]);
        uint32_t n = 0;
        if (isv) {
#pragma unroll
          for (int y = 0; y < 4; y++) n |= (uint32_t)tile[kv_v_byte(b, 4 * (j & 3) + y, t)] << (8 * y);
        } else {
          n = reinterpret_cast<const uint32_t *>(tile)[kv_k_dword(b, j & 3, t)] ^ 0x88888888u;
        }
        n = (j < 4 ? n : n >> 4) & 0x0F0F0F0Fu;
        x = make_float4(((float)(n & 255u) - 8.0f) * d, ((float)(n >> 8 & 255u) - 8.0f) * d,
                        ((float)(n >> 16 & 255u) - 8.0f) * d, ((float)(n >> 24) - 8.0f) * d);
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
  const int64_t lim = (int64_t)1 << 31;
  if (T >= lim || k_stride >= lim || v_stride >= lim || (q && (NH >= (1 << 16) || q_stride >= lim)))
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
  // A row's items over as many workgroups as give the compute units four each
  // (a row's place and cosines are found anew in each), no fewer than one item
  // a thread.
  const RopeUnits ru(r.half, r.interleaved, (int)kv->D);
  const int64_t items = kv->NKV * kv->D / 2 + (q ? NH * ru.units : 0);
  const int64_t most = (items + KT - 1) / KT, want = (4 * cus + T - 1) / T;
  const int64_t ny = std::max<int64_t>(1, std::min<int64_t>(std::min<int64_t>(most, want), 1024));
  const int part = (int)((items + ny - 1) / ny + 63) / 64 * 64;
  const dim3 grid((unsigned)std::min<int64_t>(T, 1 << 20), (unsigned)((items + part - 1) / part));
  const KvPlan p = kv_plan(kv);
  const auto go = [&](auto sym, auto vec) {
    append_kernel<decltype(sym)::value, decltype(vec)::value><<<grid, dim3(KT), 0, as_stream(stream)>>>(
        p, r, k, k_stride, v, v_stride, q, q_stride, q_out, (int)NH, (int)kv->D, T, part,
        (uint32_t)((((uint64_t)1 << 32) + ru.units - 1) / ru.units));
    return check_launch();
  };
  const auto by_vec = [&](auto sym) { return ru.vec ? go(sym, std::true_type{}) : go(sym, std::false_type{}); };
  return kv->format == W4A8_KV_Q4_SYM ? by_vec(std::true_type{}) : by_vec(std::false_type{});
}

extern "C" int kv_q4_read(const w4a8_kv *kv, float *k_out, float *v_out, int64_t T, void *stream) {
  if (int rc = kv_check(kv); rc != W4A8_OK) return rc;
  if (T < 0) return W4A8_ESHAPE;
  if (T >= ((int64_t)1 << 31)) return W4A8_ERANGE;
  if (!aligned16(k_out) || !aligned16(v_out)) return W4A8_EALIGN;
  if (k_out && k_out == v_out) return W4A8_EALIAS;
  if (T == 0 || kv->B == 0 || (!k_out && !v_out)) return W4A8_OK;
  int cus = 0;
  if (int rc = check_device(&cus); rc != W4A8_OK) return rc;
  const int64_t gx = std::min<int64_t>((T + KT / 64 - 1) / (KT / 64), 1 << 20);
  // a row's lanes over several waves while rows are few
  const int64_t waves = kv->NKV * kv->D / 2 / 64 + 1, want = (4 * cus + gx - 1) / gx;
  const dim3 grid((unsigned)gx, (unsigned)std::min<int64_t>(waves, want));
  const KvPlan p = kv_plan(kv);
  const auto go = [&](auto sym) {
    read_kernel<decltype(sym)::value><<<grid, dim3(KT), 0, as_stream(stream)>>>(p, k_out, v_out, (int)kv->D, T);
    return check_launch();
  };
  return kv->format == W4A8_KV_Q4_SYM ? go(std::true_type{}) : go(std::false_type{});
}
