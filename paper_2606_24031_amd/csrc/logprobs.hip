// Log probabilities of given tokens, entropy and top alternatives, read off
// the output head's logits (the decode head of Sec. 5.2) in one pass.
//
// A row is cut into S spans, one workgroup each (S = 1 once the rows fill the
// compute units); every wave streams its share of a span in chunks of 16
// values a lane, the next chunk's loads under way, and keeps
//   - per lane the softmax statistics (m, z, w): the maximum so far, the sum
//     of exp(l - m) WITHOUT the maximum's own 1, and sum exp(l - m) (l - m).
//     With z kept apart from the 1, log Z = log1p(z) is accurate to fp32 for a
//     confident row too, whose log Z may be 1e-6;
//   - per wave the n largest logits: a list in LDS of candidates that beat a
//     threshold, cut back to the n best (by counting, for each candidate, the
//     larger ones) when it fills.  The first threshold is the n-th largest of
//     the 64 lane maxima of the first chunk: n lanes hold a value at least as
//     large, so it is below nothing that belongs to the n best.  After that a
//     random row sends a candidate every few hundred values.
// Bound by HBM: 4 bytes a logit, read once, about 14 VALU ops a value.
#include <algorithm>
#include <cfloat>

#include "w4a8_dev.h"
#include "w4a8_host.h"

namespace w4a8 {

namespace {

constexpr int LT = 256;
constexpr int LW = LT / 64;
constexpr int UG = 4;                    // 4-value groups of a lane's chunk
constexpr int CHUNK = 64 * UG;           // groups of a wave's chunk
constexpr int CAP = 192;                 // candidates of a wave's list
constexpr int NTOP_MAX = 32;
constexpr float FAR = -1e30f;            // logits further below the maximum have probability 0

typedef unsigned long long u64;

// Larger value first, then the lower index: one unsigned comparison.  NaN is
// above every number, -0 equals 0, an absent element is 0.
__device__ __forceinline__ u64 comp_of(float x, uint32_t idx) {
  const uint32_t b = __builtin_bit_cast(uint32_t, x + 0.0f);
  const uint32_t key = x != x ? 0xFFFFFFFFu : b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
  return (u64)key << 32 | (0xFFFFFFFFu - idx);
}
__device__ __forceinline__ float comp_value(u64 c) {
  const uint32_t key = (uint32_t)(c >> 32);
  if (key == 0xFFFFFFFFu) return __builtin_nanf("");
  return __builtin_bit_cast(float, key & 0x80000000u ? key ^ 0x80000000u : ~key);
}
__device__ __forceinline__ uint32_t comp_index(u64 c) { return 0xFFFFFFFFu - (uint32_t)c; }

struct Stat {
  float m, z, w;
  __device__ void init() { m = -FLT_MAX; z = -1.0f; w = 0.0f; }   // 1 + z = 0: nothing seen
};

__device__ __forceinline__ float exp_f(float d) { return __builtin_amdgcn_exp2f(d * 1.44269504f); }

// a and b over disjoint values; the larger maximum's 1 stays out of the sum.
__device__ __forceinline__ Stat merge(Stat a, Stat b) {
  const bool sw = b.m > a.m;
  const float m = sw ? b.m : a.m, lm = sw ? a.m : b.m;
  const float z = sw ? b.z : a.z, lz = sw ? a.z : b.z;
  const float w = sw ? b.w : a.w, lw = sw ? a.w : b.w;
  const float d = fmaxf(lm - m, FAR), f = exp_f(d), t = 1.0f + lz;
  Stat r;
  r.m = m;
  r.z = fmaf(t, f, z);
  r.w = fmaf(f, fmaf(d, t, lw), w);
  return r;
}
__device__ __forceinline__ Stat wave_merge(Stat s) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    Stat b;
    b.m = __shfl_xor(s.m, o);
    b.z = __shfl_xor(s.z, o);
    b.w = __shfl_xor(s.w, o);
    s = merge(s, b);
  }
  return s;
}

// A wave's list of candidates (wave-uniform fields; buf in LDS, CAP entries).
struct Top {
  u64 *buf;
  u64 thr;        // a candidate has to be larger
  float thrf;     // thr's value (-infinity before there is one)
  int n, count;

  __device__ void init(u64 *b, int n_) {
    buf = b;
    n = n_;
    thr = 0;
    thrf = -INFINITY;
    count = 0;
  }
  __device__ __forceinline__ void set(u64 t) {
    if (t > thr) {
      thr = t;
      thrf = comp_value(t);
    }
  }
  // Keeps the n largest, in order.  Entries are distinct, so ranks are too.
  __device__ void cut() {
    const int lane = threadIdx.x & 63;
    u64 e[CAP / 64];
    int rank[CAP / 64];
#pragma unroll
    for (int k = 0; k < CAP / 64; k++) {
      e[k] = lane + 64 * k < count ? buf[lane + 64 * k] : 0;
      rank[k] = 0;
    }
    for (int j = 0; j < count; j++) {
      const u64 x = buf[j];
#pragma unroll
      for (int k = 0; k < CAP / 64; k++) rank[k] += x > e[k] ? 1 : 0;
    }
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int k = 0; k < CAP / 64; k++)
      if (e[k] && rank[k] < n) buf[rank[k]] = e[k];
    __builtin_amdgcn_wave_barrier();
    count = min(count, n);
    if (count == n) set(buf[n - 1]);
  }
  // One candidate of each lane with `c` above the threshold (0: none).
  __device__ __forceinline__ void push(u64 c) {
    u64 mask = __ballot(c > thr);
    if (!mask) return;
    if (count > CAP - 64) {
      cut();
      mask = __ballot(c > thr);
    }
    if (c > thr)
      buf[count + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32),
                                            __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0))] = c;
    count += __popcll(mask);
  }
  // A first threshold: just below the n-th largest of the lanes' own maxima.
  __device__ void seed(u64 own) {
    const uint32_t lo = (uint32_t)own, hi = (uint32_t)(own >> 32);
    int rank = 0;
    for (int j = 0; j < 64; j++) {
      const u64 o = (u64)(uint32_t)__builtin_amdgcn_readlane((int)hi, j) << 32 |
                    (uint32_t)__builtin_amdgcn_readlane((int)lo, j);
      rank += o > own ? 1 : 0;
    }
    const u64 at = __ballot(rank == n - 1 && own != 0);
    if (!at) return;                         // fewer than n lanes hold a value
    const int l = __ffsll((long long)at) - 1;
    set(((u64)(uint32_t)__builtin_amdgcn_readlane((int)hi, l) << 32 |
         (uint32_t)__builtin_amdgcn_readlane((int)lo, l)) - 1);
  }
};

// One row's result from its statistics (bad: NaN or +infinity among the
// logits); top: its n best in order, written by the wave's lanes.
struct Out {
  const float *row;
  const int32_t *targets;
  float *logprob, *entropy;
  int32_t *ids;
  float *top;
};
__device__ __forceinline__ void write_row(const Out &o, int64_t t, int V, int n, Stat s, bool bad,
                                          const u64 *best) {
  const int lane = threadIdx.x & 63;
  const float nan = __builtin_nanf("");
  const bool none = !(1.0f + s.z > 0.0f);      // nothing but -infinity
  const float lz = log1pf(s.z);
  const auto logp = [&](float l) {
    return bad ? nan : none ? -INFINITY : (l - s.m) - lz;
  };
  if (lane == 0) {
    if (o.targets) {
      const int64_t g = o.targets[t];
      o.logprob[t] = g < 0 || g >= V ? 0.0f : logp(o.row[g]);
    }
    if (o.entropy) o.entropy[t] = bad ? nan : none ? 0.0f : lz - s.w / (1.0f + s.z);
  }
  if (lane < n) {
    const u64 c = best[lane];
    o.ids[t * n + lane] = (int32_t)comp_index(c);
    o.top[t * n + lane] = logp(comp_value(c));
  }
}

// A span's result in the workspace: 16 bytes of statistics, then n candidates.
struct Part {
  float m, z, w;
  uint32_t bad;
};

// Merges the waves' statistics and lists; wave 0 returns the whole.
template <bool TOP>
__device__ __forceinline__ void block_merge(Stat &s, bool &bad, Top &top, u64 (*buf)[CAP],
                                            Part *sh, int *counts) {
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  s = wave_merge(s);
  if (TOP) top.cut();
  if (lane == 0) {
    sh[wave] = {s.m, s.z, s.w, bad};
    counts[wave] = TOP ? top.count : 0;
  }
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int i = 1; i < LW; i++) {
    Stat b;
    b.m = sh[i].m; b.z = sh[i].z; b.w = sh[i].w;
    s = merge(s, b);
    bad |= sh[i].bad != 0;
    if (TOP) top.push(lane < counts[i] ? buf[i][lane] : 0);
  }
  if (TOP) top.cut();
}

// Workgroup: span blockIdx % S of row blockIdx / S.  Groups of four values
// are counted from the 16-byte boundary at or below the row's start.
template <bool TOP>
__global__ __launch_bounds__(LT) void logprobs_kernel(const float *__restrict__ logits,
                                                      int64_t stride, Out o, int64_t T, int V,
                                                      int n, int S, uint8_t *__restrict__ ws,
                                                      int64_t part_bytes) {
  __shared__ u64 buf[TOP ? LW : 1][CAP];
  __shared__ Part sh[LW];
  __shared__ int counts[LW];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  for (int64_t item = blockIdx.x; item < T * S; item += gridDim.x) {
    const int64_t t = item / S;
    const int span = (int)(item - t * S);
    const float *row = logits + t * stride;
    const int a = (int)((t * stride) & 3);         // elements before the row in its first group
    const float4 *base = reinterpret_cast<const float4 *>(row - a);
    const int G = (a + V + 3) / 4;
    const int per = ((G + CHUNK - 1) / CHUNK + S - 1) / S * CHUNK;
    const int g0 = min(span * per, G), g1 = min(g0 + per, G);
    Stat s;
    s.init();
    bool bad = false;
    Top top;
    if (TOP) top.init(buf[wave], n);
    bool first = true;
    // groups that lie whole in the row
    const int whole0 = a ? 1 : 0, whole1 = (a + V) / 4;

    float4 v[UG], nx[UG];
    const auto load = [&](int c, float4 (&d)[UG]) {
      // clamped, always valid addresses; the rest is masked afterwards
#pragma unroll
      for (int u = 0; u < UG; u++) {
        const int g = min(c + u * 64 + lane, whole1 - 1);
        d[u] = whole1 > 0 ? base[g] : make_float4(0.f, 0.f, 0.f, 0.f);
      }
    };
    int c = g0 + wave * CHUNK;
    if (c < g1) load(c, v);
    for (; c < g1; c += LW * CHUNK) {
      if (c + LW * CHUNK < g1) load(c + LW * CHUNK, nx);
      const bool edge = c < whole0 || c + CHUNK > min(g1, whole1);
      float x[4 * UG];
#pragma unroll
      for (int u = 0; u < UG; u++) {
        x[4 * u] = v[u].x; x[4 * u + 1] = v[u].y; x[4 * u + 2] = v[u].z; x[4 * u + 3] = v[u].w;
      }
      uint32_t here = 0xFFFFu;
      if (edge) {
        here = 0;
#pragma unroll
        for (int u = 0; u < UG; u++)
#pragma unroll
          for (int i = 0; i < 4; i++) {
            const int g = c + u * 64 + lane, e = 4 * g + i - a;
            const bool in = g < g1 && e >= 0 && e < V;
            here |= in ? 1u << (4 * u + i) : 0u;
            if (in && g >= whole1) x[4 * u + i] = row[e];
            if (!in) x[4 * u + i] = -INFINITY;
          }
      }
      float cm = x[0];
      bool odd = false;
#pragma unroll
      for (int i = 0; i < 4 * UG; i++) {
        cm = fmaxf(cm, x[i]);
        odd |= !(x[i] < INFINITY);
      }
      bad |= odd;
      const float mn = fmaxf(s.m, cm);
      const float dm = fmaxf(s.m - mn, FAR), f = exp_f(dm), t1 = 1.0f + s.z;
      float zs = 0.0f, wsum = 0.0f;
      int same = 0;
#pragma unroll
      for (int i = 0; i < 4 * UG; i++) {
        const float d = x[i] - mn, e = exp_f(d);
        const bool eq = x[i] == mn;
        same += eq ? 1 : 0;
        zs += eq ? 0.0f : e;
        wsum = fmaf(e, fmaxf(d, FAR), wsum);
      }
      if (mn > s.m) {                              // the maximum's own 1 stays out
        s.w = fmaf(f, fmaf(dm, t1, s.w), wsum);
        s.z = fmaf(t1, f, zs + (float)(same - 1));
        s.m = mn;
      } else {
        s.w += wsum;
        s.z += zs + (float)same;
      }
      if (TOP) {
        if (__ballot(odd || !(cm < top.thrf))) {
          const auto comp = [&](int i) -> u64 {
            const uint32_t e = (uint32_t)(4 * (c + (i / 4) * 64 + lane) + (i & 3) - a);
            return here >> i & 1u ? comp_of(x[i], e) : 0;
          };
          if (first) {
            u64 own = 0;
#pragma unroll
            for (int i = 0; i < 4 * UG; i++) {
              const u64 q = comp(i);
              own = q > own ? q : own;
            }
            top.seed(own);
          }
#pragma unroll
          for (int i = 0; i < 4 * UG; i++) top.push(comp(i));
        }
        first = false;
      }
#pragma unroll
      for (int u = 0; u < UG; u++) v[u] = nx[u];
    }
    bad = __ballot(bad) != 0;
    block_merge<TOP>(s, bad, top, buf, sh, counts);
    if (wave == 0) {
      if (S == 1) {
        Out r = o;
        r.row = row;
        write_row(r, t, V, n, s, bad, buf[0]);
      } else {
        uint8_t *p = ws + item * part_bytes;
        if (lane == 0) *reinterpret_cast<Part *>(p) = {s.m, s.z, s.w, bad};
        if (TOP && lane < n)
          reinterpret_cast<u64 *>(p + sizeof(Part))[lane] = lane < top.count ? buf[0][lane] : 0;
      }
    }
    __syncthreads();
  }
}

// One workgroup a row: its S spans' statistics and candidates.
template <bool TOP>
__global__ __launch_bounds__(LT) void combine_spans_kernel(const float *__restrict__ logits,
                                                           int64_t stride, Out o, int V, int n,
                                                           int S, const uint8_t *__restrict__ ws,
                                                           int64_t part_bytes) {
  __shared__ u64 buf[TOP ? LW : 1][CAP];
  __shared__ Part sh[LW];
  __shared__ int counts[LW];
  const int64_t t = blockIdx.x;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const uint8_t *p = ws + t * S * part_bytes;
  Stat s;
  s.init();
  bool bad = false;
  for (int i = threadIdx.x; i < S; i += LT) {
    const Part q = *reinterpret_cast<const Part *>(p + i * part_bytes);
    Stat b;
    b.m = q.m; b.z = q.z; b.w = q.w;
    s = merge(s, b);
    bad |= q.bad != 0;
  }
  bad = __ballot(bad) != 0;
  Top top;
  if (TOP) {
    top.init(buf[wave], n);
    const auto cand = [&](int span, int j) -> u64 {
      return span < S ? reinterpret_cast<const u64 *>(p + span * part_bytes + sizeof(Part))[j] : 0;
    };
    // lane: a span; its candidates come in order, so once no lane's next one
    // beats the threshold the rest does not either
    for (int s0 = wave * 64; s0 < S; s0 += LT) {
      u64 c = cand(s0 + lane, 0);
      if (S - s0 >= n) top.seed(c);
      for (int j = 0; j < n; j++) {
        if (!__ballot(c > top.thr)) break;
        top.push(c);
        c = j + 1 < n ? cand(s0 + lane, j + 1) : 0;
      }
    }
  }
  block_merge<TOP>(s, bad, top, buf, sh, counts);
  if (wave == 0) {
    Out r = o;
    r.row = logits + t * stride;
    write_row(r, t, V, n, s, bad, buf[0]);
  }
}

// Spans of a row: enough for two workgroups on each of 256 compute units, of
// up to one chunk for each wave (16 KB) and more.
int spans(int64_t T, int64_t V) {
  const int64_t want = (512 + T - 1) / T, most = (V + 3 + 4 * CHUNK * LW - 1) / (4 * CHUNK * LW);
  return (int)std::max<int64_t>(1, std::min(want, most));
}
int64_t part_bytes(int64_t n) { return (int64_t)sizeof(Part) + 8 * n + (n & 1) * 8; }

}  // namespace
}  // namespace w4a8

using namespace w4a8;

static int logprobs_sizes(int64_t T, int64_t V, int64_t n_top) {
  if (T < 0 || V < 1) return W4A8_ESHAPE;
  if (V >= (1 << 24) || T >= ((int64_t)1 << 31) || n_top < 0 || n_top > NTOP_MAX || n_top > V)
    return W4A8_ERANGE;
  return W4A8_OK;
}

extern "C" size_t token_logprobs_workspace_size(int64_t T, int64_t V, int64_t n_top) {
  if (logprobs_sizes(T, V, n_top) != W4A8_OK) return 0;
  if (T == 0) return 16;
  return (size_t)std::max<int64_t>(16, T * spans(T, V) * part_bytes(n_top));
}

extern "C" int token_logprobs(const float *logits, int64_t stride, const int32_t *targets,
                              float *logprob, float *entropy, int32_t *top_ids,
                              float *top_logprobs, int64_t T, int64_t V, int64_t n_top,
                              void *workspace, size_t ws_bytes, void *stream) {
  if (!logits || !workspace || !targets != !logprob) return W4A8_ENULL;
  if (int rc = logprobs_sizes(T, V, n_top); rc != W4A8_OK) return rc;
  if (n_top > 0 && (!top_ids || !top_logprobs)) return W4A8_ENULL;
  if (stride < V) return W4A8_ESHAPE;
  if (stride >= ((int64_t)1 << 40) || (T > 0 && stride > ((int64_t)1 << 40) / T))
    return W4A8_ERANGE;
  const uintptr_t m = reinterpret_cast<uintptr_t>(targets) | reinterpret_cast<uintptr_t>(logprob) |
                      reinterpret_cast<uintptr_t>(entropy) | reinterpret_cast<uintptr_t>(top_ids) |
                      reinterpret_cast<uintptr_t>(top_logprobs);
  if (!aligned16(logits) || !aligned16(workspace) || (m & 3u)) return W4A8_EALIGN;
  if (ws_bytes < token_logprobs_workspace_size(T, V, n_top)) return W4A8_EWORKSPACE;
  if (T == 0) return W4A8_OK;
  if (int rc = check_device(); rc != W4A8_OK) return rc;
  const int S = spans(T, V);
  const int64_t pb = part_bytes(n_top);
  const Out o = {nullptr, targets, logprob, entropy, top_ids, top_logprobs};
  const dim3 grid((unsigned)std::min<int64_t>(T * S, 1 << 22));
  uint8_t *ws = reinterpret_cast<uint8_t *>(workspace);
  const hipStream_t st = as_stream(stream);
  const auto go = [&](auto top) {
    constexpr bool TOP = decltype(top)::value;
    logprobs_kernel<TOP><<<grid, dim3(LT), 0, st>>>(logits, stride, o, T, (int)V, (int)n_top, S,
                                                    ws, pb);
    int rc = check_launch();
    if (rc != W4A8_OK || S == 1) return rc;
    combine_spans_kernel<TOP><<<dim3((unsigned)T), dim3(LT), 0, st>>>(
        logits, stride, o, (int)V, (int)n_top, S, ws, pb);
    return check_launch();
  };
  return n_top > 0 ? go(std::true_type{}) : go(std::false_type{});
}
