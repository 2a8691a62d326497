// Log probabilities of given tokens, entropy and top alternatives, read off
// the output head's logits (the decode head of Sec. 5.2) in one pass.
//
// A row is cut into S spans, one workgroup each (S = 1 once the rows fill the
// compute units), and the last of them to finish joins their results, in their
// order; every wave streams its share of a span in chunks of 16
// values a lane, the next chunk's loads under way, and keeps
//   - the softmax statistics (m, z, w): the maximum so far, the sum of
//     exp(l - m) WITHOUT the maximum's own 1, and sum exp(l - m) (l - m), each
//     lane its share of the sums.  With z kept apart from the 1, log Z =
//     log1p(z) is accurate to fp32 for a confident row too, whose log Z may be
//     1e-6.  One maximum for the wave: chunks that raise it are few, and in the
//     others every value, its equal too, is one difference, exponential and
//     two sums (a maximum a lane had its 1 to look for in every chunk);
//   - per wave the n largest logits: a list in LDS of candidates that beat a
//     threshold, cut back to the n best (by counting, for each candidate, the
//     larger ones) when it fills.  The first threshold is a value that n of
//     the 64 lanes reach in the first chunk, so nothing below it belongs to
//     the n best.  After that a random row sends a candidate every few hundred
//     values.
// Bound by HBM: 4 bytes a logit, read once, about 13 VALU ops a value.  947
// rows of 151936 logits with 5 alternatives take 130 us (4.4 TB/s); one row
// with 20 takes 13 us, a chain of launch, one pass of its spans and their join.
#include <algorithm>
#include <cfloat>
#include <type_traits>

#include "share_dev.h"
#include "w4a8_dev.h"
#include "w4a8_host.h"

namespace w4a8 {

namespace {

constexpr int LT = 256;
constexpr int LW = LT / 64;
constexpr int UG = 4;                    // 4-value groups of a lane's chunk
constexpr int CHUNK = 64 * UG;           // groups of a wave's chunk
constexpr int CAP = 192;                 // candidates of a wave's list
constexpr int PAD = 8;
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

// exp(d), FAR <= d <= 0.  exp2 of the rounded product t = d log2(e) alone would
// be off by |d| 2^-24, which a confident row, whose sum hangs on a few values,
// shows in full (3e-7 in its log probability; so 5e-8): what t leaves out of d
// comes in to first order.
__device__ __forceinline__ float exp_f(float d) {
  const float t = d * 1.44269502f, e = __builtin_amdgcn_exp2f(t);
  return fmaf(e, fmaf(t, -0.693147181f, d), e);
}

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
  u64 thr;        // a candidate has to be larger; 0, or n values met are
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
      // (just below -infinity's key lie NaN's bits)
      thrf = (uint32_t)(t >> 32) < 0x007FFFFFu ? -INFINITY : comp_value(t);
    }
  }
  // Entries of buf larger than each of e (eight at a time: the list is padded
  // with zeros, which are larger than nothing).
  template <int N> __device__ __forceinline__ void ranks(const u64 (&e)[N], int (&rank)[N]) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int k = 0; k < N; k++) rank[k] = 0;
    if (lane < 8) buf[count + lane] = 0;
    __builtin_amdgcn_wave_barrier();
#pragma unroll 1
    for (int j = 0; j < count; j += 8) {
      u64 x[8];
#pragma unroll
      for (int i = 0; i < 8; i++) x[i] = buf[j + i];
#pragma unroll
      for (int i = 0; i < 8; i++)
#pragma unroll
        for (int k = 0; k < N; k++) rank[k] += x[i] > e[k] ? 1 : 0;
    }
    __builtin_amdgcn_wave_barrier();
  }
  // Keeps the n largest, in order.  Entries are distinct, so ranks are too.
  template <int N> __device__ __forceinline__ void cut_of() {
    const int lane = threadIdx.x & 63;
    u64 e[N];
    int rank[N];
#pragma unroll
    for (int k = 0; k < N; k++) e[k] = lane + 64 * k < count ? buf[lane + 64 * k] : 0;
    ranks<N>(e, rank);
#pragma unroll
    for (int k = 0; k < N; k++)
      if (e[k] && rank[k] < n) buf[rank[k]] = e[k];
    __builtin_amdgcn_wave_barrier();
    count = min(count, n);
    // below the n-th, so that n values lie above it in a list filled anew too
    // (no borrow from the value: an index is below 2^24, its part not 0)
    if (count == n) set(buf[n - 1] - 1);
  }
  __device__ __forceinline__ void cut() {
    if (count <= 64) cut_of<1>();
    else cut_of<CAP / 64>();
  }
  __device__ __forceinline__ void append(u64 c, bool take, u64 mask) {
    if (take)
      buf[count + __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32),
                                            __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0))] = c;
    count += __popcll(mask);
  }
  // One candidate of each lane with `c` above the threshold (0: none).
  __device__ __forceinline__ void push(u64 c) {
    u64 mask = __ballot(c > thr);
    if (!mask) return;
    if (count > CAP - 64) {
      cut();
      mask = __ballot(c > thr);
    }
    append(c, c > thr, mask);
  }
  // N of each lane, those that take(i) names with candidates comp(i), where
  // they fit; else false, and nothing has changed.
  template <int N, typename F, typename G>
  __device__ __forceinline__ bool push_all(F &&take, G &&comp) {
    u64 mask[N];
    int total = count;
#pragma unroll
    for (int i = 0; i < N; i++) {
      mask[i] = __ballot(take(i));
      total += __popcll(mask[i]);
    }
    if (total > CAP) return false;
#pragma unroll
    for (int i = 0; i < N; i++)
      if (mask[i]) append(comp(i), mask[i] >> (threadIdx.x & 63) & 1, mask[i]);
    return true;
  }
  // A first threshold from the lanes' own maxima: the largest 16-bit prefix of
  // a value that n lanes reach, found bit by bit.
  __device__ __forceinline__ void seed(u64 own) {
    const uint32_t key = (uint32_t)(own >> 48);
    uint32_t at = 0;
#pragma unroll
    for (int bit = 15; bit >= 0; bit--) {
      const uint32_t t = at | 1u << bit;
      if (__popcll(__ballot(key >= t)) >= n) at = t;
    }
    if (at) set(((u64)at << 48) - 1);        // (0: fewer than n lanes hold a value)
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
__device__ __forceinline__ void block_merge(Stat &s, bool &bad, Top &top, u64 (*buf)[CAP + PAD],
                                            Part *sh, int *counts, u64 *thrs) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (lane == 0) {
    sh[wave] = {s.m, s.z, s.w, bad};
    counts[wave] = TOP ? top.count : 0;
    if (TOP) thrs[wave] = top.thr;
  }
  __syncthreads();
  if (wave != 0) return;
#pragma unroll
  for (int i = 1; i < LW; i++) {
    Stat b;
    b.m = sh[i].m; b.z = sh[i].z; b.w = sh[i].w;
    s = merge(s, b);
    bad |= sh[i].bad != 0;
    // n values of one wave lie above its threshold, so it holds for all
    if (TOP) top.set(thrs[i]);
  }
  if (TOP) {
    // the lists' first 64 at once, over a threshold that n lanes' best reach
    u64 c[LW], own = 0;
#pragma unroll
    for (int i = 0; i < LW; i++) {
      c[i] = lane < counts[i] ? buf[i][lane] : 0;
      own = c[i] > own ? c[i] : own;
    }
    const int mine = counts[0];
    top.seed(own);
    const uint32_t least = max((uint32_t)(top.thr >> 32), 1u);
    u64 more[CAP / 64 - 1];                       // of the own list, which is written over
#pragma unroll
    for (int k = 0; k < CAP / 64 - 1; k++) more[k] = lane + 64 * (k + 1) < mine ? buf[0][lane + 64 * (k + 1)] : 0;
    top.count = 0;
    if (!top.push_all<LW>([&](int i) { return (uint32_t)(c[i] >> 32) >= least; },
                          [&](int i) { return c[i]; })) {
#pragma unroll 1
      for (int i = 0; i < LW; i++) top.push(i == 0 ? c[0] : lane < counts[i] ? buf[i][lane] : 0);
    }
    if (mine > 64) {
#pragma unroll
      for (int k = 0; k < CAP / 64 - 1; k++) top.push(more[k]);
    }
#pragma unroll 1
    for (int i = 1; i < LW; i++)
#pragma unroll 1
      for (int j = 64; j < counts[i]; j += 64) top.push(j + lane < counts[i] ? buf[i][j + lane] : 0);
    top.cut();
  }
}

// 4-byte words of a span's result.
__host__ __device__ constexpr int part_words(int n) { return 4 + 2 * (n + (n & 1)); }

// A row's S spans, each thread's in turn.
template <bool TOP>
__device__ __forceinline__ void join_spans(Rsrc rs, int words, const Out &o, int64_t t, int V, int n,
                                           int S, u64 (*buf)[CAP + PAD], Part *sh, int *counts,
                                           u64 *thrs) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  Stat s;
  s.init();
  bool bad = false;
  Top top;
  if (TOP) top.init(buf[wave], n);
#pragma unroll 1
  for (int s0 = wave * 64; s0 < S; s0 += LT) {
    const bool in = s0 + lane < S;
    const int at = min(s0 + lane, S - 1) * words;
    const v4f q = shared4(rs, at);
    u64 c[16];
    if (TOP) {
#pragma unroll
      for (int j = 0; j < 16; j += 2) {          // (part_words rounds n up to even)
        const v4u x = __builtin_bit_cast(v4u, shared4(rs, at + 4 + 2 * min(j, (n - 1) & ~1)));
        c[j] = in && j < n ? (u64)x[1] << 32 | x[0] : 0;
        c[j + 1] = in && j + 1 < n ? (u64)x[3] << 32 | x[2] : 0;
      }
    }
    Stat b;
    b.m = q[0]; b.z = q[1]; b.w = q[2];
    if (in) {
      s = merge(s, b);
      bad |= q[3] != 0.0f;
    }
    if (TOP) {
      if (S - s0 >= n) top.seed(c[0]);
      // the candidates come in order: where the first 16 do not fit the list,
      // or there are more, one by one until no lane's beats the threshold
      const uint32_t least = max((uint32_t)(top.thr >> 32), 1u);
      int j = top.push_all<16>([&](int i) { return (uint32_t)(c[i] >> 32) >= least; },
                               [&](int i) { return c[i]; }) ? 16 : 0;
#pragma unroll 1
      for (; j < n; j++) {
        const u64 x = __builtin_bit_cast(u64, shared2(rs, at + 4 + 2 * j));
        if (!__ballot(in && x > top.thr)) break;
        top.push(in ? x : 0);
      }
    }
  }
  bad = __ballot(bad) != 0;
  s = wave_merge(s);
  if (S > 64) {
    block_merge<TOP>(s, bad, top, buf, sh, counts, thrs);
  } else if (wave == 0) {                          // the other waves have had none
    if (TOP) top.cut();
  }
  if (wave == 0) write_row(o, t, V, n, s, bad, buf[0]);
}

// Workgroup: span blockIdx % S of row blockIdx / S.  Groups of four values
// are counted from the 16-byte boundary at or below the row's start.
template <bool TOP, bool SPLIT>
__global__ __launch_bounds__(LT, 4) void logprobs_kernel(const float *__restrict__ logits,
                                                      int64_t stride, Out o, int64_t T, int V,
                                                      int n, int S, int *count, uint8_t *ws) {
  __shared__ __align__(16) u64 buf[TOP ? LW : 1][CAP + PAD];
  __shared__ Part sh[LW];
  __shared__ int counts[LW];
  __shared__ u64 thrs[LW];
  __shared__ int flag;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  for (int64_t item = blockIdx.x; item < T * S; item += gridDim.x) {
    const int64_t t = SPLIT ? item / S : item;
    const int span = SPLIT ? (int)(item - t * S) : 0;
    const float *row = logits + t * stride;
    const int a = (int)((t * stride) & 3);         // elements before the row in its first group
    const float4 *base = reinterpret_cast<const float4 *>(row - a);
    const int G = (a + V + 3) / 4;
    const int per = ((G + CHUNK - 1) / CHUNK + S - 1) / S * CHUNK;
    const int g0 = min(span * per, G), g1 = min(g0 + per, G);
    float m = -INFINITY, z = 0.0f, w = 0.0f;       // m is the wave's, z and w are the lane's shares
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
      if (TOP) {
        if (__ballot(odd || !(cm < top.thrf))) {
          const auto at = [&](int i) { return (uint32_t)(4 * (c + (i / 4) * 64 + lane) + (i & 3) - a); };
          if (first) {
            u64 own = 0;
#pragma unroll
            for (int i = 0; i < 4 * UG; i++)
              if (here >> i & 1u) {
                const u64 q = comp_of(x[i], at(i));
                own = q > own ? q : own;
              }
            top.seed(own);
          }
          // by the value alone: one more of the threshold's own value does no harm
          const float least = top.thrf;
          if (__ballot(odd) ||
              !top.push_all<4 * UG>([&](int i) { return (here >> i & 1u) && x[i] >= least; },
                                    [&](int i) { return comp_of(x[i], at(i)); })) {
            // more than the list takes: one by one, read again (kept out of the
            // unrolled code, which a short row is bound by fetching)
#pragma unroll 1
            for (int i = 0; i < 4 * UG; i++) {
              const int g = c + (i / 4) * 64 + lane, e = 4 * g + (i & 3) - a;
              const bool in = g < g1 && e >= 0 && e < V;
              top.push(in ? comp_of(row[e], (uint32_t)e) : 0);
            }
          }
        }
        first = false;
      }
      if (__ballot(cm > m)) {                      // a new maximum: its own 1 stays out
        float mn = cm;
#pragma unroll
        for (int k = 32; k > 0; k >>= 1) mn = fmaxf(mn, __shfl_xor(mn, k));
        const float dm = fmaxf(m - mn, FAR), f = exp_f(dm);
        const float t1 = lane == 0 && m > -INFINITY ? z + 1.0f : z;     // the former one's goes in
        w = f * fmaf(dm, t1, w);
        z = f * t1;
        m = mn;
        bool out = lane == __ffsll((long long)__ballot(cm == mn)) - 1;
#pragma unroll
        for (int i = 0; i < 4 * UG; i++) {
          const bool eq = out && x[i] == mn;
          if (eq) x[i] = -INFINITY;
          out = out && !eq;
        }
      }
      float zs = 0.0f, wsum = 0.0f;
#pragma unroll
      for (int i = 0; i < 4 * UG; i++) {
        const float d = fmaxf(x[i] - m, FAR), e = exp_f(d);
        zs += e;
        wsum = fmaf(e, d, wsum);
      }
      z += zs;
      w += wsum;
#pragma unroll
      for (int u = 0; u < UG; u++) v[u] = nx[u];
    }
    bad = __ballot(bad) != 0;
#pragma unroll
    for (int k = 32; k > 0; k >>= 1) {
      z += __shfl_xor(z, k);
      w += __shfl_xor(w, k);
    }
    Stat s;
    s.init();
    if (m > -INFINITY) {
      s.m = m; s.z = z; s.w = w;
    }
    block_merge<TOP>(s, bad, top, buf, sh, counts, thrs);
    Out r = o;
    r.row = row;
    if constexpr (!SPLIT) {
      if (wave == 0) write_row(r, t, V, n, s, bad, buf[0]);
    } else {
      // the last span of the row to get here joins them all
      const int words = part_words(n);
      const Rsrc rs = shared_at(ws + t * S * words * 4);
      if (wave == 0) {
        if (lane == 0)
          share(rs, span * words, v4f{s.m, s.z, s.w, bad ? 1.0f : 0.0f});
        if (TOP && lane < n) {
          const u64 c = lane < top.count ? buf[0][lane] : 0;
          share(rs, span * words + 4 + 2 * lane, __builtin_bit_cast(v2f, c));
        }
      }
      if (last_of(count + t, S, &flag)) join_spans<TOP>(rs, words, r, t, V, n, S, buf, sh, counts, thrs);
    }
    __syncthreads();
  }
}

// Spans of a row: enough for two workgroups on each of 256 compute units, of
// up to one chunk for each wave (16 KB) and more.
int spans(int64_t T, int64_t V) {
  const int64_t want = (512 + T - 1) / T, most = (V + 3 + 4 * CHUNK * LW - 1) / (4 * CHUNK * LW);
  return (int)std::max<int64_t>(1, std::min(want, most));
}
constexpr int64_t COUNTERS = 512 * 4;            // an arrival count a row, before the parts

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
  const int64_t S = T == 0 ? 1 : spans(T, V);
  return S == 1 ? 16 : (size_t)(COUNTERS + T * S * part_words((int)n_top) * 4);
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
  const Out o = {nullptr, targets, logprob, entropy, top_ids, top_logprobs};
  const dim3 grid((unsigned)std::min<int64_t>(T * S, 1 << 22));
  int *count = reinterpret_cast<int *>(workspace);
  uint8_t *ws = reinterpret_cast<uint8_t *>(workspace) + COUNTERS;
  const auto go = [&](auto top, auto split) {
    logprobs_kernel<decltype(top)::value, decltype(split)::value>
        <<<grid, dim3(LT), 0, as_stream(stream)>>>(logits, stride, o, T, (int)V, (int)n_top, S, count, ws);
    return check_launch();
  };
  const std::true_type yes;
  const std::false_type no;
  if (n_top > 0) return S > 1 ? go(yes, yes) : go(yes, no);
  return S > 1 ? go(no, yes) : go(no, no);
}
