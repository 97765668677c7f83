// Log probabilities, entropy and the likeliest tokens of logits rows (include/wt_serve.h).
//
// One reading of each row, spread over a cluster of CTAs where rows are few.  Per row, with
// x = (l - m) log2(e) / t for the largest logit m:
//
//   s = sum over all but one of the largest of 2^x,      log S = log1p(s)
//   w = sum of x 2^x,                                    H = log1p(s) - ln 2 w / (1 + s)
//
// The largest logit's own 1 stays out of s, so that a sharp row keeps its entropy and its likeliest token's
// log probability to fp32's precision: nothing is subtracted (w <= 0).  A thread keeps (m, s, w) of what it has
// seen; two of them, m1 >= m2, join as s1 + f (s2 + 1) and w1 + f (w2 + d (s2 + 1)), d = (m2 - m1) log2(e) / t,
// f = 2^d: threads, warps and CTAs in a fixed order.
//
// Alternatives: a warp keeps the 32 largest (logit, token) it has seen, one a lane, in order.  The warps of a CTA
// share the best of their n_top-th logits: what lies under it is not among the row's n_top, whatever the timing.
// A candidate is found by one comparison of 16 logits' maximum; n ln(V / n) of a row's V are taken up.  At the
// end each of up to 256 candidates counts those above it, first among the warps, then among the CTAs.
#include <cooperative_groups.h>

#include <algorithm>

#include "wt_serve.cuh"

namespace wt {

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kVecs = 4;  // 16-byte vectors of a lane in flight
constexpr int kTop = WT_LOGPROBS_MAX_TOP;
static_assert(kTop == 32, "one candidate a lane");

typedef unsigned long long Key;  // order of the logit, then ~token: the larger comes first; 0: none

__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);  // -0 is 0
  return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t o) { return __uint_as_float(o ^ (o >> 31 ? 0x80000000u : 0xffffffffu)); }
__device__ __forceinline__ Key key_of(float v, int token) { return (Key)order_of(v) << 32 | (uint32_t)~token; }

struct Sums {
  float m;    // largest logit
  int first;  // its first token
  float s, w;
};

// d = (m2 - m1) k stays above -200, where 2^d is 0 and d times it, too
__device__ __forceinline__ Sums join(const Sums &a, const Sums &b, float k) {
  const bool ab = a.m > b.m || (a.m == b.m && a.first < b.first) || !(b.m > -INFINITY);
  const Sums &x = ab ? a : b, &y = ab ? b : a;
  const bool some = y.m > -INFINITY;
  const float d = some ? fmaxf((y.m - x.m) * k, -200.0f) : -200.0f, f = exp2_approx(d), n = y.s + 1.0f;
  return {x.m, x.first, x.s + f * n, x.w + f * (y.w + d * n)};
}

__device__ __forceinline__ Sums shuffle(const Sums &a, int o) {
  return {__shfl_xor_sync(0xffffffffu, a.m, o), __shfl_xor_sync(0xffffffffu, a.first, o), __shfl_xor_sync(0xffffffffu, a.s, o),
          __shfl_xor_sync(0xffffffffu, a.w, o)};
}

// Into the warp's list (descending over the lanes).
__device__ __forceinline__ void insert(Key &mine, Key c, int lane) {
  const Key up = __shfl_up_sync(0xffffffffu, mine, 1);
  if (mine < c) mine = lane && up < c ? up : c;
}

template <bool TOP>
__global__ void __launch_bounds__(kThreads) logprobs_kernel(const wt_logprobs_desc d, int *status) {
  __shared__ Sums warp_sums[kWarps];
  __shared__ Sums cta_sums;
  __shared__ Key cand[kWarps * kTop];  // of the warps; then, in the first CTA, of the CTAs
  __shared__ Key best[kTop];           // of the CTA
  __shared__ unsigned floor_order;
  cg::cluster_group cl = cg::this_cluster();
  const int C = cl.num_blocks(), c = cl.block_rank();
  const int row = blockIdx.x / C, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const float *l = d.logits + (int64_t)row * d.ldl;
  const float t = d.temp ? d.temp[row] : 1.0f;
  const bool draw = t > 0.0f;
  // Beyond the largest number any factor sends every logit but the largest to 0, and one above 0 a logit of
  // -infinity, whatever the temperature.
  const float k = draw ? fmaxf(fminf(1.4426950408889634f / t, 3.4028234e38f), 1.1754944e-38f) : 1.0f;
  if (TOP) {
    if (tid == 0) floor_order = 0;
    for (int i = tid; i < kWarps * kTop; i += kThreads) cand[i] = 0;
    for (int i = tid; i < kTop; i += kThreads) best[i] = 0;
    __syncthreads();
  }

  // The row's vectors start at the 16-byte boundary at or before it: `off` elements of the first are not its.
  const int off = (int)(reinterpret_cast<uintptr_t>(l) / 4 % 4);
  const int64_t vecs = ((int64_t)d.vocab + off + 3) / 4, per = (vecs + C - 1) / C;
  const int64_t lo = c * per, hi = min(vecs, lo + per);
  Sums a = {-INFINITY, INT32_MAX, 0.0f, 0.0f};
  Key list = 0;
  float least = -3.4028234e38f;  // a candidate is at least that: neither NaN nor -infinity
  for (int64_t j0 = lo; j0 < hi; j0 += kThreads * kVecs) {
    float v[kVecs][4];
    const int64_t j1 = j0 + warp * 32 * kVecs + lane;  // a warp's vectors lie together, in ascending order
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int64_t j = j1 + i * 32, e0 = 4 * j - off;
      if (j < hi && e0 >= 0 && e0 + 4 <= d.vocab) {
        const float4 x = __ldcs(reinterpret_cast<const float4 *>(l + e0));
        v[i][0] = x.x, v[i][1] = x.y, v[i][2] = x.z, v[i][3] = x.w;
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i][e] = j < hi && e0 + e >= 0 && e0 + e < d.vocab ? __ldcs(l + e0 + e) : -INFINITY;
      }
    }
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) top = fmaxf(top, fmaxf(fmaxf(v[i][0], v[i][1]), fmaxf(v[i][2], v[i][3])));
    const int e1 = (int)(4 * j1 - off);  // token of v[0][0]
    int skip = -1;  // the new largest one's place
    if (top > a.m) {
#pragma unroll
      for (int i = kVecs - 1; i >= 0; --i)
#pragma unroll
        for (int e = 3; e >= 0; --e)
          if (v[i][e] == top) skip = i * 4 + e;
      if (a.m > -INFINITY) {
        const float dd = fmaxf((a.m - top) * k, -200.0f), f = exp2_approx(dd), n = a.s + 1.0f;
        a.w = f * (a.w + dd * n);
        a.s = f * n;
      }
      a.m = top;
      a.first = e1 + (skip >> 2) * 128 + (skip & 3);
    }
    const float mz = a.m > -INFINITY ? a.m : 0.0f;
    float s[2] = {0.0f, 0.0f}, w[2] = {0.0f, 0.0f};
    if (skip >= 0) {
#pragma unroll
      for (int i = 0; i < kVecs; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = (v[i][e] - mz) * k, p = i * 4 + e == skip ? 0.0f : exp2_approx(x);
          s[e & 1] += p;
          w[e & 1] += p * fmaxf(x, -200.0f);
        }
    } else {
#pragma unroll
      for (int i = 0; i < kVecs; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float x = (v[i][e] - mz) * k, p = exp2_approx(x);
          s[e & 1] += p;
          w[e & 1] += p * fmaxf(x, -200.0f);  // 0 where p is
        }
    }
    a.s += s[0] + s[1];
    a.w += w[0] + w[1];

    if (TOP) {
      if (__any_sync(0xffffffffu, top >= least)) {
        least = fmaxf(least, logit_of(max(*reinterpret_cast<volatile unsigned *>(&floor_order), order_of(-3.4028234e38f))));
        Key last = __shfl_sync(0xffffffffu, list, d.n_top - 1);
        bool more = false;
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const Key mine = v[i][e] >= least ? key_of(v[i][e], e1 + i * 128 + e) : 0;
            unsigned who = __ballot_sync(0xffffffffu, mine > last);
            while (who) {
              const int from = __ffs(who) - 1;
              insert(list, __shfl_sync(0xffffffffu, mine, from), lane);
              last = __shfl_sync(0xffffffffu, list, d.n_top - 1);
              who = __ballot_sync(0xffffffffu, mine > last) & ~((2u << from) - 1);
              more = true;
            }
          }
        if (more && last) {
          const uint32_t o = (uint32_t)(last >> 32);
          least = fmaxf(least, logit_of(o));
          if (lane == 0) atomicMax(&floor_order, o);
        }
      }
    }
  }

  // the warps' sums, in order
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const Sums b = shuffle(a, o);
    a = lane & o ? join(b, a, k) : join(a, b, k);
  }
  if (lane == 0) warp_sums[warp] = a;
  if (TOP && lane < d.n_top) cand[warp * kTop + lane] = list;
  __syncthreads();
  if (tid == 0) {
    a = warp_sums[0];
    for (int i = 1; i < kWarps; ++i) a = join(a, warp_sums[i], k);
    cta_sums = a;
  }
  // a candidate's place is the number of those above it
  auto choose = [&](Key mine, int n, auto put) {
    if (!mine) return;
    int above = 0;
    for (int i = 0; i < n; ++i) above += cand[i] > mine;
    if (above < d.n_top) put(above, mine);
  };
  if (TOP) choose(cand[tid], kWarps * kTop, [&](int at, Key mine) { best[at] = mine; });
  static_assert(kWarps * kTop == kThreads && kMaxCluster <= kWarps, "a candidate a thread");
  cl.sync();
  if (c == 0) {
    a = cta_sums;
    for (int q = 1; q < C; ++q) a = join(a, *cl.map_shared_rank(&cta_sums, q), k);
    const bool bad = draw && (a.m == INFINITY || a.s != a.s), none = !(a.m > -INFINITY);
    const float log_s = log1pf(a.s);
    auto logp = [&](float x, int token) -> float {
      if (bad) return NAN;
      if (none || !(x > -INFINITY)) return -INFINITY;
      if (!draw) return token == a.first ? 0.0f : -INFINITY;
      return (x - a.m) / t - log_s;
    };
    if (tid == 0 && d.entropy) d.entropy[row] = bad ? NAN : none || !draw ? 0.0f : log_s - 0.69314718055994531f * a.w / (1.0f + a.s);
    for (int i = tid; i < d.n_given; i += kThreads) {
      const int token = d.given[(int64_t)row * d.given_stride + i];
      float lp = 0.0f;
      if (token >= d.vocab) {
        if (status) atomicCAS(status, 0, kStatusInvalid);
      } else if (token >= 0) {
        lp = logp(l[token], token);
      }
      d.given_lp[(int64_t)row * d.n_given + i] = lp;
    }
    if (TOP) {
      auto put = [&](int at, Key key) {
        const int token = (int)~(uint32_t)key;
        d.top[(int64_t)row * d.n_top + at] = key ? token : -1;
        d.top_lp[(int64_t)row * d.n_top + at] = key ? logp(logit_of((uint32_t)(key >> 32)), token) : bad ? NAN : -INFINITY;
      };
      if (C > 1) {
        const int q = tid / kTop, i = tid % kTop;
        const Key mine = q < C ? cl.map_shared_rank(best, q)[i] : 0;
        __syncthreads();  // the warps' candidates have been read
        cand[tid] = mine;
        if (tid < kTop) best[tid] = 0;  // no other CTA reads it
        __syncthreads();
        choose(mine, C * kTop, [&](int at, Key key) { best[at] = key; });
        __syncthreads();
      }
      if (tid < d.n_top) put(tid, best[tid]);
    }
  }
  cl.sync();  // no CTA leaves while the first may still read its numbers
}

template <bool TOP>
cudaError_t run(const wt_logprobs_desc &d, int cluster, int *status, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(d.rows * cluster));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)cluster;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, logprobs_kernel<TOP>, d, status);
}

}  // namespace

cudaError_t launch_logprobs(const wt_logprobs_desc &d, int *status, cudaStream_t s) {
  // Parts of at least 4096 logits, one for each vector a lane has in flight, and as many CTAs as eight to an SM hold.
  int c = 1;
  while (c < kMaxCluster && (int64_t)d.rows * c < 6ll * num_sms() && d.vocab / (2 * c) >= 4096) c *= 2;
  return d.n_top ? run<true>(d, c, status, s) : run<false>(d, c, status, s);
}

}  // namespace wt
