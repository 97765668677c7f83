// Probabilities of logits rows and verification of drafted tokens (include/wt_serve.h).
//
// Both walk rows of a vocabulary with a cluster of CTAs per row, so that a single row is spread
// over several SMs: each CTA takes a contiguous part of the row, and the few numbers that the whole
// row decides (largest logit and sum; 64-bit weight sums) cross the cluster through distributed
// shared memory.
#include <cooperative_groups.h>

#include "wt_device.cuh"
#include "wt_serve.h"

namespace wt {

namespace {

namespace cg = cooperative_groups;

constexpr int kStatusInvalid = -1;  // WT_EINVAL
constexpr int kThreads = 512;
constexpr int kWarps = kThreads / 32;
constexpr int kHeld = 32;  // logits of a row part that a thread keeps in registers
constexpr int kMaxCluster = 8;

__device__ __forceinline__ void note_invalid(int *status) {
  if (status) atomicCAS(status, 0, kStatusInvalid);
}

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ unsigned long long warp_sum(unsigned long long v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// The part of a row of n elements that CTA c of C takes: whole groups of 4 elements, evenly.
__device__ __forceinline__ void row_part(int n, int c, int C, int &lo, int &hi) {
  const int groups = (n + 3) / 4, per = (groups + C - 1) / C;
  lo = min(n, c * per * 4);
  hi = min(n, lo + per * 4);
}

// ------------------------------------------------------------------ probabilities
// p = exp((l - m) / t) / S.  One read and one write of each element: a thread keeps its logits in
// registers between the maximum, the sum and the store.  Each CTA takes exponentials against its own
// maximum; the row's maximum and sum come from one exchange of (maximum, sum) pairs, and the CTA's
// exponentials are scaled by exp((m_cta - m) / t) / S.  Bound: HBM.
struct RowPart {
  float m;    // the part's largest logit
  float s;    // sum of exp((l - m) / t) over it
  int first;  // first index of m
};

__global__ void __launch_bounds__(kThreads, 1) probs_kernel(const wt_probs_desc d) {
  __shared__ float red_f[kWarps];
  __shared__ int red_i[kWarps];
  __shared__ RowPart part;
  cg::cluster_group cl = cg::this_cluster();
  const int C = cl.num_blocks(), c = cl.block_rank();
  const int row = blockIdx.x / C, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const float *l = d.logits + (int64_t)row * d.ldl;
  float *p = d.p + (int64_t)row * d.ldp;
  const float t = d.temp ? d.temp[row] : 1.0f;
  const bool draw = t > 0.0f;
  int lo, hi;
  row_part(d.vocab, c, C, lo, hi);

  float v[kHeld];
  float m = -INFINITY;
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int i = lo + k * kThreads + tid;
    v[k] = i < hi ? l[i] : -INFINITY;
    m = fmaxf(m, v[k]);
  }
  for (int i = lo + kHeld * kThreads + tid; i < hi; i += kThreads) m = fmaxf(m, l[i]);
  m = warp_max(m);
  if (lane == 0) red_f[warp] = m;
  __syncthreads();
  m = red_f[0];
#pragma unroll
  for (int w = 1; w < kWarps; ++w) m = fmaxf(m, red_f[w]);
  __syncthreads();

  if (!draw) {
    // the first index of the part's maximum
    int first = INT32_MAX;
#pragma unroll
    for (int k = kHeld - 1; k >= 0; --k) {
      const int i = lo + k * kThreads + tid;
      if (i < hi && v[k] == m) first = i;
    }
    for (int i = lo + kHeld * kThreads + tid; i < hi && first == INT32_MAX; i += kThreads)
      if (l[i] == m) first = i;
    first = __reduce_min_sync(0xffffffffu, first);
    if (lane == 0) red_i[warp] = first;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kWarps; ++w) first = min(first, red_i[w]);
      part = {m, 0.0f, first};
    }
    cl.sync();
    float mr = -INFINITY;
    int at = -1;
    for (int q = 0; q < C; ++q) {
      const RowPart r = *cl.map_shared_rank(&part, q);
      if (r.m > mr) mr = r.m, at = r.first;
    }
    for (int i = lo + tid; i < hi; i += kThreads) p[i] = i == at ? 1.0f : 0.0f;
    cl.sync();
    return;
  }

  float s = 0.0f;
  const float mz = m > -INFINITY ? m : 0.0f;
  // a logit of -infinity is no token, whatever the temperature
  auto e = [&](float x) { return x == -INFINITY ? 0.0f : expf((x - mz) / t); };
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    v[k] = e(v[k]);
    s += v[k];
  }
  for (int i = lo + kHeld * kThreads + tid; i < hi; i += kThreads) s += e(l[i]);
  s = warp_sum(s);
  if (lane == 0) red_f[warp] = s;
  __syncthreads();
  if (tid == 0) {
    s = 0.0f;
    for (int w = 0; w < kWarps; ++w) s += red_f[w];
    part = {m, s, 0};
  }
  cl.sync();
  float mr = -INFINITY, sr = 0.0f;
  for (int q = 0; q < C; ++q) mr = fmaxf(mr, cl.map_shared_rank(&part, q)->m);
  for (int q = 0; q < C; ++q) {
    const RowPart r = *cl.map_shared_rank(&part, q);
    if (r.m > -INFINITY || r.s != 0.0f) sr += r.s * (r.m == mr ? 1.0f : expf((r.m - mr) / t));
  }
  // a row of -infinity alone: zeros
  const float f = mr == -INFINITY && sr == 0.0f ? 0.0f : (m == mr ? 1.0f : m > -INFINITY ? expf((m - mr) / t) : 0.0f);
  // NaN anywhere makes the sum NaN, and with it every element
  const float inv = mr == -INFINITY && sr == 0.0f ? 1.0f : sr;
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    const int i = lo + k * kThreads + tid;
    if (i < hi) p[i] = v[k] * f / inv;
  }
  for (int i = lo + kHeld * kThreads + tid; i < hi; i += kThreads) p[i] = e(l[i]) * f / inv;
  cl.sync();  // no CTA leaves while another may still read its part
}

// ------------------------------------------------------------------ verification
// Weights are integers, w(v) = floor(min(x, 1) 2^40): their sums are exact, so neither the split of a
// row over CTAs, warps and lanes nor the order of additions changes which token is drawn.  A warp
// takes a contiguous piece of its CTA's part; the piece that holds the drawn token is found from the
// pieces' sums, and only its warp looks at its elements again.
__device__ __forceinline__ unsigned long long weight(float x) {
  return x > 0.0f ? (unsigned long long)(fminf(x, 1.0f) * 1099511627776.0f) : 0ull;  // NaN: 0
}

struct Sums {
  unsigned long long w, p;  // the part's sums of the weights, and of p's own
};

__global__ void __launch_bounds__(kThreads) verify_kernel(const wt_verify_desc d, int *status) {
  __shared__ Sums warp_sums[kWarps];
  __shared__ Sums cta_sums;
  cg::cluster_group cl = cg::this_cluster();
  const int C = cl.num_blocks(), c = cl.block_rank();
  const int b = blockIdx.x / C, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  int n0 = d.begin[b], n1 = d.begin[b + 1];
  if (n0 < 0 || n1 < n0 || n1 > d.n_drafted || n1 - n0 > d.max_draft) {
    if (tid == 0) note_invalid(status);
    n0 = min(max(n0, 0), d.n_drafted);
    n1 = min(max(n1, n0), min(d.n_drafted, n0 + d.max_draft));
  }
  const int n = n1 - n0;
  // Every warp finds the first refused draft for itself: lane i looks at draft i.
  int acc = n, last = -1;
  for (int i0 = 0; i0 < n; i0 += 32) {
    const int i = i0 + lane;
    bool stays = true;
    int tok = -1;
    if (i < n) {
      tok = d.drafted[n0 + i];
      if (tok < 0 || tok >= d.vocab) {
        stays = false;
        tok = -1;
        if (warp == 0) note_invalid(status);
      } else {
        const float pd = d.p[(int64_t)(n0 + b + i) * d.ldp + tok];
        const float qd = d.q ? d.q[(int64_t)(n0 + i) * d.ldq + tok] : 1.0f;
        stays = __fmul_rn(d.u[n0 + i], qd) < pd;
      }
    }
    const unsigned bad = __ballot_sync(0xffffffffu, !stays);
    if (bad) {
      const int f = __ffs(bad) - 1;
      acc = i0 + f;
      last = __shfl_sync(0xffffffffu, tok, f);
      break;
    }
  }
  const bool refused = acc < n;
  const float *p = d.p + (int64_t)(n0 + b + acc) * d.ldp;
  const float *q = refused && d.q ? d.q + (int64_t)(n0 + acc) * d.ldq : nullptr;
  const int gone = refused && !d.q ? last : -1;  // a certain draft leaves nothing of its token

  int lo, hi;
  row_part(d.vocab, c, C, lo, hi);
  const int per = ((hi - lo + kWarps - 1) / kWarps + 31) / 32 * 32;
  const int wlo = min(hi, lo + warp * per), whi = min(hi, wlo + per);
  unsigned long long sw = 0, sp = 0;
#pragma unroll 4
  for (int i = wlo + lane; i < whi; i += 32) {
    const float x = p[i];
    const float r = q ? x - q[i] : i == gone ? 0.0f : x;
    sw += weight(r);
    sp += weight(x);
  }
  sw = warp_sum(sw);
  sp = warp_sum(sp);
  if (lane == 0) warp_sums[warp] = {sw, sp};
  __syncthreads();
  if (tid == 0) {
    Sums s = {0, 0};
    for (int w = 0; w < kWarps; ++w) s.w += warp_sums[w].w, s.p += warp_sums[w].p;
    cta_sums = s;
  }
  cl.sync();
  unsigned long long before_w = 0, before_p = 0, all_w = 0, all_p = 0;
  for (int k = 0; k < C; ++k) {
    const Sums s = *cl.map_shared_rank(&cta_sums, k);
    if (k < c) before_w += s.w, before_p += s.p;
    all_w += s.w, all_p += s.p;
  }
  cl.sync();
  const bool plain = all_w == 0;  // nothing left of the residual: p itself
  const unsigned long long S = plain ? all_p : all_w;
  const float u = d.u_draw[b];
  const unsigned long long um = !(u > 0.0f) ? 0ull : u >= 1.0f ? (1ull << 24) - 1 : (unsigned long long)(u * 16777216.0f);
  const unsigned long long limit = um * (S >> 24) + ((um * (S & 0xffffffull)) >> 24);
  unsigned long long before = plain ? before_p : before_w;
  for (int w = 0; w < warp; ++w) before += plain ? warp_sums[w].p : warp_sums[w].w;
  const unsigned long long mine = plain ? warp_sums[warp].p : warp_sums[warp].w;
  int token = -1;
  if (S > 0 && before <= limit && limit < before + mine) {
    unsigned long long run = before;
    for (int i0 = wlo; i0 < whi; i0 += 32) {
      const int i = i0 + lane;
      unsigned long long w = 0;
      if (i < whi) {
        const float x = p[i];
        w = weight(plain ? x : q ? x - q[i] : i == gone ? 0.0f : x);
      }
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long up = __shfl_up_sync(0xffffffffu, w, o);
        if (lane >= o) w += up;
      }
      const unsigned over = __ballot_sync(0xffffffffu, run + w > limit);
      if (over) {
        token = i0 + __ffs(over) - 1;
        break;
      }
      run += __shfl_sync(0xffffffffu, w, 31);
    }
  }
  // one warp of the cluster drew; where nothing could be drawn, CTA 0 writes -1
  if (token >= 0 && lane == 0) d.tokens[(int64_t)b * (d.max_draft + 1) + acc] = token;
  if (c == 0) {
    if (tid == 0) {
      d.accepted[b] = acc;
      if (S == 0) d.tokens[(int64_t)b * (d.max_draft + 1) + acc] = -1;
    }
    for (int i = tid; i <= d.max_draft; i += kThreads)
      if (i != acc) d.tokens[(int64_t)b * (d.max_draft + 1) + i] = i < acc ? d.drafted[n0 + i] : -1;
  }
}

// CTAs per row: enough to give every SM work, of at least 2048 elements each.
int row_cluster(int rows, int vocab) {
  int c = 1;
  while (c < kMaxCluster && (int64_t)rows * c < num_sms() && vocab / (2 * c) >= 2048) c *= 2;
  // a thread keeps kHeld elements: longer parts are read twice
  while (c < kMaxCluster && vocab > c * kThreads * kHeld) c *= 2;
  return c;
}

template <typename... A>
cudaError_t launch_cluster(void (*k)(A...), int rows, int cluster, cudaStream_t s, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * cluster));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = (unsigned)cluster;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k, args...);
}

}  // namespace

cudaError_t launch_probs(const wt_probs_desc &d, cudaStream_t s) {
  return launch_cluster(probs_kernel, d.rows, row_cluster(d.rows, d.vocab), s, d);
}

cudaError_t launch_verify(const wt_verify_desc &d, int *status, cudaStream_t s) {
  return launch_cluster(verify_kernel, d.n_req, row_cluster(d.n_req, d.vocab), s, d, status);
}

}  // namespace wt
