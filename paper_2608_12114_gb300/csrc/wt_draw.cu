// Probabilities of logits rows and verification of drafted tokens (include/wt_serve.h).
//
// Both walk rows of a vocabulary with a cluster of CTAs per row, so that a single row is spread
// over several SMs: each CTA takes a contiguous part of the row, and the few numbers that the whole
// row decides (largest logit and sum; 64-bit weight sums) cross the cluster through distributed
// shared memory.
#include <cooperative_groups.h>

#include "wt_serve.cuh"

namespace wt {

namespace {

namespace cg = cooperative_groups;

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
  lo = min((int64_t)n, (int64_t)c * per * 4);
  hi = min((int64_t)n, (int64_t)lo + per * 4);
}

// ------------------------------------------------------------------ probabilities
// p = 2^((l - m) log2(e) / t) / S.  One read and one write of each element: the part of a row that a
// CTA takes lies in its shared memory between the maximum, the sum and the store (what does not fit,
// from 458,752 logits on, is read again).  Each CTA takes exponentials against its own maximum; the
// row's maximum and sum come from one exchange of (maximum, sum) pairs, and the CTA's exponentials
// are scaled by 2^((m_cta - m) log2(e) / t) / S.  Rows on 16-byte boundaries arrive as one bulk copy, which
// needs no registers, three CTAs of 64 KB to an SM.  Bound: HBM, with loads, exponentials and stores of
// the CTAs on an SM in step: 257 rows of 128256 (264 MB) 58 us, 4.5 TB/s.  Slower, same rows: the part in
// registers 242 us, 512 threads 66, parts of 32 KB in clusters of 16 72, one CTA per SM with three rows
// in turn 96 (clusters of 8 at one CTA per SM leave a fifth of the SMs over).
constexpr int kPThreads = 256;
constexpr int kPWarps = kPThreads / 32;
constexpr int kPartGoal = 16384;   // logits of a part where the cluster may grow: 64 KB
constexpr int kPartMost = 57344;   // logits that fit a CTA's shared memory

struct RowPart {
  float m;    // the part's largest logit
  float s;    // sum of the part's exponentials
  int first;  // first index of m
};

// 2^(2 x): the square keeps subnormal results, without the tests that the function's own way takes, at twice
// its relative error, 2^-21 at most.  A probability is off by that, by its sum's (the same and the additions'),
// and by 3 2^-24 ln 2 of its exponent for the roundings of x: over 257 rows of 128256 6.5e-8 in the 2-norm,
// elementary fp32 operations 8.4e-8.
__device__ __forceinline__ float exp2_twice(float x) {
  const float y = exp2_approx(x);
  return y * y;
}

__global__ void __launch_bounds__(kPThreads, 3) probs_kernel(const wt_probs_desc d, const int held_most, int *status) {
  extern __shared__ __align__(128) uint8_t dyn[];
  float *sv = reinterpret_cast<float *>(dyn);
  __shared__ float red_f[kPWarps];
  __shared__ int red_i[kPWarps];
  __shared__ RowPart part;
  __shared__ __align__(8) uint64_t bar_mem;
  __shared__ int aborted;
  cg::cluster_group cl = cg::this_cluster();
  const int C = cl.num_blocks(), c = cl.block_rank();
  const int row = blockIdx.x / C, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  int lo, hi;
  row_part(d.vocab, c, C, lo, hi);
  const float *l = d.logits + (int64_t)row * d.ldl + lo;
  float *p = d.p + (int64_t)row * d.ldp + lo;
  const int n = hi - lo, held = min(n, held_most);
  const float t = d.temp ? d.temp[row] : 1.0f;
  const bool draw = t > 0.0f;

  const bool vec_in = reinterpret_cast<uintptr_t>(l) % 16 == 0;
  if (vec_in) {
    const uint32_t bar = smem_u32(&bar_mem);
    if (tid == 0) {
      aborted = 0;
      mbar_init(bar, 1);
      mbar_fence_init();
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      const uint32_t bytes = (uint32_t)(held & ~3) * 4;
      mbar_expect_tx(bar, bytes);
      const uint64_t pol = l2_evict_first_policy();
      for (uint32_t o = 0; o < bytes; o += 32768)
        bulk_g2s(smem_u32(sv) + o, reinterpret_cast<const uint8_t *>(l) + o, min(32768u, bytes - o), bar, pol);
    }
    __syncthreads();
    if (tid < (held & 3)) sv[(held & ~3) + tid] = l[(held & ~3) + tid];
    if (!bounded_wait(bar, 0, &aborted, status)) {
      // the copy must not land in another CTA's shared memory: give it as long again
      const long long t0 = clock64();
      while (!mbar_try_wait(bar, 0) && clock64() - t0 < kWaitCycles) {
      }
    }
  } else {
#pragma unroll 8
    for (int i = tid; i < held; i += kPThreads) sv[i] = l[i];
  }
  __syncthreads();

  const int held4 = held / 4;
  const float4 *sv4 = reinterpret_cast<const float4 *>(sv);
  float m = -INFINITY;
#pragma unroll 4
  for (int i = tid; i < held4; i += kPThreads) {
    const float4 v = sv4[i];
    m = fmaxf(m, fmaxf(fmaxf(v.x, v.y), fmaxf(v.z, v.w)));
  }
  for (int i = held4 * 4 + tid; i < n; i += kPThreads) m = fmaxf(m, i < held ? sv[i] : l[i]);
  m = warp_max(m);
  if (lane == 0) red_f[warp] = m;
  __syncthreads();
  m = red_f[0];
#pragma unroll
  for (int w = 1; w < kPWarps; ++w) m = fmaxf(m, red_f[w]);
  __syncthreads();

  if (!draw) {
    // the first index of the part's maximum
    int first = INT32_MAX;
    for (int i = tid; i < n && first == INT32_MAX; i += kPThreads)
      if ((i < held ? sv[i] : l[i]) == m) first = i + lo;
    first = __reduce_min_sync(0xffffffffu, first);
    if (lane == 0) red_i[warp] = first;
    __syncthreads();
    if (tid == 0) {
      for (int w = 1; w < kPWarps; ++w) first = min(first, red_i[w]);
      part = {m, 0.0f, first};
    }
    cl.sync();
    float mr = -INFINITY;
    int at = -1;
    for (int q = 0; q < C; ++q) {
      const RowPart r = *cl.map_shared_rank(&part, q);
      if (r.m > mr) mr = r.m, at = r.first;
    }
    cluster_arrive();
    for (int i = tid; i < n; i += kPThreads) p[i] = i + lo == at ? 1.0f : 0.0f;
    cluster_wait();
    return;
  }

  // log2(e) / 2 t.  Beyond the largest number any factor sends every logit but the largest to 0, and one
  // above 0 a logit of -infinity, whatever the temperature.
  const float k = fmaxf(fminf(0.72134752044448170f / t, 3.4028234e38f), 1.1754944e-38f);
  const float mz = m > -INFINITY ? m : 0.0f;
  auto e = [&](float x) { return exp2_twice((x - mz) * k); };
  float s = 0.0f;
#pragma unroll 4
  for (int i = tid; i < held4; i += kPThreads) {
    float4 v = sv4[i];
    v.x = e(v.x), v.y = e(v.y), v.z = e(v.z), v.w = e(v.w);
    s += (v.x + v.y) + (v.z + v.w);
    reinterpret_cast<float4 *>(sv)[i] = v;
  }
  for (int i = held4 * 4 + tid; i < n; i += kPThreads) {
    const float v = e(i < held ? sv[i] : l[i]);
    s += v;
    if (i < held) sv[i] = v;
  }
  s = warp_sum(s);
  if (lane == 0) red_f[warp] = s;
  __syncthreads();
  if (tid == 0) {
    s = 0.0f;
    for (int w = 0; w < kPWarps; ++w) s += red_f[w];
    part = {m, s, 0};
  }
  cl.sync();
  float mr = -INFINITY, sr = 0.0f;
  RowPart all[kMaxCluster];
#pragma unroll
  for (int q = 0; q < kMaxCluster; ++q) {
    all[q] = q < C ? *cl.map_shared_rank(&part, q) : RowPart{-INFINITY, 0.0f, 0};
    mr = fmaxf(mr, all[q].m);
  }
  cluster_arrive();  // before the stores: a barrier after them would wait for them to be done
  auto scale = [&](float mc) { return mc == mr ? 1.0f : mc > -INFINITY ? exp2_twice((mc - mr) * k) : 0.0f; };
#pragma unroll
  for (int q = 0; q < kMaxCluster; ++q)
    if (all[q].s != 0.0f) sr += all[q].s * scale(all[q].m);
  // a row of -infinity alone has the sum 0: zeros.  NaN anywhere makes the sum NaN, and every element.
  const float f = sr == 0.0f ? 0.0f : scale(m) / sr;
  if (reinterpret_cast<uintptr_t>(p) % 16 == 0) {
#pragma unroll 4
    for (int i = tid; i < held4; i += kPThreads) {
      float4 v = sv4[i];
      v.x *= f, v.y *= f, v.z *= f, v.w *= f;
      __stcs(reinterpret_cast<float4 *>(p) + i, v);
    }
    for (int i = held4 * 4 + tid; i < held; i += kPThreads) p[i] = sv[i] * f;
  } else {
    for (int i = tid; i < held; i += kPThreads) p[i] = sv[i] * f;
  }
  for (int i = held + tid; i < n; i += kPThreads) p[i] = e(l[i]) * f;
  cluster_wait();  // no CTA leaves while another may still read its part
}

// ------------------------------------------------------------------ verification
// Weights are integers, w(v) = floor(min(x, 1) 2^40): their sums are exact, so neither the split of a
// row over CTAs, warps and lanes nor the order of additions changes which token is drawn.  A warp
// takes chunks of 512 elements, each lane 4 vectors of p and of q in flight; the chunk that holds the
// drawn token is found from the chunks' sums, and only that chunk is looked at again, in order.
// Bound: HBM for many requests, the chain of dependent reads (offsets, drafted tokens, their
// probabilities, the rows) for few: 64 requests' rows of 128256 (57 MB) 17 us, one request 6.  Loops
// stay short because a call runs each instruction once or twice, and fetching long unrolled code cost
// more than it saved (13.8 us for one request).
constexpr int kVThreads = 512;
constexpr int kVWarps = kVThreads / 32;
constexpr int kChunk = 512;
constexpr int kMaxChunks = (WT_VERIFY_MAX_VOCAB + kChunk - 1) / kChunk + 1;

// The mantissa shifted into place: conversions to 64-bit integers run at a sixteenth of the rate.
__device__ __forceinline__ unsigned long long weight(float x) {
  const uint32_t b = __float_as_uint(fminf(x, 1.0f));
  const unsigned long long m = (unsigned long long)((b & 0x7fffffu) | 0x800000u) << 17;
  return x > 0.0f ? m >> min(127u - (b >> 23), 63u) : 0ull;  // NaN: 0
}

// Inclusive running sums of w over the warp.  Returns the first lane whose sum, after `run`, exceeds
// limit (32: none) and adds to run what lies before that lane.
__device__ __forceinline__ int first_over(unsigned long long w, unsigned long long &run, unsigned long long limit, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const unsigned long long up = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += up;
  }
  const unsigned over = __ballot_sync(0xffffffffu, run + w > limit);
  const int f = over ? __ffs(over) - 1 : 32;
  const unsigned long long add = __shfl_sync(0xffffffffu, w, f ? f - 1 : 0);
  if (f) run += add;
  return f;
}

__global__ void __launch_bounds__(kVThreads, 2) verify_kernel(const wt_verify_desc d, int *status) {
  __shared__ unsigned long long chunk_sum[kMaxChunks];
  __shared__ unsigned long long cta_sum;
  cg::cluster_group cl = cg::this_cluster();
  const int C = cl.num_blocks(), c = cl.block_rank();
  const int b = blockIdx.x / C, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  int n0 = d.begin[b], n1 = d.begin[b + 1];
  const float u = d.u_draw[b];
  if (n0 < 0 || n1 < n0 || n1 > d.n_drafted || n1 - n0 > d.max_draft) {
    if (tid == 0) note_invalid(status);
    n0 = min(max(n0, 0), d.n_drafted);
    n1 = min(max(n1, n0), n0 + min(d.max_draft, d.n_drafted - n0));
  }
  const int n = n1 - n0;
  // Every warp finds the first refused draft for itself: lane i looks at draft i.
  int acc = n, last = -1;
  for (int i0 = 0; i0 < n; i0 += 32) {
    const int i = i0 + lane;
    bool stays = true;
    int tok = -1;
    if (i < n) {
      const float ui = d.u[n0 + i];
      tok = d.drafted[n0 + i];
      if (tok < 0 || tok >= d.vocab) {
        stays = false;
        tok = -1;
        if (warp == 0) note_invalid(status);
      } else {
        const float pd = d.p[(int64_t)(n0 + b + i) * d.ldp + tok];
        const float qd = d.q ? d.q[(int64_t)(n0 + i) * d.ldq + tok] : 1.0f;
        stays = __fmul_rn(ui, qd) < pd;
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
  int gone = refused && !d.q ? last : -1;  // a certain draft leaves nothing of its token

  int lo, hi;
  row_part(d.vocab, c, C, lo, hi);
  const int chunks = (hi - lo + kChunk - 1) / kChunk;
  const bool vec = reinterpret_cast<uintptr_t>(p + lo) % 16 == 0 && (!q || reinterpret_cast<uintptr_t>(q + lo) % 16 == 0);
  // The four elements from i on (i - lo a multiple of 4): what is left of p, 0 past the part's end.
  auto left4 = [&](int i, float (&x)[4]) {
    if (vec && i + 4 <= hi) {
      const float4 a = __ldg(reinterpret_cast<const float4 *>(p + i));
      const float4 r = q ? __ldg(reinterpret_cast<const float4 *>(q + i)) : make_float4(0, 0, 0, 0);
      x[0] = a.x - r.x, x[1] = a.y - r.y, x[2] = a.z - r.z, x[3] = a.w - r.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = i + e < hi ? __ldg(p + i + e) - (q ? __ldg(q + i + e) : 0.0f) : 0.0f;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (i + e == gone) x[e] = 0.0f;
  };
  unsigned long long S = 0, before = 0;
  // a second time, from p alone, where the residual leaves nothing
  for (int pass = 0; pass < 2 && S == 0; ++pass) {
    if (pass) {
      cluster_wait();  // everyone has read the first sums
      q = nullptr;
      gone = -1;
    }
#pragma unroll 1
    for (int k = warp; k < chunks; k += kVWarps) {
      float x[kChunk / 128][4];
#pragma unroll
      for (int j = 0; j < kChunk / 128; ++j) left4(lo + k * kChunk + j * 128 + lane * 4, x[j]);
      unsigned long long s = 0;
#pragma unroll
      for (int j = 0; j < kChunk / 128; ++j) s += (weight(x[j][0]) + weight(x[j][1])) + (weight(x[j][2]) + weight(x[j][3]));
      s = warp_sum(s);
      if (lane == 0) chunk_sum[k] = s;
    }
    __syncthreads();
    if (warp == 0) {
      unsigned long long s = 0;
      for (int k = lane; k < chunks; k += 32) s += chunk_sum[k];
      s = warp_sum(s);
      if (lane == 0) cta_sum = s;
    }
    cl.sync();
    before = 0;
#pragma unroll
    for (int k = 0; k < kMaxCluster; ++k)
      if (k < C) {
        const unsigned long long s = *cl.map_shared_rank(&cta_sum, k);
        if (k < c) before += s;
        S += s;
      }
    cluster_arrive();
  }
  const unsigned long long um = !(u > 0.0f) ? 0ull : u >= 1.0f ? (1ull << 24) - 1 : (unsigned long long)(u * 16777216.0f);
  const unsigned long long limit = um * (S >> 24) + ((um * (S & 0xffffffull)) >> 24);
  int32_t *out = d.tokens + (int64_t)b * (d.max_draft + 1);
  if (warp == 0 && S > 0 && before <= limit && limit < before + cta_sum) {
    // the first chunk whose running sum passes the limit, then the vector, then the element
    unsigned long long run = before;
    int at = 0;
    for (int k0 = 0; k0 < chunks; k0 += 32) {
      const int f = first_over(k0 + lane < chunks ? chunk_sum[k0 + lane] : 0ull, run, limit, lane);
      if (f < 32) {
        at = k0 + f;
        break;
      }
    }
#pragma unroll 1
    for (int j = 0; j < kChunk / 128; ++j) {
      const int i = lo + at * kChunk + j * 128 + lane * 4;
      float x[4];
      left4(i, x);
      unsigned long long w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = weight(x[e]);
      const int f = first_over((w[0] + w[1]) + (w[2] + w[3]), run, limit, lane);
      if (f == 32) continue;
      if (lane == f) {
        int e = 0;
        while (e < 3 && (run += w[e]) <= limit) ++e;
        out[acc] = i + e;
      }
      break;
    }
  }
  if (c == 0) {
    if (tid == 0) {
      d.accepted[b] = acc;
      if (S == 0) out[acc] = -1;
    }
    for (int i = tid; i <= d.max_draft; i += kVThreads)
      if (i != acc) out[i] = i < acc ? d.drafted[n0 + i] : -1;
  }
  cluster_wait();  // no CTA leaves while another may still read its sum
}

// CTAs per row: enough to give every SM work, of at least 2048 elements each.
int row_cluster(int rows, int vocab) {
  int c = 1;
  while (c < kMaxCluster && (int64_t)rows * c < num_sms() && vocab / (2 * c) >= 2048) c *= 2;
  return c;
}

template <typename... A>
cudaError_t launch_cluster(void (*k)(A...), int rows, int cluster, int threads, size_t smem, cudaStream_t s, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(rows * cluster));
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
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

cudaError_t draw_prepare() {
  return cudaFuncSetAttribute(probs_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPartMost * 4);
}

cudaError_t launch_probs(const wt_probs_desc &d, int *status, cudaStream_t s) {
  int c = row_cluster(d.rows, d.vocab);
  while (c < kMaxCluster && d.vocab > c * kPartGoal) c *= 2;
  const int part = (int)(((int64_t)d.vocab + 4 * c - 1) / (4 * c) * 4), held = part < kPartMost ? part : kPartMost;
  return launch_cluster(probs_kernel, d.rows, c, kPThreads, (size_t)held * 4, s, d, held, status);
}

cudaError_t launch_verify(const wt_verify_desc &d, int *status, cudaStream_t s) {
  return launch_cluster(verify_kernel, d.n_req, row_cluster(d.n_req, d.vocab), kVThreads, 0, s, d, status);
}

}  // namespace wt
