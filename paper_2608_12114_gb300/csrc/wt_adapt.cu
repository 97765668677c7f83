// Low-rank adapters of many requests beside a shared projection (include/wt_serve.h):
// y[t] = base[t] + scale_s B_s (A_s x[t]), s = slot[t].
//
// One launch, one cluster of 8 CTAs per work item (projection, slot, up to kTile tokens of that
// slot).  The cluster computes v = A x with each CTA taking an eighth of K, exchanges the partial
// sums through distributed shared memory (always added in the order of the CTAs), and then each CTA
// takes an eighth of the M outputs.  A and B are read once per item, B's lines being fetched into L2
// while A is read; x and y cross once.  The slot map lies in device memory, so the items are found
// there too: every CTA counts the tokens of each slot and picks its own.  Bound: HBM for prompts,
// latency (two dependent reads and a cluster barrier) for decode steps.
//
// Products run on the tensor cores.  A x: 16-bit operands, exact products, fp32 sums.  B v: B is
// exact in tf32 (both 16-bit types fit), and v, held in fp32, is split into two tf32 numbers, so that
// v enters with 22 bits and y keeps fp32's precision; one 16-bit number would leave 2^-9 of the update.
#include <algorithm>
#include <type_traits>

#include <cooperative_groups.h>

#include "wt_device.cuh"
#include "wt_serve.h"

namespace wt {

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256;
constexpr int kWarps = 8;
constexpr int kCluster = 8;
constexpr int kStatusInvalid = -1;

__device__ __forceinline__ void mma_tf32(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t to_tf32(float f) {
  uint32_t r;
  asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(r) : "f"(f));
  return r;
}

// Two 16-bit numbers of a word as fp32 bits (exact, and exact in tf32).
template <int DT>
__device__ __forceinline__ void widen(uint32_t w, uint32_t &lo, uint32_t &hi) {
  if constexpr (DT == WT_BF16) {
    lo = w << 16;
    hi = w & 0xffff0000u;
  } else {
    float a, b;
    asm("{\n\t.reg .f16 x, y;\n\tmov.b32 {x, y}, %2;\n\tcvt.f32.f16 %0, x;\n\tcvt.f32.f16 %1, y;\n\t}"
        : "=f"(a), "=f"(b)
        : "r"(w));
    lo = __float_as_uint(a);
    hi = __float_as_uint(b);
  }
}

// Elements [k, k + 8) of a row of n elements, zeros past its end.
template <bool VEC>
__device__ __forceinline__ uint4 load8(const uint16_t *row, int k, int n) {
  if (k >= n) return make_uint4(0, 0, 0, 0);
  if constexpr (VEC) {
    return __ldg(reinterpret_cast<const uint4 *>(row + k));
  } else {
    uint16_t e[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) e[i] = k + i < n ? __ldg(row + k + i) : (uint16_t)0;
    return make_uint4(e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16, e[4] | (uint32_t)e[5] << 16,
                      e[6] | (uint32_t)e[7] << 16);
  }
}

// The first `keep` elements of 8, zeros for the others.
__device__ __forceinline__ uint4 keep8(const uint4 &v, int keep) {
  return keep >= 8 ? v : and4(v, byte_mask(0, 2 * keep));
}

struct Item {
  int slot;   // S: tokens without an adapter
  int count;  // tokens
};

// MT: 16-row tiles of the rank (R <= 16 MT).  WT: groups of 16 tokens, each with 8 / WT warps.
template <int DT, int MT, int WT>
__global__ void __launch_bounds__(kThreads) adapt_kernel(const __grid_constant__ AdaptLaunch L, int *status) {
  constexpr int kTile = 16 * WT;
  constexpr int kR = 16 * MT;
  constexpr int WK = kWarps / WT;  // warps that share a group of tokens
  extern __shared__ __align__(16) uint8_t smem[];
  float *part = reinterpret_cast<float *>(smem);          // [WK][kTile][kR] the warps' sums, then [kTile][kR] in part 0
  float *vfull = part + WK * kTile * kR;                  // [kTile][kR + 4] v of the whole cluster
  int *cnt = reinterpret_cast<int *>(vfull + kTile * (kR + 4));  // [S + 1]
  __shared__ Item s_item;
  __shared__ int s_first;             // ordinal, within the slot, of the item's first token
  __shared__ int tok[kTile];
  __shared__ int wsum[kWarps];
  cg::cluster_group cl = cg::this_cluster();
  const int c = cl.block_rank();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  // the projection and the item of this cluster
  int pi = 0;
  uint32_t w = blockIdx.x / kCluster;
  while (pi + 1 < L.n && w >= L.p[pi].items) w -= L.p[pi++].items;
  const AdaptProj &P = L.p[pi];
  const wt_adapt_desc &d = P.d;
  const int T = d.T, K = d.K, M = d.M, S = d.S, R = d.R;

  auto slot_of = [&](int t) {
    const int s = __ldg(d.slot + t);
    if (s >= S) return -1;
    return s;
  };
  const bool copy = d.base != d.y;  // tokens without adapter have work only where y is not base
  for (int s = tid; s <= S; s += kThreads) cnt[s] = 0;
  if (tid == 0) s_item = {-1, 0};
  __syncthreads();
  for (int t = tid; t < T; t += kThreads) {
    const int s = __ldg(d.slot + t);
    if (s >= S && c == 0 && status) atomicCAS(status, 0, kStatusInvalid);
    if (s >= 0 && s < S) atomicAdd(cnt + s, 1);
    else if (copy) atomicAdd(cnt + S, 1);
  }
  __syncthreads();
  if (warp == 0) {
    int seen = 0;
    for (int s0 = 0; s0 <= S; s0 += 32) {
      const int s = s0 + lane;
      const int n = s <= S ? cnt[s] : 0, tiles = (n + kTile - 1) / kTile;
      int run = tiles;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += up;
      }
      const int before = seen + run - tiles;
      if ((int)w >= before && (int)w < before + tiles) {
        s_first = ((int)w - before) * kTile;
        s_item = {s, min(kTile, n - s_first)};
      }
      seen += __shfl_sync(0xffffffffu, run, 31);
    }
  }
  __syncthreads();
  const Item item = s_item;
  if (item.slot < 0) return;  // the whole cluster: no work for this item
  const int first = s_first;
  // its tokens: those of the slot with ordinals first .. first + count - 1, in order
  for (int t0 = 0, seen = 0; t0 < T && seen < first + item.count; t0 += kThreads) {
    const int t = t0 + tid;
    bool mine = false;
    if (t < T) {
      const int s = slot_of(t);
      mine = item.slot == S ? s < 0 : s == item.slot;
    }
    const unsigned bal = __ballot_sync(0xffffffffu, mine);
    if (lane == 0) wsum[warp] = __popc(bal);
    __syncthreads();
    int at = seen + __popc(bal & ((1u << lane) - 1));
    int all = seen;
    for (int q = 0; q < kWarps; ++q) {
      if (q < warp) at += wsum[q];
      all += wsum[q];
    }
    if (mine && at >= first && at < first + item.count) tok[at - first] = t;
    seen = all;
    __syncthreads();
  }

  const int q = lane & 3, g = lane >> 2;
  const int wt = warp / WK, wk = warp % WK;
  // outputs of this CTA: whole groups of 16
  const int mper = ((M + 15) / 16 + kCluster - 1) / kCluster * 16;
  const int m0 = min(M, c * mper), m1 = min(M, m0 + mper);
  int r = 0;  // the slot's rank
  const uint16_t *A = nullptr, *B = nullptr;
  if (item.slot < S) {
    r = d.rank ? __ldg(d.rank + item.slot) : R;
    if (r < 0 || r > R) {
      if (tid == 0 && c == 0 && status) atomicCAS(status, 0, kStatusInvalid);
      r = min(max(r, 0), R);
    }
    A = static_cast<const uint16_t *>(d.A) + (int64_t)item.slot * d.a_slot;
    B = static_cast<const uint16_t *>(d.B) + (int64_t)item.slot * d.b_slot;
  }

  if (r > 0) {
    // B's rows of this CTA on their way into L2
    {
      const uint64_t lo = reinterpret_cast<uint64_t>(B + (int64_t)m0 * R), hi = reinterpret_cast<uint64_t>(B + (int64_t)m1 * R);
      for (uint64_t a = (lo & ~127ull) + 128ull * tid; a < hi; a += 128ull * kThreads)
        if (a >= lo) asm volatile("prefetch.global.L2 [%0];" ::"l"(a));
    }
    // v^T = A x^T over this CTA's part of K: M = rank, N = tokens, 32 elements of K a step.  A lane
    // holds 8 consecutive elements of a row; which k a lane's registers stand for is the same for
    // both operands, so the sum is the same.
    float acc[MT][2][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[i][j][k] = 0.0f;
    const int steps = (K + 31) / 32, per = (steps + kCluster - 1) / kCluster;
    const int s0 = min(steps, c * per), s1 = min(steps, s0 + per);
    const uint16_t *xr[2];
    bool xok[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int t = wt * 16 + j * 8 + g;
      xok[j] = t < item.count;
      xr[j] = static_cast<const uint16_t *>(d.x) + (xok[j] ? (int64_t)tok[t] * d.ldx : 0);
    }
    auto shrink = [&](auto vec) {
      constexpr bool V = decltype(vec)::value;
      for (int s = s0 + wk; s < s1; s += WK) {
        const int k = s * 32 + q * 8;
        uint4 xv[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) xv[j] = xok[j] ? load8<V>(xr[j], k, K) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          if (i * 16 >= r) break;
          const int r0 = i * 16 + g, r1 = r0 + 8;
          const uint4 a0 = r0 < r ? load8<V>(A + (int64_t)r0 * K, k, K) : make_uint4(0, 0, 0, 0);
          const uint4 a1 = r1 < r ? load8<V>(A + (int64_t)r1 * K, k, K) : make_uint4(0, 0, 0, 0);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            mma16816<DT>(acc[i][j], a0.x, a1.x, a0.y, a1.y, xv[j].x, xv[j].y);
            mma16816<DT>(acc[i][j], a0.z, a1.z, a0.w, a1.w, xv[j].z, xv[j].w);
          }
        }
      }
    };
    if (P.vec & 1) shrink(std::true_type{});
    else shrink(std::false_type{});
    // c0, c1: rank g, tokens 2 q, 2 q + 1; c2, c3: rank g + 8
    float *mine = part + wk * kTile * kR;
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          mine[(wt * 16 + j * 8 + 2 * q + (e & 1)) * kR + i * 16 + g + (e >> 1) * 8] = acc[i][j][e];
    __syncthreads();
    for (int i = tid; i < kTile * kR; i += kThreads) {
      float s = part[i];
      for (int k = 1; k < WK; ++k) s += part[k * kTile * kR + i];
      part[i] = s;
    }
    cl.sync();
    const float scale = d.scale ? __ldg(d.scale + item.slot) : 1.0f;
    for (int i = tid; i < kTile * kR; i += kThreads) {
      float s = 0.0f;
#pragma unroll
      for (int k = 0; k < kCluster; ++k) s += cl.map_shared_rank(part, k)[i];
      // ranks past the slot's: zero, also where x is infinite
      vfull[i / kR * (kR + 4) + i % kR] = i % kR < r ? s * scale : 0.0f;
    }
    cl.sync();
  }

  // y^T: M = tokens (16 of this warp), N = outputs.  A lane's eight accumulators of two N tiles are
  // four consecutive outputs of two tokens, so y moves in 16-byte vectors.
  constexpr int kSteps = 2 * MT;  // 8 elements of the rank each
  uint32_t vh[kSteps][4], vl[kSteps][4];
#pragma unroll
  for (int s = 0; s < kSteps; ++s)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      // a0: (token g, k q), a1: (g + 8, q), a2: (g, q + 4), a3: (g + 8, q + 4); k = q and q + 4 of
      // step s stand for elements of the rank that B's lanes hold side by side
      const int t = wt * 16 + g + (e & 1) * 8, k = (s >> 2) * 32 + q * 8 + (s & 3) * 2 + (e >> 1);
      // kSteps below 4: the lane's 8 elements span the rank in chunks of 2 kSteps
      const int kk = kSteps >= 4 ? k : q * (2 * kSteps) + s * 2 + (e >> 1);
      const float v = r > 0 ? vfull[t * (kR + 4) + kk] : 0.0f;
      vh[s][e] = to_tf32(v);
      vl[s][e] = fabsf(__uint_as_float(vh[s][e])) < INFINITY ? to_tf32(v - __uint_as_float(vh[s][e])) : 0u;
    }
  const int ta = wt * 16 + g, tb = ta + 8;
  const bool oka = ta < item.count, okb = tb < item.count;
  const int64_t ia = oka ? tok[ta] : 0, ib = okb ? tok[tb] : 0;
  const bool yvec = (P.vec & 4) != 0;
  for (int m = m0 + wk * 16; m < m1; m += WK * 16) {
    float acc[2][4];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[j][e] = 0.0f;
    if (r > 0) {
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        // column n of N tile j is output m + 4 (n / 2) + 2 j + n % 2
        const int mo = m + 4 * (g >> 1) + 2 * j + (g & 1);
        const uint16_t *br = B + (int64_t)mo * R;
        const bool ok = mo < m1;
#pragma unroll
        for (int s4 = 0; s4 < (kSteps + 3) / 4; ++s4) {
          if (s4 * 32 >= r) break;
          constexpr int kEl = kSteps >= 4 ? 8 : 2 * kSteps;  // elements of a lane
          const int k = kSteps >= 4 ? s4 * 32 + q * 8 : q * kEl;
          uint32_t bw[4] = {0, 0, 0, 0};
          if (ok && k < r) {
            if (P.vec & 2) {
              if constexpr (kEl == 8) {
                const uint4 v = keep8(__ldg(reinterpret_cast<const uint4 *>(br + k)), r - k);
                bw[0] = v.x, bw[1] = v.y, bw[2] = v.z, bw[3] = v.w;
              } else {
                const uint2 v = __ldg(reinterpret_cast<const uint2 *>(br + k));
                const uint4 z = keep8(make_uint4(v.x, v.y, 0, 0), r - k);
                bw[0] = z.x, bw[1] = z.y;
              }
            } else {
              const uint4 v = load8<false>(br, k, min(r, k + kEl));
              bw[0] = v.x, bw[1] = v.y, bw[2] = v.z, bw[3] = v.w;
            }
          }
#pragma unroll
          for (int s = 0; s < (kSteps < 4 ? kSteps : 4); ++s) {
            uint32_t b0, b1;
            widen<DT>(bw[s], b0, b1);
            mma_tf32(acc[j], vl[s4 * 4 + s], b0, b1);
            mma_tf32(acc[j], vh[s4 * 4 + s], b0, b1);
          }
        }
      }
    }
    // acc[j][0, 1]: token g, outputs m + 4 q + 2 j, + 1; acc[j][2, 3]: token g + 8
    const int mo = m + 4 * q;
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      if (!(e ? okb : oka)) continue;
      const int64_t t = e ? ib : ia;
      const float *bp = d.base ? d.base + t * d.ldbase + mo : nullptr;
      float *yp = d.y + t * d.ldy + mo;
      const float o[4] = {acc[0][2 * e], acc[0][2 * e + 1], acc[1][2 * e], acc[1][2 * e + 1]};
      if (yvec && mo + 4 <= m1) {
        float4 v = bp ? *reinterpret_cast<const float4 *>(bp) : make_float4(0, 0, 0, 0);
        v.x += o[0], v.y += o[1], v.z += o[2], v.w += o[3];
        *reinterpret_cast<float4 *>(yp) = v;
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k)
          if (mo + k < m1) yp[k] = (bp ? bp[k] : 0.0f) + o[k];
      }
    }
  }
}

template <int MT, int WT>
size_t adapt_smem(int S) {
  constexpr int kTile = 16 * WT, kR = 16 * MT, WK = kWarps / WT;
  return sizeof(float) * (WK * kTile * kR + kTile * (kR + 4)) + sizeof(int) * (S + 1);
}

template <int DT, int MT, int WT>
cudaError_t run(const AdaptLaunch &L, int *status, cudaStream_t s) {
  uint32_t items = 0;
  int S = 0;
  for (int i = 0; i < L.n; ++i) {
    items += L.p[i].items;
    S = std::max(S, L.p[i].d.S);
  }
  if (items == 0) return cudaSuccess;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(items * kCluster);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = adapt_smem<MT, WT>(S);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = kCluster;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, adapt_kernel<DT, MT, WT>, L, status);
}

template <int DT, int WT>
cudaError_t run_rank(const AdaptLaunch &L, int max_R, int *status, cudaStream_t s) {
  if (max_R <= 16) return run<DT, 1, WT>(L, status, s);
  if (max_R <= 32) return run<DT, 2, WT>(L, status, s);
  if (max_R <= 64) return run<DT, 4, WT>(L, status, s);
  return run<DT, 8, WT>(L, status, s);
}

template <int DT, int MT, int WT>
cudaError_t prepare_one() {
  return cudaFuncSetAttribute(adapt_kernel<DT, MT, WT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              (int)adapt_smem<MT, WT>(WT_ADAPT_MAX_SLOTS));
}
template <int DT, int WT>
cudaError_t prepare_rank() {
  cudaError_t e = prepare_one<DT, 1, WT>();
  if (e == cudaSuccess) e = prepare_one<DT, 2, WT>();
  if (e == cudaSuccess) e = prepare_one<DT, 4, WT>();
  if (e == cudaSuccess) e = prepare_one<DT, 8, WT>();
  return e;
}

}  // namespace

// Tokens of one work item: 16, or 64 where there are so many tokens that reading a slot's A and B
// once per 16 of them would cost more than x and y.
int adapt_tile(int max_T) { return max_T >= 256 ? 64 : 16; }

cudaError_t adapt_prepare() {
  cudaError_t e = prepare_rank<WT_BF16, 1>();
  if (e == cudaSuccess) e = prepare_rank<WT_BF16, 4>();
  if (e == cudaSuccess) e = prepare_rank<WT_F16, 1>();
  if (e == cudaSuccess) e = prepare_rank<WT_F16, 4>();
  return e;
}

cudaError_t launch_adapt(const AdaptLaunch &L, int max_R, int max_T, int *status, cudaStream_t s) {
  const bool wide = adapt_tile(max_T) == 64;
  if (L.p[0].d.dtype == WT_BF16)
    return wide ? run_rank<WT_BF16, 4>(L, max_R, status, s) : run_rank<WT_BF16, 1>(L, max_R, status, s);
  return wide ? run_rank<WT_F16, 4>(L, max_R, status, s) : run_rank<WT_F16, 1>(L, max_R, status, s);
}

}  // namespace wt
