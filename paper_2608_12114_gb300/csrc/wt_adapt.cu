// Low-rank adapters of many requests beside a shared projection (include/wt_serve.h):
// y[t] = base[t] + scale_s B_s (A_s x[t]), s = slot[t].
//
// Few tokens (below 256): one launch, one cluster of C = 8 CTAs (4 or 2 where there are more items than
// SMs can hold at 8) per work item (projection, slot, up to 16 tokens of that slot).  The cluster
// computes v = A x with each CTA taking a C-th of K, exchanges the partial
// sums through distributed shared memory (always added in the order of the CTAs), and then each CTA
// takes a C-th of the M outputs.  A and B are read once per item, B's lines being fetched into L2
// while A is read; x and y cross once.  The slot map lies in device memory, so the items are found
// there too: every CTA counts the tokens of each slot and picks its own.  Bound: latency
// (two dependent reads and a cluster barrier).  More tokens: three launches, see below.
//
// Products run on the tensor cores.  A x: 16-bit operands, exact products, fp32 sums.  B v: B is
// exact in tf32 (both 16-bit types fit), and v, held in fp32, is split into two tf32 numbers, so that
// v enters with 22 bits and y keeps fp32's precision; one 16-bit number would leave 2^-9 of the update.
#include <algorithm>
#include <type_traits>

#include <cooperative_groups.h>

#include "wt_serve.cuh"

namespace wt {

namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 256;
constexpr int kWarps = 8;
constexpr int kMostCluster = 8;

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

// The same off the 16-byte grid: with 8 elements of the row on either side, from the two vectors that hold
// them (rows of 2731 elements, 463 tokens: 26 us with 8 loads of an element each, 21 so).  The kernel
// for few tokens keeps the 8 loads, which are in flight together and take less code.
__device__ __forceinline__ uint4 load8_shifted(const uint16_t *row, int k, int n) {
  if (k < 8 || k + 16 > n) return load8<false>(row, k, n);
  const uint64_t at = reinterpret_cast<uint64_t>(row + k), lo = at & ~(uint64_t)15;
  const uint4 *v = reinterpret_cast<const uint4 *>(lo);
  return shift_bytes(__ldg(v), __ldg(v + 1), (uint32_t)(at - lo));
}

// The first `keep` elements of 8, zeros for the others.
__device__ __forceinline__ uint4 keep8(const uint4 &v, int keep) {
  return keep >= 8 ? v : and4(v, byte_mask(0, 2 * keep));
}

struct Item {
  int slot;   // S: tokens without an adapter
  int count;  // tokens
};

// Elements [k, k + 8) of a row of B of which the first r count, as 4 words; with EL 4, [k, k + 4) as 2.
template <int EL>
__device__ __forceinline__ void load_b(uint32_t (&w)[4], const uint16_t *row, int k, int r, bool vec) {
  w[0] = w[1] = w[2] = w[3] = 0;
  if (k >= r) return;
  uint4 v;
  if (!vec) {
    v = load8<false>(row, k, min(r, k + EL));
  } else if constexpr (EL == 8) {
    v = keep8(__ldg(reinterpret_cast<const uint4 *>(row + k)), r - k);
  } else {
    const uint2 h = __ldg(reinterpret_cast<const uint2 *>(row + k));
    v = keep8(make_uint4(h.x, h.y, 0, 0), r - k);
  }
  w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
}

// v as two tf32 numbers; the lower of an infinite one means nothing.
__device__ __forceinline__ void split(float v, uint32_t &hi, uint32_t &lo) {
  hi = to_tf32(v);
  lo = fabsf(__uint_as_float(hi)) < INFINITY ? to_tf32(v - __uint_as_float(hi)) : 0u;
}

// MT: 16-row tiles of the rank (R <= 16 MT).
template <int DT, int MT>
__global__ void __launch_bounds__(kThreads, MT <= 2 ? 2 : 1) adapt_kernel(const __grid_constant__ AdaptLaunch L, int *status) {
  constexpr int kTile = 16;  // tokens of an item
  constexpr int kR = 16 * MT;
  constexpr int WK = kWarps;
  extern __shared__ __align__(16) uint8_t smem[];
  float *part = reinterpret_cast<float *>(smem);          // [WK][kTile][kR] the warps' sums, then [kTile][kR] in part 0
  float *vfull = part + WK * kTile * kR;                  // [kTile][kR + 4] v of the whole cluster
  int *cnt = reinterpret_cast<int *>(vfull + kTile * (kR + 4));  // [S + 1]
  __shared__ Item s_item;
  __shared__ int s_first;             // ordinal, within the slot, of the item's first token
  __shared__ int tok[kTile];
  __shared__ int wsum[kWarps];
  cg::cluster_group cl = cg::this_cluster();
  const int c = cl.block_rank(), C = cl.num_blocks();
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;

  // the projection and the item of this cluster
  int pi = 0;
  uint32_t w = blockIdx.x / C;
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
  const int wk = warp;
  // outputs of this CTA: whole groups of 16
  const int mper = ((M + 15) / 16 + C - 1) / C * 16;
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

  constexpr int kSteps = 2 * MT, kEl = kSteps >= 4 ? 8 : 2 * kSteps;  // steps of 8 ranks; a lane's neighbouring elements
  const int ta = g, tb = ta + 8;
  const bool oka = ta < item.count, okb = tb < item.count;
  const int64_t ia = tok[oka ? ta : 0], ib = tok[okb ? tb : 0];
  // Where all of base, y and B load in vectors, a warp's first kHold groups of 16 outputs have their base
  // (and B, at ranks up to 32) on its way before v is computed, by loads without a branch: each group
  // waiting for its own took 1820 cycles, half of a call for one token.
  constexpr int kHold = MT == 1 ? 4 : 2;
  constexpr bool kHoldB = MT <= 2;
  const bool fast = d.base && r > 0 && (P.vec & 6) == 6 && M % 16 == 0;
  float4 held[kHold][2];
  uint32_t heldb[kHoldB ? kHold : 1][2][kEl / 2];
  const uint16_t *brow = B + (int64_t)(4 * (g >> 1) + (g & 1)) * R;  // column g of N tile j: output 4 (g / 2) + 2 j + g % 2
  auto hold = [&](int mb) {
#pragma unroll
    for (int u = 0; u < kHold; ++u) {
      const int m = min(mb + u * WK * 16, m1 - 16);
      held[u][0] = *reinterpret_cast<const float4 *>(d.base + ia * d.ldbase + m + 4 * q);
      held[u][1] = *reinterpret_cast<const float4 *>(d.base + ib * d.ldbase + m + 4 * q);
      if constexpr (kHoldB) {
        const int k = q * kEl < R ? q * kEl : 0;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const uint16_t *src = brow + (int64_t)(m + 2 * j) * R + k;
          if constexpr (kEl == 8) {
            const uint4 v = __ldg(reinterpret_cast<const uint4 *>(src));
            heldb[u][j][0] = v.x, heldb[u][j][1] = v.y, heldb[u][j][2] = v.z, heldb[u][j][3] = v.w;
          } else {
            const uint2 v = __ldg(reinterpret_cast<const uint2 *>(src));
            heldb[u][j][0] = v.x, heldb[u][j][1] = v.y;
          }
        }
      }
    }
  };
  if (fast && m0 < m1) hold(m0 + wk * 16);

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
    const int steps = (K + 31) / 32, per = (steps + C - 1) / C;
    const int s0 = min(steps, c * per), s1 = min(steps, s0 + per);
    const uint16_t *xr[2];
    bool xok[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int t = j * 8 + g;
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
          mine[(j * 8 + 2 * q + (e & 1)) * kR + i * 16 + g + (e >> 1) * 8] = acc[i][j][e];
    __syncthreads();
    const int sums = item.count * kR;  // rows of absent tokens mean nothing
    for (int i = tid; i < sums; i += kThreads) {
      float s = part[i];
      for (int k = 1; k < WK; ++k) s += part[k * kTile * kR + i];
      part[i] = s;
    }
    cl.sync();
    const float scale = d.scale ? __ldg(d.scale + item.slot) : 1.0f;
    for (int i = tid; i < sums; i += kThreads) {
      float s = 0.0f;
#pragma unroll
      for (int k = 0; k < kMostCluster; ++k)
        if (k < C) s += cl.map_shared_rank(part, k)[i];
      // ranks past the slot's: zero, also where x is infinite
      vfull[i / kR * (kR + 4) + i % kR] = i % kR < r ? s * scale : 0.0f;
    }
    cluster_arrive();  // the other CTAs' sums have been read; each waits for this before it leaves
    __syncthreads();
  }

  // y^T: M = tokens (16), N = outputs.  A lane's eight accumulators of two N tiles are four consecutive
  // outputs of two tokens, so y moves in 16-byte vectors.
  uint32_t vh[kSteps][4], vl[kSteps][4];
#pragma unroll
  for (int s = 0; s < kSteps; ++s)
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      // a0: (token g, k q), a1: (g + 8, q), a2: (g, q + 4), a3: (g + 8, q + 4); k = q and q + 4 of
      // step s stand for elements of the rank that B's lanes hold side by side
      const int t = g + (e & 1) * 8, k = (s >> 2) * 32 + q * 8 + (s & 3) * 2 + (e >> 1);
      // kSteps below 4: the lane's 8 elements span the rank in chunks of 2 kSteps
      const int kk = kSteps >= 4 ? k : q * (2 * kSteps) + s * 2 + (e >> 1);
      const float v = r > 0 ? vfull[t * (kR + 4) + kk] : 0.0f;
      split(v, vh[s][e], vl[s][e]);
    }
  if (fast) {
    for (int mb = m0 + wk * 16; mb < m1; mb += kHold * WK * 16) {
      if (mb != m0 + wk * 16) hold(mb);
#pragma unroll
      for (int u = 0; u < kHold; ++u) {
        const int m = mb + u * WK * 16;
        float acc[2][4];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[j][e] = 0.0f;
#pragma unroll
        for (int s4 = 0; s4 < (kSteps + 3) / 4; ++s4) {
          if (s4 * 32 >= r) break;
          const int k = s4 * 32 + q * kEl;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            uint32_t bw[4];
            if constexpr (kHoldB) {
              const uint4 v = keep8(make_uint4(heldb[u][j][0], heldb[u][j][1], kEl == 8 ? heldb[u][j][kEl / 2 - 2] : 0,
                                               kEl == 8 ? heldb[u][j][kEl / 2 - 1] : 0), max(r - k, 0));
              bw[0] = v.x, bw[1] = v.y, bw[2] = v.z, bw[3] = v.w;
            } else {
              load_b<kEl>(bw, brow + (int64_t)(min(m, m1 - 16) + 2 * j) * R, k, r, true);
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
        // acc[j][0, 1]: token g, outputs m + 4 q + 2 j, + 1; acc[j][2, 3]: token g + 8
        if (m < m1) {
          float4 y0 = held[u][0], y1 = held[u][1];
          y0.x += acc[0][0], y0.y += acc[0][1], y0.z += acc[1][0], y0.w += acc[1][1];
          y1.x += acc[0][2], y1.y += acc[0][3], y1.z += acc[1][2], y1.w += acc[1][3];
          if (oka) *reinterpret_cast<float4 *>(d.y + ia * d.ldy + m + 4 * q) = y0;
          if (okb) *reinterpret_cast<float4 *>(d.y + ib * d.ldy + m + 4 * q) = y1;
        }
      }
    }
    cluster_wait();
    return;
  }
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
          uint32_t bw[4];
          load_b<kEl>(bw, br, s4 * 32 + q * kEl, ok ? r : 0, (P.vec & 2) != 0);
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
  if (r > 0) cluster_wait();
}


// ------------------------------------------------------------------ prompts
// Many tokens: x and y are most of the bytes, so the work is cut into three launches of many CTAs
// each.  adapt_plan_kernel sorts the tokens by slot and cuts them into items of up to 64 tokens of one
// slot.  adapt_shrink_kernel computes v = scale A x of an item, a cluster of 4 or 8 CTAs splitting K, with
// x and A staged in shared memory by 16-byte cp.async.  adapt_expand_kernel adds B v, a CTA taking
// several tiles of 64 tokens x 64 outputs of an item, with the base and B of the next tile always on
// their way to shared memory.  Measured for 4001 f16 tokens of two projections of 6912 outputs, ranks up to
// 64: 111 us, of which the expand kernel takes 82 (base to y alone, as torch copies it, 85); in one launch,
// as for few tokens, 350.  bf16 takes 130, as its third part of v leaves room for two CTAs to an SM at
// ranks 33 to 64, and 104 at ranks up to 32; f16 at ranks up to 128, one CTA to an SM, 156.
//
// v crosses between the two as 16-bit parts that add up to it, so that the second product's operands
// need no conversion: bf16 in three parts (24 bits); f16 in two (22 bits), after a power of two for
// each token has brought its largest finite v to 2^14, far from f16's ends; the power is taken back in fp32.
// Bound: HBM (base and y).
constexpr int kItem = 64;     // tokens of an item
constexpr int kMTile = kAdaptMTile;   // outputs of a tile of the expand kernel
constexpr int kPlanThreads = 1024;
static_assert(kPlanThreads == 32 * 32, "a lane for each warp");
constexpr int kEThreads = 256;  // the expand kernel, up to three to an SM: products run while other CTAs wait for a tile
constexpr int kEAcross = kMTile / 32;  // warps side by side in a tile
constexpr int kSThreads = 128;
constexpr int kSK = 64;       // elements of K of a stage
constexpr int kSStages = 3;   // 55 KB at rank 64: four CTAs per SM
template <int DT>
constexpr int kParts = DT == WT_BF16 ? 3 : 2;
constexpr int kSPitch = kSK * 2 + 16;

__device__ __forceinline__ int *plan_of(const AdaptWide &W, int plan) { return W.plans + (int64_t)plan * W.plan_ints; }
// A plan: items (an int4 of slot, first place, tokens, 0), their number, then the tokens in order.
__device__ __forceinline__ int4 item_of(const int *plan, int i) { return reinterpret_cast<const int4 *>(plan)[1 + i]; }

__global__ void __launch_bounds__(kPlanThreads) adapt_plan_kernel(const __grid_constant__ AdaptLaunch L,
                                                                  const __grid_constant__ AdaptWide W, int *status) {
  extern __shared__ int cnt[];  // [S + 1] tokens, then the next place, of each slot
  __shared__ int wsum[32][2];
  const wt_adapt_desc &d = L.p[W.plan_proj[blockIdx.x]].d;
  const int T = d.T, S = d.S, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool copy = d.base != d.y;
  int *plan = plan_of(W, blockIdx.x);
  int4 *items = reinterpret_cast<int4 *>(plan) + 1;
  int *order = plan + W.order_at;
  for (int s = tid; s <= S; s += kPlanThreads) cnt[s] = 0;
  __syncthreads();
  auto place = [&](int t) {  // a token's slot; -1: nothing to do
    const int s = __ldg(d.slot + t);
    return s >= 0 && s < S ? s : copy ? S : -1;
  };
  // Adds a warp's tokens to the counts of their slots, one atomic a slot (a prompt's tokens share one: with
  // an atomic each the kernel took 8.7 us for 4001 tokens, this way 7.3); returns the token's place before the
  // addition.
  auto add = [&](int s) {
    const unsigned peers = __match_any_sync(0xffffffffu, s);
    const int leader = __ffs(peers) - 1;
    int first = 0;
    if (lane == leader && s >= 0) first = atomicAdd(cnt + s, __popc(peers));
    return __shfl_sync(0xffffffffu, first, leader) + __popc(peers & ((1u << lane) - 1));
  };
  for (int t = tid; t - lane < T; t += kPlanThreads) {
    if (t < T && __ldg(d.slot + t) >= S && status) atomicCAS(status, 0, kStatusInvalid);
    add(t < T ? place(t) : -1);
  }
  __syncthreads();
  // places and items of the slots, by a scan over the slots
  int tokens = 0, tiles = 0;
  for (int s0 = 0; s0 <= S; s0 += kPlanThreads) {
    const int s = s0 + tid, n = s <= S ? cnt[s] : 0, m = (n + kItem - 1) / kItem;
    int a = n, b = m;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int ua = __shfl_up_sync(0xffffffffu, a, o), ub = __shfl_up_sync(0xffffffffu, b, o);
      if (lane >= o) a += ua, b += ub;
    }
    if (lane == 31) wsum[warp][0] = a, wsum[warp][1] = b;
    __syncthreads();
    int ta = tokens, tb = tiles, at = tokens + a - n, it = tiles + b - m;
    {
      const int wa = wsum[lane][0], wb = wsum[lane][1];  // 32 warps
      at += __reduce_add_sync(0xffffffffu, lane < warp ? wa : 0), it += __reduce_add_sync(0xffffffffu, lane < warp ? wb : 0);
      ta += __reduce_add_sync(0xffffffffu, wa), tb += __reduce_add_sync(0xffffffffu, wb);
    }
    if (s <= S) cnt[s] = at;
    for (int k = 0; k < m; ++k) items[it + k] = make_int4(s, at + k * kItem, min(kItem, n - k * kItem), 0);
    tokens = ta, tiles = tb;
    __syncthreads();
  }
  if (tid == 0) plan[0] = tiles;
  // Which tokens share an item does not change their results, so their order within a slot is free.
  for (int t = tid; t - lane < T; t += kPlanThreads) {
    const int s = t < T ? place(t) : -1, at = add(s);
    if (s >= 0) order[at] = t;
  }
}

__device__ __forceinline__ void cp16(uint32_t dst, const void *src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void sts128(uint32_t dst, const uint4 &v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(dst), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}

// MT: 16-row tiles of the rank, as for adapt_kernel.  A warp takes 16 tokens.
template <int DT, int MT>
__global__ void __launch_bounds__(kSThreads) adapt_shrink_kernel(const __grid_constant__ AdaptLaunch L,
                                                                 const __grid_constant__ AdaptWide W, int *status) {
  constexpr int kR = 16 * MT;
  constexpr int kStage = (kItem + kR) * kSPitch;
  extern __shared__ __align__(16) uint8_t smem[];
  __shared__ int tok[kItem];
  cg::cluster_group cl = cg::this_cluster();
  const int c = cl.block_rank(), C = cl.num_blocks(), tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q = lane & 3, g = lane >> 2;
  int pi = 0;
  uint32_t w = blockIdx.x / C;
  while (pi + 1 < L.n && w >= L.p[pi].items) w -= L.p[pi++].items;
  const AdaptProj &P = L.p[pi];
  const wt_adapt_desc &d = P.d;
  const int *plan = plan_of(W, W.plan[pi]);
  griddep_wait();
  if ((int)w >= plan[0]) return;  // the whole cluster
  const int4 item = item_of(plan, w);
  const int slot = item.x, count = item.z, K = d.K, R = d.R;
  if (slot >= d.S) return;
  int r = d.rank ? __ldg(d.rank + slot) : R;
  if (r < 0 || r > R) {
    if (tid == 0 && c == 0 && status) atomicCAS(status, 0, kStatusInvalid);
    r = min(max(r, 0), R);
  }
  if (r == 0) return;
  if (tid < kItem) tok[tid] = tid < count ? plan[W.order_at + item.y + tid] : -1;
  __syncthreads();

  const uint16_t *A = static_cast<const uint16_t *>(d.A) + (int64_t)slot * d.a_slot;
  const uint16_t *x = static_cast<const uint16_t *>(d.x);
  const int steps = (K + kSK - 1) / kSK, per = (steps + C - 1) / C;
  const int s0 = min(steps, c * per), s1 = min(steps, s0 + per);
  const uint32_t base = smem_u32(smem);
  // Stage s: 8 vectors a row; a thread takes vector tid % 8 of rows tid / 8 + 16 i, tokens first, then
  // ranks.  Absent tokens, ranks past the slot's and elements past K are zeros.
  const int row = tid >> 3, col = (tid & 7) * 8;
  const uint16_t *xp[kItem / 16];
#pragma unroll
  for (int i = 0; i < kItem / 16; ++i) xp[i] = tok[row + 16 * i] >= 0 ? x + (int64_t)tok[row + 16 * i] * d.ldx : nullptr;
  const bool vec = (P.vec & 1) != 0;
  auto fetch = [&](int s) {
    if (s < s1) {
      const uint32_t dst = base + (uint32_t)((s - s0) % kSStages) * kStage + row * kSPitch + col * 2;
      const int k = s * kSK + col;
#pragma unroll
      for (int i = 0; i < kItem / 16 + MT; ++i) {
        const uint16_t *src;
        if (i < kItem / 16) {
          src = xp[i];
        } else {
          const int a = row + 16 * (i - kItem / 16);
          if (16 * (i - kItem / 16) >= r) break;
          src = a < r ? A + (int64_t)a * K : nullptr;
        }
        if (src && k < K && vec) cp16(dst + i * 16 * kSPitch, src + k);
        else sts128(dst + i * 16 * kSPitch, src ? load8_shifted(src, k, K) : make_uint4(0, 0, 0, 0));
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < kSStages - 1; ++i) fetch(s0 + i);

  float acc[MT][2][4];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int k = 0; k < 4; ++k) acc[i][j][k] = 0.0f;
  for (int s = s0; s < s1; ++s) {
    asm volatile("cp.async.wait_group %0;" ::"n"(kSStages - 2) : "memory");
    __syncthreads();
    fetch(s + kSStages - 1);
    const uint32_t xs = base + (uint32_t)((s - s0) % kSStages) * kStage, as = xs + kItem * kSPitch;
#pragma unroll
    for (int k = 0; k < kSK / 16; ++k) {
      uint32_t xf[4];  // tokens 0-7 and 8-15 of the warp, each in two halves of 8 elements
      ldsm4(xf, xs + (warp * 16 + (lane & 7) + (lane >> 4) * 8) * kSPitch + k * 32 + ((lane >> 3) & 1) * 16);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        if (i * 16 >= r) break;
        uint32_t af[4];
        ldsm4(af, as + (i * 16 + (lane & 15)) * kSPitch + k * 32 + (lane >> 4) * 16);
        mma16816<DT>(acc[i][0], af[0], af[1], af[2], af[3], xf[0], xf[1]);
        mma16816<DT>(acc[i][1], af[0], af[1], af[2], af[3], xf[2], xf[3]);
      }
    }
  }
  asm volatile("cp.async.wait_group 0;" ::: "memory");
  __syncthreads();
  // this CTA's sums, [kItem][kR], over the stages
  float *part = reinterpret_cast<float *>(smem);
  static_assert(kItem * kR * 4 <= kSStages * kStage, "fits the stages");
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        part[(warp * 16 + j * 8 + 2 * q + (e & 1)) * kR + i * 16 + g + (e >> 1) * 8] = acc[i][j][e];
  cl.sync();
  // a C-th of the tokens each, 8 lanes to a token: the CTAs' sums in their order; ranks past the slot's
  // are zero
  const float scale = d.scale ? __ldg(d.scale + slot) : 1.0f;
  const int own = kItem / C, t = min(c * own + (tid >> 3), kItem - 1), k0 = (tid & 7) * (kR / 8);
  const bool mine = (tid >> 3) < own;  // with 8 CTAs half the threads have a token
  float v[kR / 8], top = 0.0f;
#pragma unroll
  for (int k = 0; k < kR / 8; ++k) v[k] = 0.0f;
  auto gather = [&](auto n) {
#pragma unroll
    for (int j = 0; j < decltype(n)::value; ++j) {
      const float2 *src = reinterpret_cast<const float2 *>(cl.map_shared_rank(part, j) + t * kR + k0);
#pragma unroll
      for (int k = 0; k < kR / 8; k += 2) {
        const float2 f = src[k / 2];
        v[k] += f.x;
        v[k + 1] += f.y;
      }
    }
  };
  if (C == 8) gather(std::integral_constant<int, 8>{});
  else gather(std::integral_constant<int, 4>{});
#pragma unroll
  for (int k = 0; k < kR / 8; ++k) {
    v[k] = k0 + k < r ? v[k] * scale : 0.0f;
    if (fabsf(v[k]) < INFINITY) top = fmaxf(top, fabsf(v[k]));
  }
  cl.sync();
  uint16_t *out = W.v + W.v_at[pi] + (int64_t)(item.y + t) * kR + k0;
  const int64_t part_at = (int64_t)d.T * kR;
  if constexpr (DT == WT_F16) {
#pragma unroll
    for (int o = 1; o < 8; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    // 2^(14 - exponent of the largest finite one), within what fp32 can take back; 1 where all are zeros,
    // infinities or NaN
    const int e = top > 0.0f ? min(max((int)(__float_as_uint(top) >> 23) - 127, -112), 127) : 14;
    const float up = __uint_as_float((uint32_t)(127 + 14 - e) << 23);
    if (mine && t < count && (tid & 7) == 0) W.back[W.back_at[pi] + item.y + t] = __uint_as_float((uint32_t)(127 - 14 + e) << 23);
#pragma unroll
    for (int k = 0; k < kR / 8; ++k) v[k] *= up;
  }
  if (!mine || t >= count) return;
#pragma unroll
  for (int i = 0; i < kParts<DT>; ++i)
#pragma unroll
    for (int k = 0; k < kR / 8; k += 2) {
      uint32_t w;
      float f0, f1;
      if constexpr (DT == WT_BF16) {
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(v[k + 1]), "f"(v[k]));
      } else {
        asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(v[k + 1]), "f"(v[k]));
      }
      uint32_t b0, b1;
      widen<DT>(w, b0, b1);
      f0 = __uint_as_float(b0), f1 = __uint_as_float(b1);
      // what the next part holds; nothing after an infinite one
      v[k] = fabsf(f0) < INFINITY ? v[k] - f0 : 0.0f;
      v[k + 1] = fabsf(f1) < INFINITY ? v[k + 1] - f1 : 0.0f;
      *reinterpret_cast<uint32_t *>(out + i * part_at + k) = w;
    }
}

// Shared memory of the expand kernel: a ring of tiles (base, 4 vectors that only their thread reads;
// then the kMTile rows of B), and the item's v.  Three CTAs fit an SM up to rank 32, and to rank 64 in f16.
template <int DT, int MT>
struct Expand {
  static constexpr int stages = 2;
  static constexpr uint32_t pitch = 32 * MT + 16, base = kEThreads * 64, stage = base + kMTile * pitch;
  static constexpr uint32_t v = stages * stage, part = kItem * pitch;
  static constexpr size_t smem = v + kParts<DT> * part;
};
static_assert(Expand<WT_BF16, 4>::smem <= 232448 && Expand<WT_BF16, 8>::smem <= 232448, "shared memory of one CTA");

template <int DT, int MT>
__global__ void __launch_bounds__(kEThreads, MT == 8 ? 1 : 3) adapt_expand_kernel(const __grid_constant__ AdaptLaunch L,
                                                                   const __grid_constant__ AdaptWide W) {
  using X = Expand<DT, MT>;
  constexpr int kR = 16 * MT;
  extern __shared__ __align__(16) uint8_t smem[];
  int pi = 0;
  uint32_t w = blockIdx.x;
  while (pi + 1 < L.n && w >= L.p[pi].items * L.p[pi].m_groups) {
    w -= L.p[pi].items * L.p[pi].m_groups;
    ++pi;
  }
  const AdaptProj &P = L.p[pi];
  const wt_adapt_desc &d = P.d;
  const int *plan = plan_of(W, W.plan[pi]);
  const int at_item = w / P.m_groups, group = w - at_item * P.m_groups;
  griddep_wait();
  if (at_item >= plan[0]) return;
  const int4 item = item_of(plan, at_item);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q = lane & 3, g = lane >> 2;
  const int slot = item.x, count = item.z, M = d.M;
  // the warp's 16 tokens; in a tile it takes 32 outputs: 2 groups of 16, of which a lane has 4 outputs of
  // two tokens
  const int t0 = warp / kEAcross * 16 + g;
  int64_t tt[2];
  float back[2] = {1.0f, 1.0f};
  const int r = slot >= d.S ? 0 : min(max(d.rank ? __ldg(d.rank + slot) : d.R, 0), d.R);
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const int t = t0 + 8 * e;
    tt[e] = t < count ? plan[W.order_at + item.y + t] : -1;
    // the shrink kernel leaves v and what it was divided by only where there are ranks
    if (DT == WT_F16 && t < count && r > 0) back[e] = W.back[W.back_at[pi] + item.y + t];
  }
  const int ksteps = (r + 15) / 16;
  const bool yvec = (P.vec & 4) != 0, bvec = (P.vec & 2) != 0;
  const int tiles = (M + kMTile - 1) / kMTile, tile0 = group * P.group_tiles, tile1 = min(tiles, tile0 + P.group_tiles);
  const uint32_t base = smem_u32(smem);
  const uint16_t *B = static_cast<const uint16_t *>(d.B) + (int64_t)slot * d.b_slot;
  auto fetch = [&](int tile) {
    if (tile < tile1) {
      const uint32_t st = base + (uint32_t)((tile - tile0) % X::stages) * X::stage;
      if (yvec && d.base) {
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int m = tile * kMTile + warp % kEAcross * 32 + j * 16 + 4 * q;
            if (tt[e] >= 0 && m + 4 <= M)
              cp16(st + (j * 2 + e) * (kEThreads * 16) + tid * 16, d.base + tt[e] * d.ldbase + m);
          }
      }
      // Output 4 a + 2 n + b of a group of 16 goes to row 8 n + 2 a + b: the rows of N tile n, in which a
      // lane's four accumulators of two tiles are neighbouring outputs.  Absent ones are zeros.
      // Two neighbouring lanes take 32 bytes of a row.
      const int row = (tid >> 1) & (kMTile - 1), m = tile * kMTile + row;
      const int to = (row & ~15) | (row & 2) << 2 | (row & 12) >> 1 | (row & 1);
      const uint16_t *src = B + (int64_t)m * d.R;
      const uint32_t dst = st + X::base + to * X::pitch;
      for (int k = ((tid & 1) + tid / (2 * kMTile) * 2) * 8; k < ksteps * 16; k += kEThreads / kMTile * 8) {
        if (bvec && m < M && k + 8 <= r) cp16(dst + k * 2, src + k);
        else sts128(dst + k * 2, m < M ? load8<false>(src, k, r) : make_uint4(0, 0, 0, 0));
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  if (r > 0) {
    // v of the item; absent tokens are zeros
    const uint16_t *v = W.v + W.v_at[pi] + (int64_t)item.y * kR;
    for (int i = tid; i < kParts<DT> * kItem * ksteps * 2; i += kEThreads) {
      const int pt = i / (kItem * 2 * ksteps), t = i / (2 * ksteps) % kItem, k = i % (2 * ksteps) * 8;
      const uint32_t dst = base + X::v + pt * X::part + t * X::pitch + k * 2;
      if (t < count) cp16(dst, v + pt * (int64_t)d.T * kR + (int64_t)t * kR + k);
      else sts128(dst, make_uint4(0, 0, 0, 0));
    }
  }
#pragma unroll
  for (int i = 0; i < X::stages - 1; ++i) fetch(tile0 + i);

  for (int tile = tile0; tile < tile1; ++tile) {
    asm volatile("cp.async.wait_group %0;" ::"n"(X::stages - 2) : "memory");
    __syncthreads();
    fetch(tile + X::stages - 1);  // where the tile before lay
    const uint32_t st = base + (uint32_t)((tile - tile0) % X::stages) * X::stage;
    float acc[2][2][4];
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[j][n][e] = 0.0f;
#pragma unroll 1
    for (int s = 0; s < ksteps; ++s) {
      uint32_t a[kParts<DT>][4];
#pragma unroll
      for (int i = 0; i < kParts<DT>; ++i)
        ldsm4(a[i], base + X::v + i * X::part + (warp / kEAcross * 16 + (lane & 15)) * X::pitch + s * 32 + (lane >> 4) * 16);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        uint32_t b[4];  // N tiles 0 and 1, each in two halves of 8 ranks
        ldsm4(b, st + X::base + (warp % kEAcross * 32 + j * 16 + (lane & 7) + (lane >> 4) * 8) * X::pitch + s * 32 + ((lane >> 3) & 1) * 16);
#pragma unroll
        for (int i = kParts<DT> - 1; i >= 0; --i) {  // the smallest part first
          mma16816<DT>(acc[j][0], a[i][0], a[i][1], a[i][2], a[i][3], b[0], b[1]);
          mma16816<DT>(acc[j][1], a[i][0], a[i][1], a[i][2], a[i][3], b[2], b[3]);
        }
      }
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int m = tile * kMTile + warp % kEAcross * 32 + j * 16 + 4 * q;
        if (tt[e] < 0) continue;
        float o[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) o[k] = acc[j][k >> 1][2 * e + (k & 1)] * back[e];
        float *yp = d.y + tt[e] * d.ldy + m;
        if (yvec && m + 4 <= M) {
          if (d.base) {
            const uint4 b = lds128(st + (j * 2 + e) * (kEThreads * 16) + tid * 16);
            o[0] += __uint_as_float(b.x), o[1] += __uint_as_float(b.y), o[2] += __uint_as_float(b.z), o[3] += __uint_as_float(b.w);
          }
          __stcs(reinterpret_cast<float4 *>(yp), make_float4(o[0], o[1], o[2], o[3]));
        } else {
#pragma unroll
          for (int k = 0; k < 4; ++k)
            if (m + k < M) yp[k] = (d.base ? d.base[tt[e] * d.ldbase + m + k] : 0.0f) + o[k];
        }
      }
  }
}

// `after`: the kernel waits on the device for the one before it in this call, so it may be launched
// while that one ends.
template <typename... A>
cudaError_t launch(void (*k)(A...), unsigned grid, int threads, int cluster, size_t smem, bool after, cudaStream_t s,
                   const A &...args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3((unsigned)threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at[2];
  int n = 0;
  if (cluster > 1) {
    at[n].id = cudaLaunchAttributeClusterDimension;
    at[n].val.clusterDim.x = (unsigned)cluster;
    at[n].val.clusterDim.y = at[n].val.clusterDim.z = 1;
    ++n;
  }
  if (after) {
    at[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = at;
  cfg.numAttrs = (unsigned)n;
  return cudaLaunchKernelEx(&cfg, k, args...);
}

int most_slots(const AdaptLaunch &L) {
  int S = 0;
  for (int i = 0; i < L.n; ++i) S = std::max(S, L.p[i].d.S);
  return S;
}

template <int MT>
constexpr size_t few_smem(int S) {
  return sizeof(float) * (kWarps * 16 * 16 * MT + 16 * (16 * MT + 4)) + sizeof(int) * (S + 1);
}
template <int MT>
constexpr size_t shrink_smem() {
  return (size_t)kSStages * (kItem + 16 * MT) * kSPitch;
}

template <int DT, int MT>
cudaError_t run_few(const AdaptLaunch &L, int *status, cudaStream_t s) {
  uint32_t items = 0;
  int64_t tokens = 0, slots = 0;
  for (int i = 0; i < L.n; ++i) {
    items += L.p[i].items;
    tokens += L.p[i].d.T;
    slots += L.p[i].d.S;
  }
  if (items == 0) return cudaSuccess;
  // 48 tokens of 24 adapters through three projections: 11.7 us in clusters of 4 (432 CTAs), 18.4 of 8;
  // one token 5.8 us in a cluster of 8, 7.2 of 4.  Above rank 32 an SM holds one CTA, but the number of
  // items is a bound, which is near only where slots have several tokens each, over all projections (106
  // tokens of 4 adapters of rank 64: 18 us in clusters of 4, 26 of 8; 34 tokens of up to 38 adapters, in
  // fact 4: 20 and 14).
  const int per_sm = MT <= 2 ? 3 : tokens >= 4 * slots ? 1 : 2;
  int c = kMostCluster;
  while (c > 2 && (int64_t)items * c > per_sm * num_sms()) c /= 2;
  return launch(adapt_kernel<DT, MT>, items * (unsigned)c, kThreads, c, few_smem<MT>(most_slots(L)), false, s, L, status);
}

template <int DT, int MT>
cudaError_t run_wide(const AdaptLaunch &L, const AdaptWide &W, int *status, cudaStream_t s) {
  uint32_t items = 0, tiles = 0;
  for (int i = 0; i < L.n; ++i) {
    items += L.p[i].items;
    tiles += L.p[i].items * L.p[i].m_groups;
  }
  if (items == 0) return cudaSuccess;
  cudaError_t e = launch(adapt_plan_kernel, (unsigned)W.n_plans, kPlanThreads, 1, sizeof(int) * (most_slots(L) + 1), false, s, L, W, status);
  if (e == cudaSuccess) {
    // 8 CTAs to an item while all of them are resident: long rows of few items
    const int c = (int64_t)items * 8 <= 4 * num_sms() ? 8 : 4;
    e = launch(adapt_shrink_kernel<DT, MT>, items * (unsigned)c, kSThreads, c, shrink_smem<MT>(), true, s, L, W, status);
  }
  if (e == cudaSuccess) e = launch(adapt_expand_kernel<DT, MT>, tiles, kEThreads, 1, Expand<DT, MT>::smem, true, s, L, W);
  return e;
}

template <int DT, int MT>
cudaError_t prepare_one() {
  cudaError_t e = cudaFuncSetAttribute(adapt_kernel<DT, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)few_smem<MT>(WT_ADAPT_MAX_SLOTS));
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(adapt_shrink_kernel<DT, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)shrink_smem<MT>());
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(adapt_expand_kernel<DT, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Expand<DT, MT>::smem);
  return e;
}
template <int DT>
cudaError_t prepare_type() {
  cudaError_t e = prepare_one<DT, 1>();
  if (e == cudaSuccess) e = prepare_one<DT, 2>();
  if (e == cudaSuccess) e = prepare_one<DT, 4>();
  if (e == cudaSuccess) e = prepare_one<DT, 8>();
  return e;
}

template <int DT>
cudaError_t run_type(const AdaptLaunch &L, const AdaptWide *W, int max_R, int *status, cudaStream_t s) {
  switch (adapt_rank_tiles(max_R)) {
    case 1: return W ? run_wide<DT, 1>(L, *W, status, s) : run_few<DT, 1>(L, status, s);
    case 2: return W ? run_wide<DT, 2>(L, *W, status, s) : run_few<DT, 2>(L, status, s);
    case 4: return W ? run_wide<DT, 4>(L, *W, status, s) : run_few<DT, 4>(L, status, s);
    default: return W ? run_wide<DT, 8>(L, *W, status, s) : run_few<DT, 8>(L, status, s);
  }
}

}  // namespace

cudaError_t adapt_prepare() {
  const cudaError_t e = prepare_type<WT_BF16>();
  return e == cudaSuccess ? prepare_type<WT_F16>() : e;
}

cudaError_t launch_adapt(const AdaptLaunch &L, const AdaptWide *W, int max_R, int *status, cudaStream_t s) {
  return L.p[0].d.dtype == WT_BF16 ? run_type<WT_BF16>(L, W, max_R, status, s) : run_type<WT_F16>(L, W, max_R, status, s);
}

}  // namespace wt
