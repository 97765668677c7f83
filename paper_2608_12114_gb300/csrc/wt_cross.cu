// Attention of each request's tokens to a memory of its own (include/wt_serve.h): the kernel for few rows, and
// the merge.
//
// A CTA takes an equal share of all requests' cells (CrossPlan), so unequal memories keep no SM waiting.  Each of
// its 4 warps streams its own tiles of 16 states through a ring of its own in shared memory (16-byte cp.async),
// with m16n8k16 MMAs on them, against 16 or 32 (token, head-in-group) rows:
//
//   p = 2^(s - m),  s = scale log2(e) q.k,  O += p v,  l += p,  m moving as kSlack says
//
// and parts join as softmax splits: O = sum_i 2^(m_i - m) O_i, l alike, out = O / l.  The maximum passes over NaN
// scores, so a part whose sum is NaN says so in its m.  States that are not kept, or past the memory, arrive as
// zeros and their scores are masked, so what stands there never reaches a product.
#include <algorithm>

#include "wt_cross.cuh"

namespace wt {

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kKeys = 16;   // states of a warp's tile
constexpr int kStages = 2;  // tiles of a warp's ring
constexpr int kCell = kWarps * kKeys;

template <int DT, int ND, int MT>
__global__ void __launch_bounds__(kThreads, MT > 1 ? 2 : ND == 4 ? 4 : 3) cross_few_kernel(const __grid_constant__ CrossPlan P) {
  constexpr int kPitch = ND * 32 + 16;            // bytes of a staged row: 8 rows hit 8 different bank groups
  constexpr int kTileBytes = 2 * kKeys * kPitch;  // K rows, then V rows
  constexpr int kRows = 16 * MT;
  extern __shared__ __align__(128) uint8_t smem[];
  const wt_cross_desc &d = P.d;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q = lane & 3, g = lane >> 2;
  const int G = P.G, D = d.head_dim;
  const uint32_t ring = smem_u32(smem) + warp * kStages * kTileBytes;
  const int chunks = D / 8;  // 16-byte pieces of a row
  const int row_lane = lane / chunks, in_lane = lane - row_lane * chunks, row_step = 32 / chunks, in_step = 32 - row_step * chunks;
  const int ksteps = (D + 15) / 16;
  const float sl = d.scale * 1.4426950408889634f;

  const Share share = share_of<kThreads>(P);
  int b = share.b;
  long long first = share.first;
  Asker a = {};
  if (share.lo < share.hi) a = asker_of(P, b, false);
  for (long long cell = share.lo; cell < share.hi;) {
    while (cell >= first + a.cells(d.kv_heads)) {
      first += a.cells(d.kv_heads);
      a = asker_of(P, ++b, false);
    }
    const Segment sg = segment_at(P, a, first, cell, share);
    cell += sg.cells;
    const int rows = a.n * G, row0 = sg.row_tile * kRows;
    const int k0 = sg.tile0 * kCell, k1 = min(a.len, k0 + sg.tiles * kCell);
    const int tiles = max(0, (k1 - k0 + kKeys - 1) / kKeys);

    if (D % 16) {
      // the last 8 columns stay zero: no copy touches them
      for (int i = tid; i < kWarps * kStages * 2 * kKeys; i += kThreads)
        *reinterpret_cast<uint4 *>(smem + i * kPitch + D * 2) = make_uint4(0, 0, 0, 0);
      __syncthreads();
    }
    const uint8_t *k_of = static_cast<const uint8_t *>(d.k) + 2 * (a.mem * d.mem_stride + sg.hk * d.mem_head);
    const uint8_t *v_of = static_cast<const uint8_t *>(d.v) + 2 * (a.mem * d.mem_stride + sg.hk * d.mem_head);
    const int64_t state_bytes = 2 * d.mem_stride;
    // Tile i of this warp (tiles warp, warp + 4, ...); bit r of `there`: state r counts.  What keep says is read a
    // tile ahead of its copies.
    auto kept = [&](int i) -> bool {
      const int key = k0 + (warp + i * kWarps) * kKeys + lane;
      return lane < kKeys && key < k1 && (!d.keep || __ldg(d.keep + (int64_t)a.mem + key));
    };
    bool next = kept(0);
    uint32_t there[kStages];
    auto fetch = [&](int i, uint32_t &found) {
      const int tile = warp + i * kWarps;
      if (tile < tiles) {
        found = __ballot_sync(0xffffffffu, next);
        next = kept(i + 1);
        const int key0 = k0 + tile * kKeys;
        const uint32_t dst = ring + (i % kStages) * kTileBytes;
        int row = row_lane, in = in_lane;  // rows 0-15: K, 16-31: V
#pragma unroll 4
        for (int c = 0; c < chunks; ++c) {
          const bool ok = found >> (row & 15) & 1;
          const uint8_t *src = (row < kKeys ? k_of : v_of) + (int64_t)(key0 + (row & 15)) * state_bytes + in * 16;
          cp16(dst + row * kPitch + in * 16, ok ? src : d.q, ok);
          row += row_step;
          in += in_step;
          if (in >= chunks) in -= chunks, ++row;
        }
      }
      cp_commit();
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fetch(i, there[i]);

    // queries as A operands
    uint32_t qf[MT][ND][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = row0 + i * 16 + g + e * 8;
        const bool ok = r < rows;
        const uint16_t *src = static_cast<const uint16_t *>(d.q) +
                              (ok ? (int64_t)(a.t0 + r / G) * d.q_stride + (int64_t)(sg.hk * G + r % G) * D : 0);
#pragma unroll
        for (int k = 0; k < ND; ++k)
#pragma unroll
          for (int f = 0; f < 2; ++f) {
            const int col = k * 16 + f * 8 + q * 2;
            qf[i][k][e + 2 * f] = ok && col < D ? *reinterpret_cast<const uint32_t *>(src + col) : 0u;
          }
      }

    float o[MT][2 * ND][4], m[MT][2], l[MT][2];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
#pragma unroll
      for (int j = 0; j < 2 * ND; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[i][j][e] = 0.0f;
      m[i][0] = m[i][1] = -INFINITY;
      l[i][0] = l[i][1] = 0.0f;
    }
    auto step = [&](int i, uint32_t found) {
      cp_wait<kStages - 1>();
      __syncwarp();
      const uint32_t kt = ring + (i % kStages) * kTileBytes, vt = kt + kKeys * kPitch;
      float s[MT][2][4];
#pragma unroll
      for (int z = 0; z < MT; ++z)
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[z][j][e] = 0.0f;
#pragma unroll
      for (int k = 0; k < ND; ++k) {
        if (k >= ksteps) break;
        uint32_t kf[4];  // states 0-7 and 8-15, each in two halves of 8 elements
        ldsm4(kf, kt + ((lane & 7) + (lane >> 4) * 8) * kPitch + k * 32 + ((lane >> 3) & 1) * 16);
#pragma unroll
        for (int z = 0; z < MT; ++z) {
          mma16816<DT>(s[z][0], qf[z][k][0], qf[z][k][1], qf[z][k][2], qf[z][k][3], kf[0], kf[1]);
          mma16816<DT>(s[z][1], qf[z][k][0], qf[z][k][1], qf[z][k][2], qf[z][k][3], kf[2], kf[3]);
        }
      }
      const bool all = found == 0xffffu;
      uint32_t pf[MT][4];
#pragma unroll
      for (int z = 0; z < MT; ++z) {
        float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[z][j][e] *= sl;
            if (!all && !(found >> (j * 8 + q * 2 + (e & 1)) & 1)) s[z][j][e] = -INFINITY;
            mx[e >> 1] = fmaxf(mx[e >> 1], s[z][j][e]);
          }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 1));
          mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 2));
        }
        constexpr float kGrow = kSlack + kBelow<DT>;
        const bool grown0 = mx[0] > m[z][0] + kGrow, grown1 = mx[1] > m[z][1] + kGrow;
        if (__any_sync(0xffffffffu, grown0 || grown1)) {
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float to = (e ? grown1 : grown0) ? mx[e] - kBelow<DT> : m[z][e];
            const float f = to > -INFINITY ? exp2_approx(m[z][e] - to) : 1.0f;
            m[z][e] = to;
            l[z][e] *= f;
#pragma unroll
            for (int j = 0; j < 2 * ND; ++j) {
              o[z][j][2 * e] *= f;
              o[z][j][2 * e + 1] *= f;
            }
          }
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float ref = m[z][e] > -INFINITY ? m[z][e] : 0.0f;
#pragma unroll
          for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int y = 0; y < 2; ++y) s[z][j][2 * e + y] = exp2_approx(s[z][j][2 * e + y] - ref);
        }
        // l from the rounded weights: what their roundings have in common cancels
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            pf[z][2 * j + e] = pack2<DT>(s[z][j][2 * e], s[z][j][2 * e + 1]);
            float lo, hi;
            unpack2<DT>(pf[z][2 * j + e], lo, hi);
            l[z][e] += lo + hi;
          }
      }
#pragma unroll
      for (int k = 0; k < ND; ++k) {
        if (k >= ksteps) break;
        uint32_t vf[4];  // 16 states x 16 elements
        ldsm4t(vf, vt + (lane & 15) * kPitch + k * 32 + (lane >> 4) * 16);
#pragma unroll
        for (int z = 0; z < MT; ++z) {
          mma16816<DT>(o[z][2 * k], pf[z][0], pf[z][1], pf[z][2], pf[z][3], vf[0], vf[1]);
          mma16816<DT>(o[z][2 * k + 1], pf[z][0], pf[z][1], pf[z][2], pf[z][3], vf[2], vf[3]);
        }
      }
      __syncwarp();  // every lane has read the tile before a later fetch overwrites it
    };
    const int mine = (tiles - warp + kWarps - 1) / kWarps;  // tiles of this warp
    for (int i = 0; i < mine; i += kStages)
#pragma unroll
      for (int u = 0; u < kStages; ++u)  // unrolled: the ring's slots and `there` are constants
        if (i + u < mine) {
          fetch(i + u + kStages - 1, there[(u + kStages - 1) % kStages]);
          step(i + u, there[u]);
        }
    cp_wait<0>();
    __syncthreads();

    // join the four warps: one row of tiles at a time
    constexpr int kCols = ND * 16;
    float *so = reinterpret_cast<float *>(smem);                         // [kWarps][16][kCols]
    float2 *sml = reinterpret_cast<float2 *>(so + kWarps * 16 * kCols);  // [kWarps][16]
    static_assert((kWarps * 16 * kCols + 2 * kWarps * 16) * 4 <= kWarps * kStages * kTileBytes, "fits the rings");
#pragma unroll
    for (int z = 0; z < MT; ++z) {
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float s = l[z][e];
        s += __shfl_xor_sync(0xffffffffu, s, 1);
        s += __shfl_xor_sync(0xffffffffu, s, 2);
        if (q == 0) sml[warp * 16 + g + e * 8] = make_float2(m[z][e], s);
#pragma unroll
        for (int j = 0; j < 2 * ND; ++j)
          *reinterpret_cast<float2 *>(so + (warp * 16 + g + e * 8) * kCols + j * 8 + q * 2) =
              make_float2(o[z][j][2 * e], o[z][j][2 * e + 1]);
      }
      __syncthreads();
      for (int r = warp; r < 16; r += kWarps) {
        const int row = row0 + z * 16 + r;
        if (row >= rows) break;
        float mm = -INFINITY, f[kWarps], ll = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) mm = fmaxf(mm, sml[w * 16 + r].x);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float2 v = sml[w * 16 + r];
          f[w] = v.x > -INFINITY ? exp2_approx(v.x - mm) : 0.0f;
          ll += f[w] * v.y;
        }
        if (lane * 4 < D) {
          float4 v = make_float4(0, 0, 0, 0);
#pragma unroll
          for (int w = 0; w < kWarps; ++w) {
            const float4 x = *reinterpret_cast<const float4 *>(so + (w * 16 + r) * kCols + lane * 4);
            v.x += f[w] * x.x, v.y += f[w] * x.y, v.z += f[w] * x.z, v.w += f[w] * x.w;
          }
          if (sg.whole) {
            const float inv = ll == 0.0f ? 0.0f : 1.0f / ll;
            *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(d.out) + (int64_t)(a.t0 + row / G) * d.out_stride +
                                       (sg.hk * G + row % G) * D + lane * 4) =
                make_uint2(pack2<DT>(v.x * inv, v.y * inv), pack2<DT>(v.z * inv, v.w * inv));
          } else {
            *reinterpret_cast<float4 *>(P.o + (sg.slot * kRows + z * 16 + r) * D + lane * 4) = v;
          }
        }
        if (lane == 0 && !sg.whole) P.ml[sg.slot * kRows + z * 16 + r] = make_float2(ll == ll ? mm : ll, ll);
      }
      __syncthreads();
    }
  }
}

// A warp to a (token, head): the parts of its row tile, where that has more than one.
constexpr int kMergeParts = 8;
template <int DT>
__global__ void __launch_bounds__(kThreads) cross_merge_kernel(const __grid_constant__ CrossPlan P) {
  const wt_cross_desc &d = P.d;
  const int lane = threadIdx.x & 31, b = blockIdx.y;
  const Asker a = asker_of(P, b, false);
  griddep_wait();  // launched while the kernel before it ends
  const int i = blockIdx.x * kWarps + (threadIdx.x >> 5);
  if (i >= a.n * d.heads) return;
  const int D = d.head_dim, h = i % d.heads, t = i / d.heads, hk = h / P.G;
  const int row = t * P.G + h % P.G, row_tile = row / P.rows, r = row - row_tile * P.rows;
  const long long per = P.first[d.n_req];
  const long long u0 = P.first[b] + hk * a.head_cells() + (long long)row_tile * a.key_tiles;
  const long long c0 = u0 / per, c1 = (u0 + (row_tile == a.row_tiles - 1 ? a.last : a.key_tiles) - 1) / per;
  if (c0 == c1) return;  // one CTA took it whole
  auto slot = [&](long long c) { return (2 * c + (c * per < u0)) * P.rows + r; };
  float m = -INFINITY;
  for (long long c = c0 + lane; c <= c1; c += 32) m = fmaxf(m, P.ml[slot(c)].x);
#pragma unroll
  for (int s = 16; s; s >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, s));
  float4 o = make_float4(0, 0, 0, 0);
  float l = 0.0f;
  for (long long k0 = c0; k0 <= c1; k0 += 32) {
    const float2 mine = k0 + lane <= c1 ? P.ml[slot(k0 + lane)] : make_float2(-INFINITY, 0.0f);
    // a part whose factor is 0 still counts: what is not finite in it has to show
    const float f = mine.x > -INFINITY || mine.x != mine.x ? exp2_approx(mine.x - m) : 0.0f;
    l += f * mine.y;
    const int n = (int)min(32ll, c1 - k0 + 1);
    for (int k = 0; k < n; k += kMergeParts) {
      float4 x[kMergeParts];
#pragma unroll
      for (int u = 0; u < kMergeParts; ++u)
        x[u] = k + u < n && lane * 4 < D ? *reinterpret_cast<const float4 *>(P.o + slot(k0 + k + u) * D + lane * 4)
                                         : make_float4(0, 0, 0, 0);
#pragma unroll
      for (int u = 0; u < kMergeParts; ++u) {
        const float w = __shfl_sync(0xffffffffu, f, (k + u) & 31);
        o.x += w * x[u].x, o.y += w * x[u].y, o.z += w * x[u].z, o.w += w * x[u].w;
      }
    }
  }
#pragma unroll
  for (int s = 16; s; s >>= 1) l += __shfl_xor_sync(0xffffffffu, l, s);
  if (lane * 4 < D) {
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(d.out) + (int64_t)(a.t0 + t) * d.out_stride + h * D + lane * 4) =
        make_uint2(pack2<DT>(o.x * inv, o.y * inv), pack2<DT>(o.z * inv, o.w * inv));
  }
}

template <int ND>
constexpr size_t few_smem() {
  return (size_t)kWarps * kStages * 2 * kKeys * (ND * 32 + 16);
}

template <int DT, int ND>
cudaError_t run_few(const CrossPlan &P, cudaStream_t s) {
  if (P.rows == 16) cross_few_kernel<DT, ND, 1><<<P.ctas, kThreads, few_smem<ND>(), s>>>(P);
  else cross_few_kernel<DT, ND, 2><<<P.ctas, kThreads, few_smem<ND>(), s>>>(P);
  return cudaGetLastError();
}

template <int DT>
cudaError_t run_dim(const CrossPlan &P, cudaStream_t s) {
  if (P.d.head_dim <= 64) return run_few<DT, 4>(P, s);
  if (P.d.head_dim <= 96) return run_few<DT, 6>(P, s);
  return run_few<DT, 8>(P, s);
}

template <int DT, int ND>
cudaError_t prepare_few() {
  cudaError_t e = cudaFuncSetAttribute(cross_few_kernel<DT, ND, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)few_smem<ND>());
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(cross_few_kernel<DT, ND, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)few_smem<ND>());
  return e;
}

template <int DT>
cudaError_t run_merge(const CrossPlan &P, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(((int64_t)P.d.max_new * P.d.heads + kWarps - 1) / kWarps), (unsigned)P.d.n_req);
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, cross_merge_kernel<DT>, P);
}

}  // namespace

int cross_few_resident(int rows, int head_dim) { return rows > 16 ? 2 : head_dim <= 64 ? 4 : 3; }

cudaError_t cross_prepare() {
  cudaError_t e = prepare_few<WT_BF16, 4>();
  if (e == cudaSuccess) e = prepare_few<WT_BF16, 6>();
  if (e == cudaSuccess) e = prepare_few<WT_BF16, 8>();
  if (e == cudaSuccess) e = prepare_few<WT_F16, 4>();
  if (e == cudaSuccess) e = prepare_few<WT_F16, 6>();
  if (e == cudaSuccess) e = prepare_few<WT_F16, 8>();
  return e;
}

cudaError_t launch_cross_few(const CrossPlan &P, cudaStream_t s) {
  return P.d.dtype == WT_BF16 ? run_dim<WT_BF16>(P, s) : run_dim<WT_F16>(P, s);
}

cudaError_t launch_cross_merge(const CrossPlan &P, cudaStream_t s) {
  return P.d.dtype == WT_BF16 ? run_merge<WT_BF16>(P, s) : run_merge<WT_F16>(P, s);
}

}  // namespace wt
