// Attention of each request's tokens to a memory of its own (include/wt_serve.h): the kernel for few rows, and
// the merge.
//
// A CTA takes an equal share of all requests' cells (CrossPlan), so unequal memories keep no SM waiting.  Each of
// its 4 warps streams its own tiles of 32 states (16 of more than 64 elements: 8 KB either way) through a ring of
// its own in shared memory, on from one row tile into the next: a head of a group of four, or of two, or every
// fourth of one head's.  (48 requests' tokens, 20 heads of 64, whose 128 bytes of a state lie side by side: 50.5 us,
// and 65.1 with all warps at one head.)  Rows, (token, head-in-group) pairs, are columns of the m16n8k16 MMAs, 8 to a
// block, so that a single token's product is not 16 rows of which one counts:
//
//   S^T = K Q^T,   P^T = 2^(S^T - m),   O^T += V^T P^T,   l += column sums of P^T
//
// with s = scale log2(e) q.k and m moving as kSlack says; P^T turns from a result into an operand by movmatrix.  P is
// rounded to the memory's type, as the MMA takes both operands in one type, and l sums the rounded weights: what their
// roundings have in common cancels.
// Parts join as softmax splits: O = sum_i 2^(m_i - m) O_i, l alike, out = O / l.  The maximum passes over NaN
// scores, so a part whose sum is NaN says so in its m.
//
// Where a row has so many states that the MMAs' sums would fall short, a warp sets its O^T and l aside in the workspace
// (cross_fold) and begins anew; at the row tile's end it adds them.
//
// Tiles come as TMA boxes.  States that are not kept, and what a memory's last tile holds behind it, are masked in S
// and cleared in V.  (13 requests' beams of 32 heads of 80, three in ten states left out: leaving those out of the
// copies, row by row with cp.async, 31.3 us, as boxes 29.3.)
#include <algorithm>
#include <type_traits>

#include "wt_cross.cuh"
#include "wt_tmem.cuh"

namespace wt {

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kStages = 3;           // tiles of a warp's ring
constexpr uint32_t kTileBytes = 8192;  // K, then V; each in halves of 64 elements, rows of 128 bytes, swizzled
constexpr int kJoinRows = 4;         // rows that the warps join at a time

template <int DH>
constexpr int kKeys = DH == 1 ? 32 : 16;  // states of a tile
template <int DH>
constexpr size_t few_smem() {
  return kWarps * kStages * kTileBytes + kWarps * kJoinRows * (DH * 64 * 4 + 8) + kWarps * kStages * (8 + 4) + 16 + 1024;
}

__device__ __forceinline__ uint32_t movmatrix(uint32_t x) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
  return r;
}

// A warp's tiles in order: of every cell of the CTA's share, its own, where the memory reaches it.
struct Tiles : Walk {
  int i, first_key, by;  // its tiles so far; key of a cell's first tile of this warp; from cell to cell
  __device__ Tiles(const CrossPlan &p, const Share &share, int key) : Walk(p, share), i(0), first_key(key), by(p.keys) {}
  __device__ bool segment() {  // the next row tile
    i = 0;
    return next();
  }
  // state of the next tile of the row tile; false: none left
  __device__ bool tile(int &key0) {
    if (i >= g.tiles) return false;
    key0 = (g.tile0 + i) * by + first_key;
    if (key0 >= a.len) return false;
    ++i;
    return true;
  }
};

// DH: 64-element halves of head_dim; NQ: blocks of 8 rows.
template <int DT, int DH, int NQ, bool KEEP>
__global__ void __launch_bounds__(kThreads, 2)
    cross_few_kernel(const __grid_constant__ CUtensorMap kmap, const __grid_constant__ CUtensorMap vmap, const __grid_constant__ CrossPlan P) {
  constexpr int kT = kKeys<DH>, NK = kT / 16, ND = DH * 4, kRows = 8 * NQ;
  constexpr uint32_t kHalfTile = kT * 128, kV = DH * kHalfTile;  // V behind K
  static_assert(2 * kV == kTileBytes, "a tile");
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t *after = smem_raw + (base - smem_u32(smem_raw)) + kWarps * kStages * kTileBytes;
  const wt_cross_desc &d = P.d;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q = lane & 3, g = lane >> 2;
  const int G = P.G, D = d.head_dim, ksteps = (D + 15) / 16;
  float *so = reinterpret_cast<float *>(after);                                   // [kWarps][kJoinRows][DH * 64]
  float2 *sml = reinterpret_cast<float2 *>(so + kWarps * kJoinRows * DH * 64);    // [kWarps][kJoinRows]
  uint64_t *bars = reinterpret_cast<uint64_t *>(sml + kWarps * kJoinRows);        // [kWarps][kStages]
  uint32_t *kept_of = reinterpret_cast<uint32_t *>(bars + kWarps * kStages);      // [kWarps][kStages]: which states count
  volatile int *abort_flag = reinterpret_cast<volatile int *>(kept_of + kWarps * kStages);
  const uint32_t ring = base + warp * kStages * kTileBytes, bar0 = smem_u32(bars + warp * kStages);
  kept_of += warp * kStages;
  if (tid == 0) *abort_flag = 0;
  if (lane == 0) {
    for (int i = 0; i < kStages; ++i) mbar_init(bar0 + 8 * i, 1);
    mbar_fence_init();
  }
  if (tid == 0 && d.max_mem > 0) {  // else there are no maps
    asm volatile("prefetch.tensormap [%0];" ::"l"(&kmap) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&vmap) : "memory");
  }
  griddep_launch();  // the merge's first loads may run beside this
  const Share share = share_of<kThreads>(P);
  // warps of a head, this warp's head of the group, and its place among the head's warps
  const int of_head = kWarps / P.together, wh = warp / of_head, wk = warp - wh * of_head;
  const float sl = d.scale * 1.4426950408889634f;

  // what is ahead of the products: the tile to ask for next, and what keep says of it
  Tiles ahead(P, share, wk * kT);
  uint32_t issued = 0, used = 0;  // tiles
  int next_key = 0;
  bool some = true, mine = false;
  auto look = [&]() {
    while (!ahead.tile(next_key))
      if (!ahead.segment()) {
        some = false;
        return;
      }
    if (KEEP) mine = lane < kT && next_key + lane < ahead.a.len && __ldg(d.keep + (int64_t)ahead.a.mem + next_key + lane);
  };
  auto issue = [&]() -> bool {
    if (!some) return false;
    const uint32_t s = issued++ % kStages, dst = ring + s * kTileBytes;
    const int state = ahead.a.mem + next_key, head = ahead.g.group * P.together + wh;
    if (lane == 0) {
      mbar_expect_tx(bar0 + 8 * s, kTileBytes);
#pragma unroll
      for (int hf = 0; hf < DH; ++hf) {
        tma_3d(dst + hf * kHalfTile, &kmap, hf * 64, head, state, bar0 + 8 * s);
        tma_3d(dst + kV + hf * kHalfTile, &vmap, hf * 64, head, state, bar0 + 8 * s);
      }
    }
    const bool kept = mine;
    look();
    return kept;
  };
  // What keep says of a tile is asked for before the tile before it is, and noted after that tile's products.
  auto note = [&](uint32_t tile, bool kept) {
    if (KEEP) {
      const uint32_t bits = __ballot_sync(0xffffffffu, kept);
      if (lane == 0) kept_of[tile % kStages] = bits;
    }
  };
  look();
  bool kept[kStages - 1];
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) kept[i] = issue();
#pragma unroll
  for (int i = 0; i < kStages - 1; ++i) note(i, kept[i]);
  __syncwarp();

  // where this lane's rows of 8 x 8 blocks lie: K as it is, V turned
  const uint32_t k_lane = ((lane & 15) * 128) | (((lane >> 4) ^ lane) & 7) * 16;
  const uint32_t v_lane = (((lane & 7) + (lane >> 4) * 8) * 128) | (((lane >> 3 & 1) ^ lane) & 7) * 16;
  Tiles now(P, share, wk * kT);
  constexpr int kFold = cross_fold(DT) / kT, kAside = NQ * (ND + 1);  // tiles; float4s of a lane: of each block O^T, then l
  static_assert(kAside * kWarps * 32 * sizeof(float4) == cross_few_fold(kRows, DH * 64), "what a CTA sets aside");
  float4 *const aside = P.fold + (int64_t)(blockIdx.x * kWarps + warp) * kAside * 32 + lane;
  while (now.segment()) {
    const Asker &a = now.a;
    const Segment &sg = now.g;
    const int hk = sg.group * P.together + wh;
    const uint32_t rows = a.n * G, row0 = sg.row_tile * kRows;

    // queries as B operands
    uint32_t qb[NQ][ND][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
      const uint32_t r = row0 + n * 8 + g;
      const bool ok = r < rows;
      const uint16_t *src = static_cast<const uint16_t *>(d.q) +
                            (ok ? (int64_t)(a.t0 + r / G) * d.q_stride + (int64_t)(hk * G + r % G) * D : 0);
#pragma unroll
      for (int k = 0; k < ND; ++k)
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          const int col = k * 16 + f * 8 + q * 2;
          qb[n][k][f] = ok && col < D ? *reinterpret_cast<const uint32_t *>(src + col) : 0u;
        }
    }
    // of rows 2q and 2q + 1 of a block: O^T, references, sums
    float o[NQ][ND][4], m[NQ][2], l[NQ][2];
#pragma unroll
    for (int n = 0; n < NQ; ++n) {
#pragma unroll
      for (int t = 0; t < ND; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][t][e] = 0.0f;
      m[n][0] = m[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.0f;
    }

    auto folded = [&]() { return now.i > kFold; };  // whether something lies aside, at tile i - 1 or after the last
    for (int key0; now.tile(key0);) {
      if (folded() && now.i % kFold == 1) {
        const bool again = now.i > 2 * kFold;
#pragma unroll
        for (int n = 0; n < NQ; ++n) {
          float4 *const at = aside + n * (ND + 1) * 32;
          float4 x = make_float4(0, 0, 0, 0);
#pragma unroll
          for (int t = 0; t < ND; ++t) {
            if (t >= ksteps) break;
            if (again) x = at[t * 32];
            at[t * 32] = make_float4(x.x + o[n][t][0], x.y + o[n][t][1], x.z + o[n][t][2], x.w + o[n][t][3]);
            o[n][t][0] = o[n][t][1] = o[n][t][2] = o[n][t][3] = 0.0f;
          }
          if (again) x = at[ND * 32];
          at[ND * 32] = make_float4(x.x + l[n][0], x.y + l[n][1], 0, 0);
          l[n][0] = l[n][1] = 0.0f;
        }
      }
      const uint32_t stage = used % kStages, kt = ring + stage * kTileBytes, vt = kt + kV;
      constexpr uint32_t kAll = kT == 32 ? 0xffffffffu : (1u << kT) - 1;
      if (!warp_wait(bar0 + 8 * stage, used / kStages & 1, abort_flag, P.status)) {  // nothing of it is used
        ++used;
        continue;
      }
      const int n = a.len - key0;
      const uint32_t found = KEEP ? kept_of[stage] : n >= kT ? kAll : (1u << n) - 1;
      if (found != kAll) {  // a weight of 0 does not hide what is not finite in V
        for (int i = lane; i < kT * 8; i += 32)
          if (!(found >> (i >> 3) & 1))
#pragma unroll
            for (int hf = 0; hf < DH; ++hf)
              asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(vt + hf * kHalfTile + i * 16), "r"(0) : "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
      }
      const uint32_t asked = issued;
      ++used;
      const bool asked_kept = issue();  // into the stage before this one: every lane has read it

      float s[NQ][NK][4];
#pragma unroll
      for (int n = 0; n < NQ; ++n)
#pragma unroll
        for (int j = 0; j < NK; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[n][j][e] = 0.0f;
#pragma unroll
      for (int k = 0; k < ND; ++k) {
        if (k >= ksteps) break;
#pragma unroll
        for (int j = 0; j < NK; ++j) {
          uint32_t kf[4];  // 16 states x 16 elements
          ldsm4(kf, (kt + (k >> 2) * kHalfTile + j * 2048 + k_lane) ^ (k & 3) * 32);
#pragma unroll
          for (int n = 0; n < NQ; ++n) mma16816<DT>(s[n][j], kf[0], kf[1], kf[2], kf[3], qb[n][k][0], qb[n][k][1]);
        }
      }
      const bool all = found == kAll;
      uint32_t pf[NQ][NK][2];
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
        for (int j = 0; j < NK; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            s[n][j][e] *= sl;
            if (!all && !(found >> (j * 16 + (e >> 1) * 8 + g) & 1)) s[n][j][e] = -INFINITY;
            mx[e & 1] = fmaxf(mx[e & 1], s[n][j][e]);
          }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 4));
          mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 8));
          mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 16));
        }
        constexpr float kGrow = kSlack + kBelow<DT>;
        const bool grown0 = mx[0] > m[n][0] + kGrow, grown1 = mx[1] > m[n][1] + kGrow;
        if (__any_sync(0xffffffffu, grown0 || grown1)) {
          float f[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float to = (e ? grown1 : grown0) ? mx[e] - kBelow<DT> : m[n][e];
            f[e] = to > -INFINITY ? exp2_approx(m[n][e] - to) : 1.0f;
            m[n][e] = to;
            l[n][e] *= f[e];
#pragma unroll
            for (int t = 0; t < ND; ++t) {
              o[n][t][e] *= f[e];
              o[n][t][2 + e] *= f[e];
            }
          }
          if (folded())
#pragma unroll 1
            for (int t = 0; t <= ND; ++t)
              if (t < ksteps || t == ND) {
                float4 &x = aside[(n * (ND + 1) + t) * 32];
                x = make_float4(x.x * f[0], x.y * f[1], x.z * f[0], x.w * f[1]);
              }
        }
        const float ref0 = m[n][0] > -INFINITY ? m[n][0] : 0.0f, ref1 = m[n][1] > -INFINITY ? m[n][1] : 0.0f;
        // l from the rounded weights: what their roundings have in common cancels
#pragma unroll
        for (int j = 0; j < NK; ++j)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t w = pack2<DT>(exp2_approx(s[n][j][2 * e] - ref0), exp2_approx(s[n][j][2 * e + 1] - ref1));
            float p0, p1;
            unpack2<DT>(w, p0, p1);
            l[n][0] += p0;
            l[n][1] += p1;
            pf[n][j][e] = movmatrix(w);
          }
      }
#pragma unroll
      for (int t = 0; t < ND; ++t) {
        if (t >= ksteps) break;
#pragma unroll
        for (int j = 0; j < NK; ++j) {
          uint32_t vf[4];  // 16 elements x 16 states
          ldsm4t(vf, (vt + (t >> 2) * kHalfTile + j * 2048 + v_lane) ^ (t & 3) * 32);
#pragma unroll
          for (int n = 0; n < NQ; ++n) mma16816<DT>(o[n][t], vf[0], vf[1], vf[2], vf[3], pf[n][j][0], pf[n][j][1]);
        }
      }
      if (issued != asked) note(asked, asked_kept);
      __syncwarp();
    }

    if (folded())
#pragma unroll
      for (int n = 0; n < NQ; ++n) {
        const float4 *const at = aside + n * (ND + 1) * 32;
#pragma unroll
        for (int t = 0; t < ND; ++t) {
          if (t >= ksteps) break;
          const float4 x = at[t * 32];
          o[n][t][0] += x.x, o[n][t][1] += x.y, o[n][t][2] += x.z, o[n][t][3] += x.w;
        }
        const float4 x = at[ND * 32];
        l[n][0] += x.x, l[n][1] += x.y;
      }

    // join the head's warps, four rows at a time
#pragma unroll
    for (int n = 0; n < NQ; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], 4);
        l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], 8);
        l[n][e] += __shfl_xor_sync(0xffffffffu, l[n][e], 16);
      }
    auto together = [&]() {
      if (of_head == 1) __syncwarp();
      else __syncthreads();
    };
#pragma unroll
    for (int h = 0; h < 2 * NQ; ++h) {
      if (row0 + h * kJoinRows >= rows) break;
      const int n = h >> 1;
      if (q >> 1 == (h & 1)) {  // rows 4 (h & 1) + 2 (q & 1) + e of block n
        const int at = warp * kJoinRows + 2 * (q & 1);
        if (g == 0) sml[at] = make_float2(m[n][0], l[n][0]), sml[at + 1] = make_float2(m[n][1], l[n][1]);
#pragma unroll
        for (int t = 0; t < ND; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) so[(at + (e & 1)) * DH * 64 + t * 16 + (e >> 1) * 8 + g] = o[n][t][e];
      }
      together();
      for (int i = wk; i < kJoinRows; i += of_head) {
        const int r = h * kJoinRows + i, part = wh * of_head * kJoinRows + i;
        const uint32_t row = row0 + r;
        if (row >= rows) break;
        float mm = -INFINITY, ll = 0.0f;
        for (int w = 0; w < of_head; ++w) mm = fmaxf(mm, sml[part + w * kJoinRows].x);
        float4 v = make_float4(0, 0, 0, 0);
        for (int w = 0; w < of_head; ++w) {
          const float2 y = sml[part + w * kJoinRows];
          const float f = y.x > -INFINITY ? exp2_approx(y.x - mm) : 0.0f;
          ll += f * y.y;
          const float4 x = lane * 4 < D ? *reinterpret_cast<const float4 *>(so + (part + w * kJoinRows) * DH * 64 + lane * 4) : v;
          v.x += f * x.x, v.y += f * x.y, v.z += f * x.z, v.w += f * x.w;
        }
        const int64_t slot = (sg.slot * P.together + wh) * kRows + r;
        if (lane * 4 < D) {
          if (sg.whole) {
            const float inv = ll == 0.0f ? 0.0f : 1.0f / ll;
            *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(d.out) + (int64_t)(a.t0 + row / G) * d.out_stride +
                                       (hk * G + row % G) * D + lane * 4) =
                make_uint2(pack2<DT>(v.x * inv, v.y * inv), pack2<DT>(v.z * inv, v.w * inv));
          } else {
            *reinterpret_cast<float4 *>(P.o + slot * D + lane * 4) = v;
          }
        }
        if (lane == 0 && !sg.whole) P.ml[slot] = make_float2(ll == ll ? mm : ll, ll);
      }
      together();
    }
  }
  if (tid == 0) note_cut(P, share, now);
  if (*abort_flag && lane == 0) {  // a copy may still be landing
    for (uint32_t i = issued > (uint32_t)kStages ? issued - kStages : 0; i < issued; ++i) {
      const long long t0 = clock64();
      while (!mbar_try_wait(bar0 + 8 * (i % kStages), i / kStages & 1) && clock64() - t0 < kWaitCycles) {
      }
    }
  }
}

// The parts of row tiles that several CTAs took: blocks (x, y) join what starts in CTA x's cells, L lanes to a row.
// The references, sums and O of 8 parts are asked for at once; of two, which many rows have, by themselves.
constexpr int kMergeParts = 8;
template <int DT, int L>
__global__ void __launch_bounds__(kThreads) cross_merge_kernel(const __grid_constant__ CrossPlan P) {
  const wt_cross_desc &d = P.d;
  const int D = d.head_dim, i = blockIdx.y * (kThreads / L) + threadIdx.x / L, wh = i / P.rows, r = i - wh * P.rows;
  const int col = threadIdx.x % L * 4;
  if (wh >= P.together || col >= D) return;
  griddep_wait();  // launched while the kernel before it runs
  const CrossCut cut = P.cuts[blockIdx.x];
  const uint32_t row = cut.row_tile * P.rows + r;
  if (cut.parts == 0 || row >= (uint32_t)cut.rows) return;
  const int c0 = blockIdx.x, c1 = c0 + cut.parts - 1;
  float m = -INFINITY, l = 0.0f;
  float4 o = make_float4(0, 0, 0, 0);
  auto join = [&](auto most, int c) {  // parts c .. c + most - 1, those up to c1
    constexpr int n = decltype(most)::value;
    float2 ml[n];
    float4 x[n];
#pragma unroll
    for (int k = 0; k < n; ++k) {
      const long long at = ((2ll * (c + k) + (c + k == c0 && cut.second)) * P.together + wh) * P.rows + r;
      ml[k] = c + k <= c1 ? P.ml[at] : make_float2(-INFINITY, 0.0f);
      x[k] = c + k <= c1 ? *reinterpret_cast<const float4 *>(P.o + at * D + col) : make_float4(0, 0, 0, 0);
    }
    float to = m;
#pragma unroll
    for (int k = 0; k < n; ++k) to = fmaxf(to, ml[k].x);
    const float by = m > -INFINITY ? exp2_approx(m - to) : 0.0f;
    m = to;
    l *= by, o.x *= by, o.y *= by, o.z *= by, o.w *= by;
#pragma unroll
    for (int k = 0; k < n; ++k) {
      // a part whose factor is 0 still counts: what is not finite in it has to show
      const float f = ml[k].x > -INFINITY || ml[k].x != ml[k].x ? exp2_approx(ml[k].x - m) : 0.0f;
      l += f * ml[k].y;
      o.x += f * x[k].x, o.y += f * x[k].y, o.z += f * x[k].z, o.w += f * x[k].w;
    }
  };
  if (cut.parts == 2) {
    join(std::integral_constant<int, 2>(), c0);
  } else {
    for (int c = c0; c <= c1; c += kMergeParts) join(std::integral_constant<int, kMergeParts>(), c);
  }
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  const int hk = cut.group * P.together + wh;
  *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(d.out) + (int64_t)(cut.t0 + row / P.G) * d.out_stride + (hk * P.G + row % P.G) * D + col) =
      make_uint2(pack2<DT>(o.x * inv, o.y * inv), pack2<DT>(o.z * inv, o.w * inv));
}

template <int DT, int DH, int NQ>
cudaError_t run_few(const CrossPlan &P, const CrossMaps &m, cudaStream_t s) {
  const CUtensorMap &k = *reinterpret_cast<const CUtensorMap *>(m.k), &v = *reinterpret_cast<const CUtensorMap *>(m.v);
  if (P.d.keep) cross_few_kernel<DT, DH, NQ, true><<<P.ctas, kThreads, few_smem<DH>(), s>>>(k, v, P);
  else cross_few_kernel<DT, DH, NQ, false><<<P.ctas, kThreads, few_smem<DH>(), s>>>(k, v, P);
  return cudaGetLastError();
}

template <int DT, int DH>
cudaError_t run_rows(const CrossPlan &P, const CrossMaps &m, cudaStream_t s) {
  if (P.rows == 8) return run_few<DT, DH, 1>(P, m, s);
  if constexpr (DH == 1)
    if (P.rows == 32) return run_few<DT, DH, 4>(P, m, s);
  return run_few<DT, DH, 2>(P, m, s);
}

template <int DT, int DH, int NQ>
cudaError_t prepare_few() {
  cudaError_t e = cudaFuncSetAttribute(cross_few_kernel<DT, DH, NQ, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)few_smem<DH>());
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(cross_few_kernel<DT, DH, NQ, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)few_smem<DH>());
  return e;
}

template <int DT, int DH>
cudaError_t prepare_dim() {
  cudaError_t e = prepare_few<DT, DH, 1>();
  if (e == cudaSuccess) e = prepare_few<DT, DH, 2>();
  if constexpr (DH == 1)
    if (e == cudaSuccess) e = prepare_few<DT, DH, 4>();
  return e;
}

template <int DT>
cudaError_t run_merge(const CrossPlan &P, cudaStream_t s) {
  const int lanes = P.d.head_dim <= 64 ? 16 : 32, most = (int)std::min<int64_t>(P.rows, (int64_t)P.d.max_new * P.G);
  cudaLaunchConfig_t cfg = {};
  // rows of a head stand `rows` apart, so with several heads all count
  cfg.gridDim = dim3((unsigned)P.ctas - 1, (unsigned)(((P.together > 1 ? P.together * P.rows : most) * lanes + kThreads - 1) / kThreads));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, lanes == 16 ? cross_merge_kernel<DT, 16> : cross_merge_kernel<DT, 32>, P);
}

}  // namespace

cudaError_t cross_prepare() {
  cudaError_t e = prepare_dim<WT_BF16, 1>();
  if (e == cudaSuccess) e = prepare_dim<WT_BF16, 2>();
  if (e == cudaSuccess) e = prepare_dim<WT_F16, 1>();
  if (e == cudaSuccess) e = prepare_dim<WT_F16, 2>();
  return e;
}

int cross_few_keys(int head_dim) { return head_dim <= 64 ? kKeys<1> : kKeys<2>; }

cudaError_t launch_cross_few(const CrossPlan &P, const CrossMaps &m, cudaStream_t s) {
  if (P.d.dtype == WT_BF16) return P.d.head_dim <= 64 ? run_rows<WT_BF16, 1>(P, m, s) : run_rows<WT_BF16, 2>(P, m, s);
  return P.d.head_dim <= 64 ? run_rows<WT_F16, 1>(P, m, s) : run_rows<WT_F16, 2>(P, m, s);
}

cudaError_t launch_cross_merge(const CrossPlan &P, cudaStream_t s) {
  return P.d.dtype == WT_BF16 ? run_merge<WT_BF16>(P, s) : run_merge<WT_F16>(P, s);
}

}  // namespace wt
