// Attention of each request's tokens to a memory of its own, for many rows: on the 5th-generation tensor cores.
//
//   S = Q K^T,   P = 2^(scale log2(e) S - m),   O += P V,   l += row sums of P
//
// A CTA takes an equal share of the cells of all requests (CrossPlan), one per SM: for each row tile that it meets
// a run of key tiles of 128 states, against two streams of 128 (token, head-in-group) rows.  Where a row tile has
// one such stream of rows only, the streams take its even and its odd key tiles and are joined at the end, in
// tensor memory.
//
//   producer warp    TMA boxes of Q (two tiles), and of K and V into a ring (128-byte swizzle)
//   MMA warp         S_i = Q_i K^T for the two streams i, then O_i += P_i V as each P_i arrives
//   two warpgroups   one per stream; a thread owns a row: it reads the row of S from tensor memory, takes the
//                    exponentials and writes P (16-bit) as the next product's A operand: over S, or for heads of up
//                    to 64, whose O leaves room, beside it, so that the next S is made meanwhile
//   a warp           clears the rows of V that are not in the memory, or not kept: a weight of 0 does not hide
//                    what is not finite.  Without a mask that is a memory's last tile alone.  Such a tile lands
//                    on a barrier of its own, and this warp makes the arrival that others wait for.
//
// The reference m of a row moves as kSlack says, and O is then rescaled in tensor memory.  P is rounded to the
// memory's type (the MMA takes both operands in one type); l sums the rounded weights, so that what their roundings have
// in common cancels, as in the kernel for few rows.  (Sums of the weights before their rounding took 32.9 us for the
// targets below and 250 for the long memories, where this took 36.1 and 257; but where many weights are one number, results were off by its rounding,
// every element the same way, and a request's as soon as another request had more tokens.)
//
// After every kFold tiles of a stream a row's O goes from tensor memory to what was set aside in the workspace
// (cross_fold), and the next product begins it anew; a reference that moves takes along what lies there.  (One GB300:
// the targets below, which have nothing to fold, 36.7 us with this code and 36.1 without; the long memories 260 and 257,
// and 266 where they fold each 8192 states, 279 each 4096.)
//
// Bound: the softmax warps, two to a scheduler, whose chains (read S, maximum, exponentials, write P) hide one
// another's latencies only in part.  2 requests of up to 1024 tokens, 32 heads over 8 of 128, against up to 16384 states: 260 us,
// 1.37 PFLOP/s; 6 requests of up to 448 tokens, 20 heads of 64, against up to 1500: 37 us, of which HBM needs 6 and
// the products 5.
//
// Every mbarrier wait is bounded; a timeout records WT_ETIMEDOUT and every role stops.
#include "wt_cross.cuh"
#include "wt_tmem.cuh"

namespace wt {

namespace {

constexpr int kKeysT = 128;    // states of a tile
constexpr int kThreads = 384;  // warps 0-3, 4-7: softmax of stream 0, 1; 8: producer; 9: MMA, TMEM; 10: clearing
// Registers a thread after the split: 128 of S, and its exponentials, for softmax.  The launch gives
// 3 x 168 to the three warpgroups together.
constexpr int kRegsSoftmax = 224, kRegsRest = 56;
static_assert(2 * kRegsSoftmax + kRegsRest <= 3 * 168, "what the launch has");
constexpr uint32_t kTmemCols = 512;
// Tensor memory of stream i: S (128 columns), P (64), O.  Two halves of a head: P over S.
template <int DH>
struct Cols {
  static constexpr bool apart = DH == 1;
  static constexpr uint32_t s = DH == 1 ? 256 : 128;  // from S_0 to S_1
  static constexpr uint32_t p = DH == 1 ? 128 : 0;    // from S to P
  static constexpr uint32_t o0 = DH == 1 ? 192 : 256, o = DH == 1 ? 256 : 128;
};

template <int DH>  // 64-element halves of head_dim
struct Geo {
  static constexpr uint32_t stage = DH * kHalf;
  static constexpr int stages = DH == 2 ? 5 : 8;
  static constexpr uint32_t ring = 2 * stage;  // after the two Q tiles
  static constexpr uint32_t bars = ring + stages * stage;
  static constexpr int nbars = 3 * stages + 14;
  // (m, l) of the rows of both streams of one row tile: with two halves in the second Q tile's place, which such
  // a row tile does not use, behind the 4 KB that its first warp turns rows in
  static constexpr uint32_t join = DH == 2 ? stage + 4096 : bars + nbars * 8 + 16;
  static constexpr size_t smem = bars + nbars * 8 + 16 + (DH == 2 ? 0 : 2 * 128 * 8) + 1024;
};
static_assert(Geo<2>::stage / 4 >= 4096 + 2 * 128 * 8, "rows turned, and join");
static_assert(Geo<2>::smem + 256 <= 232448, "shared memory of one CTA, and share_of's");

// Whether V of a key tile has rows to clear.
template <bool KEEP>
__device__ __forceinline__ bool to_clear(const Asker &a, int tile) {
  return KEEP || a.len - tile * kKeysT < kKeysT;
}

template <int DT, int DH, bool KEEP>
__global__ void __launch_bounds__(kThreads, 1)
    cross_wide_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                      const __grid_constant__ CUtensorMap vmap, const __grid_constant__ CrossPlan P) {
  using X = Geo<DH>;
  using C = Cols<DH>;
  constexpr int kFold = cross_fold(DT) / kKeysT;  // key tiles of a stream
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t *gbase = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t full0 = base + X::bars, empty0 = full0 + X::stages * 8, raw0 = empty0 + X::stages * 8;
  const uint32_t q_full = raw0 + X::stages * 8, q_empty = q_full + 8;
  const uint32_t s_full = q_empty + 8, p_full = s_full + 16, o_full = p_full + 16;  // [2] each
  const uint32_t p_half = o_full + 16, fin = p_half + 16, meet = fin + 8, s_free = meet + 8;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(gbase + X::bars + X::nbars * 8);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 2);
  float2 *join = reinterpret_cast<float2 *>(gbase + X::join);
  int *status = P.status;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;

  if (threadIdx.x == 0) {
    for (const CUtensorMap *m : {&qmap, &kmap, &vmap}) asm volatile("prefetch.tensormap [%0];" ::"l"(m) : "memory");
    for (int s = 0; s < X::stages; ++s) {
      mbar_init(full0 + 8 * s, 1);
      mbar_init(empty0 + 8 * s, 1);
      mbar_init(raw0 + 8 * s, 1);
    }
    mbar_init(q_full, 1);
    mbar_init(q_empty, 256);
    mbar_init(fin, 1);
    mbar_init(meet, 256);
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full + 8 * i, 1);
      mbar_init(p_full + 8 * i, 128);
      mbar_init(p_half + 8 * i, 128);
      mbar_init(o_full + 8 * i, 1);
      mbar_init(s_free + 8 * i, 128);
    }
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  griddep_launch();  // the merge's first loads may run beside this
  const Share share = share_of<kThreads>(P);  // has the barriers of all that was set up above
  fence_after();
  const uint32_t tmem = *tmem_slot;

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsRest));
    // ---------------- producer
    if (warp == 8 && lane == 0) {
      uint32_t it = 0, seg = 0, q_loads = 0;
      uint32_t raw = 0, raw_parity = 0;  // bit s: stage s's load is to be cleared; parity of its next such load
      bool live = true;
      auto load = [&](const CUtensorMap *map, int head, int state, bool clear) {
        const uint32_t s = it % X::stages;
        if (it >= X::stages && !bounded_wait(empty0 + 8 * s, ((it / X::stages) - 1) & 1, abort_flag, status)) return false;
        const uint32_t bar = (clear ? raw0 : full0) + 8 * s, dst = base + X::ring + s * X::stage;
        mbar_expect_tx(bar, X::stage);
#pragma unroll
        for (int hf = 0; hf < DH; ++hf) tma_3d(dst + hf * kHalf, map, hf * 64, head, state, bar);
        ++it;
        raw = clear ? raw | 1u << s : raw & ~(1u << s);
        if (clear) raw_parity ^= 1u << s;
        return true;
      };
      for (Walk w(P, share); live && w.next(); ++seg) {
        const Segment &g = w.g;
        if (seg && !bounded_wait(q_empty, (seg - 1) & 1, abort_flag, status)) break;
        const int qtiles = g.half ? 1 : 2, lead = (g.half ? 2 : 1) + C::apart;  // key tiles whose K is loaded ahead of their V
        mbar_expect_tx(q_full, (uint32_t)qtiles * DH * P.half * 128);
        ++q_loads;
        for (int i = 0; i < qtiles; ++i)
#pragma unroll
          for (int hf = 0; hf < DH; ++hf)
            tma_3d(base + (i * DH + hf) * kHalf, &qmap, hf * 64, g.group * P.G, w.a.t0 + (g.row_tile * 2 + i) * P.tile_tokens, q_full);
        const int state0 = w.a.mem + g.tile0 * kKeysT;
        for (int j = 0; j < min(lead, g.tiles) && live; ++j) live = load(&kmap, g.group, state0 + j * kKeysT, false);
        for (int j = 0; j < g.tiles && live; ++j) {
          live = load(&vmap, g.group, state0 + j * kKeysT, to_clear<KEEP>(w.a, g.tile0 + j));
          if (live && j + lead < g.tiles) live = load(&kmap, g.group, state0 + (j + lead) * kKeysT, false);
        }
      }
      if (*abort_flag) {
        // drain: copies of the last stages may still be landing
        const uint32_t first = it > (uint32_t)X::stages ? it - X::stages : 0;
        for (uint32_t j = first; j < it; ++j) {
          const long long t0 = clock64();
          const uint32_t s = j % X::stages, cleared = raw >> s & 1;
          while (!mbar_try_wait((cleared ? raw0 : full0) + 8 * s, (cleared ? ~raw_parity >> s : j / X::stages) & 1) &&
                 clock64() - t0 < kWaitCycles) {
          }
        }
        if (q_loads) {
          const long long t0 = clock64();
          while (!mbar_try_wait(q_full, (q_loads - 1) & 1) && clock64() - t0 < kWaitCycles) {
          }
        }
      }
    }
    // ---------------- MMA issuer: the warp keeps together, so that addresses stay in uniform registers
    if (warp == 9) {
      constexpr uint32_t kBf = DT == WT_BF16 ? 1u : 0u;
      constexpr uint32_t kIqk = idesc(kBf, kKeysT, 0);
      const int dim_steps = (P.d.head_dim + 15) / 16;
      const uint32_t ipv = idesc(kBf, dim_steps * 16, 1);
      uint32_t it = 0, seg = 0, np[2] = {0, 0}, ns[2] = {0, 0};
      bool live = true;
      uint32_t stage = 0;
      auto next = [&]() {  // the ring's next tile has landed, and its rows are clear
        const uint32_t s = it % X::stages;
        if (!warp_wait(full0 + 8 * s, (it / X::stages) & 1, abort_flag, status)) return live = false;
        fence_after();
        stage = s;
        ++it;
        return true;
      };
      auto release = [&](uint32_t bar) {
        if (elect_one()) commit(bar);
        __syncwarp();
      };
      auto scores = [&](int i, int tile_q, uint32_t s) {
        // where P lies apart, S may be written once it has been read
        if (C::apart) {
          if (ns[i] && !warp_wait(s_free + 8 * i, (ns[i] - 1) & 1, abort_flag, status)) return live = false;
          ++ns[i];
          fence_after();
        }
        const uint32_t q = desc_k(base + tile_q * X::stage), k = desc_k(base + X::ring + s * X::stage);
        if (elect_one()) {
#pragma unroll
          for (int e = 0; e < DH * 4; ++e) {
            const uint32_t off = ((e >> 2) * kHalf + (e & 3) * 32) >> 4;
            if (e < dim_steps) umma_ss(tmem + i * C::s, q + off, k + off, kIqk, e != 0);
          }
          commit(s_full + 8 * i);
        }
        __syncwarp();
        return true;
      };
      auto values = [&](int i, uint32_t s, bool first) {  // false: no P came
        const uint32_t v = desc_mn(base + X::ring + s * X::stage);
        // the first half of the states as soon as its P is there
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          if (!warp_wait((hf ? p_full : p_half) + 8 * i, np[i] & 1, abort_flag, status)) return live = false;
          fence_after();
          if (elect_one()) {
#pragma unroll
            for (int e = hf * 4; e < hf * 4 + 4; ++e)
              umma_ts(tmem + C::o0 + i * C::o, tmem + i * C::s + C::p + e * 8, v + e * (2048 >> 4), ipv, !first || e != 0);
            if (hf) commit(o_full + 8 * i);
          }
          __syncwarp();
        }
        ++np[i];
        return true;
      };
      for (Walk w(P, share); live && w.next(); ++seg) {
        const Segment &g = w.g;
        if (!warp_wait(q_full, seg & 1, abort_flag, status)) break;
        fence_after();
        // the K tile of both streams, or in half row tiles of stream i
        auto keys = [&](int i) {
          if (!next()) return false;
          const uint32_t ks = stage;
          if (g.half) {
            if (!scores(i, 0, ks)) return false;
          } else if (!scores(0, 0, ks) || !scores(1, 1, ks)) {
            return false;
          }
          release(empty0 + 8 * ks);
          return true;
        };
        const int first = g.half ? 2 : 1;  // tiles that start the streams
        auto anew = [&](int j) { return (g.half ? j >> 1 : j) % kFold == 0; };  // O starts with this product
        for (int j = 0; j < min(first, g.tiles) && keys(j); ++j) {
        }
        if (!live) break;
        for (int j = 0; j < g.tiles; ++j) {
          const bool more = j + first < g.tiles;
          if (C::apart && g.half) {  // the next S before this P V
            if (more && !keys(j & 1)) break;
            if (!next()) break;
            const uint32_t vs = stage;
            if (!values(j & 1, vs, anew(j))) break;
            release(empty0 + 8 * vs);
          } else if (C::apart) {
            // stream by stream: neither waits for what the other does next
            uint32_t ks = 0;
            if (more) {
              if (!next()) break;
              ks = stage;
              if (!scores(0, 0, ks)) break;
            }
            if (!next()) break;
            const uint32_t vs = stage;
            if (!values(0, vs, anew(j))) break;
            if (more) {
              if (!scores(1, 1, ks)) break;
              release(empty0 + 8 * ks);
            }
            if (!values(1, vs, anew(j))) break;
            release(empty0 + 8 * vs);
          } else if (g.half) {
            if (!next()) break;
            const uint32_t vs = stage;
            if (!values(j & 1, vs, anew(j))) break;
            release(empty0 + 8 * vs);
            if (more && !keys(j & 1)) break;
          } else {
            if (!next()) break;
            const uint32_t vs = stage;
            if (!values(0, vs, anew(j))) break;
            if (more) {
              if (!next()) break;
              scores(0, 0, stage);
            }
            if (!values(1, vs, anew(j))) break;
            release(empty0 + 8 * vs);
            if (more) {
              scores(1, 1, stage);
              release(empty0 + 8 * stage);
            }
          }
        }
      }
      // the last products must have finished before tensor memory is released
      if (it > 0) {
        release(fin);
        const long long t0 = clock64();
        while (!mbar_try_wait(fin, 0) && clock64() - t0 < kWaitCycles) {
        }
      }
    }
    // ---------------- clearing: the ring's tiles in the producer's order, those of V to clear alone
    if (warp == 10) {
      uint32_t it = 0, parity = 0;  // bit s: of stage s's next tile to clear
      bool live = true;
      for (Walk w(P, share); live && w.next();) {
        const Segment &g = w.g;
        const int lead = (g.half ? 2 : 1) + C::apart;
        it += min(lead, g.tiles);
        for (int j = 0; j < g.tiles && live; ++j) {
          if (to_clear<KEEP>(w.a, g.tile0 + j)) {
            const uint32_t s = it % X::stages;
            const int state0 = (g.tile0 + j) * kKeysT;
            uint32_t kept[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const int at = state0 + c * 32 + lane;
              kept[c] = __ballot_sync(0xffffffffu, at < w.a.len && (!KEEP || __ldg(P.d.keep + (int64_t)w.a.mem + at)));
            }
            live = warp_wait(raw0 + 8 * s, parity >> s & 1, abort_flag, status);
            parity ^= 1u << s;
            if (live) {
              const uint32_t v = base + X::ring + s * X::stage + (lane & 7) * 16;
#pragma unroll
              for (int c = 0; c < 4; ++c)
                if (kept[c] != 0xffffffffu)
                  for (int r = lane >> 3; r < 32; r += 4)
                    if (!(kept[c] >> r & 1))
#pragma unroll
                      for (int hf = 0; hf < DH; ++hf)
                        asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(v + hf * kHalf + (c * 32 + r) * 128), "r"(0)
                                     : "memory");
              asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
              __syncwarp();
              if (lane == 0) mbar_arrive(full0 + 8 * s);
            }
          }
          ++it;
          if (j + lead < g.tiles) ++it;
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    // ---------------- softmax: a thread owns row threadIdx.x % 128 of stream i
    const int i = warp >> 2, r = threadIdx.x & 127;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // 32 lanes of tensor memory per warp
    const uint32_t S = tmem + lanes + i * C::s, O = tmem + lanes + C::o0 + i * C::o;
    const float scale_log2 = P.d.scale * 1.4426950408889634f;
    // set aside: [head_dim / 4][row], so that a warp's accesses are of neighbours, then l
    float4 *const aside = P.fold + (int64_t)(blockIdx.x * 2 + i) * ((DH * 16 + 1) * 128) + r;
    static_assert(2 * (DH * 16 + 1) * 128 * sizeof(float4) == cross_wide_fold(DH * 64), "what a CTA sets aside");
    uint32_t done = 0, done_other = 0;  // tiles of this stream, and of the other, over all segments
    uint32_t seg = 0, met = 0;
    bool live = true;
    Walk w(P, share);
    for (; live && w.next(); ++seg) {
      const Segment &g = w.g;
      // The segment's queries have landed, so every thread has released those before (q_empty).
      if (!warp_wait(q_full, seg & 1, abort_flag, status)) break;
      const int n = g.half ? (g.tiles + 1 - i) / 2 : g.tiles;
      const uint8_t *keep = P.d.keep + (int64_t)w.a.mem;
      // what keep says of a tile is read a tile ahead
      uint32_t ahead[4] = {1, 1, 1, 1};
      auto look = [&](int j) {
        if (!KEEP) return;
        const int at = (g.tile0 + (g.half ? 2 * j + i : j)) * kKeysT + lane;
#pragma unroll
        for (int c = 0; c < 4; ++c) ahead[c] = at + c * 32 < w.a.len ? __ldg(keep + at + c * 32) : 0;
      };
      look(0);
      float m = 0.0f, l0 = 0.0f, l1 = 0.0f;
      // O and l of the tiles before j, a multiple of kFold, to what was set aside; or of the last ones from there to O
      auto fold = [&](int j, bool last) {
        const bool again = last || j > kFold;
        constexpr int kCols = 64;  // whose accesses are on their way together
#pragma unroll 1
        for (int c = 0; c < P.d.head_dim; c += kCols) {
          float4 *const at = aside + c / 4 * 128;
          float4 x[kCols / 4];
#pragma unroll
          for (int k = 0; k < kCols / 4; ++k) x[k] = again && c + 4 * k < P.d.head_dim ? at[k * 128] : make_float4(0, 0, 0, 0);
          if (c == 0) {
            live = warp_wait(o_full + 8 * i, (done + j - 1) & 1, abort_flag, status);
            fence_after();
          }
#pragma unroll
          for (int e = 0; e < kCols; e += 32) {
            uint32_t o[32];
            tmem_ld32(O + c + e, o);
            wait_ld();
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              float4 &y = x[e / 4 + k];
              y.x += __uint_as_float(o[4 * k]), y.y += __uint_as_float(o[4 * k + 1]);
              y.z += __uint_as_float(o[4 * k + 2]), y.w += __uint_as_float(o[4 * k + 3]);
              if (!last && c + e + 4 * k < P.d.head_dim) at[(e / 4 + k) * 128] = y;
              o[4 * k] = __float_as_uint(y.x), o[4 * k + 1] = __float_as_uint(y.y);
              o[4 * k + 2] = __float_as_uint(y.z), o[4 * k + 3] = __float_as_uint(y.w);
            }
            if (last) tmem_st32(O + c + e, o);
          }
        }
        if (last) wait_st();
        fence_before();
        float &l = aside[DH * 16 * 128].x;
        l0 += again ? l1 + l : l1;
        l1 = 0.0f;
        if (!last) l = l0, l0 = 0.0f;
      };
      for (int j = 0; j < n; ++j) {
        if (j && j % kFold == 0) {
          fold(j, false);
          if (!live) break;
        }
        const int keys = w.a.len - (g.tile0 + (g.half ? 2 * j + i : j)) * kKeysT;
        uint32_t gone[4];
        if (KEEP) {
#pragma unroll
          for (int c = 0; c < 4; ++c) gone[c] = __ballot_sync(0xffffffffu, ahead[c] == 0);
          look(j + 1);
        }
        if (!warp_wait(s_full + 8 * i, (done + j) & 1, abort_flag, status)) {
          live = false;
          break;
        }
        fence_after();
        float v[128];
        {
          uint32_t u[128];
#pragma unroll
          for (int c = 0; c < 4; ++c) tmem_ld32(S + c * 32, u + c * 32);
          wait_ld();
#pragma unroll
          for (int c = 0; c < 128; ++c) v[c] = __uint_as_float(u[c]);
        }
        if (C::apart) {
          fence_before();
          mbar_arrive(s_free + 8 * i);
        }
        if (KEEP) {
#pragma unroll
          for (int c = 0; c < 128; ++c)
            if (gone[c >> 5] >> (c & 31) & 1) v[c] = -INFINITY;
        } else if (keys < kKeysT) {
#pragma unroll
          for (int c = 0; c < 128; ++c)
            if (c >= keys) v[c] = -INFINITY;
        }
        float mx0 = v[0], mx1 = v[1], mx2 = v[2], mx3 = v[3];
#pragma unroll
        for (int c = 4; c < 124; c += 8) {
          mx0 = max3(mx0, v[c], v[c + 4]);
          mx1 = max3(mx1, v[c + 1], v[c + 5]);
          mx2 = max3(mx2, v[c + 2], v[c + 6]);
          mx3 = max3(mx3, v[c + 3], v[c + 7]);
        }
        mx0 = max3(mx0, v[124], v[125]);
        mx1 = max3(mx1, v[126], v[127]);
        const float top = max3(max3(mx0, mx1, mx2), mx3, mx3) * scale_log2;
        const bool grown = top > m + (kSlack + kBelow<DT>);
        if (j == 0) {
          m = top > -INFINITY ? top - kBelow<DT> : -INFINITY;  // also where all are NaN: their p are NaN against any reference
        } else if (__any_sync(0xffffffffu, grown)) {
          // O of this row, once the product before has been added to it, against the new reference
          if (!warp_wait(o_full + 8 * i, (done + j - 1) & 1, abort_flag, status)) {
            live = false;
            break;
          }
          fence_after();
          const float f = grown ? exp2_approx(m - (top - kBelow<DT>)) : 1.0f;
          if (grown) m = top - kBelow<DT>;
          l0 *= f;
          l1 *= f;
          if (j >= kFold) {
#pragma unroll 4
            for (int c = 0; c < P.d.head_dim; c += 4) {
              float4 &x = aside[c / 4 * 128];
              x = make_float4(x.x * f, x.y * f, x.z * f, x.w * f);
            }
            aside[DH * 16 * 128].x *= f;
          }
#pragma unroll 1
          for (int c = 0; c < DH * 64; c += 32) {
            uint32_t o[32];
            tmem_ld32(O + c, o);
            wait_ld();
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
            tmem_st32(O + c, o);
          }
        }
        const float ref = m > -INFINITY ? m : 0.0f;  // no score above -infinity yet
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          uint32_t u[32];
#pragma unroll
          for (int k = 0; k < 64; k += 2) {
            const int c = hf * 64 + k;
            fma_x2(v[c], v[c + 1], scale_log2, -ref);
            v[c] = exp2_approx(v[c]);
            v[c + 1] = exp2_approx(v[c + 1]);
            u[k / 2] = pack2<DT>(v[c], v[c + 1]);
            float p0, p1;
            unpack2<DT>(u[k / 2], p0, p1);
            add_x2(l0, l1, p0, p1);
          }
          // where P lies apart, the product before may still read it
          if (C::apart && hf == 0 && done + j > 0) {
            live = warp_wait(o_full + 8 * i, (done + j - 1) & 1, abort_flag, status);
            fence_after();
          }
          tmem_st32(S + C::p + hf * 32, u);
          wait_st();
          fence_before();
          mbar_arrive((hf ? p_full : p_half) + 8 * i);
        }
        if (!live) break;
      }
      if (!live) break;
      done += n;
      const int n_other = g.half ? g.tiles - n : n;
      done_other += n_other;
      float l = l0 + l1;
      if (n == 0) m = -INFINITY;
      if (n > 0 && !warp_wait(o_full + 8 * i, (done - 1) & 1, abort_flag, status)) break;
      if (n > kFold) {
        done -= n;
        fold(n, true);
        done += n;
        l = l0;
      }
      // Two streams of one row tile: both numbers of a row, and each takes half of the columns of both.
      float f = 1.0f, f_other = 0.0f;
      if (g.half) {
        join[i * 128 + r] = make_float2(n == 0 ? -INFINITY : l == l ? m : l, l);
        mbar_arrive(meet);
        if (!warp_wait(meet, met++ & 1, abort_flag, status)) break;
        if (n_other > 0 && !warp_wait(o_full + 8 * (1 - i), (done_other - 1) & 1, abort_flag, status)) break;
        const float2 other = join[(1 - i) * 128 + r];
        const float mm = fmaxf(m, other.x);
        f = m > -INFINITY ? exp2_approx(m - mm) : 0.0f;
        f_other = n_other == 0 ? 0.0f : other.x != other.x ? other.x : other.x > -INFINITY ? exp2_approx(other.x - mm) : 0.0f;
        m = mm;
        l = l * f + (n_other ? other.y * f_other : 0.0f);
      }
      fence_after();
      // Rows out, 32 columns at a time, turned in shared memory so that neighbouring lanes write one row.  The
      // queries have been read by then, and their place is this stream's until q_empty.
      const int part0 = g.half ? 0 : i * P.half;  // in the row tile
      const uint32_t row0 = g.row_tile * P.rows + part0;
      const int rows = min(P.half, (int)(w.a.n * P.G - row0));  // of the tile; may be none
      const uint32_t turn = base + i * X::stage + (warp & 3) * (X::stage / 4);
      static_assert(32 * 128 <= X::stage / 4, "32 rows of 32 columns");
      const float inv = l == 0.0f ? 0.0f : 1.0f / l;
      const int c0 = g.half ? i * DH * 32 : 0, c1 = g.half ? c0 + DH * 32 : DH * 64;
      const uint32_t O0 = tmem + lanes + C::o0;
#pragma unroll 1
      for (int c = c0; c < c1 && c < P.d.head_dim; c += 32) {
        uint32_t o[32];
        if (n > 0) {
          tmem_ld32(O + c, o);
        } else {
#pragma unroll
          for (int k = 0; k < 32; ++k) o[k] = 0;
        }
        wait_ld();
        if (g.half) {
          if (n_other > 0) {
            uint32_t x[32];
            tmem_ld32(O0 + (1 - i) * C::o + c, x);
            wait_ld();
#pragma unroll
            for (int k = 0; k < 32; ++k)
              o[k] = __float_as_uint(__uint_as_float(o[k]) * f + __uint_as_float(x[k]) * f_other);
          }
        }
        if (g.whole) {
          // 16 words a row: 4 lanes write 64 bytes of a row
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            uint32_t p[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              p[e] = pack2<DT>(__uint_as_float(o[8 * k + 2 * e]) * inv, __uint_as_float(o[8 * k + 2 * e + 1]) * inv);
            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(turn + lane * 64 + (k ^ ((lane >> 1) & 3)) * 16), "r"(p[0]),
                         "r"(p[1]), "r"(p[2]), "r"(p[3])
                         : "memory");
          }
          __syncwarp();
          const int col = c + (lane & 3) * 8;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int t = k * 8 + (lane >> 2), at = (warp & 3) * 32 + t;
            const uint4 v = lds128(turn + t * 64 + ((lane ^ (t >> 1)) & 3) * 16);
            if (at < rows && col < P.d.head_dim) {
              const uint32_t row = row0 + at;
              *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(P.d.out) + (int64_t)(w.a.t0 + row / P.G) * P.d.out_stride +
                                         (g.group * P.G + row % P.G) * P.d.head_dim + col) = v;
            }
          }
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k)
            asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(turn + lane * 128 + (k ^ (lane & 7)) * 16), "r"(o[4 * k]),
                         "r"(o[4 * k + 1]), "r"(o[4 * k + 2]), "r"(o[4 * k + 3])
                         : "memory");
          __syncwarp();
          const int col = c + (lane & 7) * 4;
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const int t = k * 4 + (lane >> 3), at = (warp & 3) * 32 + t;
            const uint4 v = lds128(turn + t * 128 + ((lane ^ t) & 7) * 16);
            if (at < rows && col < P.d.head_dim)
              *reinterpret_cast<uint4 *>(P.o + (g.slot * P.rows + part0 + at) * P.d.head_dim + col) = v;
          }
        }
        __syncwarp();
      }
      if (!g.whole && r < rows && (!g.half || i == 0))
        P.ml[g.slot * P.rows + part0 + r] = make_float2(l == l ? m : l, l);
      fence_before();
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // before the next queries land there
      if (g.half) {  // the other stream's sums have been read
        mbar_arrive(meet);
        if (!warp_wait(meet, met++ & 1, abort_flag, status)) break;
      }
      mbar_arrive(q_empty);
    }
    if (threadIdx.x == 0) note_cut(P, share, w);
  }
  fence_before();
  __syncthreads();
  if (warp == 9) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

template <int DT, int DH>
cudaError_t run(const CrossPlan &P, const CrossMaps &m, cudaStream_t s) {
  const CUtensorMap &q = *reinterpret_cast<const CUtensorMap *>(m.q), &k = *reinterpret_cast<const CUtensorMap *>(m.k),
                    &v = *reinterpret_cast<const CUtensorMap *>(m.v);
  if (P.d.keep) cross_wide_kernel<DT, DH, true><<<P.ctas, kThreads, Geo<DH>::smem, s>>>(q, k, v, P);
  else cross_wide_kernel<DT, DH, false><<<P.ctas, kThreads, Geo<DH>::smem, s>>>(q, k, v, P);
  return cudaGetLastError();
}

template <int DT, int DH>
cudaError_t prepare_one() {
  const cudaError_t e = cudaFuncSetAttribute(cross_wide_kernel<DT, DH, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Geo<DH>::smem);
  return e != cudaSuccess ? e
                          : cudaFuncSetAttribute(cross_wide_kernel<DT, DH, false>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                 (int)Geo<DH>::smem);
}

}  // namespace

cudaError_t cross_wide_prepare() {
  cudaError_t e = prepare_one<WT_BF16, 1>();
  if (e == cudaSuccess) e = prepare_one<WT_BF16, 2>();
  if (e == cudaSuccess) e = prepare_one<WT_F16, 1>();
  if (e == cudaSuccess) e = prepare_one<WT_F16, 2>();
  return e;
}

cudaError_t launch_cross_wide(const CrossPlan &P, const CrossMaps &m, cudaStream_t s) {
  if (P.d.dtype == WT_BF16) return P.d.head_dim <= 64 ? run<WT_BF16, 1>(P, m, s) : run<WT_BF16, 2>(P, m, s);
  return P.d.head_dim <= 64 ? run<WT_F16, 1>(P, m, s) : run<WT_F16, 2>(P, m, s);
}

}  // namespace wt
