// The shared prefix of wt_attend on the 5th-generation tensor cores (tcgen05): all queries of the
// batch that use a kv head against that head's keys, as one matrix product after another,
//
//   S = Q K^T,   P = 2^(scale log2(e) S - m),   O += P V,   l += row sums of P,
//
// which reads the prefix once for the whole batch.  Rows are (token, head-in-group) pairs, 128 of
// them (whole tokens) a tile; keys come in tiles of 128.  A CTA takes one contiguous range of the
// key tiles of all kv heads (crossing from one head to the next where it must) for two row tiles, and
// leaves O (fp32, not divided), m and l of each part for the merge.  CTAs that take the same keys for
// other rows are neighbours in the grid, so a key tile crosses HBM once and is then found in L2.
//
//   producer warp    TMA boxes of Q (two tiles), and of K and V into a ring (128-byte swizzle)
//   MMA thread       S_i = Q_i K^T for the two streams i, then O_i += P_i V as each P_i arrives
//   two warpgroups   one per stream; a thread owns a row: it reads the row of S from tensor memory,
//                    takes the exponentials and writes P (16-bit) back over S, where it is the next
//                    product's A operand
//
// The two streams are two row tiles against the same keys, or, where there is one row tile only, the
// even and the odd key tiles of the range, so that one stream's products run beside the other's
// exponentials.  The reference m of a row (set below its maximum for f16: kBelow) moves only when the
// maximum has grown by more than 8 (in log2): O is then rescaled in tensor memory; until then p stays
// where both 16-bit types hold it as precisely.  P is rounded to the caches' type (the MMA takes both operands in one type);
// l is summed in fp32 from the rounded values, so that what all keys' roundings have in common cancels
// (equal scores give the mean of the values, whatever the reference).
//
// Bound: the products.  768 rows against 32768 keys of 8 heads of 128: 71 us, 1.4 PFLOP/s of the 1.86
// that a large library product reaches.  For few rows, HBM and then latency: 6000 keys of 8 heads against 96 rows take
// 13 us, of which HBM needs 4.
//
// Every mbarrier wait is bounded; a timeout records WT_ETIMEDOUT and every role stops.
#include "wt_tmem.cuh"

namespace wt {

namespace {

constexpr int kRowsT = 128;  // rows of a tile (UMMA M)
constexpr int kKeysT = 128;  // keys of a tile
constexpr int kThreads = 384;  // warps 0-3, 4-7: softmax of stream 0, 1; 8: producer; 9: MMA, TMEM; 10, 11: idle
// Registers a thread after the split: 128 of S, and its exponentials, for softmax.  The launch gives
// 3 x 168 to the three warpgroups together.
constexpr int kRegsSoftmax = 224, kRegsRest = 56;
static_assert(2 * kRegsSoftmax + kRegsRest <= 3 * 168, "what the launch has");
constexpr uint32_t kTmemCols = 512;    // S_0, S_1 (128 columns each), O_0, O_1

template <int DH>  // 64-element halves of head_dim
struct Geo {
  static constexpr uint32_t stage = DH * kHalf;
  static constexpr int stages = DH == 2 ? 5 : 8;
  static constexpr uint32_t ring = 2 * stage;  // after the two Q tiles
  static constexpr uint32_t bars = ring + stages * stage;
  static constexpr int nbars = 2 * stages + 11;
  static constexpr size_t smem = bars + nbars * 8 + 16 + 1024;
};
static_assert(Geo<2>::smem <= 232448, "shared memory of one CTA");

// The segments of a CTA's range of key tiles: one for each kv head it meets.
struct Segment {
  int head, tile0, n;  // first key tile within the head, tiles
};

template <int DT, int DH>
__global__ void __launch_bounds__(kThreads, 1)
    attend_prefix_kernel(const __grid_constant__ CUtensorMap qmap, const __grid_constant__ CUtensorMap kmap,
                         const __grid_constant__ CUtensorMap vmap, const __grid_constant__ PrefixPlan P, int *status) {
  using X = Geo<DH>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t *gbase = smem_raw + (base - smem_u32(smem_raw));
  const uint32_t full0 = base + X::bars, empty0 = full0 + X::stages * 8;
  const uint32_t q_full = empty0 + X::stages * 8, q_empty = q_full + 8;
  const uint32_t s_full = q_empty + 8, p_full = s_full + 16, o_full = p_full + 16;  // [2] each
  const uint32_t p_half = o_full + 16, fin = p_half + 16;
  uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(gbase + X::bars + X::nbars * 8);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(tmem_slot + 2);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rb = blockIdx.x % P.row_blocks, grp = blockIdx.x / P.row_blocks;
  const bool apart = P.apart != 0;  // one row tile; streams are the even and odd key tiles
  const int w0 = grp * P.len, w1 = min(P.kv_heads * P.tiles, w0 + P.len);
  auto segment = [&](int w) -> Segment {
    const int head = w / P.tiles, t0 = w - head * P.tiles;
    return {head, t0, min(P.tiles - t0, w1 - w)};
  };

  if (threadIdx.x == 0) {
    for (int s = 0; s < X::stages; ++s) {
      mbar_init(full0 + 8 * s, 1);
      mbar_init(empty0 + 8 * s, 1);
    }
    mbar_init(q_full, 1);
    mbar_init(q_empty, 256);
    mbar_init(fin, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(s_full + 8 * i, 1);
      mbar_init(p_full + 8 * i, 128);
      mbar_init(p_half + 8 * i, 128);
      mbar_init(o_full + 8 * i, 1);
    }
    *abort_flag = 0;
    mbar_fence_init();
  }
  if (warp == 9) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                 "r"(kTmemCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  fence_before();
  __syncthreads();
  fence_after();
  griddep_launch();  // the own keys' kernel may take SMs as they come free
  const uint32_t tmem = *tmem_slot;
  const int lead = apart ? 2 : 1;  // key tiles whose K is loaded ahead of their V

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsRest));
    // ---------------- producer
    if (warp == 8 && lane == 0) {
      uint32_t it = 0, seg = 0;
      bool live = true;
      auto load = [&](const CUtensorMap *map, int head, int tile) {
        const uint32_t s = it % X::stages;
        if (it >= X::stages && !bounded_wait(empty0 + 8 * s, ((it / X::stages) - 1) & 1, abort_flag, status)) return false;
        const uint32_t bar = full0 + 8 * s, dst = base + X::ring + s * X::stage;
        mbar_expect_tx(bar, X::stage);
#pragma unroll
        for (int hf = 0; hf < DH; ++hf) tma_3d(dst + hf * kHalf, map, hf * 64, head, tile * kKeysT, bar);
        ++it;
        return true;
      };
      uint32_t q_loads = 0;
      for (int w = w0; w < w1 && live; ++seg) {
        const Segment g = segment(w);
        w += g.n;
        if (seg && !bounded_wait(q_empty, (seg - 1) & 1, abort_flag, status)) break;
        const int qtiles = apart ? 1 : 2;
        mbar_expect_tx(q_full, (uint32_t)qtiles * DH * P.tile_rows * 128);
        ++q_loads;
        for (int i = 0; i < qtiles; ++i)
#pragma unroll
          for (int hf = 0; hf < DH; ++hf)
            tma_3d(base + (i * DH + hf) * kHalf, &qmap, hf * 64, g.head * P.G, (rb * 2 + i) * P.tile_tokens, q_full);
        for (int j = 0; j < min(lead, g.n) && live; ++j) live = load(&kmap, g.head, g.tile0 + j);
        for (int j = 0; j < g.n && live; ++j) {
          live = load(&vmap, g.head, g.tile0 + j);
          if (live && j + lead < g.n) live = load(&kmap, g.head, g.tile0 + j + lead);
        }
      }
      if (*abort_flag) {
        // drain: copies of the last stages may still be landing
        const uint32_t first = it > (uint32_t)X::stages ? it - X::stages : 0;
        for (uint32_t j = first; j < it; ++j) {
          const long long t0 = clock64();
          while (!mbar_try_wait(full0 + 8 * (j % X::stages), (j / X::stages) & 1) && clock64() - t0 < kWaitCycles) {
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
    // (one thread alone, with its descriptors built at each product, spent twice the products' time on
    // issuing them: 113 us for 32768 keys and 768 rows of 8 heads, this way 79)
    if (warp == 9) {
      constexpr uint32_t kBf = DT == WT_BF16 ? 1u : 0u;
      constexpr uint32_t kIqk = idesc(kBf, kKeysT, 0), kIpv = idesc(kBf, DH * 64, 1);
      uint32_t it = 0, seg = 0, np[2] = {0, 0};
      bool live = true;
      uint32_t stage = 0;
      auto next = [&]() {  // the ring's next tile has landed
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
      auto scores = [&](int i, uint32_t s) {
        const uint32_t q = desc_k(base + (apart ? 0 : i) * X::stage), k = desc_k(base + X::ring + s * X::stage);
        if (elect_one()) {
#pragma unroll
          for (int e = 0; e < DH * 4; ++e) {
            const uint32_t off = ((e >> 2) * kHalf + (e & 3) * 32) >> 4;
            if (e < P.dim_steps) umma_ss(tmem + i * 128, q + off, k + off, kIqk, e != 0);
          }
          commit(s_full + 8 * i);
        }
        __syncwarp();
      };
      auto values = [&](int i, uint32_t s, bool first) {  // false: no P came
        const uint32_t v = desc_mn(base + X::ring + s * X::stage);
        // the first half of the keys as soon as its P is there
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          if (!warp_wait((hf ? p_full : p_half) + 8 * i, np[i] & 1, abort_flag, status)) return live = false;
          fence_after();
          if (elect_one()) {
#pragma unroll
            for (int e = hf * 4; e < hf * 4 + 4; ++e)
              umma_ts(tmem + 256 + i * 128, tmem + i * 128 + e * 8, v + e * (2048 >> 4), kIpv, !first || e != 0);
            if (hf) commit(o_full + 8 * i);
          }
          __syncwarp();
        }
        ++np[i];
        return true;
      };
      for (int w = w0; w < w1 && live; ++seg) {
        const Segment g = segment(w);
        w += g.n;
        if (!warp_wait(q_full, seg & 1, abort_flag, status)) break;
        fence_after();
        if (!apart) {
          if (!next()) break;
          scores(0, stage);
          scores(1, stage);
          release(empty0 + 8 * stage);
          for (int j = 0; j < g.n; ++j) {
            if (!next()) break;
            const uint32_t vs = stage;
            const bool more = j + 1 < g.n;
            if (!values(0, vs, j == 0)) break;
            if (more) {
              if (!next()) break;
              scores(0, stage);
            }
            if (!values(1, vs, j == 0)) break;
            release(empty0 + 8 * vs);
            if (more) {
              scores(1, stage);
              release(empty0 + 8 * stage);
            }
          }
        } else {
          for (int j = 0; j < min(2, g.n) && next(); ++j) {
            scores(j, stage);
            release(empty0 + 8 * stage);
          }
          if (!live) break;
          for (int j = 0; j < g.n; ++j) {
            if (!next()) break;
            const uint32_t vs = stage;
            if (!values(j & 1, vs, j < 2)) break;
            release(empty0 + 8 * vs);
            if (j + 2 < g.n) {
              if (!next()) break;
              scores(j & 1, stage);
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
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsSoftmax));
    // ---------------- softmax: a thread owns row threadIdx.x % 128 of stream i
    const int i = warp >> 2, r = threadIdx.x & 127;
    const uint32_t lanes = (uint32_t)(warp & 3) << 21;  // 32 lanes of tensor memory per warp
    const uint32_t S = tmem + lanes + i * 128, O = tmem + lanes + 256 + i * 128;
    uint32_t done = 0;  // tiles of this stream over all segments
    uint32_t seg = 0;
    bool live = true;
    for (int w = w0; w < w1 && live; ++seg) {
      const Segment g = segment(w);
      w += g.n;
      // The segment's queries have landed, so every thread has released those before (q_empty).  A stream
      // without a tile here waits for nothing else: ahead of the other it would release queries that are
      // still in use, and the producer would announce the next ones in a phase that has its arrival.
      if (!warp_wait(q_full, seg & 1, abort_flag, status)) break;
      const int n = apart ? (g.n + 1 - i) / 2 : g.n;
      float m = 0.0f, l0 = 0.0f, l1 = 0.0f;
      for (int j = 0; j < n; ++j) {
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
        const int keys = P.prefix_len - (g.tile0 + (apart ? 2 * j + i : j)) * kKeysT;
        if (keys < kKeysT) {
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
        const float top = max3(max3(mx0, mx1, mx2), mx3, mx3) * P.scale_log2;
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
            fma_x2(v[c], v[c + 1], P.scale_log2, -ref);
            v[c] = exp2_approx(v[c]);
            v[c + 1] = exp2_approx(v[c + 1]);
            u[k / 2] = pack2<DT>(v[c], v[c + 1]);
            float r0, r1;
            unpack2<DT>(u[k / 2], r0, r1);
            add_x2(l0, l1, r0, r1);
          }
          tmem_st32(S + hf * 32, u);
          wait_st();
          fence_before();
          mbar_arrive((hf ? p_full : p_half) + 8 * i);
        }
      }
      if (!live) break;
      // This stream's rows to the workspace, 32 columns at a time, turned in shared memory so that 8 lanes
      // write 128 bytes of a row (a lane writing its own row touched 32 lines with each store: 3.3 us of a
      // decode step's 8).  The queries have been read by then, and their place is this stream's until
      // q_empty.
      const int row0 = apart ? 0 : (rb * 2 + i) * P.tile_rows;
      const int rows = min(P.tile_rows, P.rows - row0);  // of the tile; may be none
      const int64_t tile_at = ((int64_t)(grp + g.head) * P.qtiles + (apart ? i : rb * 2 + i)) * kRowsT;
      if (n > 0) {
        if (!warp_wait(o_full + 8 * i, (done + n - 1) & 1, abort_flag, status)) break;
        fence_after();
        const uint32_t turn = base + i * X::stage + (warp & 3) * (X::stage / 4);
        static_assert(32 * 128 <= X::stage / 4, "32 rows of 32 columns");
#pragma unroll 1
        for (int c = 0; c < DH * 64; c += 32) {
          uint32_t o[32];
          tmem_ld32(O + c, o);
          wait_ld();
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
            if (at < rows && col < P.head_dim) *reinterpret_cast<uint4 *>(P.o + (tile_at + at) * P.head_dim + col) = v;
          }
          __syncwarp();
        }
        fence_before();
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // before the next queries land there
      }
      mbar_arrive(q_empty);
      const float l = l0 + l1;
      if (r < rows) P.ml[tile_at + r] = make_float2(n == 0 ? -INFINITY : l == l ? m : l, l);
      done += n;
    }
  }
  fence_before();
  __syncthreads();
  if (warp == 9) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

template <int DT, int DH>
cudaError_t run(const PrefixPlan &P, const PrefixMaps &m, int *status, cudaStream_t s) {
  attend_prefix_kernel<DT, DH><<<(unsigned)(P.row_blocks * P.groups), kThreads, Geo<DH>::smem, s>>>(
      *reinterpret_cast<const CUtensorMap *>(m.q), *reinterpret_cast<const CUtensorMap *>(m.k),
      *reinterpret_cast<const CUtensorMap *>(m.v), P, status);
  return cudaGetLastError();
}

template <int DT, int DH>
cudaError_t prepare_one() {
  return cudaFuncSetAttribute(attend_prefix_kernel<DT, DH>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              (int)Geo<DH>::smem);
}

}  // namespace

cudaError_t prefix_prepare() {
  cudaError_t e = prepare_one<WT_BF16, 1>();
  if (e == cudaSuccess) e = prepare_one<WT_BF16, 2>();
  if (e == cudaSuccess) e = prepare_one<WT_F16, 1>();
  if (e == cudaSuccess) e = prepare_one<WT_F16, 2>();
  return e;
}

cudaError_t launch_attend_prefix(const PrefixPlan &P, const PrefixMaps &m, int dtype, int *status, cudaStream_t s) {
  if (dtype == WT_BF16) return P.head_dim <= 64 ? run<WT_BF16, 1>(P, m, status, s) : run<WT_BF16, 2>(P, m, status, s);
  return P.head_dim <= 64 ? run<WT_F16, 1>(P, m, status, s) : run<WT_F16, 2>(P, m, status, s);
}

}  // namespace wt
