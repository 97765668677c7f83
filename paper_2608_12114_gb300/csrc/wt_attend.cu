// Attention of a batch over a prefix that all its requests share and over each request's own paged
// cache (include/wt_serve.h): the warp kernel and the merge.
//
// Keys are split over CTAs (and over the warps of a CTA); each part gives, per (token, head), the
// sum O of p v, the sum l of p and the reference m the p were taken against, p = 2^(s - m) with
// s = scale log2(e) q.k.  Parts are joined exactly as softmax splits: O = sum_i 2^(m_i - m) O_i,
// l = sum_i 2^(m_i - m) l_i, m = max m_i, out = O / l; a part without a key has m = -infinity, and
// a token without any gets zeros.  The maximum passes over NaN scores, so a part whose sum is NaN says so
// in its m: a NaN query or key makes the token NaN on every route.
//
// attend_warp_kernel takes a CTA per (rows, kv head, keys of one request): rows are the (token,
// head) pairs that share a kv head, 16 or 32 of them, and each of 4 warps streams its own tiles of
// 16 keys through a ring of its own in shared memory (16-byte cp.async; one bulk copy a row, of 256
// bytes, was slower: 56 us against 47 for the own keys of 64 requests' drafts), with m16n8k16 MMAs on
// them.  The rows of absent keys arrive as zeros and their scores are masked, so what a page holds past
// its last key never reaches a product.  No warp waits for another before the end.  Bound: HBM (or
// L2) for up to 32 rows, latency for few keys: 134 MB of own keys of 64 requests (lengths up to 1024)
// take 38 us, 3.6 TB/s over all and 7 while every SM has long ones; 44 MB of 24 requests 16 us.
#include <algorithm>

#include "wt_serve.cuh"

namespace wt {

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
constexpr int kKeys = 16;    // keys of a tile
constexpr int kStages = 2;   // tiles of a warp's ring: three CTAs per SM at head_dim 128

// New tokens and own keys of request b, clamped to the descriptor.
struct Request {
  int t0, n, len;
};
__device__ __forceinline__ Request request_of(const wt_attend_desc &d, int b, int *status, bool tell) {
  int t0 = __ldg(d.begin + b), t1 = __ldg(d.begin + b + 1), len = d.max_len > 0 ? __ldg(d.len + b) : 0;
  if (t0 < 0 || t1 < t0 || t1 > d.n_tokens || t1 - t0 > d.max_new || len < 0 || len > d.max_len) {
    if (tell && status) atomicCAS(status, 0, kStatusInvalid);
    t0 = min(max(t0, 0), d.n_tokens);
    t1 = min(max(t1, t0), t0 + min(d.max_new, d.n_tokens - t0));
    len = min(max(len, 0), d.max_len);
  }
  return {t0, t1 - t0, len};
}

// ND: 16-element groups of head_dim (rounded up).  MT: tiles of 16 rows.  With one, three CTAs to an SM, and
// four of short heads (which the rows beside later tokens' keys would else bring to 160 registers and three).
template <int DT, int ND, int MT>
__global__ void __launch_bounds__(kThreads, MT > 1 ? 0 : ND == 4 ? 4 : 3) attend_warp_kernel(const __grid_constant__ AttendPlan P) {
  constexpr int kPitch = ND * 32 + 16;              // bytes of a staged row: 8 rows hit 8 different bank groups
  constexpr int kTileBytes = 2 * kKeys * kPitch;    // K rows, then V rows
  constexpr int kRows = 16 * MT;
  extern __shared__ __align__(128) uint8_t smem[];
  // Nothing here needs the prefix's parts, so this kernel may start while that one still runs; but it
  // must not end before it, because the merge waits for this kernel alone.
  struct AtEnd {
    __device__ ~AtEnd() { griddep_wait(); }
  } at_end;
  const wt_attend_desc &d = P.d;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, q = lane & 3, g = lane >> 2;
  const int G = P.G, D = d.head_dim;
  // CTAs of own keys by (request, split, row tile, kv head), then those of the prefix, where it is taken
  // here, by (split, row tile, kv head): it is a request of its own with every token of the batch.
  const int own_ctas = d.n_req * P.own_splits * P.own_tiles * d.kv_heads;
  const bool pre = (int)blockIdx.x >= own_ctas;
  const int at = pre ? blockIdx.x - own_ctas : blockIdx.x, hk = at % d.kv_heads;
  const int row_tiles = pre ? P.pre_tiles : P.own_tiles, rt = at / d.kv_heads % row_tiles;
  const int keys_of = at / (d.kv_heads * row_tiles);
  const int b = pre ? 0 : keys_of / P.own_splits;
  const int split = pre ? keys_of : keys_of % P.own_splits;
  Request rq;
  int k0, k1;
  if (pre) {
    rq = {0, d.n_tokens, 0};
    k0 = split * P.pre_len;
    k1 = (int)min(d.prefix_len, (int64_t)k0 + P.pre_len);
  } else {
    rq = request_of(d, b, P.status, hk == 0 && rt == 0 && split == 0 && tid == 0);
    k0 = split * P.own_len;
    k1 = (int)min((int64_t)rq.len, (int64_t)k0 + P.own_len);
  }
  const int rows = rq.n * G, row0 = rt * kRows;
  if (row0 >= rows) return;
  const int part = (pre ? P.own_splits : 0) + split;
  if (k0 >= k1) {  // the merge knows from the length that there is nothing
    if (P.direct)
      for (int r = row0 + (tid >> 5); r < min(rows, row0 + kRows); r += kWarps)
        if (lane * 4 < D)
          *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(d.out) + (int64_t)(rq.t0 + r / G) * d.out_stride +
                                     (hk * G + r % G) * D + lane * 4) = make_uint2(0, 0);
    return;
  }

  const uint32_t ring = smem_u32(smem) + warp * kStages * kTileBytes;
  if (D % 16) {
    // the last 8 columns stay zero: no copy touches them
    for (int i = tid; i < kWarps * kStages * 2 * kKeys; i += kThreads)
      *reinterpret_cast<uint4 *>(smem + i * kPitch + D * 2) = make_uint4(0, 0, 0, 0);
    __syncthreads();
  }

  const int tiles = (k1 - k0 + kKeys - 1) / kKeys;
  const int chunks = D / 8;  // 16-byte pieces of a row
  const int row_lane = lane / chunks, in_lane = lane - row_lane * chunks, row_step = 32 / chunks, in_step = 32 - row_step * chunks;
  const uint8_t *k_of = static_cast<const uint8_t *>(pre ? d.prefix_k : d.k_pages) + 2 * (pre ? hk * d.prefix_head : (int64_t)hk * D);
  const uint8_t *v_of = static_cast<const uint8_t *>(pre ? d.prefix_v : d.v_pages) + 2 * (pre ? hk * d.prefix_head : (int64_t)hk * D);
  const int64_t key_bytes = 2 * (pre ? d.prefix_stride : (int64_t)d.kv_heads * D);  // from a key to the next, within a page
  // Tiles start at multiples of 16 keys, so in pages of 16, 32, ... keys a tile lies in one page, its rows
  // evenly apart, and rows of 64 or 128 elements (8 or 16 lanes) keep each lane in its column.
  const bool even = (pre || d.page % kKeys == 0) && in_step == 0;
  // Tile i of this warp (tiles warp, warp + 4, ...) into its ring; bit r of `there`: key r exists.
  uint32_t there[kStages];
  auto fetch = [&](int i, uint32_t &found) {
    const int tile = warp + i * kWarps;
    if (tile < tiles) {
      const int key0 = k0 + tile * kKeys;
      const uint32_t dst = ring + (i % kStages) * kTileBytes;
      if (even) {
        int64_t first = key0;
        int n = min(kKeys, k1 - key0);
        if (!pre) {
          const int pg = key0 / d.page;
          const int page = __ldg(d.table + (int64_t)b * d.table_stride + pg);
          if (page >= 0 && page < d.n_pages) {
            first = (int64_t)page * d.page + (key0 - pg * d.page);
          } else {
            first = n = 0;
            if (P.status && lane == 0) atomicCAS(P.status, 0, kStatusInvalid);
          }
        }
        found = (1u << n) - 1;
        const int64_t off = (first + row_lane) * key_bytes + in_lane * 16, by = row_step * key_bytes;
        const uint8_t *ks = k_of + off, *vs = v_of + off;
        uint32_t to = dst + row_lane * kPitch + in_lane * 16;
        if (n == kKeys) {
#pragma unroll 4
          for (int r = row_lane; r < kKeys; r += row_step, to += row_step * kPitch, ks += by, vs += by) {
            cp16(to, ks, true);
            cp16(to + kKeys * kPitch, vs, true);
          }
        } else {
#pragma unroll 1
          for (int r = row_lane; r < kKeys; r += row_step, to += row_step * kPitch, ks += by, vs += by) {
            cp16(to, r < n ? ks : d.q, r < n);
            cp16(to + kKeys * kPitch, r < n ? vs : d.q, r < n);
          }
        }
      } else {
        // lane r knows where row r lies (rows 0-15: K, 16-31: V), and the lanes copy whole rows together
        const int key = key0 + (lane & 15);
        uint64_t src = 0;  // 0: an absent key
        if (key < k1) {
          const uint8_t *base = lane < 16 ? k_of : v_of;
          if (pre) {
            src = reinterpret_cast<uint64_t>(base + key * key_bytes);
          } else {
            const int pg = key / d.page;
            const int page = __ldg(d.table + (int64_t)b * d.table_stride + pg);
            if (page >= 0 && page < d.n_pages)
              src = reinterpret_cast<uint64_t>(base + ((int64_t)page * d.page + (key - pg * d.page)) * key_bytes);
            else if (P.status)
              atomicCAS(P.status, 0, kStatusInvalid);
          }
        }
        found = __ballot_sync(0xffffffffu, src != 0) & 0xffffu;
        int row = row_lane, in = in_lane;
#pragma unroll 4
        for (int c = 0; c < chunks; ++c) {
          const uint64_t a = __shfl_sync(0xffffffffu, src, row);
          cp16(dst + row * kPitch + in * 16, a ? reinterpret_cast<const void *>(a + in * 16) : d.q, a != 0);
          row += row_step;
          in += in_step;
          if (in >= chunks) in -= chunks, ++row;
        }
      }
    }
    cp_commit();
  };
  auto fill = [&]() {
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fetch(i, there[i]);
  };
  fill();

  // queries as A operands
  const int ksteps = (D + 15) / 16;
  uint32_t qf[MT][ND][4];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = row0 + i * 16 + g + e * 8;
      const bool ok = r < rows;
      const uint16_t *src = static_cast<const uint16_t *>(d.q) +
                            (ok ? (int64_t)(rq.t0 + r / G) * d.q_stride + (int64_t)(hk * G + r % G) * D : 0);
#pragma unroll
      for (int k = 0; k < ND; ++k)
#pragma unroll
        for (int f = 0; f < 2; ++f) {
          const int col = k * 16 + f * 8 + q * 2;
          qf[i][k][e + 2 * f] = ok && col < D ? __ldg(reinterpret_cast<const uint32_t *>(src + col)) : 0u;
        }
    }

  float o[MT][2 * ND][4], m[MT][2], l[MT][2];
  const float sl = d.scale * 1.4426950408889634f;

  // keys a row may see: all but the tail for own keys
  int sees[MT][2];
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const int r = row0 + i * 16 + g + e * 8;
      sees[i][e] = pre ? k1 : min(k1, rq.len - rq.n + 1 + r / G);
    }

  const int sees_all = pre ? k1 : min(k1, rq.len - rq.n + 1 + row0 / G);
  auto step = [&](int i, uint32_t found, bool apart) {
    const int slot = i % kStages;
    cp_wait<kStages - 1>();
    __syncwarp();
    const uint32_t kt = ring + slot * kTileBytes, vt = kt + kKeys * kPitch;
    const int key0 = k0 + (warp + i * kWarps) * kKeys;
    float s[MT][2][4];
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[a][j][e] = 0.0f;
#pragma unroll
    for (int k = 0; k < ND; ++k) {
      if (k >= ksteps) break;
      uint32_t kf[4];  // keys 0-7 and 8-15, each in two halves of 8 elements
      ldsm4(kf, kt + ((lane & 7) + (lane >> 4) * 8) * kPitch + k * 32 + ((lane >> 3) & 1) * 16);
#pragma unroll
      for (int a = 0; a < MT; ++a) {
        mma16816<DT>(s[a][0], qf[a][k][0], qf[a][k][1], qf[a][k][2], qf[a][k][3], kf[0], kf[1]);
        mma16816<DT>(s[a][1], qf[a][k][0], qf[a][k][1], qf[a][k][2], qf[a][k][3], kf[2], kf[3]);
      }
    }
    // every row sees every key of the tile, but at the end of a request
    const bool whole = found == 0xffffu && key0 + kKeys <= sees_all;
    uint32_t pf[MT][4];
#pragma unroll
    for (int a = 0; a < MT; ++a) {
      float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[a][j][e] *= sl;
          if (!whole) {
            const int r = j * 8 + q * 2 + (e & 1);
            if (!(found >> r & 1) || key0 + r >= sees[a][e >> 1]) s[a][j][e] = -INFINITY;
          }
          mx[e >> 1] = fmaxf(mx[e >> 1], s[a][j][e]);
        }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 1));
        mx[e] = fmaxf(mx[e], __shfl_xor_sync(0xffffffffu, mx[e], 2));
      }
      // The reference moves when a row's maximum has grown by more than 2^8; p then stays within what
      // both 16-bit types hold as precisely.  It starts at -infinity, so the first key seen sets it.
      constexpr float kGrow = kSlack + kBelow<DT>;
      const bool grown0 = mx[0] > m[a][0] + kGrow, grown1 = mx[1] > m[a][1] + kGrow;
      if (__any_sync(0xffffffffu, grown0 || grown1)) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float to = (e ? grown1 : grown0) ? mx[e] - kBelow<DT> : m[a][e];
          const float f = to > -INFINITY ? exp2_approx(m[a][e] - to) : 1.0f;
          m[a][e] = to;
          l[a][e] *= f;
#pragma unroll
          for (int j = 0; j < 2 * ND; ++j) {
            o[a][j][2 * e] *= f;
            o[a][j][2 * e + 1] *= f;
          }
        }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float ref = m[a][e] > -INFINITY ? m[a][e] : 0.0f;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            float &p = s[a][j][2 * e + z];
            p = exp2_approx(p - ref);
          }
      }
      // l from the rounded weights: what their roundings have in common cancels
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          pf[a][2 * j + e] = pack2<DT>(s[a][j][2 * e], s[a][j][2 * e + 1]);
          float lo, hi;
          unpack2<DT>(pf[a][2 * j + e], lo, hi);
          l[a][e] += lo + hi;
        }
    }
    if (apart && key0 + kKeys > sees_all) {  // each row adds the keys that it sees one by one
#pragma unroll 1
      for (int r = 0; r < kKeys; ++r) {
        if (!(found >> r & 1)) continue;
#pragma unroll
        for (int a = 0; a < MT; ++a)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const uint32_t w = __shfl_sync(0xffffffffu, r < 8 ? pf[a][e] : pf[a][2 + e], (lane & 28) | (r & 7) >> 1);
            float p0, p1;
            unpack2<DT>(w, p0, p1);
            const float p = r & 1 ? p1 : p0;
            if (key0 + r < sees[a][e])
#pragma unroll
              for (int j = 0; j < 2 * ND; ++j) {
                float v0, v1;
                unpack2<DT>(lds32(vt + r * kPitch + j * 16 + q * 4), v0, v1);
                o[a][j][2 * e] += p * v0;
                o[a][j][2 * e + 1] += p * v1;
              }
          }
      }
      __syncwarp();
      return;
    }
#pragma unroll
    for (int k = 0; k < ND; ++k) {
      if (k >= ksteps) break;
      uint32_t vf[4];  // 16 keys x 16 elements
      ldsm4t(vf, vt + (lane & 15) * kPitch + k * 32 + (lane >> 4) * 16);
#pragma unroll
      for (int a = 0; a < MT; ++a) {
        mma16816<DT>(o[a][2 * k], pf[a][0], pf[a][1], pf[a][2], pf[a][3], vf[0], vf[1]);
        mma16816<DT>(o[a][2 * k + 1], pf[a][0], pf[a][1], pf[a][2], pf[a][3], vf[2], vf[3]);
      }
    }
    __syncwarp();  // every lane has read the tile before a later fetch overwrites it
  };
  const int mine = (tiles - warp + kWarps - 1) / kWarps;  // tiles of this warp
  // A weight of 0 does not hide a value that is not finite (0 * infinity).  So where some row does not see
  // a key that is there, a later token's, and something in O is not finite, the warp goes through its
  // tiles once more and keeps the rows of the tiles with such keys apart.  (7 requests of up to 3 drafts:
  // 14.2 us; looking at such a tile's values before its product 14.6, with neither 14.0.)
  for (bool apart = false;; apart = true) {
#pragma unroll
    for (int a = 0; a < MT; ++a) {
#pragma unroll
      for (int j = 0; j < 2 * ND; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[a][j][e] = 0.0f;
      m[a][0] = m[a][1] = -INFINITY;
      l[a][0] = l[a][1] = 0.0f;
    }
    for (int i = 0; i < mine; i += kStages)
#pragma unroll
      for (int u = 0; u < kStages; ++u)  // unrolled: the ring's slots and `there` are constants
        if (i + u < mine) {
          fetch(i + u + kStages - 1, there[(u + kStages - 1) % kStages]);
          step(i + u, there[u], apart);
        }
    cp_wait<0>();
    if (apart || sees_all >= k1) break;
    float z[4] = {0.0f, 0.0f, 0.0f, 0.0f};  // NaN where O has NaN or an infinity
#pragma unroll
    for (int a = 0; a < MT; ++a)
#pragma unroll
      for (int j = 0; j < 2 * ND; ++j)
#pragma unroll
        for (int e = 0; e < 4; ++e) z[e] = fmaf(o[a][j][e], 0.0f, z[e]);
    const float any = (z[0] + z[1]) + (z[2] + z[3]);
    if (!__any_sync(0xffffffffu, any != any)) break;
    fill();
  }
  __syncthreads();

  // join the four warps: one row of tiles at a time
  constexpr int kCols = ND * 16;
  float *so = reinterpret_cast<float *>(smem);           // [kWarps][16][kCols]
  float2 *sml = reinterpret_cast<float2 *>(so + kWarps * 16 * kCols);  // [kWarps][16]
  static_assert((kWarps * 16 * kCols + 2 * kWarps * 16) * 4 <= kWarps * kStages * kTileBytes, "fits the rings");
#pragma unroll
  for (int a = 0; a < MT; ++a) {
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      float s = l[a][e];
      s += __shfl_xor_sync(0xffffffffu, s, 1);
      s += __shfl_xor_sync(0xffffffffu, s, 2);
      if (q == 0) sml[warp * 16 + g + e * 8] = make_float2(m[a][e], s);
#pragma unroll
      for (int j = 0; j < 2 * ND; ++j)
        *reinterpret_cast<float2 *>(so + (warp * 16 + g + e * 8) * kCols + j * 8 + q * 2) =
            make_float2(o[a][j][2 * e], o[a][j][2 * e + 1]);
    }
    __syncthreads();
    for (int r = warp; r < 16; r += kWarps) {
      const int row = row0 + a * 16 + r;
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
      const int64_t at = (int64_t)part * d.n_tokens * d.heads + (int64_t)(rq.t0 + row / G) * d.heads + hk * G + row % G;
      if (lane * 4 < D) {
        float4 v = make_float4(0, 0, 0, 0);
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float4 x = *reinterpret_cast<const float4 *>(so + (w * 16 + r) * kCols + lane * 4);
          v.x += f[w] * x.x, v.y += f[w] * x.y, v.z += f[w] * x.z, v.w += f[w] * x.w;
        }
        if (P.direct) {
          const float inv = ll == 0.0f ? 0.0f : 1.0f / ll;
          *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(d.out) + (int64_t)(rq.t0 + row / G) * d.out_stride +
                                     (hk * G + row % G) * D + lane * 4) =
              make_uint2(pack2<DT>(v.x * inv, v.y * inv), pack2<DT>(v.z * inv, v.w * inv));
        } else {
          *reinterpret_cast<float4 *>(P.o + at * D + lane * 4) = v;
        }
      }
      if (lane == 0 && !P.direct) P.ml[at] = make_float2(ll == ll ? mm : ll, ll);
    }
    __syncthreads();
  }
}

// out[t, h] = sum over the parts, WR warps (1 or 4) to a (token, head); with 4, each takes every
// fourth part.  The references and sums of 32 parts are read at once, one by each lane, and the parts'
// O eight at a time, so that few reads wait for one another (one part after another: 31 us for a
// decode step of 24 requests with 37 parts each, this way 4).
constexpr int kMergeParts = 8;
template <int DT, int WR>
__global__ void __launch_bounds__(kThreads) attend_merge_kernel(const __grid_constant__ AttendPlan P) {
  __shared__ float4 so[kWarps][32];
  const wt_attend_desc &d = P.d;
  const int lane = threadIdx.x & 31, warp = WR == 1 ? 0 : threadIdx.x >> 5;
  const int b = blockIdx.y;
  // without own keys no CTA before has looked at the requests
  const Request rq = request_of(d, b, P.status, P.own_splits == 0 && blockIdx.x == 0 && threadIdx.x == 0);
  griddep_wait();  // launched while the kernel before it ends
  const int i = WR == 1 ? blockIdx.x * kWarps + (threadIdx.x >> 5) : blockIdx.x;
  if (i >= rq.n * d.heads) return;
  const int h = i % d.heads, t = rq.t0 + i / d.heads;
  const int64_t row = (int64_t)rq.t0 * d.heads + i, rows = (int64_t)d.n_tokens * d.heads;
  const int own = P.own_splits ? (rq.len + P.own_len - 1) / P.own_len : 0;
  const int D = d.head_dim;
  // the parts: own splits, then the prefix's (those of the warp kernel, or the slots on tcgen05)
  int all = own + P.pre_splits, x0 = 0;
  const int per = P.x.apart ? 2 : 1;
  int xrow = 0;
  if (P.x.groups) {
    const PrefixPlan &x = P.x;
    const int hk = h / P.G, r = t * P.G + h % P.G, start = hk * x.tiles;
    const int g0 = start / x.len, g1 = (start + x.tiles - 1) / x.len;  // first and last range in the head
    all += (g1 - g0 + 1) * per;
    x0 = (g0 + hk) * x.qtiles;
    xrow = x.apart ? r : r / x.tile_rows * 128 + r % x.tile_rows;
  }
  // part k: its O (of D numbers), and its m and l
  auto find = [&](int k, const float2 *&ml) -> const float * {
    int64_t at;
    if (k < own + P.pre_splits) {
      at = (int64_t)(k < own ? k : P.own_splits + k - own) * rows + row;
      ml = P.ml + at;
      return P.o + at * D;
    }
    k -= own + P.pre_splits;
    // apart: the two streams of a slot are tiles of their own; else a slot's tiles are row tiles
    at = (int64_t)(x0 + (per == 2 ? (k >> 1) * P.x.qtiles + (k & 1) : k * P.x.qtiles)) * 128 + xrow;
    ml = P.x.ml + at;
    return P.x.o + at * D;
  };
  auto read = [&](int k) {
    const float2 *ml;
    find(k, ml);
    return *ml;
  };
  float2 mine = lane < all ? read(lane) : make_float2(-INFINITY, 0.0f);
  float m = mine.x;
  for (int k = lane + 32; k < all; k += 32) m = fmaxf(m, read(k).x);
#pragma unroll
  for (int s = 16; s; s >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, s));
  float4 o = make_float4(0, 0, 0, 0);
  float l = 0.0f;
  const bool cols = lane * 4 < D;
  for (int k0 = 0; k0 < all; k0 += 32) {
    if (k0) mine = k0 + lane < all ? read(k0 + lane) : make_float2(-INFINITY, 0.0f);
    // A part without a key: its O was not written.  One whose factor is 0 still counts: what is not finite in
    // it has to show.
    const bool keys = mine.x > -INFINITY || mine.x != mine.x;
    const float f = keys ? exp2_approx(mine.x - m) : 0.0f;
    if (keys) l += f * mine.y;
    const unsigned some = __ballot_sync(0xffffffffu, keys);
    for (int k = k0 + warp; k < min(all, k0 + 32); k += WR * kMergeParts) {
      float4 x[kMergeParts];
      float w[kMergeParts];
#pragma unroll
      for (int u = 0; u < kMergeParts; ++u) {
        const int kk = k + u * WR, at = kk - k0;
        const bool there = at < 32 && (some >> at & 1) && cols;
        const float2 *ml;
        x[u] = there ? *reinterpret_cast<const float4 *>(find(kk, ml) + lane * 4) : make_float4(0, 0, 0, 0);
        w[u] = __shfl_sync(0xffffffffu, f, at & 31);
      }
#pragma unroll
      for (int u = 0; u < kMergeParts; ++u)
        o.x += w[u] * x[u].x, o.y += w[u] * x[u].y, o.z += w[u] * x[u].z, o.w += w[u] * x[u].w;
    }
  }
#pragma unroll
  for (int s = 16; s; s >>= 1) l += __shfl_xor_sync(0xffffffffu, l, s);
  if constexpr (WR > 1) {
    so[warp][lane] = o;
    __syncthreads();
    if (warp) return;
#pragma unroll
    for (int w = 1; w < WR; ++w) {
      const float4 x = so[w][lane];
      o.x += x.x, o.y += x.y, o.z += x.z, o.w += x.w;
    }
  }
  if (cols) {
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    uint16_t *dst = static_cast<uint16_t *>(d.out) + (int64_t)t * d.out_stride + h * D + lane * 4;
    *reinterpret_cast<uint2 *>(dst) = make_uint2(pack2<DT>(o.x * inv, o.y * inv), pack2<DT>(o.z * inv, o.w * inv));
  }
}

template <int ND>
constexpr size_t warp_smem() {
  return (size_t)kWarps * kStages * 2 * kKeys * (ND * 32 + 16);
}

// `after`: the kernel waits on the device for the one before it in this call, so it may be launched
// while that one ends (measured a call: 1 to 4 us less, from one token to 64 requests).  Never a call's first
// kernel: it reads the caller's memory before it waits.
cudaError_t launch(void (*k)(AttendPlan), dim3 grid, size_t smem, bool after, cudaStream_t s, const AttendPlan &P) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = after ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, k, P);
}

template <int DT, int ND>
cudaError_t run_warp(const AttendPlan &P, cudaStream_t s) {
  const unsigned grid = (unsigned)(P.d.kv_heads * (P.d.n_req * P.own_splits * P.own_tiles + P.pre_splits * P.pre_tiles));
  if (grid == 0) return cudaSuccess;
  return launch(P.rows_tile == 16 ? attend_warp_kernel<DT, ND, 1> : attend_warp_kernel<DT, ND, 2>, dim3(grid), warp_smem<ND>(),
                P.x.groups != 0, s, P);
}

template <int DT>
cudaError_t run_dim(const AttendPlan &P, cudaStream_t s) {
  if (P.d.head_dim <= 64) return run_warp<DT, 4>(P, s);
  if (P.d.head_dim <= 96) return run_warp<DT, 6>(P, s);
  return run_warp<DT, 8>(P, s);
}

template <int DT, int ND>
cudaError_t prepare_warp() {
  cudaError_t e = cudaFuncSetAttribute(attend_warp_kernel<DT, ND, 1>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                       (int)warp_smem<ND>());
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(attend_warp_kernel<DT, ND, 2>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)warp_smem<ND>());
  return e;
}

}  // namespace

cudaError_t attend_prepare() {
  cudaError_t e = prepare_warp<WT_BF16, 4>();
  if (e == cudaSuccess) e = prepare_warp<WT_BF16, 6>();
  if (e == cudaSuccess) e = prepare_warp<WT_BF16, 8>();
  if (e == cudaSuccess) e = prepare_warp<WT_F16, 4>();
  if (e == cudaSuccess) e = prepare_warp<WT_F16, 6>();
  if (e == cudaSuccess) e = prepare_warp<WT_F16, 8>();
  return e;
}

cudaError_t launch_attend_warp(const AttendPlan &P, cudaStream_t s) {
  return P.d.dtype == WT_BF16 ? run_dim<WT_BF16>(P, s) : run_dim<WT_F16>(P, s);
}

template <int DT>
cudaError_t run_merge(const AttendPlan &P, cudaStream_t s) {
  const unsigned rows = (unsigned)(P.d.max_new * P.d.heads);
  // four warps to a row only where one to a row would leave SMs idle
  const bool one = (int64_t)P.d.n_tokens * P.d.heads >= 16ll * num_sms();
  return launch(one ? attend_merge_kernel<DT, 1> : attend_merge_kernel<DT, kWarps>,
                dim3(one ? (rows + kWarps - 1) / kWarps : rows, (unsigned)P.d.n_req), 0,
                P.x.groups || P.own_splits || P.pre_splits, s, P);
}

cudaError_t launch_attend_merge(const AttendPlan &P, cudaStream_t s) {
  return P.d.dtype == WT_BF16 ? run_merge<WT_BF16>(P, s) : run_merge<WT_F16>(P, s);
}

}  // namespace wt
