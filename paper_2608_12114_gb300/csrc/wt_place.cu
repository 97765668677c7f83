// Norms, rotation and placing of a step's queries, keys and values (include/wt_serve.h).
//
// A head's elements are taken in units of 8 that hold whole pairs (two runs of four elements: j .. j + 3
// and rot_dim / 2 further on, or eight neighbours), one unit a lane, so a rotation needs no other lane
// and the norm's sum of squares one exchange among the lanes of a head.  A warp takes one token's heads
// of q, k and v in turn, as many at a time as fit its lanes; a lane keeps its unit, so its four angles,
// and the norms' weights, are worked out once for all heads.
//
// The angle is exact modulo a turn: pos * turns wraps at 2^64 as the angle does at a turn, and the top 32
// bits of the product, as a signed number, are the fraction in [-1/2, 1/2) that sincospif takes.
#include <algorithm>

#include "wt_serve.cuh"

namespace wt {

namespace {

constexpr int kThreads = 128;
constexpr int kAhead = 4;  // heads of a lane whose loads are in flight together

__device__ __forceinline__ void note_invalid(int *status) {
  if (status) atomicCAS(status, 0, kStatusInvalid);
}

// Four elements of type DT as fp32, and back.
template <int DT>
__device__ __forceinline__ void load4(const void *p, int64_t at, float (&x)[4]) {
  if constexpr (DT == WT_F32) {
    const float4 v = *reinterpret_cast<const float4 *>(static_cast<const float *>(p) + at);
    x[0] = v.x, x[1] = v.y, x[2] = v.z, x[3] = v.w;
  } else {
    const uint2 v = *reinterpret_cast<const uint2 *>(static_cast<const uint16_t *>(p) + at);
    unpack2<DT>(v.x, x[0], x[1]);
    unpack2<DT>(v.y, x[2], x[3]);
  }
}
template <int DT>
__device__ __forceinline__ void store4(void *p, int64_t at, const float (&x)[4]) {
  *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(p) + at) = make_uint2(pack2<DT>(x[0], x[1]), pack2<DT>(x[2], x[3]));
}
__device__ __forceinline__ float load_norm(const void *p, int dtype, int at) {
  if (dtype == WT_F32) return __ldg(static_cast<const float *>(p) + at);
  const uint32_t w = __ldg(static_cast<const uint16_t *>(p) + at);
  float lo, hi;
  if (dtype == WT_BF16) unpack2<WT_BF16>(w, lo, hi);
  else unpack2<WT_F16>(w, lo, hi);
  return lo;
}

// How many of v[0 .. n) are at most t, where v ascends (any number up to n where it does not).  The whole
// warp looks at 32 entries at once: one load for up to 32 entries, two for 1024.
__device__ __forceinline__ int count_upto(const int32_t *v, int n, int t, int lane) {
  int lo = 0, hi = n;
  while (lo < hi) {
    const int step = (hi - lo + 31) / 32, i = lo + (lane + 1) * step - 1;
    const unsigned past = ~__ballot_sync(0xffffffffu, i < hi && __ldg(v + min(i, n - 1)) <= t);
    const int c = past ? __ffs(past) - 1 : 32;
    lo += c * step;
    hi = min(hi, lo + step - 1);
  }
  return min(lo, n);
}

template <int IN, int DT>
__global__ void __launch_bounds__(kThreads) place_kernel(const __grid_constant__ PlacePlan P) {
  const wt_place_desc &d = P.d;
  const int lane = threadIdx.x & 31;
  const int64_t w = (int64_t)blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5);
  const int D = d.head_dim, half = d.rot_dim / 2;
  if (d.begin)  // every request's numbers are looked at by one thread
    for (int64_t b = (int64_t)blockIdx.x * kThreads + threadIdx.x; b < d.n_req; b += (int64_t)gridDim.x * kThreads) {
      const int t0 = __ldg(d.begin + b), t1 = __ldg(d.begin + b + 1), len = d.len ? __ldg(d.len + b) : 0;
      if (t0 < 0 || t1 < t0 || t1 > d.n_tokens || (d.len && (len < t1 - t0 || len > d.max_len))) note_invalid(P.status);
    }
  const int t = (int)(w / P.chunks), chunk = (int)(w % P.chunks);
  if (t >= d.n_tokens) return;

  // this lane's unit of a head, and which of the warp's heads
  const int slot = lane >> P.width_log2, u = lane & ((1 << P.width_log2) - 1), slots = 32 >> P.width_log2;
  const bool in_head = u * 8 < D, turned = u * 8 < d.rot_dim;
  const bool halves = turned && !(d.flags & WT_PLACE_NEIGHBOURS);
  const int at0 = halves ? u * 4 : u * 8, at1 = halves ? half + u * 4 : u * 8 + 4;

  const int hq = d.q ? d.heads : 0, hk = d.k ? d.kv_heads : 0, hv = d.v ? d.kv_heads : 0, all = hq + hk + hv;
  const int h_end = min(all, (chunk + 1) * P.chunk_heads);
  float x0[kAhead][4], x1[kAhead][4];
  auto fetch = [&](int h, float (&a)[4], float (&b)[4]) {
    if (h < h_end && in_head) {
      const void *src = h < hq ? d.q : h < hq + hk ? d.k : d.v;
      const int64_t row = h < hq ? (int64_t)t * d.q_stride + (int64_t)h * D
                          : h < hq + hk ? (int64_t)t * d.k_stride + (int64_t)(h - hq) * D
                                        : (int64_t)t * d.v_stride + (int64_t)(h - hq - hk) * D;
      load4<IN>(src, row + at0, a);
      load4<IN>(src, row + at1, b);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) a[e] = b[e] = 0.0f;
    }
  };
  const int h0 = chunk * P.chunk_heads + slot;
#pragma unroll
  for (int i = 0; i < kAhead; ++i) fetch(h0 + i * slots, x0[i], x1[i]);

  // the token's request and place
  int place = 0;
  bool cached = false;
  int64_t row = 0;
  if (d.begin) {
    const int b = count_upto(d.begin, d.n_req + 1, t, lane) - 1;
    if (b < 0 || b >= d.n_req) return;
    const int t0 = __ldg(d.begin + b), t1 = min(max(__ldg(d.begin + b + 1), t0), d.n_tokens);
    if (t < t0 || t >= t1) return;
    if (d.len) {
      const int len = min(max(__ldg(d.len + b), 0), d.max_len);
      place = len - (t1 - max(t0, 0)) + (t - max(t0, 0));
      if (place >= 0 && d.table) {
        const int pg = place / d.page, page = __ldg(d.table + (int64_t)b * d.table_stride + pg);
        cached = page >= 0 && page < d.n_pages;
        row = ((int64_t)page * d.page + (place - pg * d.page)) * d.kv_heads;
        if (!cached && lane == 0) note_invalid(P.status);
      }
    }
  }

  float c[4], s[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) c[e] = 1.0f, s[e] = 0.0f;
  if (turned) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = u * 4 + e;
      const int64_t pos = d.pos ? (int64_t)__ldg(d.pos + (int64_t)t * d.pos_stride + d.axis[j]) : (int64_t)d.first_pos + place;
      const uint64_t turn = (uint64_t)pos * __ldg(reinterpret_cast<const unsigned long long *>(d.turns) + j);
      sincospif((float)(int32_t)(turn >> 32) * (1.0f / 2147483648.0f), &s[e], &c[e]);
    }
  }
  float wq[8], wk[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const int at = e < 4 ? at0 + e : at1 + e - 4;
    wq[e] = hq && d.q_norm && in_head ? load_norm(d.q_norm, d.norm_dtype, at) : 1.0f;
    wk[e] = hk && d.k_norm && in_head ? load_norm(d.k_norm, d.norm_dtype, at) : 1.0f;
  }
  const bool norms = (hq && d.q_norm) || (hk && d.k_norm);

  for (int h1 = h0; h1 - slot < h_end; h1 += kAhead * slots) {
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int h = h1 + i * slots;
      if (h - slot >= h_end) break;
      const bool is_q = h < hq, is_k = !is_q && h < hq + hk;
      float(&a)[4] = x0[i], (&b)[4] = x1[i];
      if (norms) {
        auto squares = [&]() {
          float r = 0.0f;
#pragma unroll
          for (int e = 0; e < 4; ++e) r += a[e] * a[e] + b[e] * b[e];
          for (int o = 1 << P.width_log2 >> 1; o; o >>= 1) r += __shfl_xor_sync(0xffffffffu, r, o);
          return r;
        };
        const bool normed = (is_q && d.q_norm) || (is_k && d.k_norm);
        float ss = squares(), eps = d.eps;
        // Squares of fp32 numbers can pass its range; such heads are scaled by a power of two first.
        const bool large = normed && ss > 1e37f, small = normed && ss < 1e-30f && eps < 1e-20f;
        if (__any_sync(0xffffffffu, large || small)) {
          const float f = large ? 0x1p-96f : small ? 0x1p96f : 1.0f;
#pragma unroll
          for (int e = 0; e < 4; ++e) a[e] *= f, b[e] *= f;
          ss = squares();
          eps = eps * f * f;
        }
        if (normed) {
          const float r = rsqrtf(ss * P.inv_dim + eps);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            a[e] *= r * (is_q ? wq[e] : wk[e]);
            b[e] *= r * (is_q ? wq[4 + e] : wk[4 + e]);
          }
        }
      }
      if (turned && (is_q || is_k)) {
        if (halves) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float y0 = a[e], y1 = b[e];
            a[e] = y0 * c[e] - y1 * s[e];
            b[e] = y1 * c[e] + y0 * s[e];
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; e += 2) {
            const int j = e / 2;
            const float y0 = a[e], y1 = a[e + 1], z0 = b[e], z1 = b[e + 1];
            a[e] = y0 * c[j] - y1 * s[j];
            a[e + 1] = y1 * c[j] + y0 * s[j];
            b[e] = z0 * c[2 + j] - z1 * s[2 + j];
            b[e + 1] = z1 * c[2 + j] + z0 * s[2 + j];
          }
        }
      }
      if (in_head && h < h_end) {
        if (is_q) {
          const int64_t to = (int64_t)t * d.out_stride + (int64_t)h * D;
          store4<DT>(d.q_out, to + at0, a);
          store4<DT>(d.q_out, to + at1, b);
        } else if (cached) {
          void *pages = is_k ? d.k_pages : d.v_pages;
          const int64_t to = (row + (is_k ? h - hq : h - hq - hk)) * D;
          store4<DT>(pages, to + at0, a);
          store4<DT>(pages, to + at1, b);
        }
      }
      fetch(h + kAhead * slots, a, b);
    }
  }
}

template <int IN, int DT>
cudaError_t run(const PlacePlan &P, unsigned grid, cudaStream_t s) {
  place_kernel<IN, DT><<<grid, kThreads, 0, s>>>(P);
  return cudaGetLastError();
}

}  // namespace

bool plan_place(PlacePlan *P) {
  const wt_place_desc &d = P->d;
  P->width_log2 = 0;
  while (8 << P->width_log2 < d.head_dim) ++P->width_log2;
  P->inv_dim = 1.0f / (float)d.head_dim;
  const int slots = 32 >> P->width_log2;
  const int64_t all = (int64_t)(d.q ? d.heads : 0) + (d.k ? d.kv_heads : 0) + (d.v ? d.kv_heads : 0);
  // A warp takes all of a token's heads where that gives every SM 32 warps, and fewer where it does not.
  const int64_t rounds = (all + slots - 1) / slots, want = 32ll * num_sms();
  const int64_t per = std::min(rounds, std::max<int64_t>(1, rounds * d.n_tokens / want));
  P->chunk_heads = (int)(per * slots);
  P->chunks = (int)((all + P->chunk_heads - 1) / P->chunk_heads);
  return (int64_t)d.n_tokens * P->chunks <= 0x7fffffffll * (kThreads / 32);
}

cudaError_t launch_place(const PlacePlan &P, cudaStream_t s) {
  const wt_place_desc &d = P.d;
  const unsigned grid = (unsigned)(((int64_t)d.n_tokens * P.chunks + kThreads / 32 - 1) / (kThreads / 32));
  if (d.dtype == WT_BF16) return d.in_dtype == WT_F32 ? run<WT_F32, WT_BF16>(P, grid, s) : run<WT_BF16, WT_BF16>(P, grid, s);
  return d.in_dtype == WT_F32 ? run<WT_F32, WT_F16>(P, grid, s) : run<WT_F16, WT_F16>(P, grid, s);
}

}  // namespace wt
