// Norms, rotation and placing of a step's queries, keys and values (include/wt_serve.h).
//
// A head's elements are taken in units of 8 that hold whole pairs (two runs of four elements: j .. j + 3
// and rot_dim / 2 further on, or eight neighbours), one unit a lane, so a rotation needs no other lane
// and the norm's sum of squares one exchange among the lanes of a head (any number of them: 30 lanes hold three
// heads of 80).  A CTA takes heads of q, k and v of one token.  All its loads are on their way before anything
// waits for one; meanwhile the token's request and page are found, and the angle of each pair is worked out once,
// by one thread, for all heads.
//
// The angle is exact modulo a turn: pos * turns wraps at 2^64 as the angle does at a turn, and the top 32
// bits of the product, as a signed number, are the fraction in [-1/2, 1/2) that sincospif takes.
#include <algorithm>
#include <type_traits>

#include "wt_serve.cuh"

namespace wt {

namespace {

constexpr int kWarps = 4;
constexpr int kThreads = 32 * kWarps;
// Heads of a lane whose loads are in flight together.  Eight CTAs to an SM, or seven with 16-bit rows: registers
// for the loads of four heads a lane.  (One GB300: 9350 tokens of 96 heads of 80 from fp32 69.7 us, 6.2 TB/s; with
// loops over a token's heads in one warp and the angles in registers 101.  CTAs of 8 warps take the same for fp32
// and 39.7 against 33.0 us for 4400 tokens of 60 heads of 128 in 16 bits, as every warp finds its request.)
constexpr int kDepth = 4;
template <int IN>
constexpr int kResident = IN == WT_F32 ? 8 : 7;

__device__ __forceinline__ void note_invalid(int *status) {
  if (status) atomicCAS(status, 0, kStatusInvalid);
}

// A run of N elements of type DT as they lie in memory, and as fp32.
template <int DT, int N>
struct Raw {
  static constexpr int kWords = DT == WT_F32 ? N : N / 2;
  uint32_t w[kWords];
  __device__ __forceinline__ void load(const void *p, int64_t at) {
    const uint8_t *src = static_cast<const uint8_t *>(p) + at * (DT == WT_F32 ? 4 : 2);
    if constexpr (kWords == 2) {
      const uint2 v = *reinterpret_cast<const uint2 *>(src);
      w[0] = v.x, w[1] = v.y;
    } else {
#pragma unroll
      for (int i = 0; i < kWords; i += 4) {
        const uint4 v = *reinterpret_cast<const uint4 *>(src + 4 * i);
        w[i] = v.x, w[i + 1] = v.y, w[i + 2] = v.z, w[i + 3] = v.w;
      }
    }
  }
  __device__ __forceinline__ void widen(float (&x)[N]) const {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if constexpr (DT == WT_F32) x[i] = __uint_as_float(w[i]);
      else if (i % 2 == 0) unpack2<DT>(w[i / 2], x[i], x[i + 1]);
  }
};
template <int DT, int N>
__device__ __forceinline__ void store_run(void *p, int64_t at, const float (&x)[N]) {
  uint32_t w[N / 2];
#pragma unroll
  for (int i = 0; i < N / 2; ++i) w[i] = pack2<DT>(x[2 * i], x[2 * i + 1]);
  uint16_t *dst = static_cast<uint16_t *>(p) + at;
  if constexpr (N == 4) *reinterpret_cast<uint2 *>(dst) = make_uint2(w[0], w[1]);
  else *reinterpret_cast<uint4 *>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
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

// W: elements of a unit.
template <int IN, int DT, int W>
__global__ void __launch_bounds__(kThreads, kResident<IN>) place_kernel(const __grid_constant__ PlacePlan P) {
  __shared__ __align__(16) float cosines[WT_PLACE_MAX_DIM / 2], sines[WT_PLACE_MAX_DIM / 2];
  __shared__ __align__(16) float weights[2][WT_PLACE_MAX_DIM];  // of q, of k
  const wt_place_desc &d = P.d;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, t = blockIdx.x;
  const int D = d.head_dim, half = d.rot_dim / 2;

  // this lane's unit of a head, and which of the heads that the warp takes together
  constexpr int R = W / 2;  // of a run
  const int units = D / W, slots = 32 / units, slot = lane / units, u = lane - slot * units;
  const bool in_head = slot < slots, turned = in_head && u * W < d.rot_dim;
  const bool halves = turned && !(d.flags & WT_PLACE_NEIGHBOURS);
  const int at0 = halves ? u * R : u * W, at1 = halves ? half + u * R : u * W + R;

  // heads of q, k and v in a row; a warp takes `slots` of them at a time, P.rounds times
  const int hq = d.q ? d.heads : 0, hk = d.k ? d.kv_heads : 0, hv = d.v ? d.kv_heads : 0, all = hq + hk + hv;
  const int h0 = (blockIdx.y * P.rounds * kWarps + warp) * slots + slot, step = kWarps * slots;
  Raw<IN, R> ra[kDepth] = {}, rb[kDepth] = {};
#pragma unroll
  for (int i = 0; i < kDepth; ++i) {
    const int h = h0 + i * step;
    if (i < P.rounds && h < all && in_head) {
      const void *src = h < hq ? d.q : h < hq + hk ? d.k : d.v;
      const int64_t row = h < hq ? (int64_t)t * d.q_stride + (int64_t)h * D
                          : h < hq + hk ? (int64_t)t * d.k_stride + (int64_t)(h - hq) * D
                                        : (int64_t)t * d.v_stride + (int64_t)(h - hq - hk) * D;
      ra[i].load(src, row + at0);
      rb[i].load(src, row + at1);
    }
  }
  // what hangs on nothing else is asked for first
  int64_t own_pos = 0;
  uint64_t turn = 0;
  if (tid < half) {
    if (d.pos) own_pos = __ldg(d.pos + (int64_t)t * d.pos_stride + d.axis[tid]);
    turn = __ldg(reinterpret_cast<const unsigned long long *>(d.turns) + tid);
  }
  const bool norms = (hq && d.q_norm) || (hk && d.k_norm);
  constexpr int kNorm = (WT_PLACE_MAX_DIM + kThreads - 1) / kThreads;
  float w_q[kNorm], w_k[kNorm];
#pragma unroll
  for (int i = 0; i < kNorm; ++i) {
    const int at = tid + i * kThreads;
    w_q[i] = norms && d.q_norm && at < D ? load_norm(d.q_norm, d.norm_dtype, at) : 0.0f;
    w_k[i] = norms && d.k_norm && at < D ? load_norm(d.k_norm, d.norm_dtype, at) : 0.0f;
  }
  if (d.begin && blockIdx.y == 0)  // every request's numbers are looked at by one thread
    for (int64_t b = (int64_t)blockIdx.x * kThreads + tid; b < d.n_req; b += (int64_t)gridDim.x * kThreads) {
      const int t0 = __ldg(d.begin + b), t1 = __ldg(d.begin + b + 1), len = d.len ? __ldg(d.len + b) : 0;
      if (t0 < 0 || t1 < t0 || t1 > d.n_tokens || (d.len && (len < t1 - t0 || len > d.max_len))) note_invalid(P.status);
    }

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
        if (!cached && tid == 0) note_invalid(P.status);
      }
    }
  }
  if (tid < half) {
    turn *= (uint64_t)(d.pos ? own_pos : (int64_t)d.first_pos + place);
    sincospif((float)(int32_t)(turn >> 32) * (1.0f / 2147483648.0f), &sines[tid], &cosines[tid]);
  }
  if (norms)
#pragma unroll
    for (int i = 0; i < kNorm; ++i) {
      const int at = tid + i * kThreads;
      if (at < D) weights[0][at] = w_q[i], weights[1][at] = w_k[i];
    }
  if (half || norms) __syncthreads();
#pragma unroll
  for (int i = 0; i < kDepth; ++i) {
    const int h = h0 + i * step;
    if (i >= P.rounds || h - slot >= all) break;
    const bool is_q = h < hq, is_k = !is_q && h < hq + hk;
    float a[R], b[R];
    ra[i].widen(a);
    rb[i].widen(b);
    {
      if (norms) {
        auto squares = [&]() {  // of the head: into its first lane, and back
          float r = 0.0f;
#pragma unroll
          for (int e = 0; e < R; ++e) r += a[e] * a[e] + b[e] * b[e];
#pragma unroll
          for (int o = 16; o; o >>= 1) {
            const float x = __shfl_down_sync(0xffffffffu, r, o);
            if (u + o < units) r += x;  // no lane's where o is not below units
          }
          return __shfl_sync(0xffffffffu, r, slot * units & 31);
        };
        const bool normed = in_head && ((is_q && d.q_norm) || (is_k && d.k_norm));
        float ss = squares(), eps = d.eps;
        // Squares of fp32 numbers can pass its range; such heads are scaled by a power of two first.
        const bool large = normed && ss > 1e37f, small = normed && ss < 1e-30f && eps < 1e-20f;
        if (__any_sync(0xffffffffu, large || small)) {
          const float f = large ? 0x1p-96f : small ? 0x1p96f : 1.0f;
#pragma unroll
          for (int e = 0; e < R; ++e) a[e] *= f, b[e] *= f;
          ss = squares();
          eps = eps * f * f;
        }
        if (normed) {
          const float r = rsqrtf(ss * P.inv_dim + eps);
          const float *w = weights[is_k];
#pragma unroll
          for (int e = 0; e < R; ++e) {
            a[e] *= r * w[at0 + e];
            b[e] *= r * w[at1 + e];
          }
        }
      }
      if (turned && (is_q || is_k)) {
        const float *c = cosines + u * R, *s = sines + u * R;
        if (halves) {
#pragma unroll
          for (int e = 0; e < R; ++e) {
            const float y0 = a[e], y1 = b[e];
            a[e] = y0 * c[e] - y1 * s[e];
            b[e] = y1 * c[e] + y0 * s[e];
          }
        } else {
#pragma unroll
          for (int e = 0; e < R; e += 2) {
            const int j = e / 2;
            const float y0 = a[e], y1 = a[e + 1], z0 = b[e], z1 = b[e + 1];
            a[e] = y0 * c[j] - y1 * s[j];
            a[e + 1] = y1 * c[j] + y0 * s[j];
            b[e] = z0 * c[R / 2 + j] - z1 * s[R / 2 + j];
            b[e + 1] = z1 * c[R / 2 + j] + z0 * s[R / 2 + j];
          }
        }
      }
      if (in_head && h < all) {
        if (is_q) {
          const int64_t to = (int64_t)t * d.out_stride + (int64_t)h * D;
          store_run<DT>(d.q_out, to + at0, a);
          store_run<DT>(d.q_out, to + at1, b);
        } else if (cached) {
          void *pages = is_k ? d.k_pages : d.v_pages;
          const int64_t to = (row + (is_k ? h - hq : h - hq - hk)) * D;
          store_run<DT>(pages, to + at0, a);
          store_run<DT>(pages, to + at1, b);
        }
      }
    }
  }
}

template <int IN, int DT, int W>
cudaError_t run(const PlacePlan &P, dim3 grid, cudaStream_t s) {
  place_kernel<IN, DT, W><<<grid, kThreads, 0, s>>>(P);
  return cudaGetLastError();
}

template <int DT>
cudaError_t run_type(const PlacePlan &P, dim3 grid, cudaStream_t s) {
  if (P.d.in_dtype == WT_F32) return run<WT_F32, DT, 8>(P, grid, s);
  return P.unit == 16 ? run<DT, DT, 16>(P, grid, s) : run<DT, DT, 8>(P, grid, s);
}

}  // namespace

void plan_place(PlacePlan *P) {
  const wt_place_desc &d = P->d;
  P->inv_dim = 1.0f / (float)d.head_dim;
  // 16-byte vectors of 16-bit rows, where a unit of two of them holds whole pairs
  P->unit = d.in_dtype != WT_F32 && d.head_dim % 16 == 0 && d.rot_dim % 16 == 0 ? 16 : 8;
  const int slots = 32 * P->unit / d.head_dim;
  const int64_t all = (int64_t)(d.q ? d.heads : 0) + (d.k ? d.kv_heads : 0) + (d.v ? d.kv_heads : 0);
  // A CTA takes as many of a token's heads as its loads in flight allow, and fewer where that would leave SMs
  // without three of them.
  const int64_t parts = (all + kWarps * slots - 1) / (kWarps * slots), ctas = 3ll * num_sms();
  const int64_t chunks = std::max((parts + kDepth - 1) / kDepth, std::min(parts, (ctas + d.n_tokens - 1) / d.n_tokens));
  P->rounds = (int)((parts + chunks - 1) / chunks);
  P->chunks = (int)((parts + P->rounds - 1) / P->rounds);
}

cudaError_t launch_place(const PlacePlan &P, cudaStream_t s) {
  const dim3 grid((unsigned)P.d.n_tokens, (unsigned)P.chunks);
  return P.d.dtype == WT_BF16 ? run_type<WT_BF16>(P, grid, s) : run_type<WT_F16>(P, grid, s);
}

}  // namespace wt
