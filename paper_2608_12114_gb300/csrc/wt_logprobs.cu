// Log probabilities, entropy and the likeliest tokens of logits rows (include/wt_serve.h).
//
// One reading of all rows.  Per row, with x = (l - m) log2(e) / t for the largest logit m:
//
//   s = sum over all but one of the largest of 2^x,      log S = log1p(s)
//   w = sum of x 2^x,                                    H = log1p(s) - ln 2 w / (1 + s)
//
// The largest logit's own 1 stays out of s, so that a sharp row keeps its entropy and its likeliest token's
// log probability to fp32's precision: nothing is subtracted.  A thread keeps four largest logits, of every
// fourth that it sees, out of its sums: of a new logit and the one kept, the smaller goes in.  Its sums are against
// a reference of its warp, the first largest logit, which moves when one is 2^8 above it (the
// move of w to another reference loses that many roundings of s).  At the end all of the
// kept ones but one go in, too.  Two parts, m1 >= m2, join as s1 + f (s2 + 1) and w1 + f (w2 + d (s2 + 1)),
// d = (m2 - m1) log2(e) / t, f = 2^d: warps and CTAs in a fixed order.  (With the thread's one largest logit as its
// reference, which half the time moved in one lane of a warp or another, the kernel was bound by its
// instructions: 2047 rows of 50021 logits took 97 us, and 67 this way, 6.1 TB/s.)
//
// The rows' 16-byte vectors, one row after another, are cut into equal shares, one a CTA, so that no number of
// rows leaves SMs idle.  A row that one CTA has whole is answered there; the parts of others go to the workspace,
// and a second kernel joins them.
//
// Alternatives: what lies under the n_top-th largest of several disjoint groups' maxima is not among the row's
// n_top, whatever the timing; so 128 groups of two of four threads' kept logits tell the CTA's warps where to look,
// from the first 4096 logits on and better after 2, 4, 8, ... times as many: some n_top / i random logits of the
// i-th 4096 are taken up.  At the end each of them counts those above it, which is its place: many comparisons
// at once, where sorting is a chain of them; where they are many, those under such a bound of their own leave
// first.  A warp that takes up more than its room sorts 32 and joins them to a list of its own: the larger of each
// and its opposite, sorted in five exchanges.
#include <algorithm>

#include "wt_serve.cuh"

namespace wt {

namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kResident = 4;  // CTAs to an SM
// Up to so many CTAs to an SM, of four turns or more each, load a turn ahead, in registers: 257 rows of 128256 with
// twenty alternatives, a row a CTA, 35.6 us against 44.0.  (More of them load beside one another's work as it is, and
// bulk copies into rings were slower: 57.)
constexpr int kFew = 3;
constexpr int kVecs = 4;      // 16-byte vectors of a lane at a time
constexpr int kTurn = kThreads * kVecs;  // vectors that a CTA takes at a time
constexpr int kTop = WT_LOGPROBS_MAX_TOP;
constexpr int kGroups = 128;
constexpr int kRoom = 3 * kTop;   // of a warp: it joins 32 to its list from 2 kTop on
constexpr int kDirect = 160;      // so many are placed as they are
constexpr float kGrow = 8.0f;     // in log2
static_assert(kTop == 32, "one candidate a lane");
static_assert(kGroups == kThreads / 2 && kGroups >= kTop, "two groups of four threads, enough of them");

typedef unsigned long long Key;  // order of the logit, then ~token: the larger comes first; 0: none

__device__ __forceinline__ uint32_t order_of(float v) {
  const uint32_t b = __float_as_uint(v + 0.0f);  // -0 is 0
  return b ^ (b >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ __forceinline__ float logit_of(uint32_t o) { return __uint_as_float(o ^ (o >> 31 ? 0x80000000u : 0xffffffffu)); }
__device__ __forceinline__ Key key_of(float v, int token) { return (Key)order_of(v) << 32 | (uint32_t)~token; }

struct Sums {
  float m;    // largest logit
  int first;  // its first token
  float s, w;
};

// d = (m2 - m1) k stays above -200, where 2^d is 0 and d times it, too
__device__ __forceinline__ Sums join(const Sums &a, const Sums &b, float k) {
  const bool ab = a.m > b.m || (a.m == b.m && a.first < b.first) || !(b.m > -INFINITY);
  const Sums &x = ab ? a : b, &y = ab ? b : a;
  const bool some = y.m > -INFINITY;
  const float d = some ? fmaxf((y.m - x.m) * k, -200.0f) : -200.0f, f = exp2_approx(d), n = y.s + 1.0f;
  return {x.m, x.first, x.s + f * n, x.w + f * (y.w + d * n)};
}

__device__ __forceinline__ Sums shuffle(const Sums &a, int o) {
  return {__shfl_xor_sync(0xffffffffu, a.m, o), __shfl_xor_sync(0xffffffffu, a.first, o), __shfl_xor_sync(0xffffffffu, a.s, o),
          __shfl_xor_sync(0xffffffffu, a.w, o)};
}

__device__ __forceinline__ float min_or_nan(float a, float b) {
  float r;
  asm("min.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// (x0, x1) * k, and (w0, w1) + (p0, p1) * (x0, x1), in one instruction each.
__device__ __forceinline__ void mul_x2(float &x0, float &x1, float k) {
  asm("{\n\t.reg .b64 x, y;\n\tmov.b64 x, {%0, %1};\n\tmov.b64 y, {%2, %2};\n\tmul.rn.f32x2 x, x, y;\n\tmov.b64 {%0, %1}, x;\n\t}"
      : "+f"(x0), "+f"(x1)
      : "f"(k));
}
__device__ __forceinline__ void fma_x2(float &w0, float &w1, float p0, float p1, float x0, float x1) {
  asm("{\n\t.reg .b64 w, p, x;\n\tmov.b64 w, {%0, %1};\n\tmov.b64 p, {%2, %3};\n\tmov.b64 x, {%4, %5};\n\t"
      "fma.rn.f32x2 w, p, x, w;\n\tmov.b64 {%0, %1}, w;\n\t}"
      : "+f"(w0), "+f"(w1)
      : "f"(p0), "f"(p1), "f"(x0), "f"(x1));
}

// The 32 largest of two ordered lists, in order.
__device__ __noinline__ Key merged(Key mine, Key other, int lane) {
  const Key opposite = __shfl_sync(0xffffffffu, other, 31 - lane);
  mine = mine > opposite ? mine : opposite;
#pragma unroll 1
  for (int o = 16; o; o >>= 1) {
    const Key x = __shfl_xor_sync(0xffffffffu, mine, o);
    mine = ((lane & o) == 0) == (mine > x) ? mine : x;
  }
  return mine;
}

// 32 keys in order, the largest first.
__device__ __noinline__ Key sorted(Key mine, int lane) {
#pragma unroll 1
  for (int n = 2; n <= 32; n *= 2)
#pragma unroll 1
    for (int o = n / 2; o; o >>= 1) {
      const Key x = __shfl_xor_sync(0xffffffffu, mine, o);
      const bool larger = ((lane & o) == 0) == ((lane & n) == 0);
      mine = larger == (mine > x) ? mine : x;
    }
  return mine;
}

// At most the n-th largest of the groups' maxima, and within 2^-12 of their range of it: by one warp, halving the
// range (counting what is above each of them kept the warp, and those that wait for it, four times as long).  Other
// warps may write larger ones meanwhile.
__device__ __noinline__ unsigned bound_of(const volatile unsigned *maxima, int n, int lane) {
  unsigned m[kGroups / 32], lo = ~0u, hi = 0;
#pragma unroll
  for (int i = 0; i < kGroups / 32; ++i) m[i] = maxima[i * 32 + lane], lo = min(lo, m[i]), hi = max(hi, m[i]);
  lo = __reduce_min_sync(0xffffffffu, lo), hi = __reduce_max_sync(0xffffffffu, hi);
#pragma unroll 2
  for (int i = 0; i < 12; ++i) {
    const unsigned mid = lo + (hi - lo + 1) / 2;
    int some = 0;
#pragma unroll
    for (int q = 0; q < kGroups / 32; ++q) some += __popc(__ballot_sync(0xffffffffu, m[q] >= mid));
    if (some >= n) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// The n-th largest, by a block of two threads to a group, into *low (~0 before).  Ends with a barrier.
__device__ __forceinline__ void block_bound(const unsigned *maxima, int n, unsigned *low) {
  const int tid = threadIdx.x;
  const unsigned mine = maxima[tid / 2];
  int above = 0;
#pragma unroll
  for (int i = 0; i < kGroups / 2; i += 4) {
    const uint4 x = *reinterpret_cast<const uint4 *>(maxima + tid % 2 * (kGroups / 2) + i);
    above += (x.x > mine) + (x.y > mine) + (x.z > mine) + (x.w > mine);
  }
  above += __shfl_xor_sync(0xffffffffu, above, 1);
  const unsigned least = __reduce_min_sync(0xffffffffu, above < n ? mine : ~0u);
  if (tid % 32 == 0) atomicMin(low, least);
  __syncthreads();
}

struct Choice {
  __align__(16) unsigned maxima[kGroups];
  unsigned low;
  int n;
};
// put(place, key) for the n_top largest of n different keys in shared memory (0: none, may stand there often, goes
// last); by a block of kThreads, which all come here together.  `room` holds n keys.
template <typename F>
__device__ __forceinline__ void place(const Key *keys, int n, int n_top, Key *room, Choice *c, F put) {
  const int tid = threadIdx.x;
  if (n > kDirect) {
    unsigned most = 0;
    for (int i = tid; i < n; i += kThreads) most = max(most, (unsigned)(keys[i] >> 32));
    most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
    if (tid % 2 == 0) c->maxima[tid / 2] = most;
    if (tid == 0) c->low = ~0u, c->n = 0;
    __syncthreads();
    block_bound(c->maxima, n_top, &c->low);
    const unsigned low = max(c->low, 1u);
    for (int i = tid; i < n; i += kThreads) {
      const Key x = keys[i];
      if ((unsigned)(x >> 32) >= low) room[atomicAdd(&c->n, 1)] = x;
    }
    __syncthreads();
    keys = room, n = c->n;
  }
  for (int i = tid; i < n; i += kThreads) {
    const Key mine = keys[i];
    int above = 0;
#pragma unroll 8
    for (int j = 0; j < n; ++j) above += keys[j] > mine;
    if (mine && above < n_top) put(above, mine);
  }
  // places that no key has
  int some = 0;
  for (int i = tid % 32; i < n; i += 32) some += keys[i] != 0;
  some = (int)__reduce_add_sync(0xffffffffu, (unsigned)some);
  for (int i = some + tid; i < n_top; i += kThreads) put(i, 0);
}

// What a row's sums answer.
struct Answer {
  const wt_logprobs_desc &d;
  int row;
  const float *l;
  Sums a;
  float t, log_s;
  bool draw, bad, none;
  __device__ Answer(const wt_logprobs_desc &desc, int r, const Sums &sums, float temp)
      : d(desc), row(r), l(desc.logits + (int64_t)r * desc.ldl), a(sums), t(temp), log_s(log1pf(sums.s)), draw(temp > 0.0f),
        bad(draw && (sums.m == INFINITY || sums.s != sums.s)), none(!(sums.m > -INFINITY)) {}
  __device__ float logp(float x, int token) const {
    if (bad) return NAN;
    if (none || !(x > -INFINITY)) return -INFINITY;
    if (!draw) return token == a.first ? 0.0f : -INFINITY;
    return (x - a.m) / t - log_s;
  }
  // by a warp
  __device__ void write(int i, int *status) const {
    const int token = i < d.n_given ? d.given[(int64_t)row * d.given_stride + i] : -1;
    write(i, token, token >= 0 && token < d.vocab ? l[token] : 0.0f, status);
  }
  // whose first 32 given tokens and their logits are in hand
  __device__ void write(int i, int token, float logit, int *status) const {
    if (i == 0 && d.entropy) d.entropy[row] = bad ? NAN : none || !draw ? 0.0f : log_s - 0.69314718055994531f * a.w / (1.0f + a.s);
    for (int g = i; g < d.n_given; g += 32) {
      if (g >= 32) {
        token = d.given[(int64_t)row * d.given_stride + g];
        if (token >= 0 && token < d.vocab) logit = l[token];
      }
      if (token >= d.vocab && status) atomicCAS(status, 0, kStatusInvalid);
      d.given_lp[(int64_t)row * d.n_given + g] = token >= 0 && token < d.vocab ? logp(logit, token) : 0.0f;
    }
  }
  __device__ void write_top(int at, Key key) const {
    if (at >= d.n_top) return;
    const int token = (int)~(uint32_t)key;
    d.top[(int64_t)row * d.n_top + at] = key ? token : -1;
    d.top_lp[(int64_t)row * d.n_top + at] = key ? logp(logit_of((uint32_t)(key >> 32)), token) : bad ? NAN : -INFINITY;
  }
};

// Beyond the largest number any factor sends every logit but the largest to 0, and one above 0 a logit of
// -infinity, whatever the temperature.
__device__ __forceinline__ float factor_of(float t) { return t > 0.0f ? fmaxf(fminf(1.4426950408889634f / t, 3.4028234e38f), 1.1754944e-38f) : 1.0f; }

// AHEAD: the next turn's vectors are on their way while one is worked on.
template <bool TOP, bool AHEAD>
__global__ void __launch_bounds__(kThreads, AHEAD ? kFew : kResident) logprobs_kernel(const __grid_constant__ LogprobsPlan P) {
  __shared__ Sums warp_sums[kWarps], row_sums;
  __shared__ Choice choice;
  __shared__ unsigned floor_order, first_bound;
  __shared__ __align__(16) Key taken[TOP ? kWarps : 1][kRoom];  // up by each warp
  __shared__ __align__(16) Key candidates[TOP ? kWarps * kRoom : 1];
  unsigned *const maxima = choice.maxima;
  __shared__ int counts[kWarps];
  const wt_logprobs_desc &d = P.d;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const long long begin = P.per * blockIdx.x, end = min((long long)d.rows * P.row_vecs, begin + P.per);
  griddep_launch();  // what joins rows may start its first loads
  for (long long at = begin; at < end;) {
    const int row = (int)quotient(at, P.row_vecs);
    const long long row0 = (long long)row * P.row_vecs;
    const int lo = (int)(at - row0), hi = (int)(min(end, row0 + P.row_vecs) - row0);
    const bool whole = lo == 0 && hi == P.row_vecs;
    const long long slot = 2 * blockIdx.x + (lo == 0 && at > begin);
    at = row0 + hi;
    const float *l = d.logits + (int64_t)row * d.ldl;
    const float t = d.temp ? d.temp[row] : 1.0f, k = factor_of(t);
    // The row's vectors start at the 16-byte boundary at or before it: `off` elements of the first are not its.
    const int off = (int)(reinterpret_cast<uintptr_t>(l) / 4 % 4);
    if (TOP) {
      __syncthreads();  // the last row's lists have been read
      if (tid == 0) floor_order = 0, first_bound = ~0u;
    }
    float kept[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, ref = -INFINITY;
    float s[2] = {0.0f, 0.0f}, w[2] = {0.0f, 0.0f};
    int first = INT32_MAX;         // a greedy row's: the first of the thread's largest logits
    Key list = 0;
    int n_taken = 0;
    // A candidate is at least `least` (neither NaN nor -infinity) and above `tie`, which n_top of the warp's logits
    // of earlier turns, so of lower tokens, are at least.
    float least = -3.4028234e38f, tie = -INFINITY;
    const bool greedy = !(t > 0.0f);
    auto load = [&](float (&v)[kVecs][4], int j0) {
      const int j1 = j0 + tid, e1 = 4 * j1 - off;  // and every kThreads-th vector from there
      if (j0 > 0 && j0 + kTurn <= hi && 4 * (j0 + kTurn) - off <= d.vocab) {  // all of them are the row's
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
          const float4 x = __ldcs(reinterpret_cast<const float4 *>(l + e1) + i * kThreads);
          v[i][0] = x.x, v[i][1] = x.y, v[i][2] = x.z, v[i][3] = x.w;
        }
      } else {
#pragma unroll
        for (int i = 0; i < kVecs; ++i) {
          const int j = j1 + i * kThreads, e0 = 4 * j - off;
          if (j < hi && e0 >= 0 && e0 + 4 <= d.vocab) {
            const float4 x = __ldcs(reinterpret_cast<const float4 *>(l + e0));
            v[i][0] = x.x, v[i][1] = x.y, v[i][2] = x.z, v[i][3] = x.w;
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[i][e] = j < hi && e0 + e >= 0 && e0 + e < d.vocab ? __ldcs(l + e0 + e) : -INFINITY;
          }
        }
      }
    };
    float ahead[kVecs][4];
    if (AHEAD) load(ahead, lo);
    for (int j0 = lo; j0 < hi; j0 += kTurn) {
      float v[kVecs][4];
      if (AHEAD) {
#pragma unroll
        for (int i = 0; i < kVecs; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) v[i][e] = ahead[i][e];
        if (j0 + kTurn < hi) load(ahead, j0 + kTurn);
      } else {
        load(v, j0);
      }
      const int e1 = 4 * (j0 + tid) - off;  // token of v[0][0]
      float top = -INFINITY;
#pragma unroll
      for (int i = 0; i < kVecs; ++i) top = fmaxf(top, fmaxf(fmaxf(v[i][0], v[i][1]), fmaxf(v[i][2], v[i][3])));
      if (__any_sync(0xffffffffu, (top - ref) * k > kGrow)) {
        float to = top;
#pragma unroll
        for (int o = 16; o; o >>= 1) to = fmaxf(to, __shfl_xor_sync(0xffffffffu, to, o));
        const float by = fmaxf((ref - to) * k, -200.0f), f = exp2_approx(by);
#pragma unroll
        for (int i = 0; i < 2; ++i) w[i] = f * (w[i] + by * s[i]), s[i] *= f;
        ref = to;
      }
      if (greedy && top > fmaxf(fmaxf(kept[0], kept[1]), fmaxf(kept[2], kept[3]))) {
#pragma unroll
        for (int i = kVecs - 1; i >= 0; --i)
#pragma unroll
          for (int e = 3; e >= 0; --e)
            if (v[i][e] == top) first = e1 + i * (4 * kThreads) + e;
      }
      const float z = ref > -INFINITY ? ref : 0.0f;
#pragma unroll
      for (int i = 0; i < kVecs; ++i)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          float x0 = min_or_nan(v[i][e], kept[e]), x1 = min_or_nan(v[i][e + 1], kept[e + 1]);
          kept[e] = fmaxf(kept[e], v[i][e]);
          kept[e + 1] = fmaxf(kept[e + 1], v[i][e + 1]);
          sub_x2(x0, x1, x0, x1, z, z);
          mul_x2(x0, x1, k);
          const float p0 = exp2_approx(x0), p1 = exp2_approx(x1);
          add_x2(s[0], s[1], p0, p1);
          fma_x2(w[0], w[1], p0, p1, fmaxf(x0, -200.0f), fmaxf(x1, -200.0f));  // 0 where p is
        }

      if (TOP) {
        const int turn = (j0 - lo) / kTurn;
        if ((turn & (turn + 1)) == 0) {  // the groups' largest so far
          float most0 = fmaxf(kept[0], kept[1]), most1 = fmaxf(kept[2], kept[3]);
          most0 = fmaxf(most0, __shfl_xor_sync(0xffffffffu, most0, 1));
          most1 = fmaxf(most1, __shfl_xor_sync(0xffffffffu, most1, 1));
          most0 = fmaxf(most0, __shfl_xor_sync(0xffffffffu, most0, 2));
          most1 = fmaxf(most1, __shfl_xor_sync(0xffffffffu, most1, 2));
          if (lane % 4 == 0) {
            reinterpret_cast<volatile unsigned *>(maxima)[tid / 4] = order_of(most0);
            reinterpret_cast<volatile unsigned *>(maxima)[kGroups / 2 + tid / 4] = order_of(most1);
          }
          if (turn == 0) {
            __syncthreads();
            block_bound(maxima, d.n_top, &first_bound);
            least = fmaxf(least, logit_of(first_bound));
          }
        } else if ((turn & (turn - 1)) == 0 && (__ffs(turn) + blockIdx.x) % kWarps == warp) {  // one of the warps looks
          const unsigned low = bound_of(maxima, d.n_top, lane);
          if (lane == 0) atomicMax(&floor_order, low);
          least = fmaxf(least, logit_of(low));
        }
        if (__any_sync(0xffffffffu, top >= least)) {
          least = fmaxf(least, logit_of(max(*reinterpret_cast<volatile unsigned *>(&floor_order), order_of(-3.4028234e38f))));
          unsigned mine = 0;  // this thread's to take up
#pragma unroll
          for (int i = 0; i < kVecs; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) mine |= v[i][e] >= least && v[i][e] > tie ? 1u << (i * 4 + e) : 0u;
          unsigned who;
          while ((who = __ballot_sync(0xffffffffu, mine != 0))) {
            const int which = __ffs(mine) - 1;
            float x = 0.0f;
#pragma unroll
            for (int i = 0; i < kVecs; ++i)
#pragma unroll
              for (int e = 0; e < 4; ++e) x = which == i * 4 + e ? v[i][e] : x;
            if (mine) taken[warp][n_taken + __popc(who & ((1u << lane) - 1))] = key_of(x, e1 + (which >> 2) * (4 * kThreads) + (which & 3));
            mine &= mine - 1;
            n_taken += __popc(who);
            while (n_taken >= 2 * kTop) {
              __syncwarp();
              list = merged(list, sorted(taken[warp][lane], lane), lane);
              n_taken -= kTop;
              const Key x0 = taken[warp][kTop + lane], x1 = taken[warp][2 * kTop + lane];
              __syncwarp();
              taken[warp][lane] = x0, taken[warp][kTop + lane] = x1;
            }
            __syncwarp();
          }
          const uint32_t o = (uint32_t)(__shfl_sync(0xffffffffu, list, d.n_top - 1) >> 32);
          if (o) {
            tie = logit_of(o);
            least = fmaxf(least, tie);
            if (lane == 0) atomicMax(&floor_order, o);
          }
        }
      }
    }

    // the warp's sums: all that its threads kept go in but one, a largest
    Sums a;
    {
      const float mine = fmaxf(fmaxf(kept[0], kept[1]), fmaxf(kept[2], kept[3]));
      float m = mine;
#pragma unroll
      for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
      const int out = __ffs(__ballot_sync(0xffffffffu, mine == m)) - 1;  // NaN is never kept
      const float z = ref > -INFINITY ? ref : 0.0f;
      bool left = lane != out;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool in = left || kept[e] != m;
        left |= !in;
        const float x = (kept[e] - z) * k, p = exp2_approx(x);
        if (in) s[0] += p, w[0] += p * fmaxf(x, -200.0f);
      }
      a.s = s[0] + s[1];
      a.w = w[0] + w[1];
      a.first = mine == m ? first : INT32_MAX;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        a.s += __shfl_xor_sync(0xffffffffu, a.s, o);
        a.w += __shfl_xor_sync(0xffffffffu, a.w, o);
      }
      a.first = __reduce_min_sync(0xffffffffu, a.first);
      a.m = m;
      // against m, which is not below the reference
      const float by = m > -INFINITY ? fmaxf((z - m) * k, -200.0f) : 0.0f, f = exp2_approx(by);
      a.w = f * (a.w + by * a.s);
      a.s *= f;
    }
    const bool flushed = __shfl_sync(0xffffffffu, list, 0) != 0;
    if (lane == 0) {
      warp_sums[warp] = a;
      counts[warp] = n_taken + (flushed ? d.n_top : 0);
    }
    __syncthreads();
    if (warp == 0) {
      a = warp_sums[lane & (kWarps - 1)];
#pragma unroll
      for (int o = 1; o < kWarps; o <<= 1) {
        const Sums b = shuffle(a, o);
        a = lane & o ? join(b, a, k) : join(a, b, k);
      }
      if (TOP && lane == 0) row_sums = a;
      if (whole) Answer(d, row, a, t).write(lane, P.status);
      else if (lane == 0) P.sums[slot] = make_float4(a.m, __int_as_float(a.first), a.s, a.w);
    }
    if (TOP) {
      int n = 0, to = 0;
#pragma unroll
      for (int i = 0; i < kWarps; ++i) {
        if (i == warp) to = n;
        n += counts[i];
      }
      for (int i = lane; i < n_taken; i += 32) candidates[to + i] = taken[warp][i];
      if (flushed && lane < d.n_top) candidates[to + n_taken + lane] = list;
      __syncthreads();
      Key *const room = taken[0];  // of no use any more
      if (whole) {
        const Answer r(d, row, row_sums, t);
        place(candidates, n, d.n_top, room, &choice, [&](int i, Key key) { r.write_top(i, key); });
      } else {
        place(candidates, n, d.n_top, room, &choice, [&](int i, Key key) { P.keys[slot * kTop + i] = key; });
      }
    } else {
      __syncthreads();  // warp_sums have been read
    }
  }
}

// The parts of rows that have more than one: a warp to a row, or a block with alternatives.
constexpr int kJoinParts = 24;  // whose alternatives are taken together
template <bool TOP>
__global__ void __launch_bounds__(kThreads) logprobs_join_kernel(const __grid_constant__ LogprobsPlan P) {
  __shared__ Sums row_sums;
  __shared__ Choice choice;
  __shared__ __align__(16) Key candidates[TOP ? (kJoinParts + 1) * kTop : 1], room[TOP ? (kJoinParts + 1) * kTop : 1], best[kTop];
  const wt_logprobs_desc &d = P.d;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long row = TOP ? blockIdx.x : (long long)blockIdx.x * kWarps + warp;
  if (row >= d.rows) return;
  const long long u0 = row * P.row_vecs, c0 = quotient(u0, P.per), c1 = quotient(u0 + P.row_vecs - 1, P.per);
  if (c0 == c1) return;  // one CTA had it whole
  const float t = d.temp ? d.temp[row] : 1.0f, k = factor_of(t);
  // the first given tokens' logits are on their way while the rest is joined
  const int token = lane < d.n_given ? d.given[row * d.given_stride + lane] : -1;
  const float logit = token >= 0 && token < d.vocab ? d.logits[row * d.ldl + token] : 0.0f;
  auto slot = [&](long long c) { return 2 * c + (c * P.per < u0); };
  griddep_wait();  // launched while the kernel before it ends
  if (!TOP || warp == 0) {
    Sums a = {-INFINITY, INT32_MAX, 0.0f, 0.0f};
    for (long long q0 = c0; q0 <= c1; q0 += 32) {
      Sums b = {-INFINITY, INT32_MAX, 0.0f, 0.0f};
      if (q0 + lane <= c1) {
        const float4 v = P.sums[slot(q0 + lane)];
        b = {v.x, __float_as_int(v.y), v.z, v.w};
      }
      const int n = (int)min(32ll, c1 - q0 + 1);
      for (int o = 1; o < n; o <<= 1) {
        const Sums x = shuffle(b, o);
        b = lane & o ? join(x, b, k) : join(b, x, k);
      }
      // lane 0 has them all
      b = {__shfl_sync(0xffffffffu, b.m, 0), __shfl_sync(0xffffffffu, b.first, 0), __shfl_sync(0xffffffffu, b.s, 0),
           __shfl_sync(0xffffffffu, b.w, 0)};
      a = q0 == c0 ? b : join(a, b, k);
    }
    if (lane == 0 && TOP) row_sums = a;
    Answer(d, (int)row, a, t).write(lane, token, logit, P.status);
  }
  if (TOP) {
    int before = 0;  // the best of the parts before
    for (long long q0 = c0; q0 <= c1; q0 += kJoinParts) {
      const int parts = (int)min((long long)kJoinParts, c1 - q0 + 1), n = before + parts * d.n_top;
      for (int i = tid; i < parts * d.n_top; i += kThreads) {
        const int q = i / d.n_top;
        candidates[before + i] = P.keys[slot(q0 + q) * kTop + (i - q * d.n_top)];
      }
      if (tid < before) candidates[tid] = best[tid];
      __syncthreads();
      if (q0 + kJoinParts > c1) {
        const Answer r(d, (int)row, row_sums, t);
        place(candidates, n, d.n_top, room, &choice, [&](int i, Key key) { r.write_top(i, key); });
      } else {
        place(candidates, n, d.n_top, room, &choice, [&](int i, Key key) { best[i] = key; });
        before = d.n_top;
        __syncthreads();
      }
    }
  }
}

}  // namespace

size_t plan_logprobs(LogprobsPlan *P) {
  const wt_logprobs_desc &d = P->d;
  // a row's vectors, wherever in a vector it starts
  P->row_vecs = (d.vocab + 6) / 4;
  const long long all = (long long)d.rows * P->row_vecs, ctas = (long long)kResident * num_sms();
  // Equal shares, of one turn of a CTA's threads at least, or whole rows, whichever takes less by this count, in
  // turns of SMs full of CTAs: a row that a CTA meets takes its turns and about two more, and parts of rows cost 12 more.
  // With alternatives parts cost 8, a share's turns half as much again, and turns of whole rows, which load ahead, less
  // where an SM has fewer CTAs.  (Shares against whole rows, us, with twenty alternatives: 40 rows of 128256 21.9, 24.4;
  // 60 24.3, 24.6; 80 27.1, 24.5; 128 33.0, 25.0; 200 42.4, 34.9; 254 46.5, 35.9; 257 46.0, 36.0; 300 53.6, 36.7; 620 81.7,
  // 89.1; 900 112.7, 92.9; 257 of 151936 50.7, 40.4; 20 of 50021 14.5, 15.1; 40 16.9, 15.5; 100 of 30000 20.4, 12.4; 10 of
  // 100000 with 32 16.6, 22.0.  Without: 128 of 128256 14.6, 12.7; 200 20.0, 24.9; 400 33.9, 32.3; 900 74.1, 72.3; 100 of
  // 30000 9.7, 5.5; 10 of 100000 6.4, 10.0.  On the wrong side: up to 10 rows of 50021 with twenty, 9 to 13 by shares and 15
  // as taken, one of 32000 8.6 and 11.4, and without alternatives what lies within 15 %.)
  const long long equal = std::max<long long>((all + ctas - 1) / ctas, kTurn), whole = (d.rows + ctas - 1) / ctas;
  const double met = 2.0 * equal / P->row_vecs, to_sm = std::min<double>(kResident, (d.rows + num_sms() - 1) / num_sms());
  const double by_shares = d.n_top ? 1.44 * equal / kTurn + met + 8.0 : (double)equal / kTurn + met + 12.0;
  const double by_rows = (double)whole * ((P->row_vecs + kTurn - 1) / kTurn + 2.0) * (d.n_top ? (1.0 + to_sm) / (1.0 + kResident) : 1.0);
  P->per = by_rows <= by_shares ? whole * P->row_vecs : equal;
  P->ctas = (int)((all + P->per - 1) / P->per);
  P->split = P->per % P->row_vecs != 0 && all > P->per;
  return P->split ? (size_t)P->ctas * 2 * (sizeof(float4) + (d.n_top ? kTop * sizeof(Key) : 0)) : 0;
}

cudaError_t launch_logprobs(const LogprobsPlan &P, cudaStream_t s) {
  const bool few = P.ctas <= kFew * num_sms() && P.per >= 4 * kTurn;
  if (P.d.n_top) (few ? logprobs_kernel<true, true> : logprobs_kernel<true, false>)<<<P.ctas, kThreads, 0, s>>>(P);
  else (few ? logprobs_kernel<false, true> : logprobs_kernel<false, false>)<<<P.ctas, kThreads, 0, s>>>(P);
  const cudaError_t e = cudaGetLastError();
  if (e != cudaSuccess || !P.split) return e;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(P.d.n_top ? P.d.rows : (P.d.rows + kWarps - 1) / kWarps));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, P.d.n_top ? logprobs_join_kernel<true> : logprobs_join_kernel<false>, P);
}

}  // namespace wt
