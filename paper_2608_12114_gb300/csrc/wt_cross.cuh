// What the kernels of attention to memories share (include/wt_serve.h): requests, and the cells of a CTA.
// Internal to the library (each translation unit gets its own copies).
#pragma once

#include "wt_serve.cuh"

namespace wt {
namespace {

// Tokens and memory of request b, clamped to the descriptor.
struct Asker {
  int t0, n;         // first token, tokens
  int mem, len;      // first state, states
  int row_tiles, key_tiles;
  int last;          // cells of the last row tile
  __device__ long long head_cells() const { return (row_tiles - 1ll) * key_tiles + last; }
  __device__ long long cells(const CrossPlan &P) const { return row_tiles ? head_cells() * P.groups : 0; }
};

__device__ __forceinline__ Asker asker_of(const CrossPlan &P, int b, bool tell) {
  const wt_cross_desc &d = P.d;
  int t0 = __ldg(d.begin + b), t1 = __ldg(d.begin + b + 1), mem = 0, len = 0;
  if (d.mem_len) mem = __ldg(d.mem_begin + b), len = __ldg(d.mem_len + b);
  if (t0 < 0 || t1 < t0 || t1 > d.n_tokens || t1 - t0 > d.max_new || mem < 0 || len < 0 || len > d.max_mem || mem + (int64_t)len > d.n_mem) {
    if (tell && P.status) atomicCAS(P.status, 0, kStatusInvalid);
    t0 = min(max(t0, 0), d.n_tokens);
    t1 = min(max(t1, t0), t0 + min(d.max_new, d.n_tokens - t0));
    mem = min(max(mem, 0), (int)d.n_mem);
    len = min(min(max(len, 0), d.max_mem), (int)d.n_mem - mem);
  }
  const int n = t1 - t0, row_tiles = (n * P.G + P.rows - 1) / P.rows;
  // tokens without a state have a tile all the same: it writes their zeros
  const int key_tiles = max(1, (len + P.keys - 1) / P.keys);
  const bool half = n * P.G - (row_tiles - 1) * P.rows <= P.half;
  return {t0, n, mem, len, row_tiles, key_tiles, half ? (key_tiles + 1) / 2 : key_tiles};
}

// This CTA's cells, and the request that the first of them lies in.
struct Share {
  long long lo, hi;  // cells of all requests in a row
  long long first;   // of request b
  int b;
};

// By the whole block, N threads.  Each thread adds up the cells of a run of requests; the runs' sums are scanned.
template <int N>
__device__ __forceinline__ Share share_of(const CrossPlan &P) {
  constexpr int kWarps = N / 32;
  __shared__ long long sums[kWarps];
  __shared__ Share found;
  const wt_cross_desc &d = P.d;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int run = (d.n_req + N - 1) / N, b0 = min(tid * run, d.n_req), b1 = min(b0 + run, d.n_req);
  long long mine = 0;
  for (int b = b0; b < b1; ++b) mine += asker_of(P, b, blockIdx.x == 0).cells(P);
  long long upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) sums[warp] = upto;
  if (tid == 0) found = {0, 0, 0, d.n_req};
  __syncthreads();
  long long all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w == warp) upto += all;
    all += sums[w];
  }
  const long long per = max((long long)P.least, quotient(all + gridDim.x - 1, gridDim.x)), lo = per * blockIdx.x, hi = min(all, lo + per);
  long long first = upto - mine;
  const bool here = lo < hi && first <= lo && lo < upto;
  if (here || blockIdx.x == 0)
    for (int b = b0; b < b1; ++b) {
      const long long n = asker_of(P, b, false).cells(P);
      if (blockIdx.x == 0) P.first[b] = first;
      if (here && first <= lo && lo < first + n) found = {lo, hi, first, b};
      first += n;
    }
  if (blockIdx.x == 0 && tid == 0) P.first[d.n_req] = per, P.first[d.n_req + 1] = all;
  __syncthreads();
  return found;
}

// One row tile's states that this CTA takes.
struct Segment {
  int group, row_tile;  // of kv heads, of rows
  int tile0, tiles;   // tiles of P.keys states
  int cells;          // as many, or half of them (P.half)
  bool half, whole;   // whole: all of the row tile's
  long long slot;     // where the part goes else
};

// The segment that starts at cell `at` of request a, whose first cell is `first`.
__device__ __forceinline__ Segment segment_at(const CrossPlan &P, const Asker &a, long long first, long long at, const Share &s) {
  Segment g;
  const long long per_head = a.head_cells();
  g.group = (int)quotient(at - first, per_head);
  const long long head = first + g.group * per_head;
  g.row_tile = (int)min(quotient(at - head, a.key_tiles), a.row_tiles - 1ll);
  const long long begin = head + (long long)g.row_tile * a.key_tiles;
  const int all = g.row_tile == a.row_tiles - 1 ? a.last : a.key_tiles;
  g.half = a.n * P.G - g.row_tile * P.rows <= P.half;
  g.cells = (int)(min(s.hi, begin + all) - at);
  g.whole = g.cells == all;
  g.tile0 = (int)(at - begin) << g.half;
  g.tiles = min(g.cells << g.half, a.key_tiles - g.tile0);
  g.slot = 2 * blockIdx.x + (begin >= s.lo && at > s.lo);
  return g;
}

}  // namespace
}  // namespace wt
