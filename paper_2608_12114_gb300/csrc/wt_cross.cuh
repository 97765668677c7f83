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
  const int n = t1 - t0, row_tiles = cross_row_tiles(n, P.G, P.rows);
  // tokens without a state have a tile all the same: it writes their zeros
  const int key_tiles = max(1, (len + P.keys - 1) / P.keys);
  const bool half = n * P.G - (row_tiles - 1) * P.rows <= P.half;
  return {t0, n, mem, len, row_tiles, key_tiles, half ? (key_tiles + 1) / 2 : key_tiles};
}

// This CTA's cells, and the place of the first of them: request, group of kv heads, row tile, cell of that.
struct Share {
  long long lo, hi;  // cells of all requests in a row
  int b, group, row_tile, at;
  Asker a;  // request b
};

// By the whole block, N threads.  Each thread adds up the cells of a run of requests; the runs' sums are scanned, and
// the thread whose run has the CTA's first cell finds its place.
template <int N>
__device__ __forceinline__ Share share_of(const CrossPlan &P) {
  constexpr int kWarps = N / 32;
  __shared__ long long sums[kWarps];
  __shared__ Share found;
  const wt_cross_desc &d = P.d;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (d.n_req <= 32) {  // each warp by itself, a request a lane
    Asker a = {};
    int mine = 0;  // cells; with tokens, heads and states whose products pass 31 bits the block counts them
    bool large = false;
    if (lane < d.n_req) {
      a = asker_of(P, lane, blockIdx.x == 0 && warp == 0);
      const long long n = a.cells(P);
      large = n >= 1 << 25;
      mine = (int)n;
    }
    if (!__any_sync(0xffffffffu, large)) {
      int upto = mine;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
      }
      const unsigned all = __shfl_sync(0xffffffffu, upto, 31), ctas = gridDim.x;
      const unsigned per = max((unsigned)P.least, (all + ctas - 1) / ctas), lo = min(all, per * blockIdx.x), hi = min(all, lo + per);
      Share s = {};
      if (lo < hi) {
        const int b = __popc(__ballot_sync(0xffffffffu, (unsigned)upto <= lo));  // requests that end before it
        s.a.t0 = __shfl_sync(0xffffffffu, a.t0, b), s.a.n = __shfl_sync(0xffffffffu, a.n, b);
        s.a.mem = __shfl_sync(0xffffffffu, a.mem, b), s.a.len = __shfl_sync(0xffffffffu, a.len, b);
        s.a.row_tiles = __shfl_sync(0xffffffffu, a.row_tiles, b), s.a.key_tiles = __shfl_sync(0xffffffffu, a.key_tiles, b);
        s.a.last = __shfl_sync(0xffffffffu, a.last, b);
        const unsigned at = lo - __shfl_sync(0xffffffffu, upto - mine, b), per_head = (unsigned)s.a.head_cells();
        s.lo = lo, s.hi = hi, s.b = b;
        s.group = at / per_head;
        const unsigned in_head = at - s.group * per_head;
        s.row_tile = min(in_head / s.a.key_tiles, s.a.row_tiles - 1u);
        s.at = in_head - s.row_tile * s.a.key_tiles;
      }
      __syncthreads();  // as below: what the block has set up is there
      return s;
    }
  }
  const int run = (d.n_req + N - 1) / N, b0 = min(tid * run, d.n_req), b1 = min(b0 + run, d.n_req);
  Asker a = {};
  long long mine = 0;
  for (int b = b0; b < b1; ++b) {
    a = asker_of(P, b, blockIdx.x == 0);
    mine += a.cells(P);
  }
  long long upto = mine;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long v = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) sums[warp] = upto;
  if (tid == 0) found = {};
  __syncthreads();
  long long all = 0;
#pragma unroll
  for (int w = 0; w < kWarps; ++w) {
    if (w == warp) upto += all;
    all += sums[w];
  }
  const long long per = max((long long)P.least, quotient(all + gridDim.x - 1, gridDim.x)), lo = per * blockIdx.x, hi = min(all, lo + per);
  long long first = upto - mine;
  if (lo < hi && first <= lo && lo < upto) {
    int b = b0;
    if (run > 1)
      for (;; ++b) {
        a = asker_of(P, b, false);
        const long long n = a.cells(P);
        if (lo < first + n) break;
        first += n;
      }
    const int group = (int)quotient(lo - first, a.head_cells());
    const long long at = lo - first - group * a.head_cells();
    const int row_tile = (int)min(quotient(at, a.key_tiles), a.row_tiles - 1ll);
    found = {lo, hi, b, group, row_tile, (int)(at - (long long)row_tile * a.key_tiles), a};
  }
  __syncthreads();
  return found;
}

// One row tile's states that a CTA takes.
struct Segment {
  int group, row_tile;  // of kv heads, of rows
  int tile0, tiles;     // tiles of P.keys states
  bool half, whole;     // half: P.half; whole: all of the row tile's
  bool cut;             // it starts in this CTA's cells and goes on behind them
  int cells;            // of the row tile
  long long slot;       // where the part goes if it is not whole
};

// The segments of a CTA, one after another; whoever needs them walks them by itself.
struct Walk {
  const CrossPlan &P;
  const Share &s;
  long long cell;  // behind the segment
  int b, at;       // at: the segment's first cell of its row tile
  int taken;       // its cells
  bool started;
  Asker a;
  Segment g;
  __device__ Walk(const CrossPlan &p, const Share &share) : P(p), s(share), cell(share.lo), b(share.b), at(share.at), started(false), a(share.a) {
    g.group = share.group, g.row_tile = share.row_tile, g.tiles = 0, g.cut = false;
  }
  __device__ __forceinline__ bool next() {
    if (cell >= s.hi) return false;
    if (started) {
      at = 0;
      if (++g.row_tile == a.row_tiles) {
        g.row_tile = 0;
        if (++g.group == P.groups) {
          g.group = 0;
          do a = asker_of(P, ++b, false);
          while (a.n == 0);
        }
      }
    }
    started = true;
    g.cells = g.row_tile == a.row_tiles - 1 ? a.last : a.key_tiles;
    g.half = a.n * P.G - g.row_tile * P.rows <= P.half;
    const int n = taken = (int)min(s.hi - cell, (long long)(g.cells - at));
    g.whole = n == g.cells;
    g.cut = at == 0 && n < g.cells;
    g.tile0 = at << g.half;
    g.tiles = min(n << g.half, a.key_tiles - g.tile0);
    g.slot = 2 * blockIdx.x + (at == 0 && cell > s.lo);
    cell += n;
    return true;
  }
};

// By one thread of every CTA at its end: the row tile that starts among its cells and goes on behind them, if any,
// for the merge.
__device__ __forceinline__ void note_cut(const CrossPlan &P, const Share &s, const Walk &w) {
  CrossCut c = {};
  if (w.g.cut) {
    const long long u0 = s.hi - w.taken;  // it is the last segment
    c.parts = (int)(quotient(u0 + w.g.cells - 1, s.hi - s.lo) - blockIdx.x + 1);
    c.second = u0 > s.lo;
    c.t0 = w.a.t0, c.rows = w.a.n * P.G;
    c.group = w.g.group, c.row_tile = w.g.row_tile;
  }
  P.cuts[blockIdx.x] = c;
}

}  // namespace
}  // namespace wt
