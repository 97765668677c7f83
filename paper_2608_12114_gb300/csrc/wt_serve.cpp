// C ABI of a serving step (include/wt_serve.h): argument checks, splits and launches.
#include <algorithm>
#include <cmath>
#include <cstdint>

#include <cuda_runtime.h>

#include "wt_kernels.h"
#include "wt_serve.h"

namespace {

using wt::serve_error;

#define CU(call)                                                    \
  do {                                                              \
    cudaError_t e_ = (call);                                        \
    if (e_ != cudaSuccess) return wt::serve_cuda_error(e_, #call);  \
  } while (0)

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

struct Lock {
  wt_handle *h;
  explicit Lock(wt_handle *hh) : h(hh) { wt::serve_lock(h); }
  ~Lock() { wt::serve_unlock(h); }
};

// One kernel that needs no workspace.
template <typename F>
int launch_alone(wt_handle *h, cudaStream_t s, F launch) {
  Lock lock(h);
  wt::ServeWorkspace w;
  if (int rc = wt::serve_workspace(h, s, 0, &w)) return rc;
  const cudaError_t e = launch();
  const int rc = wt::serve_done(h, s, w);
  CU(e);
  wt::serve_launched(h, 1);
  return rc;
}

bool aligned(const void *p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// Bytes of memory, which stay at the largest number where a product or a sum would pass 64 bits (rows of
// 2^31 at a pitch of 2^40 do): such a range runs past the end of any allocation.
struct Bytes {
  uint64_t n;
  Bytes(uint64_t v) : n(v) {}
  Bytes operator*(Bytes o) const {
    uint64_t r;
    return __builtin_mul_overflow(n, o.n, &r) ? UINT64_MAX : r;
  }
  Bytes operator+(Bytes o) const {
    uint64_t r;
    return __builtin_add_overflow(n, o.n, &r) ? UINT64_MAX : r;
  }
};

// Bytes from the first to one past the last element of `rows` rows of `row` elements, `pitch`
// elements apart.
uint64_t extent(uint64_t rows, uint64_t pitch, uint64_t row, uint64_t elem) {
  return rows == 0 || row == 0 ? 0 : ((Bytes(rows - 1) * pitch + row) * elem).n;
}
constexpr int64_t kMaxPitch = 1ll << 40;
// Tokens and lengths of rows: what a kernel adds to one (a stride over threads, a tile) stays below 2^31.
constexpr int32_t kMaxSize = 1 << 30;

int check_buffer(wt::ServeRanges *seen, const char *call, const char *name, const void *p, uint64_t n, uintptr_t align) {
  if (n == 0) return WT_OK;
  if (!p) return serve_error(WT_EINVAL, "%s: %s is NULL", call, name);
  if (!aligned(p, align)) return serve_error(WT_EINVAL, "%s: %s is not on a %d-byte boundary", call, name, (int)align);
  if (!wt::serve_range_ok(p, n, seen)) return serve_error(WT_EINVAL, "%s: %s runs past the end of its device allocation", call, name);
  return WT_OK;
}

int check_output(wt_handle *h, wt::ServeRanges *seen, const char *call, const char *name, const void *p, uint64_t n, uintptr_t align) {
  int rc = check_buffer(seen, call, name, p, n, align);
  if (rc == WT_OK && n && wt::serve_inside_mapping(h, p, n))
    rc = serve_error(WT_EINVAL, "%s: %s lies inside a read-only mapping", call, name);
  return rc;
}

// Rows of a buffer, in bytes; its extent has been checked.
struct Rows {
  const char *name;
  uintptr_t p;
  uint64_t n, pitch, row;
  Rows(const char *what, const void *at, uint64_t rows, uint64_t pitch_bytes, uint64_t row_bytes)
      : name(what), p(reinterpret_cast<uintptr_t>(at)), n(row_bytes ? rows : 0), pitch(pitch_bytes), row(row_bytes) {}
  Rows(const char *what, const void *at, uint64_t bytes) : Rows(what, at, 1, bytes, bytes) {}
  uintptr_t end() const { return p + (n - 1) * pitch + row; }
  // whether one of the rows meets [lo, hi)
  bool meets(uintptr_t lo, uintptr_t hi) const {
    const uint64_t k = lo < p + row ? 0 : (lo - p - row) / pitch + 1;  // the first row that ends past lo
    return k < n && p + k * pitch < hi;
  }
};

// Whether a byte belongs to rows of both: columns of one buffer, which only interleave, do not overlap.
bool overlap(const Rows &a, const Rows &b) {
  if (a.n == 0 || b.n == 0 || a.p >= b.end() || b.p >= a.end()) return false;
  if (a.pitch == b.pitch && a.n > 1 && b.n > 1) {
    const Rows &lo = a.p <= b.p ? a : b, &hi = a.p <= b.p ? b : a;
    const uint64_t off = (hi.p - lo.p) % a.pitch;
    return off < lo.row || a.pitch - off < hi.row;
  }
  const Rows &few = a.n <= b.n ? a : b, &many = a.n <= b.n ? b : a;
  for (uint64_t i = 0; i < few.n; ++i)
    if (many.meets(few.p + i * few.pitch, few.p + i * few.pitch + few.row)) return true;
  return false;
}

#define CHECK(expr)          \
  do {                       \
    int rc_ = (expr);        \
    if (rc_) return rc_;     \
  } while (0)

int check_adapt(wt_handle *h, wt::ServeRanges &seen, const wt_adapt_desc &d, size_t i) {
  const char *call = "wt_adapt";
  if (d.dtype != WT_BF16 && d.dtype != WT_F16)
    return serve_error(d.dtype >= WT_F32 && d.dtype <= WT_U8 ? WT_ENOTSUP : WT_EINVAL,
                       "%s: desc %zu: dtype %d: x, A and B are bf16 or f16", call, i, d.dtype);
  if (d.T < 0 || d.K < 0 || d.M < 0 || d.S < 0 || d.R < 0 || d.T > kMaxSize || d.K > kMaxSize || d.M > kMaxSize ||
      d.S > WT_ADAPT_MAX_SLOTS || d.R > WT_ADAPT_MAX_RANK)
    return serve_error(WT_EINVAL,
                       "%s: desc %zu: T %d, K %d, M %d (up to 2^30), S %d (up to %d) or R %d (up to %d) out of range", call, i,
                       d.T, d.K, d.M, d.S, WT_ADAPT_MAX_SLOTS, d.R, WT_ADAPT_MAX_RANK);
  const uint64_t T = d.T, K = d.K, M = d.M, S = d.S, R = d.R;
  if (d.ldx < d.K || d.ldy < d.M || (d.base && d.ldbase < d.M) || d.a_slot < (int64_t)(R * K) || d.b_slot < (int64_t)(M * R) ||
      d.ldx > kMaxPitch || d.ldy > kMaxPitch || d.ldbase > kMaxPitch || d.a_slot > kMaxPitch || d.b_slot > kMaxPitch)
    return serve_error(WT_EINVAL, "%s: desc %zu: a pitch is shorter than its row, or not below 2^40", call, i);
  if (T == 0 || M == 0) return WT_OK;
  CHECK(check_output(h, &seen, call, "y", d.y, extent(T, d.ldy, M, 4), 4));
  CHECK(check_buffer(&seen, call, "base", d.base, d.base ? extent(T, d.ldbase, M, 4) : 0, 4));
  if (d.base == d.y && d.ldbase != d.ldy)
    return serve_error(WT_EINVAL, "%s: desc %zu: base is y, with another pitch", call, i);
  CHECK(check_buffer(&seen, call, "slot", d.slot, 4 * T, 4));
  if (S == 0) return WT_OK;
  if (d.rank) CHECK(check_buffer(&seen, call, "rank", d.rank, 4 * S, 4));  // read where R is 0, too
  if (R == 0) return WT_OK;
  CHECK(check_buffer(&seen, call, "x", d.x, extent(T, d.ldx, K, 2), 2));
  CHECK(check_buffer(&seen, call, "A", d.A, extent(S, d.a_slot, R * K, 2), 2));
  CHECK(check_buffer(&seen, call, "B", d.B, extent(S, d.b_slot, M * R, 2), 2));
  if (d.scale) CHECK(check_buffer(&seen, call, "scale", d.scale, 4 * S, 4));
  return WT_OK;
}

// The descriptors of one launch run at once: no y of them may meet anything that one of them reads or
// another writes.  (Those of different launches follow one another.)
int check_adapt_overlap(const wt::AdaptLaunch &L) {
  for (int j = 0; j < L.n; ++j) {
    const wt_adapt_desc &d = L.p[j].d;
    const uint64_t T = d.T, K = d.K, M = d.M, R = d.R, S = R ? d.S : 0;
    const Rows y("y", d.y, T, 4 * d.ldy, 4 * M);
    const Rows reads[] = {{"base", d.base, d.base ? T : 0, 4 * (uint64_t)d.ldbase, 4 * M},
                          {"x", d.x, S ? T : 0, 2 * (uint64_t)d.ldx, 2 * K},
                          {"A", d.A, S, 2 * (uint64_t)d.a_slot, 2 * R * K},
                          {"B", d.B, S, 2 * (uint64_t)d.b_slot, 2 * M * R},
                          {"slot", d.slot, 4 * T},
                          {"rank", d.rank, d.rank ? 4 * (uint64_t)d.S : 0},
                          {"scale", d.scale, d.scale ? 4 * S : 0}};
    for (int i = 0; i < L.n; ++i) {
      const wt_adapt_desc &e = L.p[i].d;
      const Rows out("y", e.y, e.T, 4 * (uint64_t)e.ldy, 4 * (uint64_t)e.M);
      if (i < j && overlap(out, y)) return serve_error(WT_EINVAL, "wt_adapt: the y of two descriptors overlap");
      for (const Rows &r : reads) {
        if (i == j && &r == &reads[0] && d.base == d.y) continue;
        if (overlap(out, r))
          return serve_error(WT_EINVAL, "wt_adapt: y overlaps %s of %s descriptor", r.name, i == j ? "its" : "another");
      }
    }
  }
  return WT_OK;
}

int adapt_impl(wt_handle *h, const wt_adapt_desc *d, size_t n, cudaStream_t s) {
  wt::ServeContext ctx;
  CHECK(wt::serve_context(h, "wt_adapt", wt::kServeAdapt, &ctx));
  if (n && !d) return serve_error(WT_EINVAL, "wt_adapt: NULL descriptors");
  wt::ServeRanges seen;
  for (size_t i = 0; i < n; ++i) CHECK(check_adapt(h, seen, d[i], i));
  wt::AdaptLaunch L;
  // up to 8 descriptors of one type a launch; the index of the first of the next one
  auto take = [&](size_t i) {
    const int dtype = d[i].dtype;
    L.n = 0;
    for (; i < n && L.n < wt::kAdaptProjs && d[i].dtype == dtype; ++i)
      if (d[i].T && d[i].M) L.p[L.n++].d = d[i];
    return i;
  };
  for (size_t i = 0; i < n;) {
    i = take(i);
    CHECK(check_adapt_overlap(L));
  }
  for (size_t i = 0; i < n;) {
    const int dtype = d[i].dtype;
    i = take(i);
    if (L.n == 0) continue;
    int max_R = 0, max_T = 0;
    for (int k = 0; k < L.n; ++k) {
      max_R = std::max(max_R, L.p[k].d.R);
      max_T = std::max(max_T, L.p[k].d.T);
    }
    uint64_t all = 0;
    const bool planned = wt::adapt_planned(max_T);
    const int tile = planned ? 64 : 16;  // tokens of a work item
    for (int k = 0; k < L.n; ++k) {
      wt::AdaptProj &P = L.p[k];
      const wt_adapt_desc &e = P.d;
      const bool copy = e.base != e.y;
      P.items = (uint32_t)(std::min(e.S + (copy ? 1 : 0), e.T) + e.T / tile);
      all += (uint64_t)P.items * ((e.M + wt::kAdaptMTile - 1) / wt::kAdaptMTile);
      P.vec = 0;
      if (e.K % 8 == 0 && e.ldx % 8 == 0 && e.a_slot % 8 == 0 && aligned(e.x, 16) && aligned(e.A, 16)) P.vec |= 1;
      // vectors of B: 8 elements; 4 in the one-launch kernel where no rank is above 16
      const int el = !planned && max_R <= 16 ? 4 : 8;
      if (e.R % el == 0 && e.b_slot % el == 0 && aligned(e.B, 2 * el)) P.vec |= 2;
      if (e.ldy % 4 == 0 && aligned(e.y, 16) && (!e.base || (e.ldbase % 4 == 0 && aligned(e.base, 16)))) P.vec |= 4;
    }
    if (all > (1u << 27)) return serve_error(WT_EINVAL, "wt_adapt: %llu tiles of work in one launch", (unsigned long long)all);
    if (!planned) {
      CHECK(launch_alone(h, s, [&] { return wt::launch_adapt(L, nullptr, max_R, ctx.status, s); }));
      continue;
    }
    // many tokens: a plan for each distinct slot map, and v of every projection, in the workspace
    wt::AdaptWide W = {};
    int64_t items = 0, v = 0, back = 0;
    const int64_t row = 16 * wt::adapt_rank_tiles(max_R), parts = dtype == WT_BF16 ? 3 : 2;
    // tiles of outputs that a CTA takes one after another: about nine CTAs per SM in all, three waves of three
    // where three fit an SM
    const int64_t run = std::max<int64_t>(1, ceil_div((int64_t)all, 9 * wt::num_sms()));
    for (int k = 0; k < L.n; ++k) {
      const wt_adapt_desc &e = L.p[k].d;
      const int64_t tiles = ceil_div(e.M, wt::kAdaptMTile);
      L.p[k].m_groups = (uint32_t)ceil_div(tiles, run);
      L.p[k].group_tiles = (uint32_t)ceil_div(tiles, L.p[k].m_groups);
      auto same = [&](int q) {
        const wt_adapt_desc &f = L.p[W.plan_proj[q]].d;
        return f.slot == e.slot && f.T == e.T && f.S == e.S && (f.base == f.y) == (e.base == e.y);
      };
      int q = 0;
      while (q < W.n_plans && !same(q)) ++q;
      if (q == W.n_plans) W.plan_proj[W.n_plans++] = k;
      W.plan[k] = q;
      W.v_at[k] = v;
      W.back_at[k] = back;
      v += parts * e.T * row;
      back += e.T;
      items = std::max<int64_t>(items, L.p[k].items);
    }
    W.order_at = 4 * (items + 1);
    W.plan_ints = (W.order_at + max_T + 63) / 64 * 64;
    Lock lock(h);
    wt::ServeWorkspace w;
    const size_t plans = (size_t)(W.n_plans * W.plan_ints) * 4;
    CHECK(wt::serve_workspace(h, s, plans + (size_t)v * 2 + (size_t)back * 4, &w));
    W.plans = static_cast<int *>(w.p);
    W.v = reinterpret_cast<uint16_t *>(static_cast<uint8_t *>(w.p) + plans);
    W.back = reinterpret_cast<float *>(W.v + v);
    const cudaError_t e = wt::launch_adapt(L, &W, max_R, ctx.status, s);
    const int rc = wt::serve_done(h, s, w);
    CU(e);
    wt::serve_launched(h, 3);
    if (rc) return rc;
  }
  return WT_OK;
}

int check_attend(wt_handle *h, const wt_attend_desc &d) {
  const char *call = "wt_attend";
  wt::ServeRanges seen;
  if (d.dtype != WT_BF16 && d.dtype != WT_F16)
    return serve_error(d.dtype >= WT_F32 && d.dtype <= WT_U8 ? WT_ENOTSUP : WT_EINVAL,
                       "%s: dtype %d: queries and caches are bf16 or f16", call, d.dtype);
  if (d.n_req < 0 || d.n_req > 65535 || d.n_tokens < 0 || d.n_tokens > kMaxSize || d.max_new < 0 || d.prefix_len < 0 || d.prefix_len > (1 << 30) ||
      d.max_len < 0 || d.max_len > (1 << 30) || d.n_pages < 0)
    return serve_error(WT_EINVAL, "%s: n_req %d, n_tokens %d, max_new %d, prefix_len %lld, max_len %d or n_pages %d out of range",
                       call, d.n_req, d.n_tokens, d.max_new, (long long)d.prefix_len, d.max_len, d.n_pages);
  if (d.heads < 1 || d.kv_heads < 1 || d.heads > 65536 || d.heads % d.kv_heads || d.heads / d.kv_heads > 128)
    return serve_error(WT_EINVAL, "%s: heads %d is not up to 128 times kv_heads %d", call, d.heads, d.kv_heads);
  if (d.head_dim < 8 || d.head_dim % 8)
    return serve_error(WT_EINVAL, "%s: head_dim %d is not a multiple of 8", call, d.head_dim);
  if (d.head_dim > 128) return serve_error(WT_ENOTSUP, "%s: head_dim %d is above 128", call, d.head_dim);
  if (!std::isfinite(d.scale)) return serve_error(WT_EINVAL, "%s: scale is not finite", call);
  const int64_t row = (int64_t)d.heads * d.head_dim, D = d.head_dim;
  if (d.q_stride < row || d.out_stride < row || d.q_stride % 8 || d.out_stride % 8 || d.q_stride > kMaxPitch ||
      d.out_stride > kMaxPitch)
    return serve_error(WT_EINVAL, "%s: token pitches %lld and %lld are not multiples of 8 of at least heads * head_dim", call,
                       (long long)d.q_stride, (long long)d.out_stride);
  if ((int64_t)d.n_tokens * d.heads > 0x7fffffff) return serve_error(WT_EINVAL, "%s: n_tokens * heads above 2^31-1", call);
  if (d.n_req == 0 || d.n_tokens == 0 || d.max_new == 0) return WT_OK;
  CHECK(check_buffer(&seen, call, "q", d.q, extent(d.n_tokens, d.q_stride, row, 2), 16));
  CHECK(check_output(h, &seen, call, "out", d.out, extent(d.n_tokens, d.out_stride, row, 2), 16));
  CHECK(check_buffer(&seen, call, "begin", d.begin, 4 * ((uint64_t)d.n_req + 1), 4));
  const Rows out("out", d.out, d.n_tokens, 2 * (uint64_t)d.out_stride, 2 * (uint64_t)row);
  auto apart = [&](const Rows &r) {
    return overlap(out, r) ? serve_error(WT_EINVAL, "%s: out overlaps %s", call, r.name) : WT_OK;
  };
  // out may be q: a token's head is written once all that reads it has been read
  if (d.out != d.q || d.out_stride != d.q_stride)
    CHECK(apart({"q", d.q, (uint64_t)d.n_tokens, 2 * (uint64_t)d.q_stride, 2 * (uint64_t)row}));
  CHECK(apart({"begin", d.begin, 4 * ((uint64_t)d.n_req + 1)}));
  if (d.prefix_len) {
    if (d.prefix_head < D || d.prefix_head % 8 || d.prefix_stride < D || d.prefix_stride % 8 || d.prefix_head > kMaxPitch ||
        d.prefix_stride > kMaxPitch)
      return serve_error(WT_EINVAL, "%s: prefix pitches %lld and %lld are not multiples of 8 of at least head_dim", call,
                         (long long)d.prefix_stride, (long long)d.prefix_head);
    // dense either way round: [key, head, dim] or [head, key, dim]
    const uint64_t n = (Bytes(2) * (Bytes(d.prefix_len - 1) * d.prefix_stride + Bytes(d.kv_heads - 1) * d.prefix_head + D)).n;
    CHECK(check_buffer(&seen, call, "prefix_k", d.prefix_k, n, 16));
    CHECK(check_buffer(&seen, call, "prefix_v", d.prefix_v, n, 16));
    // as rows of whole keys where those lie apart, else of whole heads, or one
    const uint64_t P = d.prefix_len, H = d.kv_heads, key = 2 * ((H - 1) * d.prefix_head + D), head = 2 * ((P - 1) * d.prefix_stride + D);
    const bool keys = P > 1 && 2 * (uint64_t)d.prefix_stride >= key, heads = H > 1 && 2 * (uint64_t)d.prefix_head >= head;
    for (const void *p : {d.prefix_k, d.prefix_v})
      CHECK(apart(keys    ? Rows("the prefix", p, P, 2 * d.prefix_stride, key)
                  : heads ? Rows("the prefix", p, H, 2 * d.prefix_head, head)
                          : Rows("the prefix", p, n)));
  }
  if (d.max_len) {
    if (d.page < 1 || d.table_stride < 0 || d.table_stride > 0x7fffffff || (int64_t)d.max_len > d.table_stride * d.page)
      return serve_error(WT_EINVAL, "%s: max_len %d does not fit %lld pages of %d keys", call, d.max_len,
                         (long long)d.table_stride, d.page);
    const uint64_t n = (Bytes(d.n_pages) * d.page * d.kv_heads * D * 2).n;
    CHECK(check_buffer(&seen, call, "k_pages", d.k_pages, n, 16));
    CHECK(check_buffer(&seen, call, "v_pages", d.v_pages, n, 16));
    // the pages of max_len keys: what is beyond may belong to a wider table
    const uint64_t pages = ceil_div(d.max_len, d.page);
    CHECK(check_buffer(&seen, call, "table", d.table, extent(d.n_req, d.table_stride, pages, 4), 4));
    CHECK(check_buffer(&seen, call, "len", d.len, 4 * (uint64_t)d.n_req, 4));
    CHECK(apart({"k_pages", d.k_pages, n}));
    CHECK(apart({"v_pages", d.v_pages, n}));
    CHECK(apart({"table", d.table, (uint64_t)d.n_req, 4 * (uint64_t)d.table_stride, 4 * pages}));
    CHECK(apart({"len", d.len, 4 * (uint64_t)d.n_req}));
  }
  return WT_OK;
}

// The prefix goes to tcgen05 from 33 rows (token, head-in-group) on, where the warp kernel would read
// it more than twice, and from 17 where it is long (10 tokens of 4 heads a group behind 10475 keys: 23 us
// on the warp kernel, under 20; 42 tokens of one behind 50: 13.4 against 18.6).  Its softmax takes the
// largest product for the largest score, so the scale has to be positive; and a pitch has to fit a
// tensor map.
bool prefix_on_tcgen05(const wt_attend_desc &d) {
  const int64_t rows = (int64_t)d.n_tokens * (d.heads / d.kv_heads);
  return (rows > 32 || (rows > 16 && d.prefix_len >= 2048)) && d.scale > 0.0f && d.q_stride < (1ll << 38) && d.prefix_stride < (1ll << 38) &&
         d.prefix_head < (1ll << 38);
}

// Rows in tiles of whole tokens, and as many ranges of key tiles as make the SMs' work come out even:
// a range costs its tiles and about 3 more (first loads, the first and last product, the parts' stores).
int plan_prefix(const wt_attend_desc &d, int G, wt::PrefixPlan *x, wt::PrefixMaps *maps) {
  x->G = G;
  x->kv_heads = d.kv_heads;
  x->head_dim = d.head_dim;
  x->dim_steps = (d.head_dim + 15) / 16;
  x->prefix_len = (int)d.prefix_len;
  x->scale_log2 = d.scale * 1.4426950408889634f;
  x->tile_tokens = 128 / G;
  x->tile_rows = x->tile_tokens * G;
  x->rows = d.n_tokens * G;
  x->tiles = (int)ceil_div(d.prefix_len, 128);
  const int64_t row_tiles = ceil_div(d.n_tokens, x->tile_tokens);
  x->apart = row_tiles == 1;
  x->row_blocks = (int)ceil_div(row_tiles, 2);
  x->qtiles = x->apart ? 2 : 2 * x->row_blocks;
  const int64_t all = (int64_t)d.kv_heads * x->tiles, sms = wt::num_sms();
  if (all > (1 << 30)) return serve_error(WT_EINVAL, "wt_attend: %lld key tiles", (long long)all);
  int64_t best = INT64_MAX;
  for (int64_t waves = 1; waves <= 4; ++waves) {
    const int64_t g = std::min(all, std::max<int64_t>(1, waves * sms / x->row_blocks));
    const int64_t len = ceil_div(all, g), n = ceil_div(all, len);
    const int64_t cost = ceil_div(x->row_blocks * n, sms) * (len + 3);
    if (cost < best) best = cost, x->len = (int)len, x->groups = (int)n;
  }
  const uint64_t D = d.head_dim;
  const uint64_t qd[3] = {D, (uint64_t)d.heads, (uint64_t)d.n_tokens}, qs[2] = {2 * D, 2 * (uint64_t)d.q_stride};
  const uint32_t qb[3] = {64, (uint32_t)G, (uint32_t)x->tile_tokens};
  const uint64_t kd[3] = {D, (uint64_t)d.kv_heads, (uint64_t)d.prefix_len},
                 ks[2] = {2 * (uint64_t)d.prefix_head, 2 * (uint64_t)d.prefix_stride};
  const uint32_t kb[3] = {64, 1, 128};
  CHECK(wt::serve_tensor_map(maps->q, d.q, 3, qd, qs, qb));
  CHECK(wt::serve_tensor_map(maps->k, d.prefix_k, 3, kd, ks, kb));
  return wt::serve_tensor_map(maps->v, d.prefix_v, 3, kd, ks, kb);
}

int attend_impl(wt_handle *h, const wt_attend_desc *dp, cudaStream_t s) {
  wt::ServeContext ctx;
  CHECK(wt::serve_context(h, "wt_attend", wt::kServeAttend, &ctx));
  if (!dp) return serve_error(WT_EINVAL, "wt_attend: NULL descriptor");
  CHECK(check_attend(h, *dp));
  wt::AttendPlan P = {};
  P.d = *dp;
  wt_attend_desc &d = P.d;
  if (d.n_req == 0 || d.n_tokens == 0 || d.max_new == 0) return WT_OK;
  d.max_new = std::min(d.max_new, d.n_tokens);
  P.G = d.heads / d.kv_heads;
  P.status = ctx.status;
  const int64_t own_rows = (int64_t)d.max_new * P.G, pre_rows = (int64_t)d.n_tokens * P.G;
  wt::PrefixMaps maps;
  if (d.prefix_len && prefix_on_tcgen05(d)) CHECK(plan_prefix(d, P.G, &P.x, &maps));
  const bool pre_warp = d.prefix_len && !P.x.groups;
  // tiles of 32 rows where a request has more than 16; a prefix beside shorter ones is read once for each 16
  P.rows_tile = (d.max_len ? own_rows : pre_rows) <= 16 ? 16 : 32;
  P.own_tiles = (int)ceil_div(own_rows, P.rows_tile);
  P.pre_tiles = (int)ceil_div(pre_rows, P.rows_tile);
  // Splits, of at least 64 keys (one tile for each warp).  Own keys alone take 4 CTAs per SM, as lengths
  // differ and CTAs without keys end at once (24 requests: 30.4 us, with 2 CTAs 33.6).  Own keys and prefix
  // in one launch take one CTA per SM each (7 requests with a head for every query behind 1021 keys:
  // 13.6 us, with 4 17.1), and more where splits stay at 512 keys: 4, or for the prefix what an SM holds.
  const int64_t sms = wt::num_sms(), few = pre_warp ? 1 : 4, resident = P.rows_tile == 16 ? 3 : 2;
  auto split = [&](int64_t keys, int64_t ctas, int64_t most, int &splits, int &len) {
    const int64_t n = std::max(std::min(ceil_div(keys, 64), ceil_div(few * sms, ctas)), std::min(ceil_div(keys, 512), most));
    len = (int)(ceil_div(ceil_div(keys, n), 64) * 64);
    splits = (int)ceil_div(keys, len);
  };
  const int64_t own_ctas = (int64_t)d.n_req * d.kv_heads * P.own_tiles, pre_ctas = (int64_t)d.kv_heads * P.pre_tiles;
  if (d.max_len) split(d.max_len, own_ctas, ceil_div(4 * sms, own_ctas), P.own_splits, P.own_len);
  if (pre_warp) split(d.prefix_len, pre_ctas, std::max<int64_t>(1, resident * sms / pre_ctas), P.pre_splits, P.pre_len);
  const int64_t parts = P.own_splits + P.pre_splits, rows = (int64_t)d.n_tokens * d.heads;
  // a token's only part is its result
  P.direct = P.own_splits == 1 && !d.prefix_len;
  if ((double)d.kv_heads * ((double)d.n_req * P.own_splits * P.own_tiles + (double)P.pre_splits * P.pre_tiles) > 0x7fffffff)
    return serve_error(WT_EINVAL, "wt_attend: too many tokens, heads and keys for one launch");
  // workspace: O and (m, l) of every part
  auto take = [](size_t &at, size_t n) {
    const size_t o = at;
    at += (n + 255) / 256 * 256;
    return o;
  };
  const int64_t xrows = P.x.groups ? (int64_t)(P.x.groups + d.kv_heads - 1) * P.x.qtiles * 128 : 0;
  size_t bytes = 0;
  const size_t o = take(bytes, P.direct ? 0 : (size_t)(parts * rows * d.head_dim) * 4),
               ml = take(bytes, P.direct ? 0 : (size_t)(parts * rows) * sizeof(float2));
  const size_t xo = take(bytes, (size_t)(xrows * d.head_dim) * 4), xml = take(bytes, (size_t)xrows * sizeof(float2));
  Lock lock(h);
  wt::ServeWorkspace w;
  CHECK(wt::serve_workspace(h, s, bytes, &w));
  uint8_t *ws = static_cast<uint8_t *>(w.p);
  P.o = reinterpret_cast<float *>(ws + o);
  P.ml = reinterpret_cast<float2 *>(ws + ml);
  P.x.o = reinterpret_cast<float *>(ws + xo);
  P.x.ml = reinterpret_cast<float2 *>(ws + xml);
  cudaError_t e = cudaSuccess;
  if (P.x.groups) e = wt::launch_attend_prefix(P.x, maps, d.dtype, ctx.status, s);
  if (e == cudaSuccess && parts) e = wt::launch_attend_warp(P, s);
  if (e == cudaSuccess && !P.direct) e = wt::launch_attend_merge(P, s);
  const int rc = wt::serve_done(h, s, w);
  CU(e);
  wt::serve_launched(h, (P.x.groups != 0) + (parts != 0) + !P.direct);
  return rc;
}

int check_cross(wt_handle *h, const wt_cross_desc &d) {
  const char *call = "wt_cross";
  wt::ServeRanges seen;
  if (d.dtype != WT_BF16 && d.dtype != WT_F16)
    return serve_error(d.dtype >= WT_F32 && d.dtype <= WT_U8 ? WT_ENOTSUP : WT_EINVAL,
                       "%s: dtype %d: queries and memories are bf16 or f16", call, d.dtype);
  if (d.n_req < 0 || d.n_req > 65535 || d.n_tokens < 0 || d.n_tokens > kMaxSize || d.max_new < 0 || d.max_mem < 0 ||
      d.max_mem > kMaxSize || d.n_mem < 0 || d.n_mem > kMaxSize)
    return serve_error(WT_EINVAL, "%s: n_req %d, n_tokens %d, max_new %d, max_mem %d or n_mem %lld out of range", call, d.n_req,
                       d.n_tokens, d.max_new, d.max_mem, (long long)d.n_mem);
  if (d.heads < 1 || d.kv_heads < 1 || d.heads > 65536 || d.heads % d.kv_heads || d.heads / d.kv_heads > 128)
    return serve_error(WT_EINVAL, "%s: heads %d is not up to 128 times kv_heads %d", call, d.heads, d.kv_heads);
  if (d.head_dim < 8 || d.head_dim % 8)
    return serve_error(WT_EINVAL, "%s: head_dim %d is not a multiple of 8", call, d.head_dim);
  if (d.head_dim > 128) return serve_error(WT_ENOTSUP, "%s: head_dim %d is above 128", call, d.head_dim);
  if (!std::isfinite(d.scale)) return serve_error(WT_EINVAL, "%s: scale is not finite", call);
  const int64_t row = (int64_t)d.heads * d.head_dim, D = d.head_dim;
  if (d.q_stride < row || d.out_stride < row || d.q_stride % 8 || d.out_stride % 8 || d.q_stride > kMaxPitch ||
      d.out_stride > kMaxPitch)
    return serve_error(WT_EINVAL, "%s: token pitches %lld and %lld are not multiples of 8 of at least heads * head_dim", call,
                       (long long)d.q_stride, (long long)d.out_stride);
  if ((int64_t)d.n_tokens * d.heads > 0x7fffffff) return serve_error(WT_EINVAL, "%s: n_tokens * heads above 2^31-1", call);
  if (d.n_req == 0 || d.n_tokens == 0 || d.max_new == 0) return WT_OK;
  CHECK(check_buffer(&seen, call, "q", d.q, extent(d.n_tokens, d.q_stride, row, 2), 16));
  CHECK(check_output(h, &seen, call, "out", d.out, extent(d.n_tokens, d.out_stride, row, 2), 16));
  CHECK(check_buffer(&seen, call, "begin", d.begin, 4 * ((uint64_t)d.n_req + 1), 4));
  const Rows out("out", d.out, d.n_tokens, 2 * (uint64_t)d.out_stride, 2 * (uint64_t)row);
  auto apart = [&](const Rows &r) {
    return overlap(out, r) ? serve_error(WT_EINVAL, "%s: out overlaps %s", call, r.name) : WT_OK;
  };
  // out may be q: a token's head is written once all that reads it has been read
  if (d.out != d.q || d.out_stride != d.q_stride)
    CHECK(apart({"q", d.q, (uint64_t)d.n_tokens, 2 * (uint64_t)d.q_stride, 2 * (uint64_t)row}));
  CHECK(apart({"begin", d.begin, 4 * ((uint64_t)d.n_req + 1)}));
  if (d.max_mem == 0) return WT_OK;
  const uint64_t B = d.n_req;
  CHECK(check_buffer(&seen, call, "mem_begin", d.mem_begin, 4 * B, 4));
  CHECK(check_buffer(&seen, call, "mem_len", d.mem_len, 4 * B, 4));
  CHECK(apart({"mem_begin", d.mem_begin, 4 * B}));
  CHECK(apart({"mem_len", d.mem_len, 4 * B}));
  if (d.n_mem == 0) return WT_OK;
  if (d.mem_head < D || d.mem_head % 8 || d.mem_stride < D || d.mem_stride % 8 || d.mem_head > kMaxPitch || d.mem_stride > kMaxPitch)
    return serve_error(WT_EINVAL, "%s: memory pitches %lld and %lld are not multiples of 8 of at least head_dim", call,
                       (long long)d.mem_stride, (long long)d.mem_head);
  // either way round: [state, head, dim] or [head, state, dim]
  const uint64_t M = d.n_mem, H = d.kv_heads, n = (Bytes(2) * (Bytes(M - 1) * d.mem_stride + Bytes(H - 1) * d.mem_head + D)).n;
  CHECK(check_buffer(&seen, call, "k", d.k, n, 16));
  CHECK(check_buffer(&seen, call, "v", d.v, n, 16));
  if (d.keep) {
    CHECK(check_buffer(&seen, call, "keep", d.keep, M, 1));
    CHECK(apart({"keep", d.keep, M}));
  }
  // as rows of whole states where those lie apart, else of whole heads, or one
  const uint64_t state = 2 * ((H - 1) * d.mem_head + D), head = 2 * ((M - 1) * d.mem_stride + D);
  const bool states = M > 1 && 2 * (uint64_t)d.mem_stride >= state, heads = H > 1 && 2 * (uint64_t)d.mem_head >= head;
  for (const void *p : {d.k, d.v})
    CHECK(apart(states  ? Rows("the memory", p, M, 2 * (uint64_t)d.mem_stride, state)
                : heads ? Rows("the memory", p, H, 2 * (uint64_t)d.mem_head, head)
                        : Rows("the memory", p, n)));
  return WT_OK;
}

// Rows (token, head-in-group) of a kv head that the kernel for few rows takes at once.
int cross_few_rows(const wt_cross_desc &d) { return d.head_dim <= 64 ? 32 : 16; }

// More rows of a request go to tcgen05.  (Few against many, us, memories of 1500 states.  8 kv heads of 128: one request of 16
// rows 11.7, 12.5, of 20 18.0, 12.8; 16 requests of 16 37.4, 20.4, of 20 69.7, 20.9; 48 of 16 68.0, 63.5, of 20 121, 64.3.
// 20 heads of 64: one request of 32 rows 15.7, 12.6; 16 of 16 38.2, 42.7, of 32 62.9, 42.6; 48 of 32 104, 117.)  Its softmax takes
// the largest product for the largest score, so the scale has to be positive.
bool cross_on_tcgen05(const wt_cross_desc &d) {
  return (int64_t)d.max_new * (d.heads / d.kv_heads) > cross_few_rows(d) && d.scale > 0.0f && d.max_mem > 0;
}

int cross_impl(wt_handle *h, const wt_cross_desc *dp, cudaStream_t s) {
  wt::ServeContext ctx;
  CHECK(wt::serve_context(h, "wt_cross", wt::kServeCross, &ctx));
  if (!dp) return serve_error(WT_EINVAL, "wt_cross: NULL descriptor");
  CHECK(check_cross(h, *dp));
  wt::CrossPlan P = {};
  P.d = *dp;
  wt_cross_desc &d = P.d;
  if (d.n_req == 0 || d.n_tokens == 0 || d.max_new == 0) return WT_OK;
  if (d.max_mem == 0) d.mem_len = nullptr;
  d.max_new = std::min(d.max_new, d.n_tokens);
  d.max_mem = (int32_t)std::min<int64_t>(d.max_mem, d.n_mem);
  P.G = d.heads / d.kv_heads;
  P.status = ctx.status;
  wt::CrossMaps maps = {};
  const bool wide = cross_on_tcgen05(d);
  const uint64_t D = d.head_dim;
  // the pitch of a dimension of one says nothing, and one that fits no tensor map can only be such a one
  if (d.n_tokens == 1) d.q_stride = (int64_t)d.heads * d.head_dim;
  if (d.n_mem == 1) d.mem_stride = (int64_t)d.kv_heads * d.head_dim;
  if (d.kv_heads == 1) d.mem_head = d.head_dim;
  if (wide) {
    P.tile_tokens = 128 / P.G;
    P.half = P.tile_tokens * P.G;
    P.rows = 2 * P.half;
    P.keys = 128;
    P.together = 1;
    const uint64_t qd[3] = {D, (uint64_t)d.heads, (uint64_t)d.n_tokens}, qs[2] = {2 * D, 2 * (uint64_t)d.q_stride};
    const uint32_t qb[3] = {64, (uint32_t)P.G, (uint32_t)P.tile_tokens};
    CHECK(wt::serve_tensor_map(maps.q, d.q, 3, qd, qs, qb));
  } else {
    // A warp to a head, for as many as the heads fill, so that those who read one line after another do it
    // together; but all to one head where that would leave a warp few tiles.  (Together against one, us, memories of 1500
    // states.  20 heads of 64, the border at 5 requests: 4 11.6, 9.3; 12 16.4, 15.3; 48 61.2, 86.1.  8 heads of 128, whose
    // lines are twice as long: 16 requests 22.7, 20.0; 48 55.2, 52.4.)
    const int keys = wt::cross_few_keys(d.head_dim);
    const double tiles = (double)d.n_req * d.kv_heads * (double)ceil_div(d.max_mem, keys);
    P.together = tiles < 16.0 * wt::kCrossFewResident * wt::num_sms() ? 1 : d.kv_heads % 4 == 0 ? 4 : d.kv_heads % 2 == 0 ? 2 : 1;
    P.keys = keys * 4 / P.together;
    const int64_t most = (int64_t)d.max_new * P.G;
    P.rows = most <= 8 ? 8 : most <= 16 ? 16 : cross_few_rows(d);
  }
  if (d.max_mem > 0) {
    const uint64_t kd[3] = {D, (uint64_t)d.kv_heads, (uint64_t)d.n_mem}, ks[2] = {2 * (uint64_t)d.mem_head, 2 * (uint64_t)d.mem_stride};
    const uint32_t kb[3] = {64, 1, (uint32_t)(wide ? 128 : wt::cross_few_keys(d.head_dim))};
    CHECK(wt::serve_tensor_map(maps.k, d.k, 3, kd, ks, kb));
    CHECK(wt::serve_tensor_map(maps.v, d.v, 3, kd, ks, kb));
  }
  P.groups = d.kv_heads / P.together;
  // A memory of n cells takes least of them and joins n / least parts, at about a 24th of a cell's time each.  (Without
  // a least, by a 24th, a sixth, two thirds: one token of 8 kv heads of 128, 1500 states, 8.3, 8.2, 8.6, 11.7 us; of one, 16384
  // states, 26.4, 14.6, 15.4, 20.9; 131072 35.6, 32.0, 32.9, 45.8; 64 tokens of 4 heads over one, 4096 14.6, 14.2, 15.6, 17.5.)
  P.least = 1 + (int)std::sqrt((double)ceil_div(d.max_mem, P.keys) / 24.0);
  // No more CTAs than run at once, or than there can be cells.  (Requests' row tiles: whole ones of all tokens,
  // and one more each.)
  const double tiles = std::min((double)d.n_req * (double)ceil_div((int64_t)d.max_new * P.G, P.rows),
                                (double)d.n_tokens * P.G / P.rows + d.n_req);
  const double cells = tiles * P.groups * (double)std::max<int64_t>(1, ceil_div(d.max_mem, P.keys));
  const int resident = wide ? 1 : wt::kCrossFewResident;
  P.ctas = (int)std::max(1.0, std::min((double)resident * wt::num_sms(), cells));
  auto take = [](size_t &at, size_t n) {
    const size_t o = at;
    at += (n + 255) / 256 * 256;
    return o;
  };
  size_t bytes = 0;
  const size_t slots = 2 * (size_t)P.ctas * P.together * P.rows;
  const size_t o = take(bytes, slots * d.head_dim * 4), ml = take(bytes, slots * sizeof(float2)),
               cuts = take(bytes, (size_t)P.ctas * sizeof(wt::CrossCut)),
               fold = take(bytes, d.max_mem <= wt::cross_fold(d.dtype) ? 0
                                  : P.ctas * (wide ? wt::cross_wide_fold(d.head_dim) : wt::cross_few_fold(P.rows, d.head_dim)));
  Lock lock(h);
  wt::ServeWorkspace w;
  CHECK(wt::serve_workspace(h, s, bytes, &w));
  uint8_t *ws = static_cast<uint8_t *>(w.p);
  P.o = reinterpret_cast<float *>(ws + o);
  P.ml = reinterpret_cast<float2 *>(ws + ml);
  P.cuts = reinterpret_cast<wt::CrossCut *>(ws + cuts);
  P.fold = reinterpret_cast<float4 *>(ws + fold);
  const bool joined = d.max_mem > P.keys;  // memories of one cell: no row tile has two parts.  Else there are two CTAs at least.
  cudaError_t e = wide ? wt::launch_cross_wide(P, maps, s) : wt::launch_cross_few(P, maps, s);
  if (e == cudaSuccess && joined) e = wt::launch_cross_merge(P, s);
  const int rc = wt::serve_done(h, s, w);
  CU(e);
  wt::serve_launched(h, 1 + joined);
  return rc;
}

int probs_impl(wt_handle *h, const wt_probs_desc *d, cudaStream_t s) {
  const char *call = "wt_probs";
  wt::ServeRanges seen;
  wt::ServeContext ctx;
  CHECK(wt::serve_context(h, call, wt::kServeDraw, &ctx));
  if (!d) return serve_error(WT_EINVAL, "%s: NULL descriptor", call);
  if (d->rows < 0 || d->rows > (1 << 27) || d->vocab < 0 || d->vocab > (1 << 30) || d->ldl < d->vocab || d->ldp < d->vocab ||
      d->ldl > kMaxPitch || d->ldp > kMaxPitch)
    return serve_error(WT_EINVAL, "%s: rows %d, vocab %d or a pitch out of range", call, d->rows, d->vocab);
  if (d->rows == 0 || d->vocab == 0) return WT_OK;
  const uint64_t rows = d->rows, V = d->vocab;
  CHECK(check_buffer(&seen, call, "logits", d->logits, extent(rows, d->ldl, V, 4), 4));
  CHECK(check_output(h, &seen, call, "p", d->p, extent(rows, d->ldp, V, 4), 4));
  const Rows p("p", d->p, rows, 4 * d->ldp, 4 * V);
  if (d->p == d->logits ? d->ldp != d->ldl : overlap(p, {"logits", d->logits, rows, 4 * (uint64_t)d->ldl, 4 * V}))
    return serve_error(WT_EINVAL, "%s: p overlaps the logits", call);
  if (d->temp) CHECK(check_buffer(&seen, call, "temp", d->temp, 4 * rows, 4));
  if (d->temp && overlap(p, {"temp", d->temp, 4 * rows})) return serve_error(WT_EINVAL, "%s: p overlaps temp", call);
  return launch_alone(h, s, [&] { return wt::launch_probs(*d, ctx.status, s); });
}

int check_place(wt_handle *h, const wt_place_desc &d) {
  const char *call = "wt_place";
  wt::ServeRanges seen;
  if (d.dtype != WT_BF16 && d.dtype != WT_F16)
    return serve_error(d.dtype >= WT_F32 && d.dtype <= WT_U8 ? WT_ENOTSUP : WT_EINVAL,
                       "%s: dtype %d: caches and q_out are bf16 or f16", call, d.dtype);
  if (d.in_dtype != WT_F32 && d.in_dtype != d.dtype)
    return serve_error(d.in_dtype >= WT_F32 && d.in_dtype <= WT_U8 ? WT_ENOTSUP : WT_EINVAL,
                       "%s: in_dtype %d: q, k and v are fp32 or of the caches' type", call, d.in_dtype);
  const bool kv = d.k || d.v, norms = d.q_norm || d.k_norm;
  if (norms && d.norm_dtype != WT_F32 && d.norm_dtype != WT_BF16 && d.norm_dtype != WT_F16)
    return serve_error(d.norm_dtype >= WT_F32 && d.norm_dtype <= WT_U8 ? WT_ENOTSUP : WT_EINVAL,
                       "%s: norm_dtype %d: norms are fp32, bf16 or f16", call, d.norm_dtype);
  if (d.n_req < 0 || d.n_req >= kMaxSize || d.n_tokens < 0 || d.n_tokens > kMaxSize || d.max_len < 0 || d.max_len > kMaxSize ||
      d.n_pages < 0)
    return serve_error(WT_EINVAL, "%s: n_req %d, n_tokens %d, max_len %d or n_pages %d out of range", call, d.n_req, d.n_tokens, d.max_len,
                       d.n_pages);
  if ((d.q && (d.heads < 1 || d.heads > 65536)) || (kv && (d.kv_heads < 1 || d.kv_heads > 65536)))
    return serve_error(WT_EINVAL, "%s: heads %d or kv_heads %d is not from 1 to 65536", call, d.heads, d.kv_heads);
  if (d.head_dim < 8 || d.head_dim % 8) return serve_error(WT_EINVAL, "%s: head_dim %d is not a multiple of 8", call, d.head_dim);
  if (d.head_dim > WT_PLACE_MAX_DIM) return serve_error(WT_ENOTSUP, "%s: head_dim %d is above %d", call, d.head_dim, WT_PLACE_MAX_DIM);
  if (d.rot_dim < 0 || d.rot_dim % 8 || d.rot_dim > d.head_dim)
    return serve_error(WT_EINVAL, "%s: rot_dim %d is not a multiple of 8 up to head_dim", call, d.rot_dim);
  if (d.flags & ~WT_PLACE_NEIGHBOURS) return serve_error(WT_EINVAL, "%s: unknown flags 0x%x", call, (unsigned)d.flags);
  if (norms && !(d.eps >= 0.0f && std::isfinite(d.eps))) return serve_error(WT_EINVAL, "%s: eps is not a finite number from 0 on", call);
  const bool turned = d.rot_dim && (d.q || d.k), by_place = turned && !d.pos;
  if (by_place && (d.first_pos < 0 || d.first_pos > kMaxSize))
    return serve_error(WT_EINVAL, "%s: first_pos %d is not from 0 to 2^30", call, d.first_pos);
  if (turned && d.pos) {
    if (d.axes < 1 || d.axes > WT_PLACE_MAX_AXES || d.pos_stride < d.axes || d.pos_stride > kMaxPitch)
      return serve_error(WT_EINVAL, "%s: axes %d is not from 1 to %d, or the pitch of pos not at least that", call, d.axes, WT_PLACE_MAX_AXES);
    for (int j = 0; j < d.rot_dim / 2; ++j)
      if (d.axis[j] >= d.axes) return serve_error(WT_EINVAL, "%s: pair %d has axis %d of %d", call, j, d.axis[j], d.axes);
  }
  const uint64_t N = d.n_tokens, D = d.head_dim, H = d.q ? d.heads : 0, Hkv = kv ? d.kv_heads : 0, in = d.in_dtype == WT_F32 ? 4 : 2;
  auto pitch = [&](const void *p, int64_t stride, uint64_t heads) {
    return !p || (stride >= (int64_t)(heads * D) && stride % 8 == 0 && stride <= kMaxPitch);
  };
  if (!pitch(d.q, d.q_stride, H) || !pitch(d.q, d.out_stride, H) || !pitch(d.k, d.k_stride, Hkv) || !pitch(d.v, d.v_stride, Hkv))
    return serve_error(WT_EINVAL, "%s: a token pitch is not a multiple of 8 of at least heads * head_dim", call);
  if (!d.begin && (kv || by_place))
    return serve_error(WT_EINVAL, "%s: without begin tokens have no place: no k, no v and no rotation without pos", call);
  if (N == 0 || (!d.q && !kv) || (d.begin && d.n_req == 0)) return WT_OK;
  const uint64_t B = d.n_req, kv_row = Hkv * D, q_row = H * D, norm = d.norm_dtype == WT_F32 ? 4 : 2;
  const Rows none("", nullptr, 0);
  Rows outs[3] = {none, none, none}, reads[10] = {none, none, none, none, none, none, none, none, none, none};
  int n_reads = 0;
  // q_out may be q: what a lane writes, it alone reads, before
  const bool in_place = d.q && d.q_out == d.q && in == 2 && d.q_stride == d.out_stride;
  auto read = [&](const char *name, const void *p, uint64_t rows, uint64_t pitch_bytes, uint64_t row, uintptr_t align) -> int {
    CHECK(check_buffer(&seen, call, name, p, extent(rows, pitch_bytes, row, 1), align));
    reads[n_reads++] = Rows(name, p, rows, pitch_bytes, row);
    return WT_OK;
  };
  if (d.q) {
    CHECK(read("q", d.q, N, in * d.q_stride, in * q_row, 16));
    CHECK(check_output(h, &seen, call, "q_out", d.q_out, extent(N, d.out_stride, q_row, 2), 16));
    outs[0] = Rows("q_out", d.q_out, N, 2 * (uint64_t)d.out_stride, 2 * q_row);
    if (d.q_norm) CHECK(read("q_norm", d.q_norm, 1, 0, D * norm, norm));
  }
  if (kv) {
    if (d.page < 1 || d.table_stride < 0 || d.table_stride > 0x7fffffff || (int64_t)d.max_len > d.table_stride * d.page)
      return serve_error(WT_EINVAL, "%s: max_len %d does not fit %lld pages of %d keys", call, d.max_len, (long long)d.table_stride,
                         d.page);
    const uint64_t n = (Bytes(d.n_pages) * d.page * d.kv_heads * D * 2).n;
    if (d.k) {
      CHECK(read("k", d.k, N, in * d.k_stride, in * kv_row, 16));
      CHECK(check_output(h, &seen, call, "k_pages", d.k_pages, n, 16));
      outs[1] = Rows("k_pages", d.k_pages, n);
      if (d.k_norm) CHECK(read("k_norm", d.k_norm, 1, 0, D * norm, norm));
    }
    if (d.v) {
      CHECK(read("v", d.v, N, in * d.v_stride, in * kv_row, 16));
      CHECK(check_output(h, &seen, call, "v_pages", d.v_pages, n, 16));
      outs[2] = Rows("v_pages", d.v_pages, n);
    }
    const uint64_t pages = ceil_div(d.max_len, d.page);
    CHECK(read("table", d.table, B, 4 * (uint64_t)d.table_stride, 4 * pages, 4));
  }
  if (d.begin) CHECK(read("begin", d.begin, 1, 0, 4 * (B + 1), 4));
  if (kv || by_place) CHECK(read("len", d.len, 1, 0, 4 * B, 4));
  if (turned) {
    CHECK(read("turns", d.turns, 1, 0, 4 * (uint64_t)d.rot_dim, 8));
    if (d.pos) CHECK(read("pos", d.pos, N, 4 * (uint64_t)d.pos_stride, 4 * (uint64_t)d.axes, 4));
  }
  for (int i = 0; i < 3; ++i) {
    for (int j = 0; j < n_reads; ++j)
      if (!(i == 0 && j == 0 && in_place) && overlap(outs[i], reads[j]))
        return serve_error(WT_EINVAL, "%s: %s overlaps %s", call, outs[i].name, reads[j].name);
    for (int j = 0; j < i; ++j)
      if (overlap(outs[i], outs[j])) return serve_error(WT_EINVAL, "%s: %s overlaps %s", call, outs[i].name, outs[j].name);
  }
  return WT_OK;
}

int place_impl(wt_handle *h, const wt_place_desc *dp, cudaStream_t s) {
  wt::ServeContext ctx;
  CHECK(wt::serve_context(h, "wt_place", wt::kServePlain, &ctx));
  if (!dp) return serve_error(WT_EINVAL, "wt_place: NULL descriptor");
  CHECK(check_place(h, *dp));
  wt::PlacePlan P = {};
  P.d = *dp;
  wt_place_desc &d = P.d;
  if (d.n_tokens == 0 || (!d.q && !d.k && !d.v) || (d.begin && d.n_req == 0)) return WT_OK;
  // what is not asked for is not looked at
  if (!d.q) d.q_norm = nullptr;
  if (!d.k) d.k_norm = nullptr;
  if (!d.k && !d.v) d.table = nullptr;
  if (!d.q && !d.k) d.rot_dim = 0;  // values are not turned
  if (!d.rot_dim) d.turns = nullptr, d.pos = nullptr;
  if (!d.k && !d.v && (d.pos || !d.rot_dim || !d.q)) d.len = nullptr;
  P.status = ctx.status;
  wt::plan_place(&P);
  return launch_alone(h, s, [&] { return wt::launch_place(P, s); });
}

int logprobs_impl(wt_handle *h, const wt_logprobs_desc *d, cudaStream_t s) {
  const char *call = "wt_logprobs";
  wt::ServeRanges seen;
  wt::ServeContext ctx;
  CHECK(wt::serve_context(h, call, wt::kServePlain, &ctx));
  if (!d) return serve_error(WT_EINVAL, "%s: NULL descriptor", call);
  if (d->rows < 0 || d->rows > (1 << 27) || d->vocab < 0 || d->vocab > (1 << 30) || d->ldl < d->vocab || d->ldl > kMaxPitch)
    return serve_error(WT_EINVAL, "%s: rows %d, vocab %d or a pitch out of range", call, d->rows, d->vocab);
  if (d->n_given < 0 || d->n_given > (1 << 20) || d->n_top < 0 || d->n_top > WT_LOGPROBS_MAX_TOP ||
      (d->given && (d->given_stride < d->n_given || d->given_stride > kMaxPitch)))
    return serve_error(WT_EINVAL, "%s: n_given %d (up to 2^20), its pitch, or n_top %d (up to %d) out of range", call, d->n_given, d->n_top,
                       WT_LOGPROBS_MAX_TOP);
  wt_logprobs_desc e = *d;
  if (!e.given) e.n_given = 0;
  if (!e.top) e.n_top = 0;
  if (e.rows == 0 || (!e.n_given && !e.n_top && !e.entropy)) return WT_OK;
  const uint64_t rows = e.rows, V = e.vocab, given = 4 * (uint64_t)e.n_given, top = 4 * (uint64_t)e.n_top;
  CHECK(check_buffer(&seen, call, "logits", e.logits, extent(rows, e.ldl, V, 4), 4));
  if (e.temp) CHECK(check_buffer(&seen, call, "temp", e.temp, 4 * rows, 4));
  if (given) {
    CHECK(check_buffer(&seen, call, "given", e.given, extent(rows, e.given_stride, e.n_given, 4), 4));
    CHECK(check_output(h, &seen, call, "given_lp", e.given_lp, rows * given, 4));
  }
  if (e.entropy) CHECK(check_output(h, &seen, call, "entropy", e.entropy, 4 * rows, 4));
  if (top) {
    CHECK(check_output(h, &seen, call, "top", e.top, rows * top, 4));
    CHECK(check_output(h, &seen, call, "top_lp", e.top_lp, rows * top, 4));
  }
  const Rows outs[] = {{"given_lp", e.given_lp, rows * given}, {"entropy", e.entropy, e.entropy ? 4 * rows : 0},
                       {"top", e.top, rows * top}, {"top_lp", e.top_lp, rows * top}};
  const Rows reads[] = {{"the logits", e.logits, rows, 4 * (uint64_t)e.ldl, 4 * V}, {"temp", e.temp, e.temp ? 4 * rows : 0},
                        {"given", e.given, e.n_given ? rows : 0, 4 * (uint64_t)e.given_stride, given}};
  for (const Rows &o : outs) {
    for (const Rows &r : reads)
      if (overlap(o, r)) return serve_error(WT_EINVAL, "%s: %s overlaps %s", call, o.name, r.name);
    for (const Rows &p : outs)
      if (&p < &o && overlap(o, p)) return serve_error(WT_EINVAL, "%s: %s overlaps %s", call, o.name, p.name);
  }
  wt::LogprobsPlan P = {};
  P.d = e;
  P.status = ctx.status;
  const size_t bytes = wt::plan_logprobs(&P);
  Lock lock(h);
  wt::ServeWorkspace w;
  CHECK(wt::serve_workspace(h, s, bytes, &w));
  P.sums = static_cast<float4 *>(w.p);
  P.keys = reinterpret_cast<unsigned long long *>(P.sums + 2 * (size_t)P.ctas);
  const cudaError_t err = wt::launch_logprobs(P, s);
  const int rc = wt::serve_done(h, s, w);
  CU(err);
  wt::serve_launched(h, 1 + P.split);
  return rc;
}

int verify_impl(wt_handle *h, const wt_verify_desc *d, cudaStream_t s) {
  const char *call = "wt_verify";
  wt::ServeRanges seen;
  wt::ServeContext ctx;
  CHECK(wt::serve_context(h, call, wt::kServeDraw, &ctx));
  if (!d) return serve_error(WT_EINVAL, "%s: NULL descriptor", call);
  if (d->n_req < 0 || d->n_req > (1 << 24) || d->n_drafted < 0 || d->n_drafted > kMaxSize || d->max_draft < 0 || d->max_draft > (1 << 20) || d->vocab < 1 ||
      d->vocab > WT_VERIFY_MAX_VOCAB || d->ldp < d->vocab || d->ldp > kMaxPitch ||
      (d->q && (d->ldq < d->vocab || d->ldq > kMaxPitch)))
    return serve_error(WT_EINVAL, "%s: n_req %d, n_drafted %d, max_draft %d, vocab %d (up to %d) or a pitch out of range", call,
                       d->n_req, d->n_drafted, d->max_draft, d->vocab, WT_VERIFY_MAX_VOCAB);
  if (d->n_req == 0) return WT_OK;
  const uint64_t B = d->n_req, n = d->n_drafted;
  CHECK(check_buffer(&seen, call, "p", d->p, extent(n + B, d->ldp, d->vocab, 4), 4));
  if (d->q) CHECK(check_buffer(&seen, call, "q", d->q, extent(n, d->ldq, d->vocab, 4), 4));
  CHECK(check_buffer(&seen, call, "drafted", d->drafted, 4 * n, 4));
  CHECK(check_buffer(&seen, call, "begin", d->begin, 4 * (B + 1), 4));
  CHECK(check_buffer(&seen, call, "u", d->u, 4 * n, 4));
  CHECK(check_buffer(&seen, call, "u_draw", d->u_draw, 4 * B, 4));
  CHECK(check_output(h, &seen, call, "accepted", d->accepted, 4 * B, 4));
  CHECK(check_output(h, &seen, call, "tokens", d->tokens, 4 * B * ((uint64_t)d->max_draft + 1), 4));
  const uint64_t V = d->vocab;
  const Rows accepted("accepted", d->accepted, 4 * B), tokens("tokens", d->tokens, 4 * B * ((uint64_t)d->max_draft + 1));
  const Rows reads[] = {{"p", d->p, n + B, 4 * (uint64_t)d->ldp, 4 * V}, {"q", d->q, d->q ? n : 0, 4 * (uint64_t)d->ldq, 4 * V},
                        {"drafted", d->drafted, 4 * n},                  {"begin", d->begin, 4 * (B + 1)},
                        {"u", d->u, 4 * n},                              {"u_draw", d->u_draw, 4 * B}};
  for (const Rows &r : reads)
    for (const Rows *o : {&accepted, &tokens})
      if (overlap(*o, r)) return serve_error(WT_EINVAL, "%s: %s overlaps %s", call, o->name, r.name);
  if (overlap(accepted, tokens)) return serve_error(WT_EINVAL, "%s: accepted overlaps tokens", call);
  return launch_alone(h, s, [&] { return wt::launch_verify(*d, ctx.status, s); });
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

int wt_adapt(wt_handle *h, const wt_adapt_desc *d, size_t n, void *stream) {
  return adapt_impl(h, d, n, static_cast<cudaStream_t>(stream));
}

int wt_place(wt_handle *h, const wt_place_desc *d, void *stream) {
  return place_impl(h, d, static_cast<cudaStream_t>(stream));
}

int wt_attend(wt_handle *h, const wt_attend_desc *d, void *stream) {
  return attend_impl(h, d, static_cast<cudaStream_t>(stream));
}

int wt_cross(wt_handle *h, const wt_cross_desc *d, void *stream) {
  return cross_impl(h, d, static_cast<cudaStream_t>(stream));
}

int wt_probs(wt_handle *h, const wt_probs_desc *d, void *stream) {
  return probs_impl(h, d, static_cast<cudaStream_t>(stream));
}

int wt_logprobs(wt_handle *h, const wt_logprobs_desc *d, void *stream) {
  return logprobs_impl(h, d, static_cast<cudaStream_t>(stream));
}

int wt_verify(wt_handle *h, const wt_verify_desc *d, void *stream) {
  return verify_impl(h, d, static_cast<cudaStream_t>(stream));
}

}  // extern "C"
#pragma GCC visibility pop
