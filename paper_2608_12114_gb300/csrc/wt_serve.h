// Internal interface between wt_serve.cpp (argument checks, routing), the handle's owner
// (wt_host.cpp) and the kernels of a serving step.  Not part of the public C ABI.
#pragma once

#include <cstddef>
#include <cstdint>

#include <cuda_runtime.h>

#include "../../include/wt_serve.h"

namespace wt {

// ---------------------------------------------------------------- the handle (wt_host.cpp)
struct ServeContext {
  int device;
  int *status;  // device status word
};
// Kernels whose one-time attributes are set by the first call that may launch them (all of them in wt_open
// took 1.7 of a process's first 20 ms).
enum ServeKernels { kServeAdapt, kServeAttend, kServeDraw, kServeKernels };
int serve_prepare(int device, ServeKernels k);
// Refuses NULL and host-only handles, and prepares the call's kernels.
int serve_context(wt_handle *h, const char *call, ServeKernels kernels, ServeContext *out);
bool serve_inside_mapping(const wt_handle *h, const void *p, uint64_t n);
// Device allocations that a call has met: its small buffers often share one, and each look-up costs
// the driver's time.
struct ServeRanges {
  static constexpr int kMost = 8;
  uintptr_t lo[kMost], hi[kMost];
  int n = 0;
};
// false only when [p, p + n) starts inside a device allocation and runs past its end
bool serve_range_ok(const void *p, uint64_t n, ServeRanges *seen);
void serve_launched(wt_handle *h, int kernels);
// The handle's mutex, held from serve_workspace to serve_done.
void serve_lock(wt_handle *h);
void serve_unlock(wt_handle *h);
// A workspace of at least n bytes for calls on stream s (256-byte aligned; none for 0).  The caller makes
// the matching serve_done after its last launch (also after a failed one): wt_close waits for it.
struct ServeWorkspace {
  void *p = nullptr;
  void *entry = nullptr;
};
int serve_workspace(wt_handle *h, cudaStream_t s, size_t n, ServeWorkspace *out);
int serve_done(wt_handle *h, cudaStream_t s, const ServeWorkspace &w);
// cuTensorMapEncodeTiled of a 16-bit tensor with the 128-byte swizzle; strides in bytes for dims 1..
int serve_tensor_map(void *out, const void *base, int rank, const uint64_t *dims, const uint64_t *strides,
                     const uint32_t *box);
int serve_error(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
int serve_cuda_error(cudaError_t e, const char *what);

// ---------------------------------------------------------------- wt_adapt.cu
constexpr int kAdaptProjs = 8;  // projections of one launch
constexpr int kAdaptMTile = 64;
// Whether a launch's work is planned on the device first: from 256 tokens on, as the one-launch kernel
// looks at each token in every CTA and reads a slot again for each 16 of its tokens.  (Earlier only
// where slots have many: 106 tokens of 4 adapters of rank 64, three projections: 28 us planned, 26 not.)
constexpr bool adapt_planned(int max_T) { return max_T >= 256; }
// 16-row tiles of the rank that the kernels are built for
constexpr int adapt_rank_tiles(int max_R) { return max_R <= 16 ? 1 : max_R <= 32 ? 2 : max_R <= 64 ? 4 : 8; }
struct AdaptProj {
  wt_adapt_desc d;
  uint32_t items;    // upper bound of (slot, token tile) work items
  uint32_t m_groups, group_tiles;  // many tokens: CTAs of an item, and the tiles of kAdaptMTile outputs that each takes
  uint32_t vec;      // bit 0: A and x load in 16-byte vectors; bit 1: B does; bit 2: base and y do
};
struct AdaptLaunch {
  AdaptProj p[kAdaptProjs];
  int n;
};
// Workspace of a launch of many tokens: a plan for each distinct slot map, and v of each projection.
struct AdaptWide {
  int *plans;          // [n_plans][plan_ints]: {items, -, -, -}, items as int4, tokens from order_at on
  uint16_t *v;         // 16-bit parts of v, [2 or 3][T][16 adapt_rank_tiles] a projection, in the plan's token order
  float *back;         // [T] a projection: what its token's v was divided by (f16)
  int64_t plan_ints, order_at;
  int64_t v_at[kAdaptProjs], back_at[kAdaptProjs];
  int plan[kAdaptProjs];      // a projection's plan
  int plan_proj[kAdaptProjs]; // a plan's first projection
  int n_plans;
};
cudaError_t adapt_prepare();
cudaError_t launch_adapt(const AdaptLaunch &L, const AdaptWide *W, int max_R, int *status, cudaStream_t s);

// ---------------------------------------------------------------- wt_draw.cu
cudaError_t draw_prepare();
cudaError_t launch_probs(const wt_probs_desc &d, int *status, cudaStream_t s);
cudaError_t launch_verify(const wt_verify_desc &d, int *status, cudaStream_t s);

// ---------------------------------------------------------------- wt_attend.cu, wt_prefix.cu
// Weights p = 2^(s - m) are rounded to the caches' type.  The reference m lies kBelow under the largest
// score (in log2) that set it, and follows a larger one when that is kSlack above it: p reaches 2^15 for
// f16 and 2^8 for bf16.  f16 rounds p below 2^-14 to multiples of 2^-24.  Without the seven bits of
// kBelow, 65535 keys of weight 2^-26 in one part gave 0 in place of 2^-10; with them even 2^20 keys that
// are lost weigh less together than the result's own rounding.
constexpr float kSlack = 8.0f;
template <int DT>
constexpr float kBelow = DT == WT_F16 ? 7.0f : 0.0f;

// Partial results of one (token, head): O [head_dim] fp32 not yet divided by l, and (m, l) with m in
// units of log2 (scores times scale log2 e).
//
// The shared prefix on tcgen05 (wt_prefix.cu): the key tiles (128 keys) of all kv heads in a row,
// head after head, are cut into `groups` ranges of `len` tiles (the last may be shorter); each range
// is taken by row_blocks CTAs of two row tiles each.  The part of range g that lies in head h is slot g + h.
struct PrefixPlan {
  int row_blocks, groups, len;
  int apart;        // one row tile: the two streams take the even and the odd key tiles of a segment
  int tiles;        // key tiles of a head
  int tile_tokens, tile_rows;  // whole tokens of a row tile (up to 128 rows), and its rows
  int qtiles;       // tiles of a slot: 2 row_blocks, or the 2 streams
  int rows;         // n_tokens * G
  int kv_heads, G, head_dim, dim_steps, prefix_len;
  float scale_log2;
  float *o;         // [groups + kv_heads - 1][qtiles][128][head_dim]
  float2 *ml;       // [groups + kv_heads - 1][qtiles][128]
};
struct PrefixMaps {
  alignas(64) uint8_t q[128];  // CUtensorMaps
  alignas(64) uint8_t k[128];
  alignas(64) uint8_t v[128];
};
cudaError_t prefix_prepare();
cudaError_t launch_attend_prefix(const PrefixPlan &P, const PrefixMaps &m, int dtype, int *status, cudaStream_t s);

struct AttendPlan {
  wt_attend_desc d;
  int G;          // heads / kv_heads
  int rows_tile;  // rows (token, head-in-group) of one CTA of the warp kernel: 16 or 32
  int own_tiles, pre_tiles;  // tiles of the longest request's rows, and of all rows (for the prefix)
  int own_splits, own_len;  // own keys per split
  int pre_splits, pre_len;  // prefix keys per split of the warp kernel (0: not taken there)
  bool direct;              // one split of own keys and no prefix: the warp kernel writes the result
  PrefixPlan x;             // the prefix on tcgen05 (x.groups 0: not taken there)
  float *o;                 // [own_splits + pre_splits][n_tokens * heads][head_dim]
  float2 *ml;               // [own_splits + pre_splits][n_tokens * heads]
  int *status;
};
cudaError_t attend_prepare();
cudaError_t launch_attend_warp(const AttendPlan &P, cudaStream_t s);
cudaError_t launch_attend_merge(const AttendPlan &P, cudaStream_t s);

}  // namespace wt
