// The host code of the serving calls without a GPU: the handle, the workspaces and the launches are records of what
// they were given.  Linked with wt_serve.cpp by test_serve_plans.py.
#include <cstdarg>
#include <cstdio>

#include "../paper_2608_12114_gb300/csrc/wt_kernels.h"
#include "../paper_2608_12114_gb300/csrc/wt_serve.h"

#define HOST extern "C" __attribute__((visibility("default")))

namespace {
char error[512];
wt::PlacePlan place;
wt::CrossPlan cross;
int launches, counted;  // kernels launched, and what the handle was told of them
alignas(256) uint8_t workspace[256];
cudaError_t launched(int n = 1) {
  launches += n;
  return cudaSuccess;
}
}  // namespace

HOST const char *host_error() { return error; }
HOST const wt_place_desc *host_place() { return &place.d; }
HOST int host_cross_ctas() { return cross.ctas; }
HOST int host_row_tiles(int n, int G, int rows) { return wt::cross_row_tiles(n, G, rows); }
HOST void host_reset() { launches = counted = 0, place = {}, cross = {}; }
HOST int host_launches() { return launches; }
HOST int host_counted() { return counted; }

namespace wt {

int num_sms() { return 152; }
int serve_context(wt_handle *, const char *, ServeKernels, ServeContext *out) {
  *out = {0, nullptr};
  return WT_OK;
}
bool serve_inside_mapping(const wt_handle *, const void *, uint64_t) { return false; }
bool serve_range_ok(const void *, uint64_t, ServeRanges *) { return true; }
void serve_launched(wt_handle *, int kernels) { counted += kernels; }
void serve_lock(wt_handle *) {}
void serve_unlock(wt_handle *) {}
int serve_workspace(wt_handle *, cudaStream_t, size_t, ServeWorkspace *out) {
  out->p = workspace;
  return WT_OK;
}
int serve_done(wt_handle *, cudaStream_t, const ServeWorkspace &) { return WT_OK; }
int serve_tensor_map(void *, const void *, int, const uint64_t *, const uint64_t *, const uint32_t *) { return WT_OK; }
int serve_error(int code, const char *fmt, ...) {
  va_list a;
  va_start(a, fmt);
  vsnprintf(error, sizeof(error), fmt, a);
  va_end(a);
  return code;
}
int serve_cuda_error(cudaError_t, const char *) { return WT_ECUDA; }

cudaError_t launch_adapt(const AdaptLaunch &, const AdaptWide *, int, int *, cudaStream_t) { return launched(); }
cudaError_t launch_probs(const wt_probs_desc &, int *, cudaStream_t) { return launched(); }
cudaError_t launch_verify(const wt_verify_desc &, int *, cudaStream_t) { return launched(); }
void plan_place(PlacePlan *) {}
cudaError_t launch_place(const PlacePlan &P, cudaStream_t) {
  place = P;
  return launched();
}
size_t plan_logprobs(LogprobsPlan *) { return 0; }
cudaError_t launch_logprobs(const LogprobsPlan &, cudaStream_t) { return launched(); }
cudaError_t launch_attend_prefix(const PrefixPlan &, const PrefixMaps &, int, int *, cudaStream_t) { return launched(); }
cudaError_t launch_attend_warp(const AttendPlan &, cudaStream_t) { return launched(); }
cudaError_t launch_attend_merge(const AttendPlan &, cudaStream_t) { return launched(); }
int cross_few_keys(int head_dim) { return head_dim <= 64 ? 32 : 16; }
cudaError_t launch_cross_few(const CrossPlan &P, const CrossMaps &, cudaStream_t) {
  cross = P;
  return launched();
}
cudaError_t launch_cross_wide(const CrossPlan &P, const CrossMaps &, cudaStream_t) {
  cross = P;
  return launched();
}
cudaError_t launch_cross_merge(const CrossPlan &, cudaStream_t) { return launched(); }

}  // namespace wt
