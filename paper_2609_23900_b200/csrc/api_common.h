// What the entry points share: errors, the current device, timed launches.
#pragma once
#include <cuda_runtime.h>

#include <string>

#include "internal.h"

namespace lumo {

inline thread_local std::string g_create_err;

inline int fail(lumo_ctx* ctx, int code, const std::string& msg) {
  if (ctx) ctx->err = msg; else g_create_err = msg;
  return code;
}

inline int cuda_fail(lumo_ctx* ctx, cudaError_t e, const char* what) {
  return fail(ctx, LUMO_ERR_CUDA, std::string(what) + ": " + cudaGetErrorString(e));
}

// End of a call: the status of its last launch, and what stands in front of the next call from now on.
inline int launched(lumo_ctx* ctx, cudaError_t e, CallOrder::Kind kind, const char* what) {
  if (e != cudaSuccess) return cuda_fail(ctx, e, what);
  ctx->order.done(kind);
  return LUMO_OK;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

struct DeviceGuard {
  int prev = -1;       // device to go back to; -1: nothing was changed
  bool ok = true;
  explicit DeviceGuard(int dev) {
    int cur = -1;
    if (cudaGetDevice(&cur) != cudaSuccess) { ok = false; return; }
    if (cur == dev) return;
    prev = cur;
    if (cudaSetDevice(dev) != cudaSuccess) ok = false;
  }
  ~DeviceGuard() { if (prev >= 0) cudaSetDevice(prev); }
};

constexpr size_t kTimingPool = 16384;

// Brackets one launch with events when timing is on.
template <typename F>
cudaError_t timed(lumo_ctx* ctx, int kind, cudaStream_t st, F launch) {
  const bool on = ctx->timing && ctx->ev_kind.size() < kTimingPool;
  size_t i = ctx->ev_kind.size();
  if (on) {
    cudaError_t e = cudaEventRecord(ctx->ev_start[i], st);
    if (e != cudaSuccess) return e;
  }
  cudaError_t e = launch();
  if (on && e == cudaSuccess) {
    e = cudaEventRecord(ctx->ev_stop[i], st);
    if (e == cudaSuccess) ctx->ev_kind.push_back(kind);
  }
  return e;
}

}  // namespace lumo
