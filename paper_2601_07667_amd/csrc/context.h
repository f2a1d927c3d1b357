// The context behind the C ABI, and what its entry points share: messages, the device that is current during a call, checks.
#pragma once
#include <cstdarg>
#include <cstdio>

#include "asl_internal.h"
#include "paged.h"

struct asl_ctx {
  int device;
  int32_t max_seq_len, max_kv_heads, max_q_rows;
  void* base;
  size_t bytes;
  asl::Workspace ws;
  asl::Prof prof;
  hipStream_t side;          // second stream of asl_layer_step's fork/join (default priority)
  hipEvent_t ev_fork, ev_join;
  bool side_pending;         // a deferred asl_layer_step left work on `side` that nobody has waited for yet
  asl::PagedWorkspace paged; // asl_paged_reserve's; all null before it
  void* paged_kept[asl::kPagedKept];   // workspaces that it has outgrown: queued calls and captured graphs may use them
  int n_paged_kept;
  char err[256];
};

namespace {

inline size_t align_up(size_t x) { return (x + 255) & ~size_t(255); }

inline asl_status fail(asl_ctx* ctx, asl_status st, const char* fmt, ...) {
  if (ctx) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(ctx->err, sizeof(ctx->err), fmt, ap);
    va_end(ap);
  }
  return st;
}

inline asl_status hip_fail(asl_ctx* ctx, hipError_t e, const char* what) {
  return fail(ctx, ASL_EHIP, "%s: %s", what, hipGetErrorString(e));
}

// Makes ctx->device current for the duration of a call and restores the caller's device.
struct DeviceGuard {
  int prev = -1;
  bool switched = false;
  hipError_t err = hipSuccess;
  explicit DeviceGuard(int dev) {
    err = hipGetDevice(&prev);
    if (err == hipSuccess && prev != dev) {
      err = hipSetDevice(dev);
      switched = (err == hipSuccess);
    }
  }
  ~DeviceGuard() {
    if (switched) (void)hipSetDevice(prev);
  }
};

inline int elem_bytes(int dtype) { return dtype == ASL_BF16 ? 2 : 4; }

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace
