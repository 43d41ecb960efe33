// The context behind the C ABI and what every entry point does with it: error texts, workspace checks.
#pragma once

#include <stdarg.h>
#include <stdio.h>

#include "cc_internal.cuh"

struct cc_ctx {
  int device;
  int sm_count;
  cc::SelectRoom select_room;
  cc::DeviceStatus* d_status;
  cc::DeviceStatus* h_status;   // pinned
  long long* d_probe;           // scratch of cc_exp_rate_probe: two words per SM
  void* encode_tiled;           // cuTensorMapEncodeTiled, resolved through the runtime
  char err[256];
};

namespace cc {

inline size_t align256(size_t x) { return (x + 255) / 256 * 256; }

inline int fail(cc_ctx* ctx, int code, const char* fmt, ...) __attribute__((format(printf, 3, 4)));
inline int fail(cc_ctx* ctx, int code, const char* fmt, ...) {
  if (ctx) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(ctx->err, sizeof(ctx->err), fmt, ap);
    va_end(ap);
  }
  return code;
}

inline int cuda_fail(cc_ctx* ctx, cudaError_t e, const char* what) {
  return fail(ctx, CC_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

inline int check_ws(cc_ctx* ctx, size_t need, void* ws, size_t ws_bytes) {
  if (!ws) return fail(ctx, CC_ERR_WORKSPACE, "workspace is NULL");
  if ((uintptr_t)ws % 256) return fail(ctx, CC_ERR_WORKSPACE, "workspace is not 256-byte aligned");
  if (ws_bytes < need)
    return fail(ctx, CC_ERR_WORKSPACE, "workspace has %zu bytes, %zu needed", ws_bytes, need);
  return CC_OK;
}

inline Launch make_launch(cc_ctx* ctx, void* stream) {
  Launch L;
  L.stream = (cudaStream_t)stream;
  L.status = ctx->d_status;
  L.sm_count = ctx->sm_count;
  return L;
}

}  // namespace cc
