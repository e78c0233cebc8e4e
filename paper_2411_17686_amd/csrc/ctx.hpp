// The context behind the C ABI and the checks that all of its entry points share.
#pragma once
#include <cstdio>

#include "common.hpp"

struct ficoco_ctx {
  int device;
  hipEvent_t probe_start, probe_stop;   // measurement hook, both null when off
  int probe_kernel;
  char err[512];
};

namespace ficoco {

inline int fail(ficoco_ctx* ctx, int code, const char* what, const char* detail) {
  if (ctx) std::snprintf(ctx->err, sizeof(ctx->err), "%s: %s", what, detail ? detail : "");
  return code;
}

// The calling thread's current device must be the one the ctx was created for: every launch
// goes to the current device, and the caller's pointers and stream belong to it.
inline int check_device(ficoco_ctx* ctx, const char* fn) {
  int cur = -1;
  if (hipGetDevice(&cur) != hipSuccess) return fail(ctx, FICOCO_EHIP, fn, "hipGetDevice failed");
  if (cur != ctx->device) return fail(ctx, FICOCO_EINVAL, fn, "the current device is not the device this ctx was created for");
  return FICOCO_OK;
}

// Do the byte ranges [a, a + na) and [b, b + nb) overlap?
inline bool ranges_overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t a0 = (uintptr_t)a, b0 = (uintptr_t)b;
  return a && b && na && nb && a0 < b0 + nb && b0 < a0 + na;
}

inline int finish(ficoco_ctx* ctx, const char* fn) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return fail(ctx, FICOCO_EHIP, fn, hipGetErrorString(e));
  return FICOCO_OK;
}

}  // namespace ficoco
