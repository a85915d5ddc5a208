// Argument checks that the entry points of the trained tail and block share.
#pragma once

#include "internal.h"

namespace hapi {
namespace {

#define HIP_TRY(expr)                                                                  \
  do {                                                                                 \
    hipError_t e_ = (expr);                                                            \
    if (e_ != hipSuccess)                                                              \
      return fail(HAPI_E_DEVICE, "%s failed: %s", #expr, hipGetErrorString(e_));       \
  } while (0)

constexpr int64_t kAlign = 256;

int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

// The tensors of a call lie on the current device, and so must its stream.
int check_stream(void *stream) {
  int dev = -1, cur = -1;
  HIP_TRY(hipStreamGetDevice(static_cast<hipStream_t>(stream), &dev));
  HIP_TRY(hipGetDevice(&cur));
  if (dev != cur) return fail(HAPI_E_INVAL, "desc->stream belongs to device %d, current device is %d", dev, cur);
  return HAPI_OK;
}

int check_workspace(const void *ws, size_t have, int64_t need) {
  if (need > 0 && (!ws || (int64_t)have < need))
    return fail(HAPI_E_NOMEM, "workspace of %zu bytes, %lld needed", have, (long long)need);
  if ((uintptr_t)ws % kAlign) return fail(HAPI_E_INVAL, "workspace must be 256-byte aligned");
  return HAPI_OK;
}

int check_ptr(const void *p, size_t align, const char *name) {
  if (!p) return fail(HAPI_E_INVAL, "%s is NULL", name);
  if ((uintptr_t)p % align) return fail(HAPI_E_INVAL, "%s must be %zu-byte aligned", name, align);
  return HAPI_OK;
}
#define TRY(expr)                    \
  do {                               \
    const int r_ = (expr);           \
    if (r_ != HAPI_OK) return r_;    \
  } while (0)

}  // namespace
}  // namespace hapi
