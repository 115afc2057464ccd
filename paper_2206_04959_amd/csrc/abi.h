// Argument checks shared by the C entry points (host side).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "merak_stage.h"

namespace merak {

inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p % a) == 0; }

inline int check_ptr(const void* p) {
  if (!p) return MERAK_ERR_INVALID_ARG;
  if (!aligned(p, 16)) return MERAK_ERR_ALIGN;
  return MERAK_OK;
}

}  // namespace merak

#define TRY(expr)               \
  do {                          \
    int r_ = (expr);            \
    if (r_ != MERAK_OK) return r_; \
  } while (0)

#define HIP_TRY(expr)                          \
  do {                                         \
    hipError_t e_ = (expr);                    \
    if (e_ != hipSuccess) return MERAK_ERR_HIP; \
  } while (0)
