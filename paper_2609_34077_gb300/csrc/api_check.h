// What the C ABI's files beside api.cu share: error returns with a message, and alignment tests. Not part of the C
// ABI.
#pragma once

#include <cuda_runtime.h>
#include <stdarg.h>
#include <stdio.h>

#include "internal.h"

namespace mcft {

__attribute__((format(printf, 2, 3))) inline mcft_status fail(mcft_status st, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  return set_error_message(st, buf);
}

inline mcft_status cuda_fail(cudaError_t e, const char* where) {
  return fail(e == cudaErrorMemoryAllocation ? MCFT_ERR_OOM : MCFT_ERR_CUDA, "%s: %s", where, cudaGetErrorString(e));
}

inline bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

}  // namespace mcft
