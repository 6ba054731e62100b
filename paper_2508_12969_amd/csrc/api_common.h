// Small pieces of argument checking that the files of entry points share.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "layout.h"

namespace ca {

inline int fail(int status, const char* what) {
  set_error("%s", what);
  return status;
}

inline int hip_fail(hipError_t e, const char* where) {
  set_error("%s: %s", where, hipGetErrorString(e));
  return CA_ERR_HIP;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int elem_size(int32_t dtype) { return dtype == CA_BF16 ? 2 : 4; }

// Do the byte ranges [a, a + na) and [b, b + nb) share a byte?
inline bool ranges_overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
  return a0 < b0 + (uintptr_t)nb && b0 < a0 + (uintptr_t)na;
}

// Makes sure the layout's tables are on the current device (api.cpp).
int ensure_uploaded(ca_layout* L, hipStream_t stream);

}  // namespace ca
