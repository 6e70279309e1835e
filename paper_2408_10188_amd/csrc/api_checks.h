// What the files of the C-ABI layer share: the error message of the calling thread and the checks of common arguments.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/mmsp.h"

namespace mmsp {

constexpr int64_t kMaxExtent = (int64_t)1 << 30;   // rows and positions are int32 inside the kernels

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

mmsp_status fail(mmsp_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
mmsp_status check_shape(const mmsp_shape* s);
mmsp_status device_result(hipError_t e, const char* what);

}  // namespace mmsp
