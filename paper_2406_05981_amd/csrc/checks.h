// Checks of arguments that the entry points share.
#ifndef SHIFTADD_CHECKS_H
#define SHIFTADD_CHECKS_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "shiftadd.h"

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

inline int check_dims(int q, int N, int K) {
    if (q < 1 || q > SA_MAX_Q) return SA_ERR_Q;
    if (N < 1 || K < 8 || (K & 7)) return SA_ERR_SHAPE;
    // every element count that the kernels index must fit comfortably; one
    // plane of packed keys stays below 2^31 bytes (32-bit per-lane offsets)
    if ((int64_t)q * N * K > (int64_t)1 << 36) return SA_ERR_SHAPE;
    if ((int64_t)N * (K / 8) >= (int64_t)1 << 31) return SA_ERR_SHAPE;
    return SA_OK;
}

inline int launch_status() { return hipGetLastError() == hipSuccess ? SA_OK : SA_ERR_HIP; }

#endif
