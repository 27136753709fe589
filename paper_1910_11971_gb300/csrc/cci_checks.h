// cci_checks.h -- argument checks that the entry points share (host only).
#pragma once

#include <cstddef>
#include <cstdint>

#include <cuda_runtime.h>

#include "cci.h"

namespace cci {

constexpr int64_t kMaxElems = int64_t(1) << 62;

inline bool aligned(const void *p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

inline size_t elem_size(int dtype) { return dtype == CCI_F32 ? 4 : 2; }

inline bool valid_dtype(int dtype) { return dtype == CCI_F32 || dtype == CCI_BF16; }

// a*b without overflow past kMaxElems (all inputs >= 0)
inline bool mul_ok(int64_t a, int64_t b)
{
    if (a == 0 || b == 0) return true;
    return a <= kMaxElems / b;
}

inline cci_status check_group(int64_t Cout, int G, int K)
{
    if (G < 1 || G > 256 || K < 1 || K > G) return CCI_ERR_GROUP;
    if (Cout % G != 0) return CCI_ERR_GROUP;
    return CCI_OK;
}

inline cci_status to_status(cudaError_t e) { return e == cudaSuccess ? CCI_OK : CCI_ERR_CUDA; }

}  // namespace cci
