// Transforms with a weight for each node type (linear_typed.hip: entry points and rows; linear_typed_dw.hip: weight gradients).
#pragma once

#include "packed.h"
#include "sar_internal.h"

namespace sar {

// The rows of type t: [ptr[t], ptr[t + 1]), cut to what the tensors have, so that no pointer array leads outside of them.  Without
// an array there is one type, which has all rows.
struct Types {
    const int32_t* ptr;
    int T;
    int64_t n;
    __device__ inline void span(int t, int64_t& lo, int64_t& hi) const
    {
        if (ptr == nullptr) {
            lo = 0, hi = n;
            return;
        }
        lo = min(max((int64_t)ptr[t], (int64_t)0), n);
        hi = min(max((int64_t)ptr[t + 1], lo), n);
    }
};

// dW[t] (+)= X_t^T dZ_t for every type.  X [n, K] of dtype or packed, dZ [n, F] of dtype; work: typed_dw_bytes.
struct TypedDw {
    const void* X;
    const int8_t* Xq;
    const uint8_t* Xe;
    const void* dZ;
    float* dW;
    Types types;
    int K, F, accumulate;
    float* partial;
};
size_t typed_dw_bytes(int64_t n, int K, int F, int T);
int typed_dw(int dtype, const TypedDw& g, hipStream_t st);

}  // namespace sar
