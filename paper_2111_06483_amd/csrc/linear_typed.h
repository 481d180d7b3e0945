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

// Calls of few rows (linear_typed_few.hip): whether they are, and one launch each, or one for both of a backward pass.
bool few_blocks(const Types& types, int N);
bool few_rows_dw(int64_t n, int T, int K, int F);
struct TypedRows {
    const void* A;         // [n, C]
    const float* W;        // [T, K, F]
    void* out;             // [n, N]
    Types types;
    int C, N, K, F;
};
int few_product(int dtype, bool trans, const TypedRows& a, hipStream_t st);
int few_dw(int dtype, const TypedDw& g, hipStream_t st);
int few_dw_and_dx(int dtype, const TypedDw& g, const TypedRows& a, hipStream_t st);

// Operands of fp32 products are multiplied by 2^24 before they are cut into pieces of bf16, and sums by what takes that back where they are added up.  An
// fp32 value is a multiple of 2^-149, so its pieces are then multiples of 2^-125, each a normal bf16 value, and a value keeps its bits however small it
// is (unscaled, the last bits of a value below 2^-110 have no bf16 value).  What this takes away is the other end: of values from 2^104 and sums from 2^80
// on, which are formed again from the operands as all that are not finite are.  (A multiplication a value:
// of four types, 237500 x 256 -> 256, 194.0 us for 192.6, backward 410 for 407; 8000 rows, one launch, 19.5 for 18.8; 60000 x 400 -> 400, backward from 8 bits,
// 312 for 302.)
constexpr float kUp = 0x1p24f, kDown = 0x1p-24f;

// What rows an operand has: pieces of a value, values a thread takes of a row, and their bytes.
struct F32Rows {
    using T = float;
    static constexpr int kPieces = 3, kCols = 2;
};
struct Bf16Rows {
    using T = bf16_t;
    static constexpr int kPieces = 1, kCols = 2;
};
struct PackedRows {
    static constexpr int kPieces = 1, kCols = 4;
};

struct DwArgs {
    const void* X;
    const int8_t* Xq;
    const uint8_t* Xe;
    const void* dZ;
    float* partial;        // [workgroups + T, K, F]
    Types types;
    int K, F;
    int64_t share;         // rows of a workgroup
};

// A value of X as fp32.
template <typename XR>
__device__ inline float x_value(const DwArgs& a, int64_t row, int c)
{
    if constexpr (XR::kCols == 4) {
        return (float)a.Xq[row * packed_stride(a.K) + c] * step_of(a.Xe[row * packed_steps(a.K) + c / kPackBlock]);
    } else if constexpr (sizeof(typename XR::T) == 4) {
        return static_cast<const float*>(a.X)[row * a.K + c];
    } else {
        return bf16_to_f32(static_cast<const bf16_t*>(a.X)[row * a.K + c]);
    }
}
template <typename ZR>
__device__ inline float z_value(const DwArgs& a, int64_t row, int c)
{
    if constexpr (sizeof(typename ZR::T) == 4) return static_cast<const float*>(a.dZ)[row * a.F + c];
    else return bf16_to_f32(static_cast<const bf16_t*>(a.dZ)[row * a.F + c]);
}


}  // namespace sar
