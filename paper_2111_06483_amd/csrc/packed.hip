// Rows kept in 8 bits between the forward and the backward pass.
//
// What the backward pass of a layer needs of its input are sums over many rows (dW = X^T dZ, layer norm's gradients), in which the
// rounding of single values averages out; it is the input kept for them that fills the memory.  The form (packed.h): blocks of 32 values of a
// row, whole numbers of 8 bits, a power of two as the block's step.
//   - Whole numbers, not 8-bit floating point: of normally distributed values the root mean square error is 0.8% of their deviation
//     (32 values, the largest 2 to 3 deviations: steps of 1/64 to 1/32 of one), of e4m3 2.6%.
//   - A power of two, not the largest value / 127: x / step and q step are then exact, so the one rounding is that to a whole number
//     and the same row has the same bytes wherever it is packed; and q step has 7 bits, hence IS a bf16 value.  The
//     products of the backward pass feed the matrix cores from packed rows with no rounding at all, where a step of 24
//     bits would cost a second one.  The price: steps are up to twice as long as they need to be (1.4 times on average).
//   - 32 values: one more byte per block; a single large value spoils no more than its block.
// Both kernels are bound by memory: a lane moves 16 bytes of the row and 4 or 8 of the packed one, rows one after the other in one
// index space, so that short and odd rows leave no lanes idle but those behind a row's last piece.  1734375 x 256, bf16: 243 us to pack, 208 to unpack, 5.5 and
// 6.5 TB/s (a large copy: 4.8); 306250 x 100, fp32: 39 and 25 us.
#include "packed.h"
#include "sar_internal.h"

namespace sar {

namespace {

constexpr int kUnits = 4;                    // pieces a thread
constexpr int kThreads = 256;

// A workgroup takes kUnits * kThreads units, a unit being a piece's place in a row of `per_row` places (whole blocks).
template <typename T, bool PACK>
__global__ __launch_bounds__(kThreads) void k_packed(T* X, int8_t* q, uint8_t* e, int64_t n, int K, uint32_t per_row)
{
    constexpr int N = Cols<T>::N;
    const int64_t first = (int64_t)blockIdx.x * (kUnits * kThreads);
    const int64_t row0 = first / per_row;
    const uint32_t rest = (uint32_t)(first - row0 * per_row);
    const int stride = packed_stride(K), steps = packed_steps(K);
    uint4 x[kUnits];
    typename PackedCols<N>::Raw y[kUnits];
    int64_t row[kUnits];
    int c[kUnits];
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        const uint32_t at = rest + u * kThreads + threadIdx.x;
        const uint32_t r = at / per_row;
        row[u] = row0 + r;
        c[u] = (int)(at - r * per_row) * N;
        // (rows behind the last one are read as the last one: the lanes of a block stay together)
        const int64_t i = min(row[u], n - 1);
        if constexpr (PACK) x[u] = Cols<T>::load(X + i * K, c[u], K, (n - i) * K);
        else y[u] = PackedCols<N>::load(q + i * stride, e + i * steps, c[u], stride);
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
        if (row[u] >= n) continue;
        float v[N];
        if constexpr (PACK) {
            Cols<T>::values(x[u], c[u], K, v);
            store_packed<T>(q + row[u] * stride, e + row[u] * steps, c[u], K, v);
        } else {
            PackedCols<N>::values(y[u], c[u], stride, v);
            Cols<T>::store(X + row[u] * K, c[u], K, v);
        }
    }
}

template <typename T, bool PACK>
int run(T* X, int8_t* q, uint8_t* e, int64_t n, int K, hipStream_t st)
{
    const uint32_t per_row = (uint32_t)packed_steps(K) * (kPackBlock / Cols<T>::N);
    const int64_t units = n * per_row, wgs = (units + kUnits * kThreads - 1) / (kUnits * kThreads);
    if (wgs > most_workgroups(kThreads)) return fail(SAR_ERR_UNSUPPORTED, "packed rows: %lld rows of %d values are too many for one launch", (long long)n, K);
    k_packed<T, PACK><<<(unsigned)wgs, kThreads, 0, st>>>(X, q, e, n, K, per_row);
    SAR_LAUNCH_CHECK();
    return SAR_OK;
}

int check_args(const void* X, const void* q, const void* e, int dtype, int64_t n, int K)
{
    if (dtype != SAR_F32 && dtype != SAR_BF16) return fail(SAR_ERR_UNSUPPORTED, "dtype %d is neither SAR_F32 nor SAR_BF16", dtype);
    SAR_CHECK_ARG(n >= 0 && K >= 1, "n = %lld rows of K = %d values", (long long)n, K);
    if (K > kMostPackedWidth) return fail(SAR_ERR_UNSUPPORTED, "packed rows of K = %d values (at most %d)", K, kMostPackedWidth);
    if (n == 0) return SAR_OK;
    SAR_CHECK_ARG(X && q && e, "null pointer (X, q, e)");
    return check_packed("q", q, e);
}

}  // namespace

int check_packed(const char* what, const void* q, const void* e)
{
    SAR_CHECK_ARG((q == nullptr) == (e == nullptr), "%s: packed rows need both their numbers and their steps", what);
    SAR_CHECK_ARG((reinterpret_cast<uintptr_t>(q) & 15) == 0, "%s: packed rows must be 16-byte aligned", what);
    return SAR_OK;
}

}  // namespace sar

using namespace sar;

extern "C" int sar_pack(const void* X, int dtype, int64_t n, int K, int8_t* q, uint8_t* e, void* stream)
{
    SAR_TRY(check_args(X, q, e, dtype, n, K));
    if (n == 0) return SAR_OK;
    return dtype == SAR_F32 ? run<float, true>(static_cast<float*>(const_cast<void*>(X)), q, e, n, K, as_stream(stream))
                            : run<bf16_t, true>(static_cast<bf16_t*>(const_cast<void*>(X)), q, e, n, K, as_stream(stream));
}

extern "C" int sar_unpack(const int8_t* q, const uint8_t* e, int dtype, int64_t n, int K, void* X, void* stream)
{
    SAR_TRY(check_args(X, q, e, dtype, n, K));
    if (n == 0) return SAR_OK;
    int8_t* const qm = const_cast<int8_t*>(q);
    uint8_t* const em = const_cast<uint8_t*>(e);
    return dtype == SAR_F32 ? run<float, false>(static_cast<float*>(X), qm, em, n, K, as_stream(stream))
                            : run<bf16_t, false>(static_cast<bf16_t*>(X), qm, em, n, K, as_stream(stream));
}
