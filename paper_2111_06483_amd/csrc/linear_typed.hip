// Products of rows with the weight of their type: Z = X W_t and dX = dZ W_t^T for rows sorted by type, of any numbers.
//
// Both are rows (contraction index contiguous) times a small operand B [C, N] per type.
//   - Few rows (linear_typed_few.hip): latency.  One launch.
//   - Otherwise a first launch (k_typed_lay) lays B out in pieces of bf16, in the order in which a wavefront's lanes want them: fp32 rows three pieces a
//     weight (24 bits, linear_pieces.h; products to within 2^-23, linear_split.hip), bf16 rows two (as in linear.hip: the weight to 16 bits, below 2^-117 to
//     within 2^-134; the result is rounded to 8), T K F values; and lists the row blocks of every type, as many as its rows need, which the
//     workgroups of the main launch (k_typed_rows) share: 128 rows and up to 256 columns at a time, four wavefronts, the pieces by asynchronous
//     copies to LDS, two buffers, a barrier a stage.  (Tried, with no gain beyond a twentieth either way: 256 rows by eight
//     wavefronts, rows by asynchronous copies as well, both two stages ahead.)
//   - Columns are dealt to the column tiles by turns (`column_of`), so that a lane ends up with four neighbours of a row and writes them at once:
//     a wavefront's store covers whole lines, with no turn through LDS.
// fp32 sums: the matrix unit cuts (does not round) when it adds, so a chunk's 16 products are summed from zero there and added to the
// running sum by vector instructions, which round to nearest; and every other chunk is multiplied by -B and subtracted, so that what is
// cut leans to neither side.  bf16 products are added there: a unit of 2^-23 of the sum for eight terms, 2^-10 of the longest
// contraction's (65536), which is rounded to 8 bits.  A result that is not finite (infinities and NaN have no such pieces, and numbers are scaled up first, kUp) sends the wavefront's tile back to the fp32 matrix instruction, from
// the operands themselves.
// What bounds them (256 -> 256, four types): fp32, 237500 rows, 187 us = 166 TFLOP/s: the six products, 998 TFLOP/s of bf16 (a large library product in
// bf16 reaches 1170, one in fp32 154); bf16, 867187 rows, 276 us: its two products 823 TFLOP/s, its 888 MB 3.2 TB/s, neither alone (195 and 185 us).
#include "linear_typed_rows.h"

namespace sar {

namespace {

size_t round256(size_t b) { return (b + 255) / 256 * 256; }

int check_shape(int64_t n, int K, int F, int T)
{
    SAR_CHECK_ARG(n >= 0 && K >= 1 && F >= 1, "typed products: n = %lld rows, K = %d, F = %d", (long long)n, K, F);
    SAR_CHECK_ARG(T >= 1, "typed products: T = %d types", T);
    if (n > 0x7fffffff - 256 || K > 65536 || F > 65536 || T > 65535)
        return fail(SAR_ERR_UNSUPPORTED, "typed products: n = %lld rows (below 2^31 - 256), K = %d, F = %d (at most 65536), T = %d types (at most 65535)",
                    (long long)n, K, F, T);
    // (the launch that lays them out: a thread for two or three pieces of 16 bytes, and a workgroup for each type)
    if (std::max(lay_bytes(K, F, T), lay_bytes(F, K, T)) / (2 * 16 * 256) + T > (size_t)most_workgroups(256))
        return fail(SAR_ERR_UNSUPPORTED, "typed products: %d x %d weights of %d types are too many for one launch", K, F, T);
    return SAR_OK;
}

size_t work_bytes_of(int64_t n, int K, int F, int T)
{
    return round256(std::max(std::max(lay_bytes(K, F, T), lay_bytes(F, K, T)) + list_bytes(n, T), typed_dw_bytes(n, K, F, T)));
}

int check_call(int dtype, int64_t n, int K, int F, int T, const void* ptr, const void* work, size_t work_bytes)
{
    if (dtype != SAR_F32 && dtype != SAR_BF16) return fail(SAR_ERR_UNSUPPORTED, "dtype %d is neither SAR_F32 nor SAR_BF16", dtype);
    SAR_TRY(check_shape(n, K, F, T));
    SAR_CHECK_ARG(ptr || T == 1, "typed products: type_ptr is null with T = %d types", T);
    const size_t need = work_bytes_of(n, K, F, T);
    SAR_CHECK_ARG(work && work_bytes >= need, "typed products: work has %zu bytes, needs %zu", work ? work_bytes : 0, need);
    SAR_CHECK_ARG((reinterpret_cast<uintptr_t>(work) & 15) == 0, "typed products: work must be 16-byte aligned");
    return SAR_OK;
}

bool few_bwd(const Types& types, int K, int F) { return few_rows_dw(types.n, types.T, K, F) && few_blocks(types, K); }

// The backward pass of both entry points (ptr null: one type); with rows, dX too.
int typed_bwd(const void* X, const int8_t* Xq, const uint8_t* Xe, const void* dZ, const float* W, const int32_t* ptr, int T, int accumulate,
              float* dW, void* dX, bool rows, int dtype, int64_t n, int K, int F, void* work, hipStream_t st)
{
    SAR_TRY(check_packed("Xq", Xq, Xe));
    SAR_CHECK_ARG(!(X && Xq), "typed products: X and Xq are both given");
    if (n > 0) {
        SAR_CHECK_ARG(dZ || (!dW && !dX), "null pointer (dZ)");
        SAR_CHECK_ARG(!dW || X || Xq, "null pointer (X or Xq)");
        SAR_CHECK_ARG(!dX || W, "null pointer (W)");
        SAR_CHECK_ARG(!dX || dX != dZ, "typed products: dX must not alias dZ");
        SAR_CHECK_ARG(!dX || !dW || dW != W, "typed products: dW must not alias W");
    }
    const Types types{ptr, T, n};
    const TypedDw g{X, Xq, Xe, dZ, dW, types, K, F, accumulate, static_cast<float*>(work)};
    const size_t size = (size_t)n * K * (dtype == SAR_F32 ? 4 : 2);
    if (dW && dX && n > 0 && few_bwd(types, K, F) && apart(dX, size, X, size) && apart(dX, size, Xq, (size_t)n * packed_stride(K)) &&
        apart(dX, size, Xe, (size_t)n * packed_steps(K)))
        return few_dw_and_dx(dtype, g, {dZ, W, dX, types, F, K, K, F}, st);
    if (dW) SAR_TRY(typed_dw(dtype, g, st));
    if (rows && dX && n > 0)
        return dtype == SAR_F32 ? rows_product<float, true>(dZ, W, types, dX, K, F, work, st)
                                : rows_product<bf16_t, true>(dZ, W, types, dX, K, F, work, st);
    return SAR_OK;
}

}  // namespace
}  // namespace sar

using namespace sar;

extern "C" int sar_linear_typed_workspace_bytes(int64_t n, int K, int F, int T, size_t* bytes)
{
    SAR_CHECK_ARG(bytes, "bytes is null");
    SAR_TRY(check_shape(n, K, F, T));
    *bytes = work_bytes_of(n, K, F, T);
    return SAR_OK;
}

extern "C" int sar_linear_typed_fwd(const void* X, const float* W, const int32_t* type_ptr, int T, void* Z, int dtype, int64_t n, int K, int F,
                                    void* work, size_t work_bytes, void* stream)
{
    SAR_TRY(check_call(dtype, n, K, F, T, type_ptr, work, work_bytes));
    if (n == 0) return SAR_OK;
    SAR_CHECK_ARG(X && W && Z, "null pointer (X, W, Z)");
    SAR_CHECK_ARG(X != Z, "typed products: Z must not alias X");
    const Types types{type_ptr, T, n};
    return dtype == SAR_F32 ? rows_product<float, false>(X, W, types, Z, K, F, work, as_stream(stream))
                            : rows_product<bf16_t, false>(X, W, types, Z, K, F, work, as_stream(stream));
}

extern "C" int sar_linear_typed_bwd(const void* X, const int8_t* Xq, const uint8_t* Xe, const void* dZ, const float* W,
                                    const int32_t* type_ptr, int T, int accumulate, float* dW, void* dX, int dtype, int64_t n, int K, int F,
                                    void* work, size_t work_bytes, void* stream)
{
    SAR_TRY(check_call(dtype, n, K, F, T, type_ptr, work, work_bytes));
    return typed_bwd(X, Xq, Xe, dZ, W, type_ptr, T, accumulate, dW, dX, true, dtype, n, K, F, work, as_stream(stream));
}

extern "C" int sar_linear_bwd_packed(const int8_t* Xq, const uint8_t* Xe, const void* dZ, const float* W, int accumulate, float* dW, void* dX,
                                     int dtype, int64_t n, int K, int F, void* work, size_t work_bytes, void* stream)
{
    SAR_TRY(check_call(dtype, n, K, F, 1, nullptr, work, work_bytes));
    // few rows: both products in one launch; of more, dX by the kernels of sar_linear_bwd
    const bool few = few_bwd({nullptr, 1, n}, K, F);
    SAR_TRY(typed_bwd(nullptr, Xq, Xe, dZ, W, nullptr, 1, accumulate, dW, dX, few, dtype, n, K, F, work, as_stream(stream)));
    return dX && !few ? sar_linear_bwd(nullptr, dZ, W, nullptr, dX, dtype, n, K, F, nullptr, 0, stream) : SAR_OK;
}
