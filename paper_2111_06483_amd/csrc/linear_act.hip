// The transform with what stands around it in a layer: Y = act(X W + b + R) or act(X W + b) + R, and its backward pass.
//
//   a = X W + b (+ R),  Y = act(a) (+ R);   dA = dY act'(a):  dW = X^T dA,  db = sum over rows of dA,  dX = dA W^T
//
// Bias, residual and activation meet the sums in registers, in 32 bits, and are rounded once; the products are formed as in linear_typed.hip (one type).
//   - Forward, and dX of rows that are already dA: many rows by linear_kept.h, whose wavefronts keep memory busy while they multiply; operands that do not fit
//     there by linear_typed_rows.h; few rows in one launch by linear_typed_few.hip.  Activations cost instructions: GELU some 20 a value, 60 us of 867187 x 256 values.
//   - Backward: dA is formed where a product brings its rows, never in a pass of its own but where no product wants it (k_act_bwd).
//     bf16: the product for dW forms it (linear_act_dw.hip), as two pieces of bf16, and writes them for dX, which multiplies them as such: rounded to one, dA
//     would have dX off by another rounding of its own size.  fp32: the product for dX forms and
//     writes it, the one for dW reads it.  db leaves with dW.  Few rows: dW, db, dX and dA in one launch, or one
//     each where dX has many columns.
// What bounds it: forward, 867187 x 256 -> 256, bf16, GELU, a residual and its argument kept: 428 to 451 us, 4.0 TB/s of its 1.78 GB (their copy: 349), the vector
// instructions in use 63% of the time, the matrix cores 28%; 306250 x 100 -> 256, fp32, ReLU with a residual 180 us, 4.2 TB/s.  Backward, 867187 x 256 -> 256, bf16, GELU: 886
// to 925 us, of it (traced) dW 575 (2.7 GB with the two pieces of dA that it writes; vector instructions 68%), dX 394 (three products, matrix cores 59%; 2.2 GB); 306250 x 256 ->
// 256, fp32, ELU 605 to 640 us, 128 TFLOP/s of products (a large library product: 150).
#include "linear_kept.h"

namespace sar {

namespace {

constexpr int kActThreads = 256;
constexpr int kActGroups = 1024;

// dA = dY act'(a) of rows, and sums of its columns: where no product forms it.
struct ActBwdArgs {
    const void* dY;
    const void* A;
    void* dA;              // [n, F] of dtype, or null
    float* partial;        // [gridDim.x, F], or null
    int64_t n;
    int F, act, lanes;     // lanes: of a row, a power of two
};

template <typename T>
__global__ __launch_bounds__(kActThreads) void k_act_bwd(ActBwdArgs a)
{
    constexpr int N = Cols<T>::N;
    __shared__ float sums[kActThreads * N];
    const int t = threadIdx.x & (a.lanes - 1), slice = threadIdx.x / a.lanes, rows = kActThreads / a.lanes;
    const int c = (blockIdx.y * a.lanes + t) * N;
    float total[N] = {};
    for (int64_t row = (int64_t)blockIdx.x * rows + slice; row < a.n; row += (int64_t)gridDim.x * rows) {
        const int64_t at = row * a.F, left = (a.n - row) * a.F;
        float d[N];
        Cols<T>::values(Cols<T>::load(static_cast<const T*>(a.dY) + at, c, a.F, left), c, a.F, d);
        if (a.act != SAR_ACT_NONE) {
            float x[N];
            Cols<T>::values(Cols<T>::load(static_cast<const T*>(a.A) + at, c, a.F, left), c, a.F, x);
            with_act(a.act, [&](auto act) {
#pragma unroll
                for (int j = 0; j < N; ++j) d[j] = act_grad<decltype(act)::value>(d[j], x[j]);
            });
        }
#pragma unroll
        for (int j = 0; j < N; ++j) total[j] += d[j];
        if (a.dA) Cols<T>::store(static_cast<T*>(a.dA) + at, c, a.F, d);
    }
    if (!a.partial) return;
#pragma unroll
    for (int j = 0; j < N; ++j) sums[(slice * N + j) * a.lanes + t] = total[j];
    __syncthreads();
    for (int k = threadIdx.x; k < a.lanes * N; k += kActThreads) {
        const int col = (blockIdx.y * a.lanes + k % a.lanes) * N + k / a.lanes;
        if (col >= a.F) continue;
        float v = 0.f;
        for (int s = 0; s < rows; ++s) v += sums[s * a.lanes * N + k];
        a.partial[(int64_t)blockIdx.x * a.F + col] = v;
    }
}

int lanes_of(int dtype, int F)
{
    const int vec = dtype == SAR_F32 ? 4 : 8;
    int lanes = 1;
    while (lanes < 64 && lanes * vec < F) lanes <<= 1;
    return lanes;
}
int groups_of(int dtype, int64_t n, int F)
{
    const int64_t rows = kActThreads / lanes_of(dtype, F);
    return (int)std::max<int64_t>(1, std::min<int64_t>((n + rows - 1) / rows, std::max(1, std::min(kActGroups, (1 << 22) / F))));
}

// Whether a product's operand is kept: from a tile of 32 rows for every wavefront of the chip on, 65536 rows where there is one block of columns, about where the two are
// level (us kept / by the other kernel, by GELU with a residual, 16, 32, 64, 96 and 128 thousand rows: 64 -> 128 bf16 15.6 / 8.6, 17.4 / 16.1, 20.2 / 22.5, 29.0 / 29.4, 30.8 / 34.9;
// 256 -> 128 bf16 22.4 / 15.0, 24.0 / 20.9, 28.1 / 27.6, 42.8 / 43.3, 46.2 / 50.4; 128 -> 128 fp32 25.3 / 17.7, 27.2 / 22.5, 35.5 / 36.8, 52.2 / 52.2, 57.6 / 62.8; two blocks, 128 -> 256
// bf16, 19.3 / 18.6, 21.5 / 23.7, 32.4 / 45.4).  256 -> 256, bf16, 867187 rows 433 / 576; 47 -> 64, half of a block empty, 400 thousand rows 108 / 50; 128 -> 70, pairs of
// neighbours, 135 / 112.
template <typename T>
bool kept(int64_t n, int C, int N)
{
    const int64_t blocks = (N + 32 * kKeptTiles - 1) / (32 * kKeptTiles);
    return n * blocks >= 256 * kKeptWaves * 32 && fits_kept<T>(C, N);
}

template <typename T>
int forward(const void* X, const float* W, int64_t n, void* Y, int K, int F, void* work, hipStream_t st, const Epilogue& e)
{
    if (kept<T>(n, K, F)) return run_kept<T, false>(X, W, n, Y, K, F, work, st, e);
    return rows_product<T, false>(X, W, Types{nullptr, 1, n}, Y, K, F, work, st, e);
}

// dX of rows of dA that are formed, or (bf16) in two pieces.
template <typename T, typename Q>
int product_of(const void* rows, const float* W, int64_t n, void* dX, int K, int F, void* work, hipStream_t st, const Q& q)
{
    if constexpr (sizeof(T) == 2) {
        if (kept<T>(n, F, K)) return run_kept<T, true>(rows, W, n, dX, K, F, work, st, NoEpilogue{}, q);
    }
    return rows_product<T, true>(rows, W, Types{nullptr, 1, n}, dX, K, F, work, st, NoEpilogue{}, q);
}

size_t rounded(size_t b) { return (b + 255) / 256 * 256; }
size_t partial_bytes(int64_t n, int F)
{
    return rounded((size_t)std::max(groups_of(SAR_F32, n, F), groups_of(SAR_BF16, n, F)) * F * sizeof(float));
}

// Scratch of either product (one after the other).
size_t product_bytes(int64_t n, int K, int F)
{
    size_t b = 0;
    (void)sar_linear_typed_workspace_bytes(n, K, F, 1, &b);
    return rounded(std::max(b, act_dw_bytes(n, K, F)));
}

int check_act(int act)
{
    if (act < SAR_ACT_NONE || act > SAR_ACT_ELU) return fail(SAR_ERR_UNSUPPORTED, "act %d is none of SAR_ACT_NONE, _RELU, _GELU, _SILU, _ELU", act);
    return SAR_OK;
}

// forward: the operand's pieces and the row blocks' list are all that it lays out.
int check_work(int dtype, int64_t n, int K, int F, bool forward, const void* work, size_t work_bytes)
{
    if (dtype != SAR_F32 && dtype != SAR_BF16) return fail(SAR_ERR_UNSUPPORTED, "dtype %d is neither SAR_F32 nor SAR_BF16", dtype);
    size_t need = 0;
    SAR_TRY(forward ? sar_linear_typed_workspace_bytes(n, K, F, 1, &need) : sar_linear_act_workspace_bytes(n, K, F, &need));
    SAR_CHECK_ARG(work && work_bytes >= need, "linear with activation: work has %zu bytes, needs %zu", work ? work_bytes : 0, need);
    SAR_CHECK_ARG((reinterpret_cast<uintptr_t>(work) & 15) == 0, "linear with activation: work must be 16-byte aligned");
    return SAR_OK;
}

template <typename T>
int act_bwd(const void* dY, const void* A, const void* X, const float* W, int act, int accumulate, float* dW, float* db, void* dX, void* dA, int64_t n,
            int K, int F, void* work, hipStream_t st)
{
    const int dtype = sizeof(T) == 4 ? SAR_F32 : SAR_BF16;
    const size_t products = product_bytes(n, K, F);
    float* const partial = reinterpret_cast<float*>(static_cast<char*>(work) + products);
    char* const high = reinterpret_cast<char*>(partial) + partial_bytes(n, F);
    const bool formed = act != SAR_ACT_NONE;
    const Types types{nullptr, 1, n};
    const bool few_dw = few_rows_dw(n, 1, K, F), few_dx = few_blocks(types, K);
    // Few rows: one launch, but for what would have no kernel there to write it (db without dW, for which there need be no X; dA without dX, or of no
    // activation).
    if (few_dw && few_dx && n > 0 && (!db || dW) && (!dA || (formed && dX)) && (dW || dX)) {
        const TypedDw g{X, nullptr, nullptr, dY, dW, types, K, F, accumulate, nullptr, formed ? A : nullptr, act, db};
        return few_act_bwd(dtype, g, {dY, W, dX, types, F, K, K, F}, dA, st);
    }
    // What forms dA of many rows: in bf16 the product for dW, which writes it for dX (two pieces, of which the first may be the caller's dA), or for who asked for it;
    // without that the product for dX; otherwise a launch of its own.  (867187 x 256 -> 256, bf16, GELU: dW writes it 886 us, of one piece, that dX had fewer bits of, 735;
    // dX alone, which forms it for either half of its columns, 625.)  One block of columns of dX that is kept forms it again for fewer bytes: 400000 rows, written / formed twice,
    // 128 -> 256 by SiLU 459 / 386, 128 -> 128 by ReLU 214 / 187, by GELU 230 / 224, with dA wanted 230 / 243; 100 -> 256 by GELU 448 / 423.
    // (Few rows' dW forms it in either type, with db.)
    constexpr bool bf16 = sizeof(T) == 2;
    const bool few = dW && few_dw && n > 0, again = formed && dW && !few_dw && bf16;
    const bool twice = bf16 && K <= 32 * kKeptTiles && kept<T>(n, F, K);
    const bool writes = again && F % 2 == 0 && n > 0 && (dA || (dX && !few_dx && !twice));
    const bool within = formed && dX && n > 0 && (few_dx ? bf16 : !writes);
    const bool reads = (dW && !few && !again) || (dX && !within);
    void* const rows = !formed ? const_cast<void*>(dY) : dA ? dA : reads ? high : nullptr;
    char* const second = high + rounded((size_t)n * F * sizeof(bf16_t));       // (bf16)
    const bool sums = db && !dW;       // (otherwise with dW)
    void* const written = formed ? (within || writes ? nullptr : rows) : dA;
    if (n > 0 && (written || sums)) {
        const int lanes = lanes_of(dtype, F), groups = groups_of(dtype, n, F);
        const ActBwdArgs a{dY, A, written, sums ? partial : nullptr, n, F, act, lanes};
        const int across = (F + lanes * Cols<T>::N - 1) / (lanes * Cols<T>::N);
        k_act_bwd<T><<<dim3(groups, across), kActThreads, 0, st>>>(a);
        SAR_LAUNCH_CHECK();
    }
    if (sums) SAR_TRY(act_sum(partial, n > 0 ? groups_of(dtype, n, F) : 0, F, accumulate, db, st));
    auto weights = [&]() -> int {
        return act_dw(dtype, {X, again ? dY : rows, again ? A : nullptr, act, dW, db, n, K, F, accumulate, work, writes ? rows : nullptr, writes && dX && !within ? second : nullptr}, st);
    };
    if (writes) SAR_TRY(weights());
    if (dX && n > 0) {
        const TypedDw none{nullptr, nullptr, nullptr, nullptr, nullptr, types, K, F, 0, nullptr, A, act};
        if (within && few_dx) {
            SAR_TRY(few_act_bwd(dtype, none, {dY, W, dX, types, F, K, K, F}, writes ? nullptr : rows, st));
        } else if (within) {
            SAR_TRY(product_of<T>(dY, W, n, dX, K, F, work, st, ActPrologue{A, rows, act}));
        } else if (writes) {
            if constexpr (bf16) SAR_TRY(product_of<T>(rows, W, n, dX, K, F, work, st, LowPieces{second}));
        } else if (kept<T>(n, F, K)) {
            SAR_TRY((run_kept<T, true>(rows, W, n, dX, K, F, work, st, NoEpilogue{})));
        } else {
            SAR_TRY((rows_product<T, true>(rows, W, types, dX, K, F, work, st)));
        }
    }
    if (few) return few_act_bwd(dtype, {X, nullptr, nullptr, dY, dW, types, K, F, accumulate, nullptr, formed ? A : nullptr, act, db}, {}, nullptr, st);
    if (dW && !writes) return weights();
    return SAR_OK;
}

}  // namespace
}  // namespace sar

using namespace sar;

extern "C" int sar_linear_act_workspace_bytes(int64_t n, int K, int F, size_t* bytes)
{
    SAR_CHECK_ARG(bytes, "bytes is null");
    size_t products = 0;
    SAR_TRY(sar_linear_typed_workspace_bytes(n, K, F, 1, &products));      // (refuses what no product takes)
    *bytes = product_bytes(n, K, F) + partial_bytes(n, F) + 2 * rounded((size_t)n * F * 2);
    return SAR_OK;
}

extern "C" int sar_linear_act_fwd(const void* X, const float* W, const float* bias, const void* res, int act, int res_after, void* Y, void* A, int dtype,
                                  int64_t n, int K, int F, void* work, size_t work_bytes, void* stream)
{
    SAR_TRY(check_act(act));
    SAR_TRY(check_work(dtype, n, K, F, true, work, work_bytes));
    if (n == 0) return SAR_OK;
    SAR_CHECK_ARG(X && W && Y, "null pointer (X, W, Y)");
    const size_t b = dtype == SAR_F32 ? 4 : 2, in = (size_t)n * K * b, out = (size_t)n * F * b;
    SAR_CHECK_ARG(apart(Y, out, X, in) && apart(Y, out, W, (size_t)K * F * 4) && apart(Y, out, A, out) && apart(X, in, A, out) && apart(W, (size_t)K * F * 4, A, out),
                  "linear with activation: Y, A must not alias X, W or each other");
    SAR_CHECK_ARG(Y == res || apart(Y, out, res, out), "linear with activation: Y overlaps res, and is not res");
    SAR_CHECK_ARG((A == res && !res_after) || !A || apart(A, out, res, out), "linear with activation: A overlaps res");
    const Epilogue e{bias, res, A, act, res_after};
    return dtype == SAR_F32 ? forward<float>(X, W, n, Y, K, F, work, as_stream(stream), e) : forward<bf16_t>(X, W, n, Y, K, F, work, as_stream(stream), e);
}

extern "C" int sar_linear_act_bwd(const void* dY, const void* A, const void* X, const float* W, int act, int accumulate, float* dW, float* db, void* dX,
                                  void* dA, int dtype, int64_t n, int K, int F, void* work, size_t work_bytes, void* stream)
{
    SAR_TRY(check_act(act));
    SAR_TRY(check_work(dtype, n, K, F, false, work, work_bytes));
    if (n > 0) {
        const size_t b = dtype == SAR_F32 ? 4 : 2, in = (size_t)n * K * b, out = (size_t)n * F * b, w = (size_t)K * F * 4;
        SAR_CHECK_ARG(dY && (act == SAR_ACT_NONE || A), "null pointer (dY, A)");
        SAR_CHECK_ARG(!dW || X, "null pointer (X)");
        SAR_CHECK_ARG(!dX || W, "null pointer (W)");
        SAR_CHECK_ARG(!dX || (apart(dX, in, dY, out) && apart(dX, in, A, out) && apart(dX, in, X, in) && apart(dX, in, W, w) && apart(dX, in, dA, out)),
                      "linear with activation: dX must not alias dY, A, X, W or dA");
        SAR_CHECK_ARG(!dA || (apart(dA, out, dY, out) && apart(dA, out, A, out) && apart(dA, out, X, in) && (!dX || apart(dA, out, W, w))),
                      "linear with activation: dA must not alias dY, A, X or W");
        SAR_CHECK_ARG(!dW || !W || apart(dW, w, W, w), "linear with activation: dW must not alias W");
    }
    return dtype == SAR_F32 ? act_bwd<float>(dY, A, X, W, act, accumulate, dW, db, dX, dA, n, K, F, work, as_stream(stream))
                            : act_bwd<bf16_t>(dY, A, X, W, act, accumulate, dW, db, dX, dA, n, K, F, work, as_stream(stream));
}
