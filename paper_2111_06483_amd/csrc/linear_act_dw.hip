// Weight and bias gradients of the transform with its activation: dW (+)= X^T dA, db (+)= sum over rows of dA, by the kernels of linear_typed_dw.h with one type.
//
// Of bf16 rows dA = dY act'(A) is formed where a workgroup brings the rows and multiplied as two pieces of bf16 (16 bits; one piece would leave dW, an
// fp32 sum, with 8), and written as such for the product that forms dX.  A workgroup's tile is rather 256 x 128 than 128 x 256: it is dA that costs instructions.
// 867187 x 256 x 256, bf16, traced: of dY as it is 249 us, by ReLU 466 (four more tensors pass), by SiLU 528, by GELU 575.  What it waits for are vector instructions, some 44
// a value of dA by GELU, which the matrix instructions of the same wavefront do not hide.  (Fewer of them elsewhere, signs and infinities: no gain that shows.)
#include "linear_typed_dw.h"

namespace sar {

namespace {

// db (+)= the sums of `groups` workgroups, in order: 32 columns a workgroup, whose 32 slices take every 32nd.
__global__ __launch_bounds__(1024) void k_act_sum(const float* partial, int groups, int F, int accumulate, float* db)
{
    __shared__ float part[32][33];
    const int k = threadIdx.x % 32, slice = threadIdx.x / 32, c = blockIdx.x * 32 + k;
    float v = 0.f;
    if (c < F)
        for (int w = slice; w < groups; w += 32) v += partial[(int64_t)w * F + c];
    part[slice][k] = v;
    __syncthreads();
    if (slice == 0 && c < F) {
        float total = 0.f;
#pragma unroll
        for (int s = 0; s < 32; ++s) total += part[s][k];
        db[c] = accumulate ? db[c] + total : total;
    }
}

int64_t most_groups_of(int64_t n, int K, int F)
{
    return std::max({most_groups(n, K, F, kChunk32, false), most_groups(n, K, F, kChunk16, false), most_groups(n, K, F, kChunk16, true)});
}

}  // namespace

int act_sum(const float* partial, int groups, int F, int accumulate, float* db, hipStream_t st)
{
    k_act_sum<<<(F + 31) / 32, 1024, 0, st>>>(partial, groups, F, accumulate, db);
    SAR_LAUNCH_CHECK();
    return SAR_OK;
}

size_t act_dw_bytes(int64_t n, int K, int F)
{
    const size_t most = most_groups_of(n, K, F);
    return ((most + 1) * K + most) * F * sizeof(float);
}

int act_dw(int dtype, const ActDw& g, hipStream_t st)
{
    const bool formed = g.pre != nullptr;
    const Shape s = shape_of(g.n, g.K, g.F, dtype == SAR_F32 ? kChunk32 : kChunk16, formed);
    float* const partial = static_cast<float*>(g.work);
    const DwArgs a{g.X, nullptr, nullptr, g.dY, partial, Types{nullptr, 1, g.n}, g.K, g.F, s.share, g.pre, g.act,
                   g.db ? partial + (s.groups + 1) * g.K * g.F : nullptr, g.formed, g.low};
    return dtype == SAR_F32 ? run_all<F32Rows, F32Sums, kChunk32 / 16, 1>(a, s, g.accumulate, g.dW, st, g.db)
           : g.formed       ? run_all<Bf16Rows, Bf16Written, kChunk16 / 16, 2>(a, s, g.accumulate, g.dW, st, g.db)
           : formed         ? run_all<Bf16Rows, Bf16Formed, kChunk16 / 16, 2>(a, s, g.accumulate, g.dW, st, g.db)
                            : run_all<Bf16Rows, Bf16Sums, kChunk16 / 16, 2>(a, s, g.accumulate, g.dW, st, g.db);
}

}  // namespace sar
