// Distillation from a teacher's top classes: the divergence of a student's softmax from the teacher's, which has its listed classes only,
// both at a temperature, and its gradient.
//
//   p = softmax of the listed scores / T, s = softmax(x / T):  loss = sum_j p_j (log p_j - log s_{c_j})
//   dx_c = g / T (s_c - sum of the p_j of class c)
//
// One pass over the student's scores each way (class_rows.h).
#include "class_rows.h"

namespace sar {

namespace {

// The listed classes of a row: what the teacher's softmax takes.
struct Teacher {
    const float* value;    // [n, k]
    const int32_t* index;  // [n, k]
    int k, C;
    float by, over;        // log2(e) / T, 1 / T
    __device__ inline bool is(int32_t c) const { return (uint32_t)c < (uint32_t)C; }
};

struct DistillJob {
    static constexpr bool kEntropy = false, kTop = false;
    struct Args {
        Teacher teacher;
        float *loss, *lse;
    };

    template <typename T, int L>
    static __device__ inline void by_lanes(const ClassRows& a, const Args& o, int64_t row, bool there, int t, const RowSums& r)
    {
        const Teacher& q = o.teacher;
        const float log = logf(r.s), base = base_of(r.m);
        if (there && t == 0 && o.lse) o.lse[row] = fmaf(base, q.over, log);
        if (!o.loss) return;
        const float* value = q.value + row * q.k;
        const int32_t* index = q.index + row * q.k;
        float most = -__builtin_inff();
        for (int j = t; j < q.k; j += L)
            if (q.is(index[j])) most = fmaxf(most, value[j]);
        const float top = base_of(lanes_largest<L>(most));
        float s = 0.f, w = 0.f;
        for (int j = t; j < q.k; j += L) {
            const int32_t c = index[j];
            if (!q.is(c)) continue;
            const float d = value[j] - top, e = exp_below(d, q.by);
            s += e;
            if (e != 0.f) w = fmaf(e, (d - (to_f32(static_cast<const T*>(a.X)[row * a.C + c]) - base)) * q.over, w);
        }
        s = lanes_sum<L>(s);
        w = lanes_sum<L>(w);
        const bool empty = r.m == -__builtin_inff() && r.s == 0.f;
        if (there && t == 0) o.loss[row] = s == 0.f ? 0.f : empty ? __builtin_inff() : w / s - logf(s) + log;
    }
    static __device__ inline float to_f32(float v) { return v; }
    static __device__ inline float to_f32(bf16_t v) { return bf16_to_f32(v); }

    template <typename T, int TPR, int R>
    static __device__ inline void in_lanes(const ClassRows& a, const Args& o, int64_t row, bool there, int t, const RowSums& r,
                                           const float (&)[R][Cols<T>::N])
    {
        by_lanes<T, TPR>(a, o, row, there, t, r);
    }
    template <typename T>
    static __device__ inline void in_wave(const ClassRows& a, const Args& o, int64_t row, const RowSums& r, const TopList&)
    {
        by_lanes<T, 64>(a, o, row, true, threadIdx.x & 63, r);
    }
};

struct GradArgs {
    ClassTiles t;
    const void* X;
    Teacher teacher;
    const float *lse, *dloss;
    void* dX;
};

// A row's share of the gradient: s = 2^(x by - lse), times g; the teacher's probabilities are e over.
struct RowGrad {
    float lse, g, top, over;
};

// The gradient of a tile without the teacher's part goes to LDS, the teacher's is subtracted there (a class that is listed twice, twice, in the
// list's order), and the tile is written as a whole.
template <typename T>
__global__ __launch_bounds__(kClassThreads) void k_distill_bwd(GradArgs a)
{
    constexpr int N = Cols<T>::N;
    __shared__ RowGrad rows[kMostTileRows];
    __shared__ __attribute__((aligned(16))) float tile[kTileValues + 8];
    const Teacher& q = a.teacher;
    for (int64_t index = blockIdx.x; index < a.t.tiles; index += gridDim.x) {
        const int64_t down = index / a.t.across, row0 = down * a.t.rows;
        const int c0 = (int)(index - down * a.t.across) * a.t.width;
        const int count = (int)min((int64_t)a.t.rows, a.t.n - row0);
        const int width = min(a.t.width, a.t.C - c0), values = count * width;
        __syncthreads();               // (the last tile has been read)
        if ((int)threadIdx.x < count) {
            const int64_t row = row0 + threadIdx.x;
            float most = -__builtin_inff(), s = 0.f;
            for (int j = 0; j < q.k; ++j)
                if (q.is(q.index[row * q.k + j])) most = fmaxf(most, q.value[row * q.k + j]);
            const float top = base_of(most);
            for (int j = 0; j < q.k; ++j)
                if (q.is(q.index[row * q.k + j])) s += exp_below(q.value[row * q.k + j] - top, q.by);
            const float lse = a.lse[row], g = a.dloss[row] * q.over;
            RowGrad r{lse * kLog2e, g, top, g / s};
            if (s == 0.f || lse == -__builtin_inff()) r = {__builtin_inff(), 0.f, 0.f, 0.f};       // no class, or no score: no gradient
            else if (lse == __builtin_inff()) r.lse = __builtin_nanf("");
            rows[threadIdx.x] = r;
        }
        __syncthreads();
        const int64_t at = row0 * a.t.C + c0;
        const T* X = static_cast<const T*>(a.X) + at;
        T* dX = static_cast<T*>(a.dX) + at;
        const int64_t left = a.t.n * a.t.C - at;
        for (int e = threadIdx.x * N; e < values; e += kClassThreads * N) {
            float x[N];
            Cols<T>::unpack(Cols<T>::load(X, e, values, left), x);
            int r = a.t.across > 1 ? 0 : tile_row(a.t, e), c = e - r * width;
            RowGrad g = rows[r];
#pragma unroll
            for (int j = 0; j < N; ++j) {
                if (e + j < values) {
                    if (c == width) c = 0, g = rows[++r];
                    ++c;
                    x[j] = g.g * __builtin_amdgcn_exp2f(fmaf(x[j], q.by, -g.lse));
                }
            }
#pragma unroll
            for (int j = 0; j < N; j += 4) *reinterpret_cast<float4*>(tile + e + j) = make_float4(x[j], x[j + 1], x[j + 2], x[j + 3]);
        }
        __syncthreads();
        if (a.t.rows > 1) {
            if ((int)threadIdx.x < count) {
                const RowGrad g = rows[threadIdx.x];
                const int64_t row = row0 + threadIdx.x;
                for (int j = 0; j < q.k; ++j) {
                    const int32_t c = q.index[row * q.k + j];
                    if (q.is(c)) tile[threadIdx.x * width + c] -= g.over * exp_below(q.value[row * q.k + j] - g.top, q.by);
                }
            }
        } else if (threadIdx.x < 64) {
            const int j = threadIdx.x;
            const int32_t c = j < q.k ? q.index[row0 * q.k + j] : -1;
            const float p = j < q.k ? rows[0].over * exp_below(q.value[row0 * q.k + j] - rows[0].top, q.by) : 0.f;
            for (uint64_t in = __ballot(q.is(c) && c >= c0 && c < c0 + width); in; in &= in - 1) {
                const int l = __builtin_ctzll(in);
                if (j == l) tile[c - c0] -= p;
                // (the next one may be the same class: behind this one's write)
                __builtin_amdgcn_wave_barrier();
                __threadfence_block();
            }
        }
        __syncthreads();
        for (int e = threadIdx.x * N; e < values; e += kClassThreads * N) {
            float x[N];
#pragma unroll
            for (int j = 0; j < N; ++j) x[j] = tile[e + j];
            Cols<T>::store(dX, e, values, x);
        }
    }
}

int check_temperature(float T)
{
    SAR_CHECK_ARG(T > 0.f && std::isfinite(T) && std::isfinite(1.f / T), "distillation: temperature %g", (double)T);
    return SAR_OK;
}

Teacher teacher_of(const float* value, const int32_t* index, int k, int C, float T) { return {value, index, k, C, kLog2e / T, 1.f / T}; }

}  // namespace
}  // namespace sar

using namespace sar;

extern "C" int sar_distill_workspace_bytes(int64_t n, int C, int k, size_t* bytes)
{
    SAR_CHECK_ARG(bytes, "bytes is null");
    SAR_TRY(check_classes("distillation", SAR_F32, n, C, k));
    *bytes = class_work_bytes(n, C, 0);
    return SAR_OK;
}

extern "C" int sar_distill_fwd(const void* X, int k, const float* top_value, const int32_t* top_index, float temperature, float* loss, float* lse,
                               int dtype, int64_t n, int C, void* work, size_t work_bytes, void* stream)
{
    SAR_TRY(check_classes("distillation", dtype, n, C, k));
    SAR_TRY(check_temperature(temperature));
    if (n == 0) return SAR_OK;
    SAR_CHECK_ARG(X && (!loss || k == 0 || (top_value && top_index)), "null pointer (X, top_value, top_index)");
    const DistillJob::Args job{teacher_of(top_value, top_index, k, C, temperature), loss, lse};
    ClassRows a{X, n, C, k, job.teacher.by, job.teacher.over, 1, C, nullptr, nullptr};
    return dtype == SAR_F32 ? run_classes<float, DistillJob>(a, job, "distillation", work, work_bytes, as_stream(stream))
                            : run_classes<bf16_t, DistillJob>(a, job, "distillation", work, work_bytes, as_stream(stream));
}

extern "C" int sar_distill_bwd(const void* X, int k, const float* top_value, const int32_t* top_index, float temperature, const float* lse,
                               const float* dloss, void* dX, int dtype, int64_t n, int C, void* stream)
{
    SAR_TRY(check_classes("distillation", dtype, n, C, k));
    SAR_TRY(check_temperature(temperature));
    if (n == 0) return SAR_OK;
    SAR_CHECK_ARG(X && lse && dloss && dX && (k == 0 || (top_value && top_index)), "null pointer (X, top_value, top_index, lse, dloss, dX)");
    const GradArgs a{class_tiles(n, C), X, teacher_of(top_value, top_index, k, C, temperature), lse, dloss, dX};
    const unsigned groups = (unsigned)std::min<int64_t>(a.t.tiles, 1 << 20);
    if (dtype == SAR_F32) k_distill_bwd<float><<<groups, kClassThreads, 0, as_stream(stream)>>>(a);
    else k_distill_bwd<bf16_t><<<groups, kClassThreads, 0, as_stream(stream)>>>(a);
    SAR_LAUNCH_CHECK();
    return SAR_OK;
}
