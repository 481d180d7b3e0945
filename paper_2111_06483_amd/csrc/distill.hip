// Distillation from a teacher's top classes: the divergence of a student's softmax from the teacher's, which has its listed classes only,
// both at a temperature, and its gradient.
//
//   p = softmax of the listed scores / T, s = softmax(x / T):  loss = sum_j p_j (log p_j - log s_{c_j})
//   dx_c = g / T (s_c - sum of the p_j of class c)
//
// One pass over the student's scores each way (class_rows.h).  The teacher's few classes meet the student's scores by gathers that are under way with the row, and in the
// gradient where the tile still is on the chip, in the list's order, so that a class that is listed twice has the same sum in every run.
// What bounds it: 1734375 x 172, bf16, eight classes: 137 us, 5.3 TB/s: memory; gradient, 4096 x 50000, bf16, 32 classes: 144 us, 5.7 TB/s; 306250 x 47, fp32, eight: 41 us, 3.4 TB/s (a
// copy of as many bytes 27.5, the gradient of log probabilities, whose workgroups have no lists and more of them fit, 28): a workgroup's reads, lists and two barriers stand one behind the
// other, with nothing of a next tile under way (lists by one lane a row 62; tiles of 40 rows, six workgroups a compute unit, a third barrier: the same).
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
    static constexpr bool kEntropy = false, kTop = false, kWide = true;
    struct Args {
        Teacher teacher;
        float *loss, *lse;
    };

    // An entry of the list, and the student's score of its class.
    struct Entry {
        bool is;
        float value, score;
    };
    template <typename T>
    static __device__ inline Entry entry_of(const ClassRows& a, const Teacher& q, int64_t row, int j)
    {
        Entry e{false, 0.f, 0.f};
        if (j >= q.k) return e;
        const int32_t c = q.index[row * q.k + j];
        e.is = q.is(c);
        e.value = q.value[row * q.k + j];
        if (e.is) e.score = value_in(static_cast<const T*>(a.X)[row * a.C + c]);
        return e;
    }
    // The first of a lane.
    template <typename T>
    static __device__ inline Entry begin(const ClassRows& a, const Args& o, int64_t row, int t)
    {
        return o.loss ? entry_of<T>(a, o.teacher, row, t) : Entry{false, 0.f, 0.f};
    }

    template <typename T, int L>
    static __device__ inline void by_lanes(const ClassRows& a, const Args& o, int64_t row, bool there, int t, const RowSums& r, const Entry& first)
    {
        const Teacher& q = o.teacher;
        const float log = logf(r.s), base = base_of(r.m);
        if (there && t == 0 && o.lse) o.lse[row] = fmaf(base, q.over, log);
        if (!o.loss) return;
        float most = first.is ? first.value : -__builtin_inff();
        for (int j = t + L; j < q.k; j += L)
            if (q.is(q.index[row * q.k + j])) most = fmaxf(most, q.value[row * q.k + j]);
        const float top = base_of(lanes_largest<L>(most));
        float s = 0.f, w = 0.f;
        auto add = [&](const Entry& x) {
            const float d = x.value - top, e = exp_below(d, q.by);
            if (!x.is) return;
            s += e;
            if (e != 0.f) w = fmaf(e, (d - (x.score - base)) * q.over, w);
        };
        add(first);
        for (int j = t + L; j < q.k; j += L) add(entry_of<T>(a, q, row, j));
        s = lanes_sum<L>(s);
        w = lanes_sum<L>(w);
        const bool empty = r.m == -__builtin_inff() && r.s == 0.f;
        if (there && t == 0) o.loss[row] = s == 0.f ? 0.f : empty ? __builtin_inff() : w / s - logf(s) + log;
    }

    template <typename T, int TPR, int R>
    static __device__ inline void in_lanes(const ClassRows& a, const Args& o, int64_t row, bool there, int t, const RowSums& r, const Entry& first,
                                           const float (&)[R][Cols<T>::N])
    {
        by_lanes<T, TPR>(a, o, row, there, t, r, first);
    }
    template <typename T>
    static __device__ inline void in_wave(const ClassRows& a, const Args& o, int64_t row, const RowSums& r, TopKey)
    {
        by_lanes<T, 64>(a, o, row, true, threadIdx.x & 63, r, begin<T>(a, o, row, threadIdx.x & 63));
    }
};

struct GradArgs {
    ClassTiles t;
    const void* X;
    Teacher teacher;
    int lanes;             // of a row's list: a power of two, k at least
    const float *lse, *dloss;
    void* dX;
};

// Over `lanes` neighbours, a power of two.
template <typename Op>
__device__ inline float over_some(float v, int lanes, Op op)
{
    if (lanes >= 2) v = op(v, __uint_as_float(lane_xor<1>(__float_as_uint(v))));
    if (lanes >= 4) v = op(v, __uint_as_float(lane_xor<2>(__float_as_uint(v))));
    if (lanes >= 8) v = op(v, __uint_as_float(lane_xor<4>(__float_as_uint(v))));
    if (lanes >= 16) v = op(v, __uint_as_float(lane_xor<8>(__float_as_uint(v))));
    if (lanes >= 32) v = op(v, __uint_as_float(lane_xor<16>(__float_as_uint(v))));
    if (lanes >= 64) v = op(v, __uint_as_float(lane_xor<32>(__float_as_uint(v))));
    return v;
}

// A row's part of the gradient: s = 2^(x by - lse), times g.
struct RowGrad {
    float lse, g;
};
// ... and a listed class's, p = g q, of the entry that this lane has: the row's lanes together.
__device__ inline RowGrad row_grad(const GradArgs& a, int64_t row, bool is, float value, float& p)
{
    const Teacher& q = a.teacher;
    const float top = base_of(over_some(is ? value : -__builtin_inff(), a.lanes, [](float x, float y) { return fmaxf(x, y); }));
    const float e = is ? exp_below(value - top, q.by) : 0.f;
    const float s = over_some(e, a.lanes, [](float x, float y) { return x + y; });
    const float lse = a.lse[row], g = a.dloss[row] * q.over;
    // no class, or no score: no gradient
    const bool none = s == 0.f || lse == -__builtin_inff();
    p = none ? 0.f : e * (g / s);
    return none ? RowGrad{__builtin_inff(), 0.f} : RowGrad{lse == __builtin_inff() ? __builtin_nanf("") : lse * kLog2e, g};
}
__device__ inline float student_part(float x, const RowGrad& r, float by) { return r.g * __builtin_amdgcn_exp2f(fmaf(x, by, -r.lse)); }

// Short rows, several a tile: what the teacher takes off goes to LDS, zeros elsewhere, and meets the student's part there.  Lists are read as they lie,
// a lane an entry, up to kEntries a thread.
constexpr int kEntries = 4;
template <typename T>
__global__ __launch_bounds__(kClassThreads) void k_distill_bwd(GradArgs a)
{
    constexpr int N = Cols<T>::N, U = kTileValues / (kClassThreads * N);
    __shared__ RowGrad rows[kMostTileRows + 1];
    __shared__ __attribute__((aligned(16))) float taught[kTileValues];
    __shared__ uint8_t named[kTileValues];
    const Teacher& q = a.teacher;
    const int j = threadIdx.x & (a.lanes - 1), group = threadIdx.x / a.lanes, groups = kClassThreads / a.lanes;
    for (int64_t index = blockIdx.x; index < a.t.tiles; index += gridDim.x) {
        const int64_t row0 = index * a.t.rows;
        const int C = a.t.C, count = (int)min((int64_t)a.t.rows, a.t.n - row0), values = count * C;
        const int64_t at = row0 * C;
        const T* X = static_cast<const T*>(a.X) + at;
        T* dX = static_cast<T*>(a.dX) + at;
        const int64_t left = a.t.n * C - at;
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = Cols<T>::load(X, (u * kClassThreads + (int)threadIdx.x) * N, values, left);
        if (index != blockIdx.x) __syncthreads();      // (the last tile has been read)
#pragma unroll
        for (int u = 0; u < kTileValues / (4 * kClassThreads); ++u)
            *reinterpret_cast<float4*>(taught + (u * kClassThreads + threadIdx.x) * 4) = make_float4(0.f, 0.f, 0.f, 0.f);
        int place[kEntries];           // of the entry's class in the tile, -1 without one
        float p[kEntries];
#pragma unroll
        for (int k = 0; k < kEntries; ++k) {
            const int r = k * groups + group;
            place[k] = -1;
            if (k * groups >= count) continue;
            const int64_t row = row0 + min(r, count - 1), entry = row * q.k + min(j, q.k - 1);
            const int32_t c = q.k > 0 ? q.index[entry] : -1;
            const float value = q.k > 0 ? q.value[entry] : 0.f;
            const bool is = j < q.k && q.is(c);
            const RowGrad g = row_grad(a, row, is, value, p[k]);
            if (r >= count) continue;
            if (j == 0) rows[r] = g;
            if (!is) continue;
            place[k] = r * C + c;
            named[place[k]] = (uint8_t)j;
        }
        __syncthreads();
        // A class that is named twice takes the sum of its entries, in the list's order, by the first of them.
#pragma unroll
        for (int k = 0; k < kEntries; ++k) {
            if (k * groups >= count) continue;
            if (__any(place[k] >= 0 && named[place[k]] != j)) {
                float sum = 0.f;
                bool first = true;
                for (int l = 0; l < q.k; ++l) {
                    const int from = ((int)threadIdx.x & 63 & ~(a.lanes - 1)) + l, other = __shfl(place[k], from);
                    const float more = __shfl(p[k], from);
                    if (other == place[k]) {
                        sum += more;
                        first &= l >= j;
                    }
                }
                p[k] = sum;
                if (!first) place[k] = -1;
            }
            if (place[k] >= 0) taught[place[k]] = p[k];
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int e = (u * kClassThreads + (int)threadIdx.x) * N;
            if (e >= values) continue;
            float x[N];
            Cols<T>::unpack(raw[u], x);
            const int r = tile_row(a.t, e), end = (r + 1) * C - e;
            if (C >= N) {
                const RowGrad g0 = rows[r], g1 = rows[r + 1];          // (behind the last row: for values that are not stored)
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] = student_part(x[i], i < end ? g0 : g1, q.by);
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) x[i] = student_part(x[i], rows[min(tile_row(a.t, e + i), count - 1)], q.by);
            }
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const float4 v = *reinterpret_cast<const float4*>(taught + e + i);
                x[i] -= v.x, x[i + 1] -= v.y, x[i + 2] -= v.z, x[i + 3] -= v.w;
            }
            Cols<T>::store(dX, e, values, x);
        }
    }
}

// Long rows, a piece of one a workgroup: the student's part is written, then the few listed classes of the piece once more, with the teacher's.
template <typename T>
__global__ __launch_bounds__(kClassThreads) void k_distill_bwd_wide(GradArgs a)
{
    constexpr int N = Cols<T>::N, U = kWideTile / (kClassThreads * N);
    const Teacher& q = a.teacher;
    const int j = threadIdx.x & 63;
    for (int64_t index = blockIdx.x; index < a.t.tiles; index += gridDim.x) {
        const int64_t row = index / a.t.across;
        const int c0 = (int)(index - row * a.t.across) * a.t.width, width = min(a.t.width, a.t.C - c0);
        const int64_t at = row * a.t.C + c0, left = a.t.n * a.t.C - at;
        const T* X = static_cast<const T*>(a.X) + at;
        T* dX = static_cast<T*>(a.dX) + at;
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = Cols<T>::load(X, (u * kClassThreads + (int)threadIdx.x) * N, width, left);
        const int32_t c = j < q.k ? q.index[row * q.k + j] : -1;
        const float value = j < q.k ? q.value[row * q.k + j] : 0.f;
        const bool in = q.is(c) && c >= c0 && c < c0 + width;
        float own = 0.f, p;
        if (threadIdx.x < 64 && in) own = value_in(X[c - c0]);
        const RowGrad g = row_grad(a, row, q.is(c), value, p);
        own = student_part(own, g, q.by);
        // (of scores in place: they have been read before any is written)
        asm volatile("s_waitcnt vmcnt(0)" : "+v"(own)::"memory");
        __syncthreads();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int e = (u * kClassThreads + (int)threadIdx.x) * N;
            float x[N];
            Cols<T>::unpack(raw[u], x);
#pragma unroll
            for (int i = 0; i < N; ++i) x[i] = student_part(x[i], g, q.by);
            Cols<T>::store(dX, e, width, x);
        }
        __syncthreads();
        if (threadIdx.x >= 64) continue;
        // a class that is named twice: the sum of its entries, in the list's order, by the first of them
        float sum = 0.f;
        int first = 64;
        for (uint64_t left_in = __ballot(in); left_in; left_in &= left_in - 1) {
            const int l = __builtin_ctzll(left_in);
            const float more = __uint_as_float((uint32_t)__builtin_amdgcn_readlane((int)__float_as_uint(p), l));
            if (__builtin_amdgcn_readlane(c, l) == c) sum += more, first = min(first, l);
        }
        if (first == j) dX[c - c0] = from_f32<T>(own - sum);
    }
}

int check_temperature(float T)
{
    SAR_CHECK_ARG(T > 0.f && std::isfinite(T) && std::isfinite(kLog2e / T), "distillation: temperature %g", (double)T);       // (the larger of its factors)
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
    SAR_TRY(check_gradient("distillation", dtype, n, C, X, dX));
    int lanes = 1;
    while (lanes < k) lanes <<= 1;
    const bool wide = C > kTileValues / 2;
    const GradArgs a{wide ? class_tiles(n, C, kWideTile, 1) : class_tiles(n, C, kTileValues, kEntries * kClassThreads / lanes), X,
                     teacher_of(top_value, top_index, k, C, temperature), wide ? 64 : lanes, lse, dloss, dX};
    const unsigned groups = (unsigned)std::min<int64_t>(a.t.tiles, 1 << 20);
    if (wide && dtype == SAR_F32) k_distill_bwd_wide<float><<<groups, kClassThreads, 0, as_stream(stream)>>>(a);
    else if (wide) k_distill_bwd_wide<bf16_t><<<groups, kClassThreads, 0, as_stream(stream)>>>(a);
    else if (dtype == SAR_F32) k_distill_bwd<float><<<groups, kClassThreads, 0, as_stream(stream)>>>(a);
    else k_distill_bwd<bf16_t><<<groups, kClassThreads, 0, as_stream(stream)>>>(a);
    SAR_LAUNCH_CHECK();
    return SAR_OK;
}
