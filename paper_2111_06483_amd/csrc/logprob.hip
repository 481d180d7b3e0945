// Log probabilities of given classes, with the distribution's entropy and its top classes, and their gradient.
//
//   m = max x, S = sum exp(x - m), U = sum exp(x - m) (x - m):  lse = m + log S, log p_c = (x_c - m) - log S, H = log S - U / S
//   dx_c = g ([c = label] - p_c) - h p_c (log p_c + H)
//
// One pass over the scores each way (class_rows.h): rows of up to 2048 classes in the registers of 1 to 64 lanes, several rows a wavefront; longer ones by a
// workgroup with the running largest, or, of few rows, by several and a second launch.  Exponentials are taken of differences from the largest, so that 32 bits hold; the
// entropy's sum is taken with them.  The gradient needs no sums: tiles of whole pieces, whatever the rows' lengths.
// What bounds it: 1734375 x 172, bf16, eight classes: 208 us, 3.5 TB/s of its 735 MB (a copy: 144): vector instructions, half of them for the
// eight classes (without any 137 us, as distill.hip's pass over the same scores); 306250 x 47, fp32, five: 20 us, 3.7 TB/s; 64 x 65536, fp32, eight: 15.1 us, two launches, 12.2
// and 3.8 under the trace (without classes 8.9).  More than eight of a bf16 row, and any of an fp32 one, are a search over the row for each: 1734375 x 172, bf16, nine 297 us, 16 421, 40 986.  Gradient, 1734375 x 172, bf16: 241 us, 5.1 TB/s.
#include "class_rows.h"

namespace sar {

namespace {

struct LogprobArgs {
    const int32_t* label;
    float *logp, *lse, *entropy, *value;
    int32_t* index;
};

// SHORT: up to eight top classes of bf16 rows that stay in registers.
template <bool SHORT>
struct LogprobJob {
    static constexpr bool kEntropy = true, kTop = true, kWide = !SHORT;
    using Args = LogprobArgs;

    // The label and its score (0, a class that is none, where it is not asked for).
    struct Label {
        int32_t cls;
        float score;
    };
    template <typename T>
    static __device__ inline Label begin(const ClassRows& a, const Args& o, int64_t row, int)
    {
        Label l{o.logp ? o.label[row] : -1, 0.f};
        if ((uint32_t)l.cls < (uint32_t)a.C) l.score = value_in(static_cast<const T*>(a.X)[row * a.C + l.cls]);
        return l;
    }

    // What a row has beside its top classes; by one lane.
    static __device__ inline void results(const ClassRows& a, const Args& o, int64_t row, const RowSums& r, const Label& l, float log)
    {
        const bool none = r.m == -__builtin_inff() && r.s == 0.f;
        if (o.lse) o.lse[row] = base_of(r.m) + log;
        if (o.entropy) o.entropy[row] = none ? 0.f : log - r.u / r.s;
        if (o.logp) o.logp[row] = (uint32_t)l.cls >= (uint32_t)a.C ? 0.f : none ? -__builtin_inff() : (l.score - base_of(r.m)) - log;
    }
    static __device__ inline void write_top(const ClassRows& a, const Args& o, int64_t row, int k, bool is, uint32_t order, int cls, const RowSums& r, float log)
    {
        o.value[row * a.k + k] = is ? (score_of(order) - base_of(r.m)) - log : -__builtin_inff();
        o.index[row * a.k + k] = is ? cls : -1;
    }
    // A bf16 score's order and its class in one number.
    static __device__ inline uint32_t short_key(float v, int c) { return (order_of(v) & 0xffff0000u) | (0xffffu - (uint32_t)c); }
    // The number of the class c among a lane's i-th piece, 0 behind the last one.
    template <typename T, int R>
    static __device__ inline uint32_t key_in_lane(const ClassRows& a, float v, int i, int c)
    {
        const uint32_t key = Cols<T>::N == 8 ? short_key(v, c) : order_of(v);
        return ends_in<T, R>(i) && c >= a.C ? 0u : key;
    }
    static __device__ inline uint32_t order_of_short(uint32_t key) { return key & 0x80000000u ? key & 0xffff0000u : key | 0xffffu; }
    static __device__ inline int class_of_short(uint32_t key) { return (int)(0xffffu - (key & 0xffffu)); }

    template <typename T, int TPR, int R>
    static __device__ inline void in_lanes(const ClassRows& a, const Args& o, int64_t row, bool there, int t, const RowSums& r, const Label& label,
                                           const float (&v)[R][Cols<T>::N])
    {
        constexpr int N = Cols<T>::N;
        const float log = logf(r.s);
        if (there && t == 0) results(a, o, row, r, label, log);
        if (a.k == 0) return;
        if constexpr (SHORT) {
            // Every lane's eight largest, sorted; the largest of the row's lanes is then taken from whichever lane has it, k times over.  (1734375 rows of 172 classes, eight
            // of them, by the search below 346 us, lists merged lane by lane 295.)
            uint32_t top[8], piece[8];
#pragma unroll
            for (int i = 0; i < R; ++i) {
#pragma unroll
                for (int j = 0; j < 8; ++j) (i == 0 ? top : piece)[j] = key_in_lane<T, R>(a, v[i][j], i, (t + i * TPR) * N + j);
                if (i == 0) {
                    sort8(top);
                } else {
                    sort8(piece);
                    merge8(top, piece);
                }
            }
            uint32_t mine[(8 + TPR - 1) / TPR] = {};
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (k >= a.k) break;
                const uint32_t best = over_lanes<TPR>(top[0], [](uint32_t x, uint32_t y) { return max(x, y); });
                const bool taken = top[0] == best;
#pragma unroll
                for (int i = 0; i + k < 7; ++i) top[i] = taken ? top[i + 1] : top[i];
                mine[k / TPR] = t == k % TPR ? best : mine[k / TPR];
            }
#pragma unroll
            for (int i = 0; i < (8 + TPR - 1) / TPR; ++i) {
                const int k = t + i * TPR;
                const uint32_t order = order_of_short(mine[i]);
                if (there && k < a.k) write_top(a, o, row, k, order > kOrderOfNone, order, class_of_short(mine[i]), r, log);
            }
            return;
        }
        // Whichever class is the largest is written and taken out, k times over.  A bf16 score's order and its class fit one number.
        uint32_t key[R][N];
#pragma unroll
        for (int i = 0; i < R; ++i)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                key[i][j] = key_in_lane<T, R>(a, v[i][j], i, (t + i * TPR) * N + j);
            }
        for (int k = 0; k < a.k; ++k) {
            uint32_t best = 0;
#pragma unroll
            for (int i = 0; i < R; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) best = max(best, key[i][j]);
            best = over_lanes<TPR>(best, [](uint32_t x, uint32_t y) { return max(x, y); });
            int cls;
            if constexpr (N == 8) {
                cls = class_of_short(best);
#pragma unroll
                for (int i = 0; i < R; ++i)
#pragma unroll
                    for (int j = 0; j < N; ++j) key[i][j] = key[i][j] == best ? 0u : key[i][j];
                best = order_of_short(best);
            } else {
                cls = 0x7fffffff;
#pragma unroll
                for (int i = R - 1; i >= 0; --i)
#pragma unroll
                    for (int j = N - 1; j >= 0; --j) cls = key[i][j] == best ? (t + i * TPR) * N + j : cls;
                cls = over_lanes<TPR>(cls, [](int x, int y) { return min(x, y); });
#pragma unroll
                for (int i = 0; i < R; ++i)
#pragma unroll
                    for (int j = 0; j < N; ++j) key[i][j] = (t + i * TPR) * N + j == cls ? 0u : key[i][j];
            }
            if (there && t == 0) write_top(a, o, row, k, best > kOrderOfNone, best, cls, r, log);
        }
    }

    template <typename T>
    static __device__ inline void in_wave(const ClassRows& a, const Args& o, int64_t row, const RowSums& r, TopKey top)
    {
        const int lane = threadIdx.x & 63;
        const float log = logf(r.s);
        if (lane == 0) results(a, o, row, r, begin<T>(a, o, row, 0), log);
        if (lane < a.k) write_top(a, o, row, lane, top != 0, order_in(top), class_in(top), r, log);
    }
};

struct GradArgs {
    ClassTiles t;
    const void* X;
    const int32_t* label;
    const float *lse, *entropy, *dlogp, *dentropy;
    void* dX;
};

// What a row's gradient takes: p = exp(x - lse), dx = -p (g + h (x - lse + H)), and g more at the label.
struct RowGrad {
    float lse, g, h, entropy;
};
__device__ inline float grad_of(float x, const RowGrad& r)
{
    const float d = x - r.lse, p = exp_below(d, kLog2e);
    return -p * fmaf(r.h, fmaxf(d, kLeast) + r.entropy, r.g);
}

// ROWS: how many rows a piece of N scores may meet: 1, 2, or any number.
template <typename T, int ROWS>
__global__ __launch_bounds__(kClassThreads) void k_logprob_bwd(GradArgs a)
{
    constexpr int N = Cols<T>::N;
    __shared__ RowGrad rows[kMostTileRows + 1];
    __shared__ int labels[kMostTileRows + 1];
    constexpr int U = kTileValues / (kClassThreads * N);
    for (int64_t index = blockIdx.x; index < a.t.tiles; index += gridDim.x) {
        const int64_t down = index / a.t.across, row0 = down * a.t.rows;
        const int c0 = (int)(index - down * a.t.across) * a.t.width;
        const int count = (int)min((int64_t)a.t.rows, a.t.n - row0);
        const int width = min(a.t.width, a.t.C - c0), values = count * width;
        const int64_t at = row0 * a.t.C + c0;
        const T* X = static_cast<const T*>(a.X) + at;
        T* dX = static_cast<T*>(a.dX) + at;
        const int64_t left = a.t.n * a.t.C - at;
        uint4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u) raw[u] = Cols<T>::load(X, (u * kClassThreads + (int)threadIdx.x) * N, values, left);
        __syncthreads();               // (the last tile's rows have been read)
        if ((int)threadIdx.x < count) {
            const int64_t row = row0 + threadIdx.x;
            const int32_t c = a.label ? a.label[row] : -1;
            const bool has = (uint32_t)c < (uint32_t)a.t.C;
            RowGrad r{a.lse[row], has && a.dlogp ? a.dlogp[row] : 0.f, a.dentropy ? a.dentropy[row] : 0.f, a.dentropy ? a.entropy[row] : 0.f};
            if (r.lse == -__builtin_inff()) r = {__builtin_inff(), 0.f, 0.f, 0.f};        // nothing but -inf: no gradient
            else if (r.lse == __builtin_inff()) r.lse = __builtin_nanf("");
            rows[threadIdx.x] = r, labels[threadIdx.x] = has ? c - c0 : -1;
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int e = (u * kClassThreads + (int)threadIdx.x) * N;
            if (e >= values) continue;
            float x[N];
            Cols<T>::unpack(raw[u], x);
            int r = a.t.rows == 1 ? 0 : tile_row(a.t, e);
            int c = e - r * width;
            if constexpr (ROWS == 1) {
                const RowGrad g = rows[r];
                const int label = labels[r] - c;
#pragma unroll
                for (int j = 0; j < N; ++j) x[j] = grad_of(x[j], g) + (j == label ? g.g : 0.f);
            } else if constexpr (ROWS == 2) {
                // (behind the last row: whatever is there, for values that are not stored)
                const RowGrad g0 = rows[r], g1 = rows[r + 1];
                const int end = width - c, l0 = labels[r] - c, l1 = labels[r + 1] + end;
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const bool next = j >= end;
                    const RowGrad g{next ? g1.lse : g0.lse, next ? g1.g : g0.g, next ? g1.h : g0.h, next ? g1.entropy : g0.entropy};
                    x[j] = grad_of(x[j], g) + (j == (next ? l1 : l0) ? g.g : 0.f);
                }
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    if (e + j < values) x[j] = grad_of(x[j], rows[r]) + (c == labels[r] ? rows[r].g : 0.f);
                    if (++c == width) c = 0, ++r;
                }
            }
            Cols<T>::store(dX, e, values, x);
        }
    }
}

template <typename T>
int logprob_bwd(const GradArgs& a, hipStream_t st)
{
    constexpr int N = Cols<T>::N;
    const unsigned groups = (unsigned)std::min<int64_t>(a.t.tiles, 1 << 20);
    if (a.t.rows == 1 || a.t.C % N == 0) k_logprob_bwd<T, 1><<<groups, kClassThreads, 0, st>>>(a);
    else if (a.t.C >= N) k_logprob_bwd<T, 2><<<groups, kClassThreads, 0, st>>>(a);
    else k_logprob_bwd<T, 0><<<groups, kClassThreads, 0, st>>>(a);
    SAR_LAUNCH_CHECK();
    return SAR_OK;
}

}  // namespace
}  // namespace sar

using namespace sar;

extern "C" int sar_logprob_workspace_bytes(int64_t n, int C, int k, size_t* bytes)
{
    SAR_CHECK_ARG(bytes, "bytes is null");
    SAR_TRY(check_classes("log probabilities", SAR_F32, n, C, k));
    *bytes = class_work_bytes(n, C, k);
    return SAR_OK;
}

extern "C" int sar_logprob_fwd(const void* X, const int32_t* label, float* logp, float* lse, float* entropy, int k, float* top_value,
                               int32_t* top_index, int dtype, int64_t n, int C, void* work, size_t work_bytes, void* stream)
{
    SAR_TRY(check_classes("log probabilities", dtype, n, C, k));
    SAR_CHECK_ARG(k == 0 || n == 0 || (top_value && top_index), "null pointer (top_value, top_index)");
    SAR_CHECK_ARG(!logp || label || n == 0, "null pointer (label)");
    if (n == 0) return SAR_OK;
    SAR_CHECK_ARG(X, "null pointer (X)");
    const ClassRows a{X, n, C, k, kLog2e, 1.f, 1, C, nullptr, nullptr};
    const LogprobArgs job{label, logp, lse, entropy, top_value, top_index};
    hipStream_t st = as_stream(stream);
    const char* const what = "log probabilities";
    if (dtype == SAR_F32) return run_classes<float, LogprobJob<false>>(a, job, what, work, work_bytes, st);
    if (k > 0 && k <= 8 && C <= kMostInLanes) return run_classes<bf16_t, LogprobJob<true>>(a, job, what, work, work_bytes, st);
    return run_classes<bf16_t, LogprobJob<false>>(a, job, what, work, work_bytes, st);
}

extern "C" int sar_logprob_bwd(const void* X, const int32_t* label, const float* lse, const float* entropy, const float* dlogp,
                               const float* dentropy, void* dX, int dtype, int64_t n, int C, void* stream)
{
    SAR_TRY(check_classes("log probabilities", dtype, n, C, 0));
    if (n == 0) return SAR_OK;
    SAR_CHECK_ARG(X && lse && dX, "null pointer (X, lse, dX)");
    SAR_CHECK_ARG(!dlogp || label, "null pointer (label)");
    SAR_CHECK_ARG(!dentropy || entropy, "null pointer (entropy)");
    SAR_TRY(check_gradient("log probabilities", dtype, n, C, X, dX));
    const GradArgs a{class_tiles(n, C), X, label, lse, entropy, dlogp, dentropy, dX};
    return dtype == SAR_F32 ? logprob_bwd<float>(a, as_stream(stream)) : logprob_bwd<bf16_t>(a, as_stream(stream));
}
