// Rows of class scores (logprob.hip, distill.hip): the largest of a row, the sum of exponentials below it and the row's top classes, in one
// pass over the scores, and the gradient's tiles.
#pragma once

#include <algorithm>
#include <cmath>

#include "packed.h"
#include "sar_internal.h"

namespace sar {

constexpr int kClassThreads = 256, kClassWaves = kClassThreads / kWave;
constexpr int kMostTop = 64;                           // a lane of a wavefront for each
constexpr float kLeast = -1e4f;                        // a difference whose exponential is zero: times that it is zero, where -inf would be NaN

// ---- over the L neighbouring lanes that share a row

template <int CTRL>
__device__ inline uint32_t dpp_of(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false); }

template <int L, typename V, typename Op>
__device__ inline V over_lanes(V v, Op op)
{
    static_assert(sizeof(V) == 4, "a register");
    auto other = [&](auto ctrl) { return __builtin_bit_cast(V, dpp_of<decltype(ctrl)::value>(__builtin_bit_cast(uint32_t, v))); };
    if constexpr (L >= 2) v = op(v, other(std::integral_constant<int, 0xB1>{}));       // lane ^ 1
    if constexpr (L >= 4) v = op(v, other(std::integral_constant<int, 0x4E>{}));       // lane ^ 2
    if constexpr (L >= 8) v = op(v, other(std::integral_constant<int, 0x141>{}));      // the other four of eight
    if constexpr (L >= 16) v = op(v, other(std::integral_constant<int, 0x140>{}));     // the other eight of sixteen
    // (a lane's own value and the one of lane ^ 16, lane ^ 32, in either order)
    const auto both = [&](auto r) {
        const uint32_t x = r[0], y = r[1];
        return op(__builtin_bit_cast(V, x), __builtin_bit_cast(V, y));
    };
    const auto word = [&] { return __builtin_bit_cast(uint32_t, v); };
    if constexpr (L >= 32) v = both(__builtin_amdgcn_permlane16_swap(word(), word(), false, false));
    if constexpr (L >= 64) v = both(__builtin_amdgcn_permlane32_swap(word(), word(), false, false));
    return v;
}
template <int L>
__device__ inline float lanes_largest(float v) { return over_lanes<L>(v, [](float a, float b) { return fmaxf(a, b); }); }
template <int L>
__device__ inline float lanes_sum(float v) { return over_lanes<L>(v, [](float a, float b) { return a + b; }); }

__device__ inline float value_in(float v) { return v; }
__device__ inline float value_in(bf16_t v) { return bf16_to_f32(v); }

// ---- a row's sums

// largest; sum of exp((x - largest) / T); sum of the same times (x - largest) / T
struct RowSums {
    float m, s, u;
};
__device__ inline float base_of(float m) { return m == -__builtin_inff() ? 0.f : m; }      // what is subtracted of a row without a score
// log2(e) / T: exponentials are taken by the base 2
__device__ inline float exp_below(float d, float by) { return __builtin_amdgcn_exp2f(d * by); }

// Sums of parts of a row, with their largest score's place moved from r.m to `to`.
__device__ inline void move_sums(RowSums& r, float to, float by, float over)
{
    const float d = fmaxf(r.m - base_of(to), kLeast), f = exp_below(r.m - base_of(to), by);
    r.u = f * (r.u + r.s * (d * over));
    r.s *= f;
    r.m = to;
}

// ---- scores in order
// A score's place among scores: numbers that ascend as the scores do (-0 and 0 alike, NaN last), never zero.
__device__ inline uint32_t order_of(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ inline float score_of(uint32_t order) { return __uint_as_float(order & 0x80000000u ? order ^ 0x80000000u : ~order); }
constexpr uint32_t kOrderOfNone = 0x007fffffu;         // that of -inf: such a class, and those behind the last one (0), are none of the top ones

// A score and its class as one number: a higher score is a larger number, of equal scores the lower class.  0: none.
typedef unsigned long long TopKey;
__device__ inline TopKey key_of(uint32_t order, int cls) { return (TopKey)order << 32 | (uint32_t)~cls; }
__device__ inline uint32_t order_in(TopKey k) { return (uint32_t)(k >> 32); }
__device__ inline int class_in(TopKey k) { return (int)~(uint32_t)k; }
__device__ inline TopKey key_at(TopKey k, int lane)        // (lane: the same for all)
{
    return (TopKey)(uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)k, lane);
}

// What lane ^ O holds, by vector instructions (through LDS a list's sort was most of a call of few rows).
template <int O>
__device__ inline uint32_t lane_xor(uint32_t v)
{
    if constexpr (O == 1) return dpp_of<0xB1>(v);
    else if constexpr (O == 2) return dpp_of<0x4E>(v);
    else if constexpr (O == 3) return dpp_of<0x1B>(v);
    else if constexpr (O == 4) return dpp_of<0x1B>(dpp_of<0x141>(v));
    else if constexpr (O == 8) return dpp_of<0x128>(v);
    else if constexpr (O == 15) return dpp_of<0x140>(v);
    else if constexpr (O == 16) {
        const auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        return threadIdx.x & 16 ? r[0] : r[1];
    } else if constexpr (O == 32) {
        const auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        return threadIdx.x & 32 ? r[0] : r[1];
    } else {
        static_assert(O == 63, "a distance that the sort has");
        return lane_xor<32>(lane_xor<16>(lane_xor<15>(v)));
    }
}
template <int O>
__device__ inline TopKey lane_xor64(TopKey k) { return (TopKey)lane_xor<O>((uint32_t)(k >> 32)) << 32 | lane_xor<O>((uint32_t)k); }

// The top classes of a wavefront's scores, the l-th in lane l.
// One candidate, the same for all lanes.
__device__ inline void insert_top(TopKey& list, TopKey c)
{
    const int lane = threadIdx.x & 63, place = __builtin_popcountll(__ballot(list > c));
    const TopKey before = (TopKey)dpp_of<0x138>((uint32_t)(list >> 32)) << 32 | dpp_of<0x138>((uint32_t)list);       // lane - 1
    if (lane > place) list = before;
    if (lane == place) list = c;
}
// Larger keys towards lane 0, along distances O, O / 2 ... 1; the other way round in lanes that `rises`.
template <int O>
__device__ inline void merge_lanes(TopKey& v, bool rises)
{
    const TopKey p = lane_xor64<O>(v);
    if ((p > v) == (((threadIdx.x & O) == 0) != rises)) v = p;
    if constexpr (O > 1) merge_lanes<O / 2>(v, rises);
}
// One candidate of every lane, sorted.
__device__ inline void sort_top(TopKey& v)
{
    const int lane = threadIdx.x;
    merge_lanes<1>(v, lane & 2);
    merge_lanes<2>(v, lane & 4);
    merge_lanes<4>(v, lane & 8);
    merge_lanes<8>(v, lane & 16);
    merge_lanes<16>(v, lane & 32);
    merge_lanes<32>(v, false);
}
// A descending list of candidates.
__device__ inline void merge_top(TopKey& list, TopKey sorted)
{
    const TopKey c = lane_xor64<63>(sorted);
    if (c > list) list = c;                // (the upper half of both, falling and then rising)
    merge_lanes<32>(list, false);
}
// Those of one candidate a lane that are beyond `last`, the k-th of the list.
__device__ inline void offer_top(TopKey& list, TopKey c, TopKey last)
{
    uint64_t in = __ballot(c > last);
    if (__builtin_popcountll(in) > 8) {                // (a sort and a merge are some eight insertions)
        sort_top(c);
        if (key_at(list, 0) == 0) list = c;
        else merge_top(list, c);
        return;
    }
    while (in) {
        const int l = __builtin_ctzll(in);
        in &= in - 1;
        insert_top(list, key_at(c, l));
    }
}

// The lists of a workgroup's first `count` wavefronts, which are in `lists` too: the first one's then has all of them.  All wavefronts.
template <int WAVES>
__device__ inline void join_lists(TopKey& top, TopKey (*lists)[kMostTop], int wave, int lane, int count)
{
#pragma unroll 1
    for (int half = WAVES / 2; half >= 1; half /= 2) {
        if (wave < half) {
            if (wave + half < count) merge_top(top, lists[wave + half][lane]);
            if (half > 1) lists[wave][lane] = top;
        }
        if (half > 1) __syncthreads();
    }
}

// ---- the eight largest of a lane's numbers; numbers that differ, or zeros

__device__ inline void falling(uint32_t& a, uint32_t& b)
{
    const uint32_t high = max(a, b);
    b = min(a, b), a = high;
}
// Sorted, by a network of 19 exchanges.
__device__ inline void sort8(uint32_t (&v)[8])
{
    constexpr int kPairs[19][2] = {{0, 2}, {1, 3}, {4, 6}, {5, 7}, {0, 4}, {1, 5}, {2, 6}, {3, 7}, {0, 1}, {2, 3},
                                   {4, 5}, {6, 7}, {2, 4}, {3, 5}, {1, 4}, {3, 6}, {1, 2}, {3, 4}, {5, 6}};
#pragma unroll
    for (int k = 0; k < 19; ++k) falling(v[kPairs[k][0]], v[kPairs[k][1]]);
}
// Falls and then rises: sorted.
__device__ inline void settle8(uint32_t (&v)[8])
{
#pragma unroll
    for (int o = 4; o >= 1; o >>= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if ((i & o) == 0) falling(v[i], v[i + o]);
}
__device__ inline void merge8(uint32_t (&v)[8], const uint32_t (&sorted)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = max(v[i], sorted[7 - i]);
    settle8(v);
}

// ---- how rows are laid over threads

// Rows of up to 32 values a lane of a wavefront stay in registers.
constexpr int kMostInLanes = 64 * 32;

struct ClassShape {
    int tpr, r;            // lanes a row, pieces a lane
};
// top: k classes are looked for; otherwise k listed ones are read, a lane each as far as they go.
inline ClassShape class_shape(int dtype, int64_t n, int C, int k, bool top)
{
    const int vec = dtype == SAR_F32 ? 4 : 8, pieces = (C + vec - 1) / vec, most = 32 / vec;
    // A piece or two are a lane's or two's, of up to three of the k classes each; otherwise four lanes or more.  (1000000 rows, bf16, us by one or two lanes / by four: log
    // probabilities, four classes without k 7 / 16, k = 3 13 / 29, sixteen classes, k = 3 19 / 29; distillation, C = k = 2 9 / 19, 4 20 / 21, 8 92 / 30.)
    int tpr = 1;
    while (tpr < 4 && (pieces > tpr || k > 3 * tpr)) tpr <<= 1;
    // 32 values a lane; of many bf16 rows 48, for half the lanes to share what is done once a row (172 classes, eight of them, 872093 rows by four lanes 111 us, by eight
    // 124, 100000 rows 17.4 and 16.9; eight listed ones, two a lane, 91 and 73; 300 classes, 500000 rows, one a lane, 62 and 72).
    auto holds = [&](int lanes) {
        return pieces <= lanes * most || (vec == 8 && pieces <= lanes * 6 && n * lanes >= 64 * 16384 && (top || k <= lanes));
    };
    while (tpr < 64 && !holds(tpr)) tpr <<= 1;
    // few rows are spread over more lanes
    while (tpr < 64 && pieces > tpr && n * tpr < 64 * 2048) tpr <<= 1;
    const int r = (pieces + tpr - 1) / tpr;
    return {tpr, r <= 4 ? r : (r + 1) / 2 * 2};
}

// Longer rows are cut into parts of whole pieces, a workgroup each; several parts a row where there are few rows, and a second launch that joins them.
// (Of 512 workgroups the lists are half as many to join as of 1024: 64 x 262144, bf16, eight classes 24 us and 28, 64 of them 36 and 59, none 14 and 15; 64 x 65536, fp32,
// eight, 15.1 and 15.8.  A row by one workgroup of 16 wavefronts, without the second launch: 20.4; of eight, 22.4.)
constexpr int64_t kWideGroups = 512;
constexpr int kMostParts = 64;                         // a lane of a wavefront for each
inline int64_t least_part(int dtype) { return (int64_t)kClassThreads * 4 * (dtype == SAR_F32 ? 4 : 8); }
inline int parts_of(int dtype, int64_t n, int C)
{
    if (C <= kMostInLanes) return 1;
    const int64_t want = (kWideGroups + n - 1) / std::max<int64_t>(n, 1), most = (C + least_part(dtype) - 1) / least_part(dtype);
    return (int)std::max<int64_t>(1, std::min<int64_t>({want, most, kMostParts}));
}
// Values of a part, a multiple of eight.
inline int64_t part_width(int C, int parts) { return ((C + parts - 1) / parts + 7) / 8 * 8; }
// Parts that any call of up to n rows has, where it has several a row.
inline int64_t most_parts(int64_t n, int C)
{
    if (C <= kMostInLanes) return 0;
    const int64_t most = std::min<int64_t>((C + least_part(SAR_F32) - 1) / least_part(SAR_F32), kMostParts), rows = std::min(n, kWideGroups);
    return most > 1 ? std::min(rows * most, rows + kWideGroups) : 0;
}

struct ClassRows {
    const void* X;         // [n, C]
    int64_t n;
    int C, k;
    float by, over;        // log2(e) / T, 1 / T
    int parts;
    int64_t width;
    RowSums* sums;         // [n, parts]
    TopKey* lists;         // [n, parts, k]
};

// Whether a row may end in the lanes' r-th pieces: the last, where lanes have as few as cover it (class_shape).
template <typename T, int R>
constexpr bool ends_in(int r) { return r >= R - (R > 4 ? 2 : 1); }

// A row's pieces of `T` in the lanes t of TPR, -inf behind the row's end.  inner: none of the workgroup's rows is so near to the tensor's end that a piece passes that.
template <typename T, int TPR, int R>
__device__ inline void row_in_lanes(const ClassRows& a, int64_t row, int t, bool inner, float (&v)[R][Cols<T>::N])
{
    constexpr int N = Cols<T>::N;
    uint4 raw[R];
    const T* x = static_cast<const T*>(a.X) + row * a.C;
    if (inner) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (t + r * TPR) * N;
            raw[r] = load16(x + (ends_in<T, R>(r) && c >= a.C ? 0 : c));
        }
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r) raw[r] = Cols<T>::load(x, (t + r * TPR) * N, a.C, (a.n - row) * a.C);
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        Cols<T>::unpack(raw[r], v[r]);
        if (!ends_in<T, R>(r)) continue;
        const int left = a.C - (t + r * TPR) * N;
#pragma unroll
        for (int j = 0; j < N; ++j) v[r][j] = j < left ? v[r][j] : -__builtin_inff();
    }
}

template <typename T, int TPR, int R, typename Job>
__global__ __launch_bounds__(kClassThreads) void k_class_rows(ClassRows a, typename Job::Args job)
{
    constexpr int N = Cols<T>::N, kRows = kClassThreads / TPR;
    for (int64_t base = (int64_t)blockIdx.x * kRows; base < a.n; base += (int64_t)gridDim.x * kRows) {
        // (worked out for every row: which of its values lie behind the end was kept through the loop, in a hundred scalar registers that there are not)
        int t = threadIdx.x % TPR;
        asm volatile("" : "+v"(t));
        const int64_t row = base + threadIdx.x / TPR;
        const bool there = row < a.n;
        float v[R][N];
        const auto other = Job::template begin<T>(a, job, min(row, a.n - 1), t);       // (what else is read of a row, under way with it)
        row_in_lanes<T, TPR, R>(a, min(row, a.n - 1), t, (a.n - base - kRows) * a.C >= N, v);
        RowSums sums{-__builtin_inff(), 0.f, 0.f};
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < N; ++j) sums.m = fmaxf(sums.m, v[r][j]);
        sums.m = lanes_largest<TPR>(sums.m);
        const float m = base_of(sums.m);
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const float d = v[r][j] - m, e = exp_below(d, a.by);
                sums.s += e;
                if constexpr (Job::kEntropy) sums.u = fmaf(e, fmaxf(d, kLeast), sums.u);
            }
        sums.s = lanes_sum<TPR>(sums.s);
        if constexpr (Job::kEntropy) sums.u = lanes_sum<TPR>(sums.u) * a.over;
        Job::template in_lanes<T, TPR, R>(a, job, min(row, a.n - 1), there, t, sums, other, v);
    }
}

// A part of a row.
template <typename T, typename Job>
__global__ __launch_bounds__(kClassThreads) void k_class_wide(ClassRows a, typename Job::Args job)
{
    constexpr int N = Cols<T>::N, U = 4;
    __shared__ RowSums wave_sums[kClassWaves];
    __shared__ TopKey wave_top[Job::kTop ? kClassWaves : 1][kMostTop];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    for (int64_t index = blockIdx.x; index < a.n * a.parts; index += gridDim.x) {
        const int64_t row = index / a.parts;
        const int part = (int)(index - row * a.parts);
        const T* x = static_cast<const T*>(a.X) + row * a.C;
        const int64_t left = (a.n - row) * a.C;
        const int64_t c0 = part * a.width, c1 = min(c0 + a.width, (int64_t)a.C);
        RowSums sums{-__builtin_inff(), 0.f, 0.f};
        TopKey top = 0;
        uint4 raw[U], next[U];
        const bool ends = c1 + N > left;           // whether the part's last piece may pass the tensor's end
        auto read = [&](int64_t at) {
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int c = (int)min(at + (i * kClassThreads + (int)threadIdx.x) * N, c1);
                next[i] = ends ? Cols<T>::load(x, c, a.C, left) : load16(x + c);
            }
        };
        read(c0);
        for (int64_t at = c0; at < c1; at += kClassThreads * N * U) {
            float v[U][N];
#pragma unroll
            for (int i = 0; i < U; ++i) raw[i] = next[i];
            read(at + kClassThreads * N * U);           // (under way meanwhile)
            float most = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < U; ++i) {
                const int64_t c = at + (i * kClassThreads + (int)threadIdx.x) * N;
                Cols<T>::unpack(raw[i], v[i]);
                if (c + N > c1) {
#pragma unroll
                    for (int j = 0; j < N; ++j)
                        if (c + j >= c1) v[i][j] = -__builtin_inff();
                }
#pragma unroll
                for (int j = 0; j < N; ++j) most = fmaxf(most, v[i][j]);
            }
            if (most > sums.m) move_sums(sums, most, a.by, 1.f);
            const float m = base_of(sums.m);
#pragma unroll
            for (int i = 0; i < U; ++i)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float d = v[i][j] - m, e = exp_below(d, a.by);
                    sums.s += e;
                    if constexpr (Job::kEntropy) sums.u = fmaf(e, fmaxf(d, kLeast), sums.u);
                }
            if constexpr (Job::kTop) {
                // Every lane's largest score that is among the wavefront's first k so far, one a lane at a time.
                if (a.k > 0) {
                    for (;;) {
                        const TopKey last = key_at(top, a.k - 1);
                        if (!__any(most > -__builtin_inff() && order_of(most) >= order_in(last))) break;
                        int cls = 0;
#pragma unroll
                        for (int i = U - 1; i >= 0; --i)
#pragma unroll
                            for (int j = N - 1; j >= 0; --j) cls = v[i][j] == most ? i * (kClassThreads * N) + j : cls;
                        const TopKey c = most > -__builtin_inff() ? key_of(order_of(most), (int)at + (int)threadIdx.x * N + cls) : 0ull;
                        const bool in = c > last;
                        if (!__any(in)) break;
                        offer_top(top, c, last);
                        most = -__builtin_inff();
#pragma unroll
                        for (int i = 0; i < U; ++i)
#pragma unroll
                            for (int j = 0; j < N; ++j) {
                                if (in && cls == i * (kClassThreads * N) + j) v[i][j] = -__builtin_inff();
                                most = fmaxf(most, v[i][j]);
                            }
                    }
                }
            }
        }
        // the wavefront's, then the workgroup's
        const float largest = lanes_largest<64>(sums.m);
        move_sums(sums, largest, a.by, 1.f);
        sums.s = lanes_sum<64>(sums.s);
        if constexpr (Job::kEntropy) sums.u = lanes_sum<64>(sums.u);
        __syncthreads();               // (what the last part left there has been read)
        if (lane == 0) wave_sums[wave] = sums;
        if constexpr (Job::kTop) wave_top[wave][lane] = top;
        __syncthreads();
        if constexpr (Job::kTop) {
            if (a.k > 0) join_lists<kClassWaves>(top, wave_top, wave, lane, kClassWaves);
        }
        if (wave != 0) continue;
        RowSums all{-__builtin_inff(), 0.f, 0.f};
        if (lane < kClassWaves) all = wave_sums[lane];
        move_sums(all, lanes_largest<64>(all.m), a.by, 1.f);
        all.s = lanes_sum<64>(all.s);
        if constexpr (Job::kEntropy) all.u = lanes_sum<64>(all.u);
        if (a.parts == 1) {
            all.u *= a.over;
            Job::template in_wave<T>(a, job, row, all, top);
        } else {
            if (lane == 0) a.sums[index] = all;
            if constexpr (Job::kTop) {
                if (lane < a.k) a.lists[index * a.k + lane] = top;
            }
        }
    }
}

// The parts of a row, by a workgroup.
constexpr int kJoinWaves = 8;
template <typename T, typename Job>
__global__ __launch_bounds__(kJoinWaves* kWave) void k_class_join(ClassRows a, typename Job::Args job)
{
    __shared__ TopKey wave_top[Job::kTop ? kJoinWaves : 1][kMostTop];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t row = blockIdx.x;
    RowSums all{-__builtin_inff(), 0.f, 0.f};
    if (wave == 0 && lane < a.parts) all = a.sums[row * a.parts + lane];
    TopKey top = 0;
    if constexpr (Job::kTop) {
        if (a.k > 0) {
            TopKey list[kMostParts / kJoinWaves];
#pragma unroll
            for (int i = 0; i < kMostParts / kJoinWaves; ++i) {
                const int p = i * kJoinWaves + wave;
                list[i] = p < a.parts && lane < a.k ? a.lists[(row * a.parts + p) * a.k + lane] : 0ull;
            }
            top = list[0];
#pragma unroll
            for (int i = 1; i < kMostParts / kJoinWaves; ++i)
                if (i * kJoinWaves + wave < a.parts) merge_top(top, list[i]);
            wave_top[wave][lane] = top;
            __syncthreads();
            join_lists<kJoinWaves>(top, wave_top, wave, lane, a.parts);
        }
    }
    if (wave != 0) return;
    move_sums(all, lanes_largest<64>(all.m), a.by, 1.f);
    all.s = lanes_sum<64>(all.s);
    all.u = lanes_sum<64>(all.u) * a.over;
    Job::template in_wave<T>(a, job, row, all, top);
}

inline size_t class_work_bytes(int64_t n, int C, int k)
{
    return (size_t)most_parts(n, C) * (sizeof(RowSums) + (size_t)k * sizeof(TopKey) + 8);
}

template <typename T, typename Job, int TPR>
int run_in_lanes(int r, const ClassRows& a, const typename Job::Args& job, hipStream_t st)
{
    constexpr int kRows = kClassThreads / TPR;
    const unsigned groups = (unsigned)std::min<int64_t>((a.n + kRows - 1) / kRows, 1 << 20);
    if (TPR < 4 || r == 1) {
        k_class_rows<T, TPR, 1, Job><<<groups, kClassThreads, 0, st>>>(a, job);
        SAR_LAUNCH_CHECK();
        return SAR_OK;
    }
    if constexpr (TPR >= 4) switch (r) {
    case 2: k_class_rows<T, TPR, 2, Job><<<groups, kClassThreads, 0, st>>>(a, job); break;
    case 3: k_class_rows<T, TPR, 3, Job><<<groups, kClassThreads, 0, st>>>(a, job); break;
    case 4: k_class_rows<T, TPR, 4, Job><<<groups, kClassThreads, 0, st>>>(a, job); break;
    default:
        if (sizeof(T) == 2 || r == 6) k_class_rows<T, TPR, 6, Job><<<groups, kClassThreads, 0, st>>>(a, job);
        else if constexpr (sizeof(T) == 4) k_class_rows<T, TPR, 8, Job><<<groups, kClassThreads, 0, st>>>(a, job);
    }
    SAR_LAUNCH_CHECK();
    return SAR_OK;
}

// One pass over the scores X [n, C] of a job; work: class_work_bytes.
template <typename T, typename Job>
int run_classes(ClassRows a, const typename Job::Args& job, const char* what, void* work, size_t work_bytes, hipStream_t st)
{
    const int dtype = sizeof(T) == 4 ? SAR_F32 : SAR_BF16;
    if (a.C <= kMostInLanes) {
        const ClassShape s = class_shape(dtype, a.n, a.C, a.k, Job::kTop);
        switch (s.tpr) {
        case 1: return run_in_lanes<T, Job, 1>(s.r, a, job, st);
        case 2: return run_in_lanes<T, Job, 2>(s.r, a, job, st);
        case 4: return run_in_lanes<T, Job, 4>(s.r, a, job, st);
        case 8: return run_in_lanes<T, Job, 8>(s.r, a, job, st);
        case 16: return run_in_lanes<T, Job, 16>(s.r, a, job, st);
        case 32: return run_in_lanes<T, Job, 32>(s.r, a, job, st);
        default: return run_in_lanes<T, Job, 64>(s.r, a, job, st);
        }
    }
    if constexpr (Job::kWide) {
        a.parts = parts_of(dtype, a.n, a.C);
        a.width = part_width(a.C, a.parts);
        if (a.parts > 1) {
            const size_t need = class_work_bytes(a.n, a.C, Job::kTop ? a.k : 0);
            SAR_CHECK_ARG(work && work_bytes >= need, "%s: work has %zu bytes, needs %zu", what, work ? work_bytes : 0, need);
            SAR_CHECK_ARG((reinterpret_cast<uintptr_t>(work) & 15) == 0, "%s: work must be 16-byte aligned", what);
            a.lists = static_cast<TopKey*>(work);
            a.sums = reinterpret_cast<RowSums*>(a.lists + a.n * a.parts * (Job::kTop ? a.k : 0));
        }
        const unsigned groups = (unsigned)std::min<int64_t>(a.n * a.parts, 1 << 20);
        k_class_wide<T, Job><<<groups, kClassThreads, 0, st>>>(a, job);
        SAR_LAUNCH_CHECK();
        if (a.parts > 1) {
            k_class_join<T, Job><<<(unsigned)a.n, kJoinWaves * kWave, 0, st>>>(a, job);
            SAR_LAUNCH_CHECK();
        }
        return SAR_OK;
    }
    return fail(SAR_ERR_UNSUPPORTED, "%s: no kernel for %d classes", what, a.C);
}

// ---- gradients: tiles of up to kTileValues scores, whole rows where they are short, a piece of one row where they are long

constexpr int kTileValues = 4096, kWideTile = 8192, kMostTileRows = 256;
struct ClassTiles {
    int64_t n;
    int C;
    int rows, width;       // of a tile
    int across;            // tiles beside each other
    int64_t tiles;
    uint32_t magic;        // ceil(2^32 / C): a place in a tile of whole rows by it is its row
};
inline ClassTiles class_tiles(int64_t n, int C, int values = kTileValues, int most_rows = kMostTileRows)
{
    ClassTiles t{n, C, 1, std::min(C, values), 0, 0, 0};
    t.rows = std::max(1, std::min(values / C, std::min(most_rows, kMostTileRows)));
    if (t.rows >= 8) t.rows = t.rows / 8 * 8;          // (whole pieces)
    t.across = (C + t.width - 1) / t.width;
    t.tiles = (n + t.rows - 1) / t.rows * t.across;
    t.magic = C > 1 ? (uint32_t)(((1ull << 32) + C - 1) / C) : 0u;
    return t;
}
__device__ inline int tile_row(const ClassTiles& t, int place) { return t.C > 1 ? (int)__umulhi((uint32_t)place, t.magic) : place; }

// Refuses a gradient that lies across the scores: in their place (a workgroup reads its scores before it writes) or beside them.
inline int check_gradient(const char* what, int dtype, int64_t n, int C, const void* X, const void* dX)
{
    const size_t bytes = (size_t)n * C * (dtype == SAR_F32 ? 4 : 2);
    SAR_CHECK_ARG(dX == X || apart(dX, bytes, X, bytes), "%s: dX overlaps X, and is not X", what);
    return SAR_OK;
}

// Refuses what no call takes.
inline int check_classes(const char* what, int dtype, int64_t n, int C, int k)
{
    if (dtype != SAR_F32 && dtype != SAR_BF16) return fail(SAR_ERR_UNSUPPORTED, "dtype %d is neither SAR_F32 nor SAR_BF16", dtype);
    SAR_CHECK_ARG(n >= 0 && C >= 1 && k >= 0, "%s: n = %lld rows of C = %d classes, k = %d", what, (long long)n, C, k);
    if (k > kMostTop) return fail(SAR_ERR_UNSUPPORTED, "%s: k = %d classes of a row (at most %d)", what, k, kMostTop);
    if (C > (1 << 30)) return fail(SAR_ERR_UNSUPPORTED, "%s: C = %d classes (at most 2^30)", what, C);
    return SAR_OK;
}

}  // namespace sar
