// Layer norm over the rows of a feature tensor, and its backward pass with the reduction of both parameters' gradients.
//
//   mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), xh = (x - mu) r, y = xh g + b
//   d = dy g:  dx = r (d - mean(d) - xh mean(d xh)),  dg = sum over rows of dy xh,  db = sum over rows of dy
//
// Both passes are bound by memory (a dozen operations a value): a row is read once, stays in registers (the deviations are taken
// from the row's own mean, not as a difference of two large sums), and is written once.  A row's lanes are a power of two that
// covers it in 16-byte pieces, so that narrow rows share a wavefront; rows of more than kWaveRow values take a workgroup.
// The backward pass keeps a lane's share of dg and db in registers over all rows that the lane meets; a workgroup's wavefronts add theirs up in
// LDS, every workgroup writes one row of partial sums, and a second launch adds those in a fixed order (few rows: columns_of_few): the result is the same
// in every run.
// 306250 x 256, fp32: forward 104 us, 6.0 TB/s (a large copy: 4.8, one of this size 5.3), with both forms in 8 bits 137; backward 177 + 5 us, 5.2 TB/s; 867187 x 256,
// bf16: 148 us, with both 230; backward from 8 bits 223; 1000003 x 47, bf16, from 8 bits 64 + 5 us, 3.5 TB/s of the bytes it needs, whose rows of 94 and 48 + 2
// bytes are no whole lines.
#include <algorithm>
#include <cmath>

#include "packed.h"
#include "sar_internal.h"

namespace sar {

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / kWave;
constexpr int kMostWidth = 8192;       // 32 values a thread of a workgroup
constexpr float kFar = 16.f;

// Sums over the TPR threads that hold a row (TPR <= 64: neighbours in a wavefront; kThreads: a workgroup, by way of `lds`).
template <int TPR, int M>
__device__ inline void row_sums(float (&v)[M], float (*lds)[kWaves])
{
    constexpr int L = TPR < kWave ? TPR : kWave;
#pragma unroll
    for (int m = 0; m < M; ++m) {
        auto dpp = [&](auto ctrl) {
            v[m] += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v[m]), decltype(ctrl)::value, 0xf, 0xf, false));
        };
        if constexpr (L >= 2) dpp(std::integral_constant<int, 0xB1>{});        // lane ^ 1
        if constexpr (L >= 4) dpp(std::integral_constant<int, 0x4E>{});        // lane ^ 2
        if constexpr (L >= 8) dpp(std::integral_constant<int, 0x141>{});       // the other four of eight
        if constexpr (L >= 16) dpp(std::integral_constant<int, 0x140>{});      // the other eight of sixteen
        if constexpr (L >= 32) v[m] += __shfl_xor(v[m], 16);
        if constexpr (L >= 64) v[m] += __shfl_xor(v[m], 32);
    }
    if constexpr (TPR > kWave) {
        __syncthreads();               // (what the last sums left there has been read)
#pragma unroll
        for (int m = 0; m < M; ++m)
            if (threadIdx.x % kWave == 0) lds[m][threadIdx.x / kWave] = v[m];
        __syncthreads();
#pragma unroll
        for (int m = 0; m < M; ++m) v[m] = (lds[m][0] + lds[m][1]) + (lds[m][2] + lds[m][3]);
    }
}

struct FwdArgs {
    const void* X;
    const float* gamma;
    const float* beta;
    void* Y;
    float* stats;
    int8_t *Xq, *Yq;
    uint8_t *Xe, *Ye;
    int64_t n;
    int D;
    float eps;
};

// The parameters of a thread's columns: `fill` where there are none and behind the row's end.
template <int N>
__device__ inline void load_params(const float* p, int c, int D, float fill, float (&v)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = fill;
    if (p == nullptr) return;
    if (c + N <= D) {
#pragma unroll
        for (int j = 0; j < N; j += 4) {
            const uint4 w = load16(p + c + j);
            v[j] = __uint_as_float(w.x), v[j + 1] = __uint_as_float(w.y), v[j + 2] = __uint_as_float(w.z), v[j + 3] = __uint_as_float(w.w);
        }
    } else {
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (c + j < D) v[j] = p[c + j];
    }
}

// NR rows a thread at once, R pieces of each.
template <typename T, int TPR, int R, int NR>
__global__ __launch_bounds__(kThreads) void k_norm_fwd(FwdArgs a)
{
    constexpr int N = Cols<T>::N, kRows = kThreads / TPR;
    __shared__ float lds[NR][kWaves];
    const int t = threadIdx.x % TPR;
    const int64_t row0 = (int64_t)blockIdx.x * (kRows * NR) + threadIdx.x / TPR;
    const int D = a.D;
    uint4 raw[NR][R];
    float v[NR][R][N], mean[NR], rstd[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
        for (int r = 0; r < R; ++r)        // (rows behind the last one are read as the last one)
        {
            const int64_t row = min(row0 + i * kRows, a.n - 1);
            raw[i][r] = Cols<T>::load(static_cast<const T*>(a.X) + row * D, (t + r * TPR) * N, D, (a.n - row) * D);
        }
    float g[R][N], b[R][N];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        load_params<N>(a.gamma, (t + r * TPR) * N, D, 1.f, g[r]);
        load_params<N>(a.beta, (t + r * TPR) * N, D, 0.f, b[r]);
    }
    const float over = 1.f / (float)D;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        mean[i] = 0.f;
#pragma unroll
        for (int r = 0; r < R; ++r) {
            Cols<T>::values(raw[i][r], (t + r * TPR) * N, D, v[i][r]);
#pragma unroll
            for (int j = 0; j < N; ++j) mean[i] += v[i][r][j];
        }
    }
    row_sums<TPR>(mean, lds);
    // (each rounded to nearest: the approximate reciprocal square root is an ulp off)
    auto deviations = [&](const float (&m)[NR], float (&r)[NR]) {
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            r[i] = 0.f;
#pragma unroll
            for (int k = 0; k < R; ++k)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    const float d = (t + k * TPR) * N + j < D ? v[i][k][j] - m[i] : 0.f;
                    r[i] = fmaf(d, d, r[i]);
                }
        }
        row_sums<TPR>(r, lds);
#pragma unroll
        for (int i = 0; i < NR; ++i) r[i] = 1.f / sqrtf(fmaf(r[i], over, a.eps));
    };
    bool any = false;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        mean[i] *= over;
        asm("" : "+v"(mean[i]));       // (rounded: not multiplied anew, unrounded, where it is subtracted)
    }
    deviations(mean, rstd);
    // A row that lies further from zero than 16 of its deviations: its mean is some units in the last place off, which count there (they would be
    // all that a constant row has left).  The deviations' own mean is added, and they are taken again.  (867187 x 256, bf16, where no row is such a
    // one: 148.6 us, without the look 146.7, with every row's mean taken twice 154; fp32 the same with and without.)
#pragma unroll
    for (int i = 0; i < NR; ++i) any |= fabsf(mean[i]) * rstd[i] > kFar;
    if (TPR > kWave ? any : __any(any)) {      // (of a row that a workgroup takes, the same for all threads)
        float left[NR], closer[NR];
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            left[i] = 0.f;
#pragma unroll
            for (int k = 0; k < R; ++k)
#pragma unroll
                for (int j = 0; j < N; ++j) left[i] += (t + k * TPR) * N + j < D ? v[i][k][j] - mean[i] : 0.f;
        }
        row_sums<TPR>(left, lds);
#pragma unroll
        for (int i = 0; i < NR; ++i) left[i] = fmaf(left[i], over, mean[i]);
        deviations(left, closer);
#pragma unroll
        for (int i = 0; i < NR; ++i)
            if (fabsf(mean[i]) * rstd[i] > kFar) mean[i] = left[i], rstd[i] = closer[i];       // (not a row that it came with)
    }
#pragma unroll
    for (int i = 0; i < NR; ++i) {
        const int64_t row = row0 + i * kRows;
        if (row >= a.n) continue;
        if (a.stats && t == 0) reinterpret_cast<float2*>(a.stats)[row] = make_float2(mean[i], rstd[i]);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const int c = (t + r * TPR) * N;
            if (a.Xq) store_packed<T>(a.Xq + row * packed_stride(D), a.Xe + row * packed_steps(D), c, D, v[i][r]);
            float y[N];
#pragma unroll
            for (int j = 0; j < N; ++j) y[j] = fmaf((v[i][r][j] - mean[i]) * rstd[i], g[r][j], b[r][j]);
            Cols<T>::store(static_cast<T*>(a.Y) + row * D, c, D, y);
            if (a.Yq) {
                // the values as they are stored, zeros behind the row's end
                if constexpr (sizeof(T) == 2) Cols<T>::unpack(Cols<T>::round(y), y);
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (c + j >= D) y[j] = 0.f;
                store_packed<T>(a.Yq + row * packed_stride(D), a.Ye + row * packed_steps(D), c, D, y);
            }
        }
    }
}

struct BwdArgs {
    const void* dY;
    const void* X;
    const int8_t* Xq;
    const uint8_t* Xe;
    const float* stats;
    const float* gamma;
    void* dX;
    float* partial;        // [workgroups, 2, D]
    float* dgamma;         // where one workgroup takes all rows, or (`few`) others take columns
    float* dbeta;
    int64_t n;
    int D;
    int accumulate;
    int groups;            // workgroups that take rows
    bool few;
};

// Few rows: both parts in one launch, workgroups behind those that take rows summing 16 columns of dgamma and dbeta each, their threads every 16th row, eight
// at a time.  With the host's 7.5 us a call: 1000 x 256, fp32, 7.5 us, by two launches 10.4; 1000 x 4096 18.7 and 19.7; 2000 x 256 10.1 and 10.4, 4000 x 256 19.1 and 10.3.
constexpr int kFewColumns = 16, kFewRows = 1024;
template <typename T, bool PACKED>
__device__ inline void columns_of_few(const BwdArgs& a, int c0)
{
    constexpr int kSlices = kThreads / kFewColumns, U = 8;
    __shared__ float part[2][kSlices][kFewColumns];
    const int k = threadIdx.x % kFewColumns, slice = threadIdx.x / kFewColumns, c = min(c0 + k, a.D - 1);
    auto value = [](const void* p, int64_t at) {
        if constexpr (sizeof(T) == 4) return static_cast<const float*>(p)[at];
        else return bf16_to_f32(static_cast<const bf16_t*>(p)[at]);
    };
    float dg = 0.f, db = 0.f;
    for (int64_t base = slice; base < a.n; base += U * kSlices) {
        float x[U], dy[U];
        float2 st[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t row = min(base + u * kSlices, a.n - 1);
            st[u] = reinterpret_cast<const float2*>(a.stats)[row];
            dy[u] = value(a.dY, row * a.D + c);
            if constexpr (PACKED) x[u] = (float)a.Xq[row * packed_stride(a.D) + c] * step_of(a.Xe[row * packed_steps(a.D) + c / kPackBlock]);
            else x[u] = value(a.X, row * a.D + c);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (base + u * kSlices >= a.n) continue;
            dg = fmaf(dy[u], (x[u] - st[u].x) * st[u].y, dg);
            db += dy[u];
        }
    }
    part[0][slice][k] = dg;
    part[1][slice][k] = db;
    __syncthreads();
    const int which = threadIdx.x / kFewColumns;
    float* out = which == 0 ? a.dgamma : a.dbeta;
    if (which > 1 || !out || c0 + k >= a.D) return;
    float v = 0.f;
#pragma unroll
    for (int s = 0; s < kSlices; ++s) v += part[which][s][k];
    out[c0 + k] = a.accumulate ? out[c0 + k] + v : v;
}

template <typename T, int TPR, int R, int NR, bool PACKED>
__global__ __launch_bounds__(kThreads) void k_norm_bwd(BwdArgs a)
{
    constexpr int N = Cols<T>::N, kRows = kThreads / TPR, kPieces = TPR * R;
    constexpr int kShare = TPR <= kWave ? kWaves : 1;                      // wavefronts that hold the same columns
    __shared__ float lds[2 * NR][kWaves];
    __shared__ float sums[kShare > 1 ? kWaves * 2 * kPieces * N : 1];
    if ((int)blockIdx.x >= a.groups) return columns_of_few<T, PACKED>(a, ((int)blockIdx.x - a.groups) * kFewColumns);
    const int t = threadIdx.x % TPR, D = a.D;
    const float over = 1.f / (float)D;
    float g[R][N], dg[R][N], db[R][N];
    uint4 within[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        load_params<N>(a.gamma, (t + r * TPR) * N, D, 1.f, g[r]);
        within[r] = Cols<T>::within((t + r * TPR) * N, D);
#pragma unroll
        for (int j = 0; j < N; ++j) dg[r][j] = db[r][j] = 0.f;
    }
    for (int64_t base = (int64_t)blockIdx.x * (kRows * NR); base < a.n; base += (int64_t)a.groups * (kRows * NR)) {
        uint4 xr[NR][R], dr[NR][R];
        typename PackedCols<N>::Raw xp[NR][R];
        float x[NR][R][N], dy[NR][R][N], s[2 * NR];
        float2 st[NR];
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const int64_t row = min(base + i * kRows + threadIdx.x / TPR, a.n - 1);
            st[i] = reinterpret_cast<const float2*>(a.stats)[row];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int c = (t + r * TPR) * N;
                if constexpr (PACKED)
                    xp[i][r] = PackedCols<N>::load(a.Xq + row * packed_stride(D), a.Xe + row * packed_steps(D), c, packed_stride(D));
                else
                    xr[i][r] = Cols<T>::load(static_cast<const T*>(a.X) + row * D, c, D, (a.n - row) * D);
                dr[i][r] = Cols<T>::load(static_cast<const T*>(a.dY) + row * D, c, D, (a.n - row) * D);
            }
        }
#pragma unroll
        for (int i = 0; i < NR; ++i) {
            const bool there = base + i * kRows + threadIdx.x / TPR < a.n;
            s[2 * i] = s[2 * i + 1] = 0.f;
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int c = (t + r * TPR) * N;
                if constexpr (PACKED) PackedCols<N>::values(xp[i][r], c, packed_stride(D), x[i][r]);
                else Cols<T>::values(xr[i][r], within[r], x[i][r]);
                Cols<T>::values(dr[i][r], within[r], dy[i][r]);
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    // (dy is zero behind a row's end; x is not looked at there, nor in a row that is not there)
                    const float h = c + j < D ? (x[i][r][j] - st[i].x) * st[i].y : 0.f;
                    const float d = dy[i][r][j] * g[r][j];
                    x[i][r][j] = h;
                    if (there) {
                        dg[r][j] = fmaf(dy[i][r][j], h, dg[r][j]);
                        db[r][j] += dy[i][r][j];
                    }
                    s[2 * i] += d;
                    s[2 * i + 1] = fmaf(d, h, s[2 * i + 1]);
                }
            }
        }
        if (a.dX) {
            row_sums<TPR>(s, lds);
#pragma unroll
            for (int i = 0; i < NR; ++i) {
                const int64_t row = base + i * kRows + threadIdx.x / TPR;
                if (row >= a.n) continue;
                const float c1 = s[2 * i] * over, c2 = s[2 * i + 1] * over;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    float o[N];
#pragma unroll
                    for (int j = 0; j < N; ++j) o[j] = st[i].y * (fmaf(dy[i][r][j], g[r][j], -c1) - x[i][r][j] * c2);
                    Cols<T>::store(static_cast<T*>(a.dX) + row * D, (t + r * TPR) * N, D, o);
                }
            }
        }
    }
    if (a.few || (a.partial == nullptr && a.dgamma == nullptr && a.dbeta == nullptr)) return;

    // a wavefront's lane groups, then a workgroup's wavefronts
    if constexpr (TPR < kWave) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < N; ++j)
#pragma unroll
                for (int o = TPR; o < kWave; o <<= 1) {
                    dg[r][j] += __shfl_xor(dg[r][j], o);
                    db[r][j] += __shfl_xor(db[r][j], o);
                }
    }
    auto put = [&](int which, int c, float v) {
        if (a.partial) {
            a.partial[((int64_t)blockIdx.x * 2 + which) * D + c] = v;
        } else if (float* out = which ? a.dbeta : a.dgamma) {
            out[c] = a.accumulate ? out[c] + v : v;
        }
    };
    if constexpr (kShare > 1) {
        const int wave = threadIdx.x / kWave;
        if (threadIdx.x % kWave < TPR) {
#pragma unroll
            for (int r = 0; r < R; ++r)
#pragma unroll
                for (int j = 0; j < N; ++j) {
                    sums[(wave * 2 + 0) * kPieces * N + (t + r * TPR) * N + j] = dg[r][j];
                    sums[(wave * 2 + 1) * kPieces * N + (t + r * TPR) * N + j] = db[r][j];
                }
        }
        __syncthreads();
        for (int k = threadIdx.x; k < 2 * kPieces * N; k += kThreads) {
            const int which = k / (kPieces * N), c = k % (kPieces * N);
            if (c >= D) continue;
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) v += sums[(w * 2 + which) * kPieces * N + c];
            put(which, c, v);
        }
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const int c = (t + r * TPR) * N + j;
                if (c < D) put(0, c, dg[r][j]), put(1, c, db[r][j]);
            }
    }
}

// dgamma, dbeta (+)= the partial sums of `groups` workgroups.  32 columns (a line) a workgroup of 1024 threads, which take every 32nd row of the
// sums, eight at a time.
__global__ __launch_bounds__(1024) void k_norm_params(const float* partial, int groups, int D, int accumulate, float* dgamma, float* dbeta)
{
    __shared__ float part[32][33];
    const int k = threadIdx.x % 32, slice = threadIdx.x / 32, c = blockIdx.x * 32 + k;
    float v = 0.f;
    if (c < 2 * D) {
        int w = slice;
        for (; w + 7 * 32 < groups; w += 8 * 32) {
            float x[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) x[u] = partial[(int64_t)(w + u * 32) * 2 * D + c];
            v += ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
        }
        for (; w < groups; w += 32) v += partial[(int64_t)w * 2 * D + c];
    }
    part[slice][k] = v;
    __syncthreads();
    if (slice == 0 && c < 2 * D) {
        float total = 0.f;
#pragma unroll
        for (int s = 0; s < 32; ++s) total += part[s][k];
        float* out = c < D ? dgamma : dbeta;
        if (out) out[c % D] = accumulate ? out[c % D] + total : total;
    }
}

// How a row of D values is laid over threads.
struct Shape {
    int tpr, r, nr;
};
Shape shape_of(int dtype, int D)
{
    const int vec = dtype == SAR_F32 ? 4 : 8, pieces = (D + vec - 1) / vec;
    int tpr = kPackBlock / vec;                     // (a block in 8 bits lies within a row's lanes)
    while (tpr < kWave && tpr < pieces) tpr <<= 1;
    int r = (pieces + tpr - 1) / tpr;
    // a thread holds up to 16 values of a row; a workgroup's 256 threads take up to 32
    if (r * vec > 16) tpr = kThreads, r = (pieces + tpr - 1) / tpr;
    int pow = 1;
    while (pow < r) pow <<= 1;
    return {tpr, pow, pow * vec <= 8 ? 2 : 1};
}

// Workgroups of the backward pass: four for every compute unit, no more than there are rows for, and of wide rows (whose sums are long) only
// so many that the sums stay within 16 MiB.  (306250 x 256 fp32, both launches: 1024 workgroups 188 us, 2048 202.)
constexpr int kBwdGroups = 1024;
int bwd_groups(int dtype, int64_t n, int D)
{
    const Shape s = shape_of(dtype, D);
    const int64_t rows = (int64_t)kThreads / s.tpr * s.nr;
    return (int)std::max<int64_t>(1, std::min<int64_t>((n + rows - 1) / rows, std::min(kBwdGroups, (1 << 21) / D)));
}

template <typename F>
int with_shape(int dtype, int D, F&& f)
{
    const Shape s = shape_of(dtype, D);
#define SAR_NORM_CASE(T, TPR, R, NR) \
    if (s.tpr == TPR && s.r == R) return f(T{}, std::integral_constant<int, TPR>{}, std::integral_constant<int, R>{}, std::integral_constant<int, NR>{})
    if (dtype == SAR_F32) {
        SAR_NORM_CASE(float, 8, 1, 2);
        SAR_NORM_CASE(float, 16, 1, 2);
        SAR_NORM_CASE(float, 32, 1, 2);
        SAR_NORM_CASE(float, 64, 1, 2);
        SAR_NORM_CASE(float, 64, 2, 2);
        SAR_NORM_CASE(float, 64, 4, 1);
        SAR_NORM_CASE(float, 256, 2, 2);
        SAR_NORM_CASE(float, 256, 4, 1);
        SAR_NORM_CASE(float, 256, 8, 1);
    } else {
        SAR_NORM_CASE(bf16_t, 4, 1, 2);
        SAR_NORM_CASE(bf16_t, 8, 1, 2);
        SAR_NORM_CASE(bf16_t, 16, 1, 2);
        SAR_NORM_CASE(bf16_t, 32, 1, 2);
        SAR_NORM_CASE(bf16_t, 64, 1, 2);
        SAR_NORM_CASE(bf16_t, 64, 2, 1);
        SAR_NORM_CASE(bf16_t, 256, 1, 2);
        SAR_NORM_CASE(bf16_t, 256, 2, 1);
        SAR_NORM_CASE(bf16_t, 256, 4, 1);
    }
#undef SAR_NORM_CASE
    return fail(SAR_ERR_UNSUPPORTED, "layer norm: no kernel for rows of %d values", D);
}

int check_shape(int dtype, int64_t n, int D)
{
    if (dtype != SAR_F32 && dtype != SAR_BF16) return fail(SAR_ERR_UNSUPPORTED, "dtype %d is neither SAR_F32 nor SAR_BF16", dtype);
    SAR_CHECK_ARG(n >= 0 && D >= 1, "layer norm: n = %lld rows of D = %d values", (long long)n, D);
    if (D > kMostWidth) return fail(SAR_ERR_UNSUPPORTED, "layer norm: rows of D = %d values (at most %d)", D, kMostWidth);
    return SAR_OK;
}

}  // namespace
}  // namespace sar

using namespace sar;

extern "C" int sar_layernorm_fwd(const void* X, const float* gamma, const float* beta, float eps, void* Y, float* stats, int dtype, int64_t n,
                                 int D, int8_t* Xq, uint8_t* Xe, int8_t* Yq, uint8_t* Ye, void* stream)
{
    SAR_TRY(check_shape(dtype, n, D));
    SAR_CHECK_ARG(eps >= 0.f && std::isfinite(eps), "layer norm: eps = %g", (double)eps);
    SAR_TRY(check_packed("Xq", Xq, Xe));
    SAR_TRY(check_packed("Yq", Yq, Ye));
    if (n == 0) return SAR_OK;
    SAR_CHECK_ARG(X && Y, "null pointer (X, Y)");
    const FwdArgs a{X, gamma, beta, Y, stats, Xq, Yq, Xe, Ye, n, D, eps};
    return with_shape(dtype, D, [&](auto T0, auto tpr, auto r, auto nr) {
        using T = decltype(T0);
        const int64_t rows = kThreads / tpr.value * nr.value, wgs = (n + rows - 1) / rows;
        if (wgs > most_workgroups(kThreads)) return fail(SAR_ERR_UNSUPPORTED, "layer norm: %lld rows are too many for one launch", (long long)n);
        k_norm_fwd<T, tpr.value, r.value, nr.value><<<(unsigned)wgs, kThreads, 0, as_stream(stream)>>>(a);
        SAR_LAUNCH_CHECK();
        return (int)SAR_OK;
    });
}

extern "C" int sar_layernorm_workspace_bytes(int64_t n, int D, size_t* bytes)
{
    SAR_CHECK_ARG(bytes, "bytes is null");
    SAR_TRY(check_shape(SAR_F32, n, D));
    *bytes = (size_t)std::max(bwd_groups(SAR_F32, n, D), bwd_groups(SAR_BF16, n, D)) * 2 * D * sizeof(float);
    return SAR_OK;
}

extern "C" int sar_layernorm_bwd(const void* dY, const void* X, const int8_t* Xq, const uint8_t* Xe, const float* stats, const float* gamma,
                                 int accumulate, void* dX, float* dgamma, float* dbeta, int dtype, int64_t n, int D, void* work,
                                 size_t work_bytes, void* stream)
{
    SAR_TRY(check_shape(dtype, n, D));
    SAR_TRY(check_packed("Xq", Xq, Xe));
    SAR_CHECK_ARG(!(X && Xq), "layer norm: X and Xq are both given");
    const bool params = dgamma || dbeta;
    if (n > 0) SAR_CHECK_ARG(dY && (X || Xq) && stats, "null pointer (dY, X or Xq, stats)");
    if ((n == 0 || !dX) && !params) return SAR_OK;
    hipStream_t st = as_stream(stream);
    // (dX in the place of an operand: that has to be read first)
    const size_t bytes = (size_t)n * D * (dtype == SAR_F32 ? 4 : 2);
    const bool few = params && n > 1 && n <= kFewRows &&
                     (!dX || (apart(dX, bytes, dY, bytes) && apart(dX, bytes, X, bytes) && apart(dX, bytes, Xq, (size_t)n * packed_stride(D)) &&
                              apart(dX, bytes, Xe, (size_t)n * packed_steps(D))));
    const int groups = n == 0 || (few && !dX) ? 0 : bwd_groups(dtype, n, D);
    // (one workgroup's sums need no second launch)
    const bool second = params && !few && groups != 1;
    if (second && groups > 0) {
        const size_t need = (size_t)groups * 2 * D * sizeof(float);
        SAR_CHECK_ARG(work && work_bytes >= need, "layer norm: work has %zu bytes, needs %zu", work ? work_bytes : 0, need);
        SAR_CHECK_ARG((reinterpret_cast<uintptr_t>(work) & 15) == 0, "layer norm: work must be 16-byte aligned");
    }
    if (groups > 0 || few) {
        const BwdArgs a{dY, X, Xq, Xe, stats, gamma, dX, second ? static_cast<float*>(work) : nullptr, second ? nullptr : dgamma,
                        second ? nullptr : dbeta, n, D, accumulate, groups, few};
        const int all = groups + (few ? (D + kFewColumns - 1) / kFewColumns : 0);
        SAR_TRY(with_shape(dtype, D, [&](auto T0, auto tpr, auto r, auto nr) {
            using T = decltype(T0);
            if (Xq) k_norm_bwd<T, tpr.value, r.value, nr.value, true><<<all, kThreads, 0, st>>>(a);
            else k_norm_bwd<T, tpr.value, r.value, nr.value, false><<<all, kThreads, 0, st>>>(a);
            SAR_LAUNCH_CHECK();
            return (int)SAR_OK;
        }));
    }
    if (second) {
        k_norm_params<<<(2 * D + 31) / 32, 1024, 0, st>>>(static_cast<const float*>(work), groups, D, accumulate, dgamma, dbeta);
        SAR_LAUNCH_CHECK();
    }
    return SAR_OK;
}
