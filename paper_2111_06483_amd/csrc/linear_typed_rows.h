// Rows times a small operand of their type, laid out in pieces: the kernels of linear_typed.hip, which says how they work, with what is done
// to a result before it is stored (`E`: nothing, or the bias, residual and activation of linear_act.hip).
#pragma once

#include <algorithm>

#include "linear_act.h"
#include "linear_pieces.h"
#include "linear_typed.h"

namespace sar {

namespace {

template <typename T>
struct Mode;
template <>
struct Mode<float> {
    static constexpr int kPieces = 3, kSteps = 2, kStage = 1;      // pieces of a weight; products of 16 a chunk; of those, how many a stage
};
template <>
struct Mode<bf16_t> {
    static constexpr int kPieces = 2, kSteps = 4, kStage = 2;
};
// Contraction values of a chunk: 128 bytes of a row.  Lanes 0..31 (half 0) hold the first 64 bytes of their rows, lanes 32..63 the others; in step s a
// lane contributes the eight values from 8 s on.
template <typename T>
constexpr int kChunk = 16 * Mode<T>::kSteps;

// How the four wavefronts share 128 rows and NT column tiles.  fp32: 32 rows and all columns each, so that a row's values are cut into pieces by
// one of them; bf16, where there is nothing to cut and reading B from LDS takes as long as multiplying (32 rows each: 64 KiB of LDS a
// chunk and wavefront for 64 products): 64 rows and half of the columns, a fragment of B for two products.
template <typename T, int NT>
struct Share {
    static constexpr int MR = sizeof(T) == 2 && NT >= 4 ? 2 : 1;       // row tiles a wavefront
    static constexpr int WC = MR, WR = 4 / WC, NW = NT / WC;           // wavefronts beside and below each other; column tiles a wavefront
    static constexpr int IL = NW < 4 ? NW : 4;
    // Column c (0..31) of column tile i: tiles in groups of four (or two) take columns by turns.
    static __host__ __device__ constexpr int column_of(int i, int c) { return i / IL * (32 * IL) + c * IL + i % IL; }
};

// A wavefront that has all columns of its rows (linear_kept.h).
template <typename T, int NT>
struct WholeShare {
    static constexpr int MR = 1, WC = 1, WR = 1, NW = NT, IL = NT < 4 ? NT : 4;
    static __host__ __device__ constexpr int column_of(int i, int c) { return i / IL * (32 * IL) + c * IL + i % IL; }
};

// ---- the small operand's pieces
//
// out [T, column blocks, chunks, steps, pieces, NT, 64 lanes] of 16 bytes: eight consecutive contraction values of a column.
struct LayArgs {
    const float* W;        // [T, K, F]
    uint4* out;
    int T, K, F, C, N, chunks, blocks;
    Types types;
    int4* list;            // the launch's list of row blocks: how many, then (type, first row, the row behind the last)
    int64_t most;          // places in it
    unsigned lay;          // workgroups that lay out weights; one for each type's rows behind them
};

// The blocks of kTileRows rows of type t, behind those of the types before it.
constexpr int kTileRows = 128;
__device__ inline void list_rows(const LayArgs& a, int t)
{
    __shared__ int64_t sums[4];
    auto blocks_of = [&](int u) {
        int64_t lo, hi;
        a.types.span(u, lo, hi);
        return (hi - lo + kTileRows - 1) / kTileRows;
    };
    int64_t before = 0;
    for (int u = threadIdx.x; u < t; u += 256) before += blocks_of(u);
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) before += (int64_t)__shfl_xor((long long)before, o);
    if (threadIdx.x % 64 == 0) sums[threadIdx.x / 64] = before;
    __syncthreads();
    before = sums[0] + sums[1] + sums[2] + sums[3];
    int64_t lo, hi;
    a.types.span(t, lo, hi);
    const int64_t mine = (hi - lo + kTileRows - 1) / kTileRows;
    // (bounds that do not ascend can ask for more blocks than there is room for: those are left out)
    for (int64_t k = threadIdx.x; k < mine && before + k < a.most; k += 256)
        a.list[1 + before + k] = make_int4(t, (int)(lo + k * kTileRows), (int)hi, 0);
    if (t == a.T - 1 && threadIdx.x == 0) a.list[0] = make_int4((int)min(before + mine, a.most), 0, 0, 0);
}

template <typename T, int NT, bool TRANS, typename SH = Share<T, NT>>
__global__ __launch_bounds__(256) void k_typed_lay(LayArgs a)
{
    constexpr int P = Mode<T>::kPieces, S = Mode<T>::kSteps;
    if (blockIdx.x >= a.lay) return list_rows(a, (int)(blockIdx.x - a.lay));
    const int64_t unit = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int lane = unit & 63, tile = (unit >> 6) % NT;
    int64_t rest = unit / (64 * NT);
    const int s = rest % S;
    rest /= S;
    const int chunk = (int)(rest % a.chunks);
    rest /= a.chunks;
    const int block = (int)(rest % a.blocks);
    const int t = (int)(rest / a.blocks);
    if (t >= a.T) return;
    const int n = block * (32 * NT) + SH::column_of(tile, lane & 31);
    const int c = chunk * kChunk<T> + (lane >> 5) * (kChunk<T> / 2) + s * 8;
    const float* W = a.W + (int64_t)t * a.K * a.F;
    float v[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        v[j] = 0.f;
        if (n < a.N && c + j < a.C) v[j] = TRANS ? W[(int64_t)n * a.F + c + j] : W[(int64_t)(c + j) * a.F + n];
        if (P == 3) v[j] *= chunk & 1 ? -kUp : kUp;
    }
    uint4* out = a.out + (((int64_t)(t * a.blocks + block) * a.chunks + chunk) * S + s) * (P * NT * 64) + tile * 64 + lane;
    if constexpr (P == 3) {
        uint4 p[3];
        split8(v, p);
#pragma unroll
        for (int k = 0; k < 3; ++k) out[k * NT * 64] = p[k];
    } else {
        uint32_t hi[4], lo[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            hi[j] = pack2_bf16(v[2 * j], v[2 * j + 1]);
            lo[j] = pack2_bf16(v[2 * j] - __uint_as_float(hi[j] << 16), v[2 * j + 1] - __uint_as_float(hi[j] & 0xffff0000u));
        }
        out[0] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        out[NT * 64] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
    }
}

// ---- rows times pieces

template <typename E>
struct RowsArgs {
    const void* A;         // [n, C]
    const uint4* B;        // as k_typed_lay leaves it
    const float* W;        // [T, K, F]
    void* out;             // [n, N]
    const int4* list;      // row blocks, as k_typed_lay leaves them
    int C, N, chunks, blocks;
    int K, F;
    E epilogue;
};

// A wavefront's tiles of 32 rows once more by the fp32 matrix instruction; column tiles from `first` on of the block that begins at n0.
template <typename T, typename SH, bool TRANS, typename E, typename P>
__device__ inline void exact_tiles(const RowsArgs<E>& a, const P& prologue, int t, int64_t i, int n0, int first, float16_t (&acc)[SH::NW])
{
    constexpr int NW = SH::NW;
    const T* row = static_cast<const T*>(a.A) + i * a.C;
    const int lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
    const float* W = a.W + (int64_t)t * a.K * a.F;
#pragma unroll
    for (int i = 0; i < NW; ++i) acc[i] = float16_t{};
    for (int k = 0; k < a.C; k += 2) {
        const bool in = k + h < a.C;
        float x = 0.f;
        if (in) {
            x = value_of(row[k + h]);
            if constexpr (P::kAny) x = formed_value<T>(prologue, x, i * a.C + k + h);
        }
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const int n = n0 + SH::column_of(first + i, c);
            float w = 0.f;
            if (in && n < a.N) w = TRANS ? W[(int64_t)n * a.F + k + h] : W[(int64_t)(k + h) * a.F + n];
            acc[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, w, acc[i], 0, 0, 0);
        }
    }
}

// The bias, residual and activation of a wavefront's tiles, which are stored: four rows of a group of column tiles at a time, from their residuals (which
// are under way some steps before) to the results, so that few values are in work at once beside the sums.
template <typename T, int IL>
struct __attribute__((packed, aligned(sizeof(T)))) Neighbours {
    uint32_t x[IL * sizeof(T) / 4];
    __device__ inline void values(float (&v)[IL]) const
    {
#pragma unroll
        for (int j = 0; j < IL; ++j) {
            if constexpr (sizeof(T) == 4) v[j] = __uint_as_float(x[j]);
            else v[j] = __uint_as_float(j % 2 ? x[j / 2] & 0xffff0000u : x[j / 2] << 16);
        }
    }
    __device__ inline void set(const float (&v)[IL])
    {
#pragma unroll
        for (int j = 0; j < IL * (int)sizeof(T) / 4; ++j) {
            if constexpr (sizeof(T) == 4) x[j] = __float_as_uint(v[j]);
            else x[j] = pack2_bf16(v[2 * j], v[2 * j + 1]);
        }
    }
};
// Where a wavefront's 32 rows lie: the first one, how many there are, the column tiles.  (Addresses are the tile's, the same for all lanes, and a lane's place
// in it: by 64 bits each they were a hundred registers.)
template <typename SH>
struct Place {
    int row0, rows, N, n0, first, lane;
    __device__ SAR_INLINE inline Place(int64_t r0, int64_t end, int N, int n0, int first, int lane)
        : row0(__builtin_amdgcn_readfirstlane((int)r0)), rows(__builtin_amdgcn_readfirstlane((int)min(end - r0, (int64_t)32))), N(N), n0(n0), first(first), lane(lane)
    {
    }
    __device__ SAR_INLINE inline int64_t tile() const { return (int64_t)row0 * N; }
    __device__ SAR_INLINE inline int column(int g) const { return n0 + SH::column_of(first + g * SH::IL, lane & 31); }
    __device__ SAR_INLINE inline int row(int r) const { return 8 * (r / 4) + 4 * (lane >> 5) + r % 4; }
};
// (a byte's place within 32 rows fits 32 bits; said so, it is added to the tile's address by the access itself)
template <typename V, typename T>
__device__ SAR_INLINE inline V* within_tile(T* base, uint32_t bytes)
{
    return reinterpret_cast<V*>(reinterpret_cast<uintptr_t>(base) + bytes);
}
// The residuals of step s: four rows of a group of column tiles.
template <typename T, typename SH>
__device__ SAR_INLINE inline void fetch_residual(const Epilogue& e, const Place<SH>& at, int s, Neighbours<T, SH::IL> (&out)[4])
{
    constexpr int IL = SH::IL;
    const int n = at.column(s / 4);
    const T* from = static_cast<const T*>(e.res) + at.tile();
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t place = (uint32_t)min(at.row(4 * (s % 4) + k), at.rows - 1) * (uint32_t)at.N;
        if (n + IL <= at.N) {
            out[k] = *within_tile<const Neighbours<T, IL>>(from, (place + (uint32_t)n) * (uint32_t)sizeof(T));
        } else {
            float v[IL];
#pragma unroll
            for (int j = 0; j < IL; ++j) v[j] = value_of(from[place + (uint32_t)min(n + j, at.N - 1)]);
            out[k].set(v);
        }
    }
}
template <typename T, typename SH, int NW>
__device__ SAR_INLINE inline void finish_tiles(const Epilogue& e, void* out, const Place<SH>& at, float16_t (&acc)[NW])
{
    constexpr int IL = SH::IL, kSteps = NW / IL * 4, kAhead = sizeof(T) == 4 ? 2 : 4;
    using V = Neighbours<T, IL>;
    const int N = at.N, rows = at.rows;
    const int64_t tile = at.tile();
    auto column = [&](int g) SAR_INLINE { return at.column(g); };
    auto row = [&](int r) SAR_INLINE { return at.row(r); };
    V res[kAhead][4];
    auto fetch = [&](int s) SAR_INLINE { fetch_residual<T, SH>(e, at, s, res[s % kAhead]); };
    auto store = [&](void* to, int g, int q, const float (&v)[4][IL]) SAR_INLINE {
        const int n = column(g);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const int i = row(4 * q + k);
            if (i >= rows || n >= N) continue;
            T* p = within_tile<T>(static_cast<T*>(to) + tile, ((uint32_t)i * (uint32_t)N + (uint32_t)n) * (uint32_t)sizeof(T));
            if (n + IL <= N) {
                V w;
                w.set(v[k]);
                *reinterpret_cast<V*>(p) = w;
            } else {
#pragma unroll
                for (int j = 0; j < IL; ++j)
                    if (n + j < N) p[j] = from_f32<T>(v[k][j]);
            }
        }
    };
    if (e.res) {
#pragma unroll
        for (int s = 0; s < kAhead - 1; ++s) fetch(s);
    }
    float bias[IL];
#pragma unroll
    for (int s = 0; s < kSteps; ++s) {
        const int g = s / 4, q = s % 4;
        if (e.res && s + kAhead - 1 < kSteps) fetch(s + kAhead - 1);
        if (q == 0) {
            const int n = column(g);
#pragma unroll
            for (int j = 0; j < IL; ++j) bias[j] = e.bias && n + j < N ? e.bias[n + j] : 0.f;
        }
        float v[4][IL];
        auto add_residual = [&]() SAR_INLINE {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                float r[IL];
                res[s % kAhead][k].values(r);
#pragma unroll
                for (int j = 0; j < IL; ++j) v[k][j] += r[j];
            }
        };
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int j = 0; j < IL; ++j) v[k][j] = acc[g * IL + j][4 * q + k] + bias[j];
        if (e.res && !e.after) add_residual();
        if (e.pre) store(e.pre, g, q, v);
        with_act(e.act, [&](auto act) SAR_INLINE {
#pragma unroll
            for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int j = 0; j < IL; ++j) v[k][j] = act_of<decltype(act)::value>(v[k][j]);
        });
        if (e.res && e.after) add_residual();
        store(out, g, q, v);
        __builtin_amdgcn_sched_barrier(0);
    }
}

// A wavefront's tiles of rows r0..r0+31 (up to `end`), column tiles from `first` on.
template <typename T, typename SH, bool TRANS, int NW, typename E, typename P>
__device__ SAR_INLINE inline void store_tiles(const RowsArgs<E>& a, const P& prologue, int t, int64_t r0, int64_t end, int n0, int first, float16_t (&acc)[NW])
{
    constexpr int IL = SH::IL;
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));         // (as above: nothing of this is carried through the products)
    const int h = lane >> 5;
    if (r0 >= end) return;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < NW; ++i) odd |= not_finite(acc[i]);
    if (__any(odd))
        exact_tiles<T, SH, TRANS>(a, prologue, t, min(r0 + (lane & 31), end - 1), n0, first, acc);

    if constexpr (E::kAny) {
        finish_tiles<T, SH, NW>(a.epilogue, a.out, Place<SH>(r0, end, a.N, n0, first, lane), acc);
        return;
    }
    // lane holds columns of its place; register r holds row 8*(r/4) + 4*h + r%4
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int64_t i = r0 + 8 * (r / 4) + 4 * h + r % 4;
        if (i >= end) continue;
        T* out = static_cast<T*>(a.out) + i * a.N;
#pragma unroll
        for (int g = 0; g < NW / IL; ++g) {
            const int n = n0 + SH::column_of(first + g * IL, lane & 31);
            const float16_t* v = &acc[g * IL];
            if (n + IL <= a.N) {
                if constexpr (sizeof(T) == 4) {
                    struct __attribute__((packed, aligned(4))) V { float x[IL]; } w;
#pragma unroll
                    for (int j = 0; j < IL; ++j) w.x[j] = v[j][r];
                    *reinterpret_cast<V*>(out + n) = w;
                } else {
                    struct __attribute__((packed, aligned(2))) V { uint32_t x[IL / 2]; } w;
#pragma unroll
                    for (int j = 0; j < IL / 2; ++j) w.x[j] = pack2_bf16(v[2 * j][r], v[2 * j + 1][r]);
                    *reinterpret_cast<V*>(out + n) = w;
                }
            } else {
#pragma unroll
                for (int j = 0; j < IL; ++j)
                    if (n + j < a.N) out[n + j] = from_f32<T>(v[j][r]);
            }
        }
    }
}

using LdsPtr = __attribute__((address_space(3))) void;
using GlobalSrc = const __attribute__((address_space(1))) void;
constexpr int kTileWaves = kTileRows / 32;

// KiB of B a stage.
template <typename T, int NT>
constexpr int kStageFrags = Mode<T>::kStage * Mode<T>::kPieces * NT;

template <typename T, int NT>
__device__ SAR_INLINE inline void copy_stage(uint4* to, const uint4* from)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int f = 0; f < (kStageFrags<T, NT> + kTileWaves - 1) / kTileWaves; ++f) {
        if (kStageFrags<T, NT> % kTileWaves && wave + f * kTileWaves >= kStageFrags<T, NT>) continue;
        __builtin_amdgcn_global_load_lds((GlobalSrc*)(from + (wave + f * kTileWaves) * 64 + lane), (LdsPtr*)(to + (wave + f * kTileWaves) * 64), 16, 0, 0);
    }
}

// A stage's products of the rows' fragments p with the pieces of B at `b`.
template <typename T, int NT, int MR, int NW, int SP>
__device__ SAR_INLINE inline void multiply_stage(const uint4* b, const uint4 (&p)[MR][Mode<T>::kStage][SP], float sign, float16_t (&acc)[MR][NW])
{
    constexpr int P = Mode<T>::kPieces, SB = Mode<T>::kStage;
    if constexpr (P == 3) {
        // a tile's products run while the sums of the tile before are added and the pieces of the next one are read
        static_assert(MR == 1 && SB == 1, "one product of 16 a stage and row tile");
        uint4 w[2][3];
        float16_t sum, last;
#pragma unroll
        for (int k = 0; k < 3; ++k) w[0][k] = b[k * NT * 64];
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            sum = float16_t{};
            if (i + 1 < NW) {
#pragma unroll
                for (int k = 0; k < 3; ++k) w[(i + 1) & 1][k] = b[(k * NT + i + 1) * 64];
            }
#pragma unroll
            for (int k = 0; k < 6; ++k)
                sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, p[0][0][kTerm[k][0]]),
                                                              __builtin_bit_cast(bf16x8_t, w[i & 1][kTerm[k][1]]), sum, 0, 0, 0);
            if (i > 0) {
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[0][i - 1][r] = fmaf(last[r], sign, acc[0][i - 1][r]);
                // (here, not where the compiler would have them: behind the stage, with all tiles' products kept until then)
                asm volatile("" : "+v"(acc[0][i - 1]));
            }
            last = sum;
#pragma unroll
            for (int k = 0; k < 6; ++k) {
                __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);                        // a product
                if (k % 2 == 0) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);       // a read
                __builtin_amdgcn_sched_group_barrier(0x002, 3, 0);                        // additions
            }
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[0][NW - 1][r] = fmaf(last[r], sign, acc[0][NW - 1][r]);
        asm volatile("" : "+v"(acc[0][NW - 1]));
    } else {
#pragma unroll
        for (int s = 0; s < SB; ++s)
#pragma unroll
            for (int i = 0; i < NW; ++i)
#pragma unroll
                for (int k = P - 1; k >= 0; --k) {
                    const uint4 w = b[((s * P + k) * NT + i) * 64];
#pragma unroll
                    for (int m = 0; m < MR; ++m)
                        acc[m][i] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, p[m][s][0]),
                                                                            __builtin_bit_cast(bf16x8_t, w), acc[m][i], 0, 0, 0);
                }
    }
}

// A stage's products, while the next stage's pieces (`from`, null where there is none) go to `to`.  (A function of its own for its arguments'
// sake: it is by them that the compiler knows the two apart.  Otherwise every first read of a stage waits for the copy that was just begun:
// 237500 x 256 -> 256, fp32, 226 us for 195.)
template <typename T, int NT, int SP, typename Fetch>
__device__ SAR_INLINE inline void stage_products(uint4* __restrict__ to, const uint4* from, const uint4* __restrict__ b,
                                                 const uint4 (&p)[Share<T, NT>::MR][Mode<T>::kStage][SP], float sign, bool works,
                                                 float16_t (&acc)[Share<T, NT>::MR][Share<T, NT>::NW], Fetch&& fetch_rows)
{
    if (from) copy_stage<T, NT>(to, from);
    fetch_rows();
    if (works) multiply_stage<T, NT, Share<T, NT>::MR, Share<T, NT>::NW>(b, p, sign, acc);
}

template <typename T, int NT, bool TRANS, typename E, typename Q>
__global__ __launch_bounds__(kTileWaves * 64, 2) void k_typed_rows(RowsArgs<E> a, Q prologue)
{
    constexpr int P = Mode<T>::kPieces, S = Mode<T>::kSteps, CH = kChunk<T>, N = Cols<T>::N, SB = Mode<T>::kStage;
    using Sh = Share<T, NT>;
    constexpr int MR = Sh::MR, NW = Sh::NW;
    constexpr int kRaw = 64 / 16;                        // 16-byte pieces of a row that a lane holds of a chunk
    constexpr int kFrags = kStageFrags<T, NT>, kSP = P == 3 ? 3 : 1;
    static_assert(S / SB == 2, "a barrier between taking a chunk's rows and handing over the next one's");
    // Bf16 rows in two pieces are multiplied in two turns a chunk, by their first pieces and by their second ones, which wait in registers that hold the next
    // chunk's rows afterwards.
    constexpr int kTurns = Q::kAny && sizeof(T) == 2 ? 2 : 1;
    static_assert(!Q::kAny || Q::kForms || sizeof(T) == 2, "two pieces of bf16");
    extern __shared__ __attribute__((aligned(16))) uint4 lds[];      // [2][kFrags][64] of B, [4][32][8] of rows
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, h = lane >> 5, wr = wave / Sh::WC, wc = wave % Sh::WC;

    // a workgroup takes every gridDim.x-th of the listed row blocks; what it multiplies first of the next one travels while it
    // finishes and stores this one
    const int total = a.list[0].x;
    struct Tile {
        int t, first, end;
    };
    auto tile_at = [&](int i) SAR_INLINE {
        const int4 v = a.list[1 + min(i, total - 1)];
        return Tile{__builtin_amdgcn_readfirstlane(v.x), __builtin_amdgcn_readfirstlane(v.y), __builtin_amdgcn_readfirstlane(v.z)};
    };
    if ((int)blockIdx.x >= total) return;

    auto pieces_of = [&](const Tile& w, int stage) SAR_INLINE {
        return a.B + (((int64_t)(w.t * a.blocks + blockIdx.y) * a.chunks) * (S / SB) + stage) * (kFrags * 64);
    };
    // Rows come by whole lines: eight lanes a row, eight rows a load, 32 rows a wavefront.  (By the lanes that multiply them, 16 bytes of
    // 64 rows a load, every line was asked for once for each of its pieces.)  They are handed to those lanes through LDS, pieces turned by the row
    // so that neither side meets a bank twice.
    auto brings = [&](const Tile& w) SAR_INLINE { return w.first + wave * 32 < w.end; };
    auto fetch_from = [&](const void* p, const Tile& w, int chunk, uint4 (&v)[kRaw]) SAR_INLINE {
        const int64_t r0 = w.first + wave * 32;
        const T* tile = static_cast<const T*>(p) + r0 * a.C;
        const uint32_t most = (uint32_t)min((int64_t)w.end - 1 - r0, (int64_t)31);
        const int c = chunk * CH + (lane & 7) * N;
        if (a.C >= N) {
            const uint32_t at = (uint32_t)min(c, a.C - N);
#pragma unroll
            for (int p = 0; p < kRaw; ++p) v[p] = load16(tile + (min((uint32_t)(8 * p + (lane >> 3)), most) * (uint32_t)a.C + at));
        } else {
#pragma unroll
            for (int p = 0; p < kRaw; ++p) v[p] = Cols<T>::load(tile + min((uint32_t)(8 * p + (lane >> 3)), most) * (uint32_t)a.C, c, a.C, a.C);
        }
    };
    uint4 pre[Q::kAny ? kRaw : 1];
    auto fetch_a = [&](const Tile& w, int chunk, uint4 (&v)[kRaw]) SAR_INLINE {
        fetch_from(a.A, w, chunk, v);
        if constexpr (Q::kForms) fetch_from(prologue.pre, w, chunk, pre);
        else if constexpr (Q::kAny) fetch_from(prologue.low, w, chunk, pre);
    };
    uint4* const rows = lds + 2 * kFrags * 64;
    uint4 later[kTurns > 1 ? kRaw : 1];
    auto to_lds = [&](const uint4 (&v)[kRaw]) SAR_INLINE {
#pragma unroll
        for (int p = 0; p < kRaw; ++p) rows[wave * 256 + (8 * p + (lane >> 3)) * 8 + ((lane & 7) ^ (lane >> 3))] = v[p];
    };
    auto hand_over = [&](const Tile& w, int chunk, uint4 (&v)[kRaw]) SAR_INLINE {
        const int c = chunk * CH + (lane & 7) * N;
        if ((chunk + 1) * CH > a.C && c + N > a.C) {
#pragma unroll
            for (int p = 0; p < kRaw; ++p) {
                auto cut = [&](uint4& u) SAR_INLINE {
                    if (c >= a.C) u = make_uint4(0u, 0u, 0u, 0u);
                    else if (a.C >= N) u = front_of_piece<T>(u, a.C - c);
                };
                cut(v[p]);
                if constexpr (Q::kAny) cut(pre[p]);
            }
        }
        if constexpr (Q::kForms) {
#pragma unroll
            for (int p = 0; p < kRaw; ++p) form_piece<T>(prologue.act, v[p], pre[p], later[kTurns > 1 ? p : 0]);
            if (prologue.formed && blockIdx.y == 0) {
#pragma unroll
                for (int p = 0; p < kRaw; ++p) {
                    const int64_t i = w.first + wave * 32 + 8 * p + (lane >> 3);
                    float u[N];
                    Cols<T>::unpack(v[p], u);
                    if (i < w.end) Cols<T>::store(static_cast<T*>(prologue.formed) + i * a.C, c, a.C, u);
                }
            }
        } else if constexpr (Q::kAny) {
#pragma unroll
            for (int p = 0; p < kRaw; ++p) later[p] = pre[p];
        }
        to_lds(v);
    };
    auto take = [&](int m, uint4 (&v)[kRaw]) SAR_INLINE {
#pragma unroll
        for (int p = 0; p < kRaw; ++p) v[p] = rows[(wr * MR + m) * 256 + (lane & 31) * 8 + ((h * kRaw + p) ^ (lane & 7))];
    };

    uint4 raw[kRaw];
    Tile tile = tile_at(blockIdx.x);
    copy_stage<T, NT>(lds, pieces_of(tile, 0));
    if (brings(tile)) {
        fetch_a(tile, 0, raw);
        hand_over(tile, 0, raw);
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    const int stages = a.chunks * (S / SB);
    int buffer = 0;
    for (int index = blockIdx.x; index < total; index += gridDim.x) {
        const bool another = index + (int)gridDim.x < total;
        const Tile after = tile_at(index + gridDim.x);
        const bool works = tile.first + wr * MR * 32 < tile.end, here = brings(tile), there = another && brings(after);
        float16_t acc[MR][NW];
#pragma unroll
        for (int m = 0; m < MR; ++m)
#pragma unroll
            for (int i = 0; i < NW; ++i) acc[m][i] = float16_t{};
        float sign = kDown * kDown;        // (fp32 products: rows' and weights' 2^24)
        for (int turn = 0; turn < a.chunks * kTurns; ++turn) {
            const int chunk = turn / kTurns;
            const bool second = kTurns > 1 && turn % kTurns == 0;         // the next turn is that of this chunk's second pieces
            const bool more = chunk + 1 < a.chunks, coming = !second && (more ? here : there);
            uint4 p[S / SB][MR][SB][kSP];
            if (works) {
#pragma unroll
                for (int m = 0; m < MR; ++m) {
                    uint4 x[kRaw];
                    take(m, x);
#pragma unroll
                    for (int s = 0; s < S; ++s) {
                        if constexpr (P == 3) {
                            float v[8] = {__uint_as_float(x[2 * s].x), __uint_as_float(x[2 * s].y), __uint_as_float(x[2 * s].z),
                                          __uint_as_float(x[2 * s].w), __uint_as_float(x[2 * s + 1].x), __uint_as_float(x[2 * s + 1].y),
                                          __uint_as_float(x[2 * s + 1].z), __uint_as_float(x[2 * s + 1].w)};
#pragma unroll
                            for (int j = 0; j < 8; ++j) v[j] *= kUp;
                            split8(v, p[s / SB][m][s % SB]);
                        } else {
                            p[s / SB][m][s % SB][0] = x[s];
                        }
                    }
                }
            }
#pragma unroll
            for (int part = 0; part < S / SB; ++part) {
                const int stage = chunk * (S / SB) + part;
                const bool again = second && part == S / SB - 1;
                const uint4* from = again ? pieces_of(tile, chunk * (S / SB)) : stage + 1 < stages ? pieces_of(tile, stage + 1) : another ? pieces_of(after, 0) : nullptr;
                stage_products<T, NT>(lds + (buffer ^ 1) * kFrags * 64, from, lds + (buffer * kFrags + wc * NW) * 64 + lane, p[part], sign, works,
                                      acc, [&]() SAR_INLINE {
                                          if (part == 0 && coming) fetch_a(more ? tile : after, more ? chunk + 1 : 0, raw);
                                      });
                if (part == S / SB - 1 && coming) hand_over(more ? tile : after, more ? chunk + 1 : 0, raw);
                if constexpr (kTurns > 1) {
                    if (again && here) to_lds(later);
                }
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                __syncthreads();
                buffer ^= 1;
            }
            sign = -sign;
        }
        const Tile done = tile;
        tile = after;
#pragma unroll
        for (int m = 0; m < MR; ++m)
            store_tiles<T, Sh, TRANS>(a, prologue, done.t, done.first + (wr * MR + m) * 32, done.end, blockIdx.y * (32 * NT), wc * NW, acc[m]);
    }
}

// Column tiles a workgroup forms at once: as few as let all workgroups run at the same time (three a compute unit of two tiles, two of more).
// 256 -> 256, fp32, by two / four / eight: 16 thousand rows 27.3 / 28.6 / 31.6 us, 32 thousand 42.8 / 34.0 / 34.0, 48 thousand 52.1 / 53.3 / 48.2; bf16
// 17.0 / 16.9 / 19.7, 22.9 / 20.7 / 20.6, 26.4 / 29.1 / 26.0.  Beyond that eight, so that rows are read once, unless half of them would lie behind the last column.
int tiles_of(int64_t n, int N)
{
    auto groups = [&](int tiles) { return (n + kTileRows - 1) / kTileRows * ((N + 32 * tiles - 1) / (32 * tiles)); };
    if (N <= 64 || groups(2) <= 256 * 3) return 2;
    return groups(4) <= 256 * 2 || (N + 127) / 128 % 2 ? 4 : 8;
}

template <typename T, int NT, bool TRANS, typename E, typename Q>
int run_rows(const RowsArgs<E>& a, const Q& prologue, LayArgs l, hipStream_t st)
{
    const int64_t units = (int64_t)l.T * l.blocks * l.chunks * Mode<T>::kSteps * NT * 64, lay = (units + 255) / 256;
    l.lay = (unsigned)lay;
    k_typed_lay<T, NT, TRANS><<<(unsigned)lay + l.T, 256, 0, st>>>(l);
    SAR_LAUNCH_CHECK();
    // as many workgroups as a compute unit holds (three of two column tiles, two of more), each with every so-manyth block; of eight, two turns of
    // them, so that no unit waits long for the last (100000 x 512 -> 512, fp32, 332 us by one turn, 302 by two, 301 by four; 237500 x 256 -> 256 197, 191, 193)
    constexpr int kGroups = NT == 2 ? 3 : NT == 4 ? 2 : 4;
    constexpr size_t shared = (size_t)(2 * kStageFrags<T, NT> + 4 * kTileWaves) * 1024;
    auto* fn = k_typed_rows<T, NT, TRANS, E, Q>;
    if (shared > 65536) SAR_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, (int)shared));
    const int64_t groups = std::min<int64_t>(l.types.n / kTileRows + l.T, std::max(1, 256 * kGroups / l.blocks));
    fn<<<dim3((unsigned)groups, l.blocks), kTileWaves * 64, shared, st>>>(a, prologue);
    SAR_LAUNCH_CHECK();
    return SAR_OK;
}

// Bytes of B's pieces for contraction C and N columns (either type, either number of tiles).
size_t lay_bytes(int C, int N, int T)
{
    const size_t f32 = (size_t)((C + 31) / 32) * 2 * 3, b16 = (size_t)((C + 63) / 64) * 4 * 2;
    return (size_t)T * ((N + 255) / 256 * 8) * std::max(f32, b16) * 1024;
}
int64_t most_tiles(int64_t n, int T) { return n / kTileRows + T; }
size_t list_bytes(int64_t n, int T) { return (size_t)(most_tiles(n, T) + 1) * sizeof(int4); }

// out [n, N] = A [n, C] B; TRANS: B = W^T.
template <typename T, bool TRANS, typename E = NoEpilogue, typename Q = NoPrologue>
int rows_product(const void* A, const float* W, const Types& types, void* out, int K, int F, void* work, hipStream_t st, const E& e = {}, const Q& q = {})
{
    // (formed bf16 rows, whose pieces take registers: four column tiles at most; 867187 x 256 -> 256, by GELU, 803 us, by eight, which spill 57, 951)
    const int C = TRANS ? F : K, N = TRANS ? K : F, NT = std::min(tiles_of(types.n, N), Q::kForms && sizeof(T) == 2 ? 4 : 8);
    if (!Q::kAny && few_blocks(types, N)) return few_product(sizeof(T) == 4 ? SAR_F32 : SAR_BF16, TRANS, {A, W, out, types, C, N, K, F}, e, st);
    const int chunks = (C + kChunk<T> - 1) / kChunk<T>, blocks = (N + 32 * NT - 1) / (32 * NT);
    const int64_t most = most_tiles(types.n, types.T);
    int4* const list = static_cast<int4*>(work);
    uint4* const pieces = static_cast<uint4*>(work) + (most + 1);
    const RowsArgs<E> a{A, pieces, W, out, list, C, N, chunks, blocks, K, F, e};
    const LayArgs l{W, pieces, types.T, K, F, C, N, chunks, blocks, types, list, most, 0};
    if constexpr (!(Q::kForms && sizeof(T) == 2)) {
        if (NT == 8) return run_rows<T, 8, TRANS>(a, q, l, st);
    }
    return NT == 2 ? run_rows<T, 2, TRANS>(a, q, l, st) : run_rows<T, 4, TRANS>(a, q, l, st);
}

}  // namespace
}  // namespace sar
