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
#include <algorithm>

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

template <typename T, int NT, bool TRANS>
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
    const int n = block * (32 * NT) + Share<T, NT>::column_of(tile, lane & 31);
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

struct RowsArgs {
    const void* A;         // [n, C]
    const uint4* B;        // as k_typed_lay leaves it
    const float* W;        // [T, K, F]
    void* out;             // [n, N]
    const int4* list;      // row blocks, as k_typed_lay leaves them
    int C, N, chunks, blocks;
    int K, F;
};

// A wavefront's tiles of 32 rows once more by the fp32 matrix instruction; column tiles from `first` on of the block that begins at n0.
template <typename T, int NT, bool TRANS>
__device__ inline void exact_tiles(const RowsArgs& a, int t, const T* row, int n0, int first, float16_t (&acc)[Share<T, NT>::NW])
{
    constexpr int NW = Share<T, NT>::NW;
    const int lane = threadIdx.x & 63, c = lane & 31, h = lane >> 5;
    const float* W = a.W + (int64_t)t * a.K * a.F;
#pragma unroll
    for (int i = 0; i < NW; ++i) acc[i] = float16_t{};
    for (int k = 0; k < a.C; k += 2) {
        const bool in = k + h < a.C;
        float x = 0.f;
        if (in) {
            if constexpr (sizeof(T) == 4) x = row[k + h];
            else x = bf16_to_f32(row[k + h]);
        }
#pragma unroll
        for (int i = 0; i < NW; ++i) {
            const int n = n0 + Share<T, NT>::column_of(first + i, c);
            float w = 0.f;
            if (in && n < a.N) w = TRANS ? W[(int64_t)n * a.F + k + h] : W[(int64_t)(k + h) * a.F + n];
            acc[i] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, w, acc[i], 0, 0, 0);
        }
    }
}

// A wavefront's tiles of rows r0..r0+31 (up to `end`), column tiles from `first` on.
template <typename T, int NT, bool TRANS, int NW>
__device__ SAR_INLINE inline void store_tiles(const RowsArgs& a, int t, int64_t r0, int64_t end, int first, float16_t (&acc)[NW])
{
    constexpr int IL = Share<T, NT>::IL;
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));         // (as above: nothing of this is carried through the products)
    const int h = lane >> 5, n0 = blockIdx.y * (32 * NT);
    if (r0 >= end) return;
    bool odd = false;
#pragma unroll
    for (int i = 0; i < NW; ++i) odd |= not_finite(acc[i]);
    if (__any(odd))
        exact_tiles<T, NT, TRANS>(a, t, static_cast<const T*>(a.A) + min(r0 + (lane & 31), end - 1) * a.C, n0, first, acc);

    // lane holds columns of its place; register r holds row 8*(r/4) + 4*h + r%4
#pragma unroll
    for (int r = 0; r < 16; ++r) {
        const int64_t i = r0 + 8 * (r / 4) + 4 * h + r % 4;
        if (i >= end) continue;
        T* out = static_cast<T*>(a.out) + i * a.N;
#pragma unroll
        for (int g = 0; g < NW / IL; ++g) {
            const int n = n0 + Share<T, NT>::column_of(first + g * IL, lane & 31);
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

template <typename T, int NT, bool TRANS>
__global__ __launch_bounds__(kTileWaves * 64, 2) void k_typed_rows(RowsArgs a)
{
    constexpr int P = Mode<T>::kPieces, S = Mode<T>::kSteps, CH = kChunk<T>, N = Cols<T>::N, SB = Mode<T>::kStage;
    using Sh = Share<T, NT>;
    constexpr int MR = Sh::MR, NW = Sh::NW;
    constexpr int kRaw = 64 / 16;                        // 16-byte pieces of a row that a lane holds of a chunk
    constexpr int kFrags = kStageFrags<T, NT>, kSP = P == 3 ? 3 : 1;
    static_assert(S / SB == 2, "a barrier between taking a chunk's rows and handing over the next one's");
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
    auto fetch_a = [&](const Tile& w, int chunk, uint4 (&v)[kRaw]) SAR_INLINE {
        const int64_t r0 = w.first + wave * 32;
        const T* tile = static_cast<const T*>(a.A) + r0 * a.C;
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
    uint4* const rows = lds + 2 * kFrags * 64;
    auto hand_over = [&](int chunk, uint4 (&v)[kRaw]) SAR_INLINE {
        const int c = chunk * CH + (lane & 7) * N;
        if ((chunk + 1) * CH > a.C && c + N > a.C) {
#pragma unroll
            for (int p = 0; p < kRaw; ++p) {
                if (c >= a.C) v[p] = make_uint4(0u, 0u, 0u, 0u);
                else if (a.C >= N) v[p] = front_of_piece<T>(v[p], a.C - c);
            }
        }
#pragma unroll
        for (int p = 0; p < kRaw; ++p) rows[wave * 256 + (8 * p + (lane >> 3)) * 8 + ((lane & 7) ^ (lane >> 3))] = v[p];
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
        hand_over(0, raw);
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
        for (int chunk = 0; chunk < a.chunks; ++chunk) {
            const bool more = chunk + 1 < a.chunks, coming = more ? here : there;
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
                const uint4* from = stage + 1 < stages ? pieces_of(tile, stage + 1) : another ? pieces_of(after, 0) : nullptr;
                stage_products<T, NT>(lds + (buffer ^ 1) * kFrags * 64, from, lds + (buffer * kFrags + wc * NW) * 64 + lane, p[part], sign, works,
                                      acc, [&]() SAR_INLINE {
                                          if (part == 0 && coming) fetch_a(more ? tile : after, more ? chunk + 1 : 0, raw);
                                      });
                if (part == S / SB - 1 && coming) hand_over(more ? chunk + 1 : 0, raw);
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
            store_tiles<T, NT, TRANS>(a, done.t, done.first + (wr * MR + m) * 32, done.end, wc * NW, acc[m]);
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

template <typename T, int NT, bool TRANS>
int run_rows(const RowsArgs& a, LayArgs l, hipStream_t st)
{
    const int64_t units = (int64_t)l.T * l.blocks * l.chunks * Mode<T>::kSteps * NT * 64, lay = (units + 255) / 256;
    l.lay = (unsigned)lay;
    k_typed_lay<T, NT, TRANS><<<(unsigned)lay + l.T, 256, 0, st>>>(l);
    SAR_LAUNCH_CHECK();
    // as many workgroups as a compute unit holds (three of two column tiles, two of more), each with every so-manyth block; of eight, two turns of
    // them, so that no unit waits long for the last (100000 x 512 -> 512, fp32, 332 us by one turn, 302 by two, 301 by four; 237500 x 256 -> 256 197, 191, 193)
    constexpr int kGroups = NT == 2 ? 3 : NT == 4 ? 2 : 4;
    constexpr size_t shared = (size_t)(2 * kStageFrags<T, NT> + 4 * kTileWaves) * 1024;
    auto* fn = k_typed_rows<T, NT, TRANS>;
    if (shared > 65536) SAR_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, (int)shared));
    const int64_t groups = std::min<int64_t>(l.types.n / kTileRows + l.T, std::max(1, 256 * kGroups / l.blocks));
    fn<<<dim3((unsigned)groups, l.blocks), kTileWaves * 64, shared, st>>>(a);
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
template <typename T, bool TRANS>
int rows_product(const void* A, const float* W, const Types& types, void* out, int K, int F, void* work, hipStream_t st)
{
    const int C = TRANS ? F : K, N = TRANS ? K : F, NT = tiles_of(types.n, N);
    if (few_blocks(types, N)) return few_product(sizeof(T) == 4 ? SAR_F32 : SAR_BF16, TRANS, {A, W, out, types, C, N, K, F}, st);
    const int chunks = (C + kChunk<T> - 1) / kChunk<T>, blocks = (N + 32 * NT - 1) / (32 * NT);
    const int64_t most = most_tiles(types.n, types.T);
    int4* const list = static_cast<int4*>(work);
    uint4* const pieces = static_cast<uint4*>(work) + (most + 1);
    const RowsArgs a{A, pieces, W, out, list, C, N, chunks, blocks, K, F};
    const LayArgs l{W, pieces, types.T, K, F, C, N, chunks, blocks, types, list, most, 0};
    return NT == 2 ? run_rows<T, 2, TRANS>(a, l, st) : NT == 4 ? run_rows<T, 4, TRANS>(a, l, st) : run_rows<T, 8, TRANS>(a, l, st);
}

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
