// Products with a weight for each node type where rows are few.
//
// Here a call is latency, a launch costs as much as the work, and the weights' pieces and lists that calls of many rows lay out first do not pay: one launch
// a call, the backward pass's two products in the same one, operands straight from memory, the contraction shared by a workgroup's wavefronts,
// which add up in LDS.  The numbers are formed as there (linear_pieces.h: fp32 as three bf16 pieces, six products, from zero, added by vector
// instructions; sums that are not finite once more by the fp32 matrix instruction).  Which kernel takes a call shows in the last bits alone.
// 2000 x 128 -> 128, bf16, 4 types: 4.3 us, 10 with pieces and lists laid out first; 300 x 256 -> 256, fp32, 5 types: forward 5.1, backward, both products, 7.3, by a launch
// each 11.2.
#include <algorithm>

#include "linear_pieces.h"
#include "linear_typed.h"

namespace sar {

namespace {

// ---- rows times weights
//
// A wavefront, or four that share the contraction, for every 32 x 32 outputs; operands from memory to registers in chunks of 64 contraction
// values, a chunk ahead, weights cut into pieces where they are multiplied.
// Which rows: block `index` of 32 of a type, type after type; false behind the last one.
__device__ inline bool few_rows_of(const Types& types, int64_t index, int& t, int64_t& first, int64_t& end)
{
    const int lane = threadIdx.x & 63;
    for (int base = 0; base < types.T; base += 64) {
        int64_t lo = 0, hi = 0;
        if (base + lane < types.T) types.span(base + lane, lo, hi);
        const int mine = (int)((hi - lo + 31) / 32);
        int upto = mine;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const int v = __shfl_up(upto, o);
            if (lane >= o) upto += v;
        }
        const uint64_t here = __ballot(index < upto);
        if (here) {
            const int l = __builtin_ctzll(here);
            t = __builtin_amdgcn_readfirstlane(base + l);
            first = __builtin_amdgcn_readfirstlane(__shfl((int)(lo + (index - (upto - mine)) * 32), l));      // (rows are fewer than 2^31)
            end = __builtin_amdgcn_readfirstlane(__shfl((int)hi, l));
            return true;
        }
        index -= __shfl(upto, 63);
    }
    return false;
}

// PARTS: wavefronts that share one block's contraction, chunk by chunk, and add up in LDS (4), or one a block (1), of a workgroup of WAVES.  `row`: which
// block of rows; `beside`: which of the groups of column tiles that a workgroup takes; `sums`: [WAVES][16][64].
template <typename T, bool TRANS, int PARTS, int WAVES>
__device__ SAR_INLINE inline void few_rows(const TypedRows& a, int64_t row_block, int beside, float* sums)
{
    constexpr int N = Cols<T>::N, kRaw = 8 / N, U = 4;                // 16-byte pieces of a row a product of 16; products a chunk
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5, share = wave % PARTS;
    const int n0 = (beside * (WAVES / PARTS) + wave / PARTS) * 32, n = n0 + (lane & 31);
    const int k_from = n0 < a.N ? share * 16 * U : a.C;               // (no columns: nothing to multiply)
    constexpr int kTurn = PARTS * 16 * U;
    int t;
    int64_t first, end;
    if (!few_rows_of(a.types, row_block, t, first, end)) return;      // (the same for all of the workgroup)
    const int64_t i = min(first + (lane & 31), end - 1);
    const T* row = static_cast<const T*>(a.A) + i * a.C;
    const int64_t left = (a.types.n - i) * a.C;
    const float* W = a.W + (int64_t)t * a.K * a.F;
    const int nc = min(n, a.N - 1);
    struct Chunk {
        uint4 x[U][kRaw];
        float w[U][8];
    };
    auto load = [&](Chunk& g, int k0) SAR_INLINE {
        const float* w = TRANS ? W + (int64_t)nc * a.F : W + nc;
        if (k0 + 16 * U <= a.C) {          // the same for all lanes: one run of loads
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = k0 + u * 16 + h * 8;
#pragma unroll
                for (int p = 0; p < kRaw; ++p) g.x[u][p] = load16(row + c + p * N);
                if constexpr (TRANS) {
#pragma unroll
                    for (int j = 0; j < 8; j += 4) {
                        const uint4 v = load16(w + c + j);
                        g.w[u][j] = __uint_as_float(v.x), g.w[u][j + 1] = __uint_as_float(v.y);
                        g.w[u][j + 2] = __uint_as_float(v.z), g.w[u][j + 3] = __uint_as_float(v.w);
                    }
                } else {
#pragma unroll
                    for (int j = 0; j < 8; ++j) g.w[u][j] = w[(int64_t)(c + j) * a.F];
                }
            }
        } else {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int c = k0 + u * 16 + h * 8;
#pragma unroll
                for (int p = 0; p < kRaw; ++p) g.x[u][p] = Cols<T>::load(row, c + p * N, a.C, left);
#pragma unroll
                for (int j = 0; j < 8; ++j) g.w[u][j] = w[(int64_t)min(c + j, a.C - 1) * (TRANS ? 1 : a.F)];
            }
        }
    };
    float16_t acc[1] = {};
    auto multiply = [&](const Chunk& g, int k0) SAR_INLINE {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int c = k0 + u * 16 + h * 8;
            if (k0 + u * 16 >= a.C) break;
            float w[8], x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = c + j < a.C ? g.w[u][j] * (sizeof(T) == 4 ? kUp : 1.f) : 0.f;
            if constexpr (sizeof(T) == 4) {
                float lo[4], hi[4];
                Cols<T>::values(g.x[u][0], c, a.C, lo);
                Cols<T>::values(g.x[u][1 % kRaw], c + 4, a.C, hi);
#pragma unroll
                for (int j = 0; j < 4; ++j) x[j] = lo[j] * kUp, x[4 + j] = hi[j] * kUp;
                uint4 p[3], q[3];
                split8(x, p);
                split8(w, q);
                float16_t sum;
                multiply_split(p, q, sum);
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[0][r] = fmaf(sum[r], kDown * kDown, acc[0][r]);
            } else {
                const uint4 m = Cols<T>::within(c, a.C), v = g.x[u][0];
                const uint4 p = make_uint4(v.x & m.x, v.y & m.y, v.z & m.z, v.w & m.w);
                uint32_t big[4], small[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    big[j] = pack2_bf16(w[2 * j], w[2 * j + 1]);
                    small[j] = pack2_bf16(w[2 * j] - __uint_as_float(big[j] << 16), w[2 * j + 1] - __uint_as_float(big[j] & 0xffff0000u));
                }
                acc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, p), __builtin_bit_cast(bf16x8_t, make_uint4(small[0], small[1], small[2], small[3])), acc[0], 0, 0, 0);
                acc[0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, p), __builtin_bit_cast(bf16x8_t, make_uint4(big[0], big[1], big[2], big[3])), acc[0], 0, 0, 0);
            }
        }
    };
    if (k_from < a.C) {
        Chunk g[2];
        load(g[0], k_from);
        for (int k0 = k_from; k0 < a.C; k0 += 2 * kTurn) {
            if (k0 + kTurn < a.C) load(g[1], k0 + kTurn);
            multiply(g[0], k0);
            if (k0 + kTurn >= a.C) break;
            if (k0 + 2 * kTurn < a.C) load(g[0], k0 + 2 * kTurn);
            multiply(g[1], k0 + kTurn);
        }
        if (__any(not_finite(acc[0]))) {
            acc[0] = float16_t{};
            for (int k0 = k_from; k0 < a.C; k0 += kTurn)
                for (int k = k0; k < min(k0 + 16 * U, a.C); k += 2) {
                    const bool in = k + h < a.C;
                    float x = 0.f, w = 0.f;
                    if (in) {
                        if constexpr (sizeof(T) == 4) x = row[k + h];
                        else x = bf16_to_f32(row[k + h]);
                        w = TRANS ? W[(int64_t)nc * a.F + k + h] : W[(int64_t)(k + h) * a.F + nc];
                    }
                    acc[0] = __builtin_amdgcn_mfma_f32_32x32x2f32(x, w, acc[0], 0, 0, 0);
                }
        }
    }
    auto store = [&](int r, float v) SAR_INLINE {
        const int64_t o = first + 8 * (r / 4) + 4 * h + r % 4;
        if (n < a.N && o < end) static_cast<T*>(a.out)[o * a.N + n] = from_f32<T>(v);
    };
    if constexpr (PARTS == 4) {
        float(*part)[16][64] = reinterpret_cast<float(*)[16][64]>(sums) + wave / PARTS * PARTS;
#pragma unroll
        for (int r = 0; r < 16; ++r) part[share][r][lane] = acc[0][r];
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int r = share * 4 + j;
            store(r, (part[0][r][lane] + part[1][r][lane]) + (part[2][r][lane] + part[3][r][lane]));
        }
    } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) store(r, acc[0][r]);
    }
}

// ---- weight gradients
//
// A workgroup for 32 x 32 weights of a type, whose wavefronts take every fourth or eighth 16 of the type's rows straight from memory
// (lanes are columns: whole lines), add up their sums in LDS and write dW.
template <typename XR, typename ZR, int WAVES>
__device__ SAR_INLINE inline void few_weights(const DwArgs& a, int accumulate, float* dW, int k0, int f0, int t, float* sums)
{
    constexpr int PX = XR::kPieces, PZ = ZR::kPieces, U = 2, kTurn = WAVES * 16;          // products of 16 rows a step
    float(*part)[16][64] = reinterpret_cast<float(*)[16][64]>(sums);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int k = min(k0 + (lane & 31), a.K - 1), f = min(f0 + (lane & 31), a.F - 1);
    int64_t lo, hi;
    a.types.span(t, lo, hi);
    float16_t acc = {};
    struct Step {
        float x[U][8], z[U][8];
    };
    auto load = [&](Step& s, int64_t r0) SAR_INLINE {
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int64_t r = min(r0 + u * kTurn + h * 8 + j, hi - 1);
                s.x[u][j] = x_value<XR>(a, r, k);
                s.z[u][j] = z_value<ZR>(a, r, f);
            }
    };
    auto multiply = [&](Step& s, int64_t r0) SAR_INLINE {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (r0 + u * kTurn >= hi) break;
            float x[8], z[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const bool in = r0 + u * kTurn + h * 8 + j < hi;
                x[j] = in ? s.x[u][j] : 0.f, z[j] = in ? s.z[u][j] : 0.f;
            }
            uint4 p[3], q[3];
            auto whole = [](const float (&v)[8]) SAR_INLINE {        // (bf16 values: not rounded)
                return make_uint4(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7]));
            };
            if constexpr (PX == 3) {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] *= kUp;
                split8(x, p);
            } else {
                p[0] = whole(x);
            }
            if constexpr (PZ == 3) {
#pragma unroll
                for (int j = 0; j < 8; ++j) z[j] *= kUp;
                split8(z, q);
            } else {
                q[0] = whole(z);
            }
            float16_t sum = {};
#pragma unroll
            for (int i = 0; i < 6; ++i)
                if (kTerm[i][0] < PX && kTerm[i][1] < PZ)
                    sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, p[kTerm[i][0] < PX ? kTerm[i][0] : 0]),
                                                                  __builtin_bit_cast(bf16x8_t, q[kTerm[i][1] < PZ ? kTerm[i][1] : 0]), sum, 0, 0, 0);
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[r] = fmaf(sum[r], (PX == 3 ? kDown : 1.f) * (PZ == 3 ? kDown : 1.f), acc[r]);
        }
    };
    const int64_t from = lo + wave * 16;
    constexpr int kNext = U * kTurn;
    if (from < hi) {
        Step s[2];
        load(s[0], from);
        for (int64_t r0 = from; r0 < hi; r0 += 2 * kNext) {
            if (r0 + kNext < hi) load(s[1], r0 + kNext);
            multiply(s[0], r0);
            if (r0 + kNext >= hi) break;
            if (r0 + 2 * kNext < hi) load(s[0], r0 + 2 * kNext);
            multiply(s[1], r0 + kNext);
        }
        if (PZ == 3 && __any(not_finite(acc))) {
            acc = float16_t{};
            for (int64_t r0 = from; r0 < hi; r0 += kTurn)
                for (int64_t r = r0; r < min(r0 + 16, hi); r += 2) {
                    const bool in = r + h < hi;
                    acc = __builtin_amdgcn_mfma_f32_32x32x2f32(in ? x_value<XR>(a, r + h, k) : 0.f, in ? z_value<ZR>(a, r + h, f) : 0.f, acc, 0, 0, 0);
                }
        }
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) part[wave][r][lane] = acc[r];
    __syncthreads();
    // lane holds column f; register r holds weight row 8*(r/4) + 4*h + r%4: two registers a wavefront
    if (f0 + (lane & 31) >= a.F) return;
#pragma unroll
    for (int j = 0; j < 16 / WAVES; ++j) {
        const int r = wave * (16 / WAVES) + j, row = k0 + 8 * (r / 4) + 4 * h + r % 4;
        if (row >= a.K) continue;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) v += part[w][r][lane];
        float* out = dW + ((int64_t)t * a.K + row) * a.F + f;
        *out = accumulate ? *out + v : v;
    }
}

// ---- launches

template <typename T, bool TRANS, int PARTS>
__global__ __launch_bounds__(256, 2) void k_typed_few(TypedRows a)
{
    __shared__ float sums[PARTS == 4 ? 4 * 16 * 64 : 1];
    few_rows<T, TRANS, PARTS, 4>(a, blockIdx.x, blockIdx.y, sums);
}

template <typename XR, typename ZR, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void k_typed_dw_few(DwArgs a, int accumulate, float* dW)
{
    __shared__ float sums[WAVES * 16 * 64];
    few_weights<XR, ZR, WAVES>(a, accumulate, dW, blockIdx.x * 32, blockIdx.y * 32, blockIdx.z, sums);
}

// Both: workgroups from `rows_from` on (as many as there are) take dX, the others dW.
template <typename XR, typename ZR, int WAVES, int PARTS>
__global__ __launch_bounds__(WAVES * 64, 2) void k_typed_few_bwd(DwArgs a, int accumulate, float* dW, TypedRows g, unsigned across, unsigned down, unsigned rows_from,
                                                                 unsigned rows, unsigned beside)
{
    __shared__ float sums[WAVES * 16 * 64];
    const unsigned i = blockIdx.x - rows_from;
    if (i < rows) {
        few_rows<typename ZR::T, true, PARTS, WAVES>(g, i / beside, i % beside, sums);
    } else {
        const unsigned w = blockIdx.x < rows_from ? blockIdx.x : blockIdx.x - rows;
        few_weights<XR, ZR, WAVES>(a, accumulate, dW, w % across * 32, w / across % down * 32, w / across / down, sums);
    }
}

int64_t row_blocks(const Types& types) { return types.n / 32 + types.T; }
// Four wavefronts a block where that is no more than four a SIMD (2000 rows 256 -> 256, fp32, 544 blocks 9.2 us, one a block 13.0; 8000 rows 25.2 and 21.4).
constexpr int kFewShared = 1024;
bool shared_blocks(const TypedRows& a) { return a.C > 64 && row_blocks(a.types) * ((a.N + 31) / 32) <= kFewShared; }
// Eight wavefronts for 32 x 32 weights where types have rows for them (2000 rows of 4 types, 256 x 256 from 8 bits, 7.2 us, by four 8.6; 300 rows of 20
// types, 400 x 512, 30.7 and 15.7).
bool eight_waves(const Types& types) { return types.n > 64 * (int64_t)types.T; }

template <typename T, bool TRANS>
int product(const TypedRows& a, hipStream_t st)
{
    const unsigned groups = (unsigned)row_blocks(a.types);
    if (shared_blocks(a)) k_typed_few<T, TRANS, 4><<<dim3(groups, (a.N + 31) / 32), 256, 0, st>>>(a);
    else k_typed_few<T, TRANS, 1><<<dim3(groups, (a.N + 127) / 128), 256, 0, st>>>(a);
    SAR_LAUNCH_CHECK();
    return SAR_OK;
}

DwArgs dw_args(const TypedDw& g) { return {g.X, g.Xq, g.Xe, g.dZ, g.partial, g.types, g.K, g.F, 0}; }

template <typename XR, typename ZR>
int weights(const TypedDw& g, hipStream_t st)
{
    const dim3 grid((g.K + 31) / 32, (g.F + 31) / 32, g.types.T);
    if (eight_waves(g.types)) k_typed_dw_few<XR, ZR, 8><<<grid, 512, 0, st>>>(dw_args(g), g.accumulate, g.dW);
    else k_typed_dw_few<XR, ZR, 4><<<grid, 256, 0, st>>>(dw_args(g), g.accumulate, g.dW);
    SAR_LAUNCH_CHECK();
    return SAR_OK;
}

// One launch for both products as long as they are about what the chip holds at once (a wavefront of the one takes the registers of the other's; bf16 from 8
// bits, together and apart: 300 x 256 -> 256 of 5 types 6.9 and 10.3 us, 2000 x 256 -> 256 of 8 types 18.1 and 23.3, 8000 x 256 -> 256 of 46 types 53.5 and 50.9, 4735 x 258 -> 400 of 46
// 80.8 and 62.2).
constexpr int64_t kBothWaves = 16384;
template <typename XR, typename ZR, int WAVES, int PARTS>
int both(const TypedDw& g, const TypedRows& a, hipStream_t st)
{
    const unsigned across = (g.K + 31) / 32, down = (g.F + 31) / 32, beside = (a.N + 32 * (WAVES / PARTS) - 1) / (32 * (WAVES / PARTS));
    const int64_t dw = (int64_t)across * down * g.types.T, dx = row_blocks(a.types) * beside;
    if ((dw + dx) * WAVES > kBothWaves) {
        SAR_TRY((weights<XR, ZR>(g, st)));
        return product<typename ZR::T, true>(a, st);
    }
    // the longer contraction first: they need not all fit at once
    k_typed_few_bwd<XR, ZR, WAVES, PARTS><<<(unsigned)(dw + dx), WAVES * 64, 0, st>>>(dw_args(g), g.accumulate, g.dW, a, across, down,
                                                                                    g.types.n < g.F ? 0u : (unsigned)dw, (unsigned)dx, beside);
    SAR_LAUNCH_CHECK();
    return SAR_OK;
}
template <typename XR, typename ZR>
int both(const TypedDw& g, const TypedRows& a, hipStream_t st)
{
    if (eight_waves(g.types)) return shared_blocks(a) ? both<XR, ZR, 8, 4>(g, a, st) : both<XR, ZR, 8, 1>(g, a, st);
    return shared_blocks(a) ? both<XR, ZR, 4, 4>(g, a, st) : both<XR, ZR, 4, 1>(g, a, st);
}

}  // namespace

// Whether a product's blocks of 32 x 32 outputs, whose wavefronts read all the weights they need anew, are few (256 -> 256, 8 thousand rows, 2032 blocks,
// fp32 21.1 us here and 23.9 by two launches, bf16 12.4 and 15.1; 16 thousand rows 36.0 and 27.3, 20.8 and 17.0).
constexpr int kFewBlocks = 2560;
bool few_blocks(const Types& types, int N) { return row_blocks(types) * ((N + 31) / 32) <= kFewBlocks; }

// Whether these take a backward pass's sums over rows.  Of one type a wavefront takes every eighth 16 rows (256 x 256, fp32: 500 rows 6.5 us and 10.6 in shares
// of the rows (linear_typed_dw.hip), 1000 rows 10.6 and 11.6, 2000 rows 19.1 and 13.9); of several, whose shares are seldom even, the largest may have a good part:
// 256 rows a type (shares as the cubes of random numbers, 256 x 256 from 8 bits: 8 types, 2000 rows 14.9 and 18.4, 4000 rows 26.5 and 21.8; 46 types, 8000 rows 38.0
// and 50.4; 64 x 100: 9.5 and 22.2, 16000 rows 16.7 and 22.5).  How long the longest type is the host does not know, and its rows are walked by the wavefronts of
// one workgroup: with 95% of 16384 rows in one of 64 types 147 us and 100 (even types 50 and 61, cubes 62 and 77), 64 x 100 133 and 29 (11 and 16, 17 and 25); of
// 128 types and more 256 x 256 is faster here even so (162 and 185).  And every 32 x 32 weights read their columns anew (1000 rows, 1024 x 1024 from 8 bits 40.5 and 43.0, 2048 x 1024
// 78.5 and 59.1).
constexpr int64_t kFewRows = 1024, kFewOfType = 256, kFewRowsOfAll = 16384, kFewColumns = 1 << 20;
bool few_rows_dw(int64_t n, int T, int K, int F)
{
    return n <= std::min(std::max(kFewRows, kFewOfType * T), kFewRowsOfAll) && n * ((K + 31) / 32) * ((F + 31) / 32) <= kFewColumns;
}

int few_product(int dtype, bool trans, const TypedRows& a, hipStream_t st)
{
    if (dtype == SAR_F32) return trans ? product<float, true>(a, st) : product<float, false>(a, st);
    return trans ? product<bf16_t, true>(a, st) : product<bf16_t, false>(a, st);
}

int few_dw(int dtype, const TypedDw& g, hipStream_t st)
{
    if (dtype == SAR_F32) return g.Xq ? weights<PackedRows, F32Rows>(g, st) : weights<F32Rows, F32Rows>(g, st);
    return g.Xq ? weights<PackedRows, Bf16Rows>(g, st) : weights<Bf16Rows, Bf16Rows>(g, st);
}

// (the same bits as by two launches)
int few_dw_and_dx(int dtype, const TypedDw& g, const TypedRows& a, hipStream_t st)
{
    if (dtype == SAR_F32) return g.Xq ? both<PackedRows, F32Rows>(g, a, st) : both<F32Rows, F32Rows>(g, a, st);
    return g.Xq ? both<PackedRows, Bf16Rows>(g, a, st) : both<Bf16Rows, Bf16Rows>(g, a, st);
}

}  // namespace sar
