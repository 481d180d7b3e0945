// Weight gradients by type: dW[t] (+)= X_t^T dZ_t over the rows of every type, X as fp32 or bf16 rows or in 8 bits (packed.h).
//
// The contraction runs along the rows, which both operands have as their slow dimension.  A workgroup of four wavefronts holds a tile of 128 x 256
// (256 x 128, 128 x 128, 128 x 64, 64 x 128) sums in registers, two or three of them a compute unit; its rows come in chunks of 16 (bf16: 32):
//   - A thread reads eight rows of two columns (four of packed rows) into registers, two chunks ahead (fp32 x fp32 in the wide tiles: one), turns them
//     into bf16 pieces along the rows (fp32: three, exact; bf16 rows and packed ones, whose values are bf16 values: one) and puts them to LDS as whole
//     fragments: 16 bytes are eight rows of a column, conflict-free to read.  (Not to write from 8 bits: of a thread's four columns two are
//     neighbours there, so lanes meet a bank twice; 25% of the LDS cycles at 867187 x 256 x 256.)  Two buffers, one barrier a chunk.
//   - fp32 x fp32 takes six products of pieces (linear_pieces.h), packed x fp32 three, packed or bf16 x bf16 one.
//   - Sums: fp32 products are summed from zero in the matrix unit over 16 rows, then added by vector instructions, every other chunk with the other
//     sign of X: the matrix unit cuts where it adds, and over a million rows that would lean to one side.  Bf16 products, as many times fewer, are
//     added to the sums there, X's sign turning every four chunks and with the workgroup.
// Rows are dealt evenly to the workgroups, whatever the types' sizes: a workgroup that meets the end of a type writes its sums and starts
// anew, so no workgroup has more rows than another.  Workgroup w writes its sums of type t to place w + t (every step along the rows goes to the
// next workgroup or the next type, so no two have the same place), and a second launch adds a type's places up in order: the result is the
// same in every run.  fp32 sums that are not finite (kUp: nor that large) are taken again there, from the operands.
// What bounds it: 237500 x 256 x 256, fp32, 210 us = 148 TFLOP/s (the six products' 890 TFLOP/s of bf16, of 1170 that a large library product reaches); bf16 from
// 8 bits, 867187 rows, 212 us: its 680 MB once would be 141, its products 97; every chunk's way from memory through registers to LDS is instructions between the
// products (the matrix cores are busy a quarter of the cycles).
#include <algorithm>

#include "linear_pieces.h"
#include "linear_typed.h"

namespace sar {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64;
constexpr int kChunk32 = 16, kChunk16 = 32;          // rows of a chunk: fp32, bf16

// Where column c of a tile's columns lies in LDS: of 64 columns the even ones first, so that the two that a thread writes go to runs of
// their own, and a lane of two neighbouring column tiles holds two neighbouring columns.
__device__ inline int place_of(int c) { return (c & ~63) | (c & 1) << 5 | (c >> 1 & 31); }
__device__ inline int column_at(int p) { return (p & ~63) | (p & 31) << 1 | (p >> 5 & 1); }

// Eight rows of kCols columns of a tile on their way from memory to LDS.  `base` is the chunk's first row, the same for all lanes; a chunk
// that is not full reads its last row again in place of those that are not there, and counts them as zeros.
template <typename R>
struct Unit {
    using T = typename R::T;
    static constexpr int kRegs = 8 * (int)sizeof(T) * 2 / 4;
    // c: column of the tensor (its rows are `width` values wide)
    static __device__ SAR_INLINE inline void load(uint32_t* w, const T* base, int group, int rows, bool full, int c, int width)
    {
        const uint32_t bytes = (uint32_t)width * sizeof(T);
        const char* p = reinterpret_cast<const char*>(base);
        if (full && width >= 2) {
            const uint32_t at = (uint32_t)min(c, width - 2) * sizeof(T) + (uint32_t)group * 8 * bytes;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if constexpr (sizeof(T) == 4) {
                    struct __attribute__((packed, aligned(4))) V { uint32_t x, y; };
                    const V v = *reinterpret_cast<const V*>(p + (at + (uint32_t)k * bytes));
                    w[2 * k] = v.x, w[2 * k + 1] = v.y;
                } else {
                    struct __attribute__((packed, aligned(2))) V { uint32_t x; };
                    w[k] = reinterpret_cast<const V*>(p + (at + (uint32_t)k * bytes))->x;
                }
            }
        } else {
            // value by value (a type's or a workgroup's last rows; rows of one value); addresses worked out here, not kept through the loop
            asm volatile("" : "+v"(c), "+v"(group));
            const uint32_t first = (uint32_t)min(c, max(width - 2, 0)) * sizeof(T), second = min(first + (uint32_t)sizeof(T), bytes - (uint32_t)sizeof(T));
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t row = (uint32_t)min(8 * group + k, rows - 1) * bytes;
                if constexpr (sizeof(T) == 4) {
                    w[2 * k] = *reinterpret_cast<const uint32_t*>(p + (row + first));
                    w[2 * k + 1] = *reinterpret_cast<const uint32_t*>(p + (row + second));
                } else {
                    const uint32_t lo = *reinterpret_cast<const uint16_t*>(p + (row + first)), hi = *reinterpret_cast<const uint16_t*>(p + (row + second));
                    w[k] = lo | hi << 16;
                }
            }
        }
    }
    // ... and into out[piece * stride], out[piece * stride + 32], the two columns' fragments
    static __device__ SAR_INLINE inline void put(uint32_t* w, uint4* out, int stride, int group, int rows, bool full, int c, int width, bool negate)
    {
        if (!full) {
#pragma unroll
            for (int k = 0; k < kRegs; ++k)
                if (8 * group + k * 8 / kRegs >= rows) w[k] = 0u;
        }
        if (c == width - 1) {          // the two values end with the row's last
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if constexpr (sizeof(T) == 4) w[2 * k] = w[2 * k + 1];
                else w[k] >>= 16;
            }
        }
        if constexpr (sizeof(T) == 4) {
            const float scale = negate ? -kUp : kUp;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                float v[8];
                uint4 p[3];
#pragma unroll
                for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(w[2 * k + j]) * scale;
                split8(v, p);
#pragma unroll
                for (int t = 0; t < 3; ++t) out[t * stride + 32 * j] = p[t];
            }
        } else {
            const uint32_t flip = negate ? 0x80008000u : 0u;
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                uint32_t p[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) p[k] = __builtin_amdgcn_perm(w[2 * k + 1], w[2 * k], j ? 0x07060302u : 0x05040100u) ^ flip;
                out[32 * j] = make_uint4(p[0], p[1], p[2], p[3]);
            }
        }
    }
};
struct PackedUnit {
    static constexpr int kRegs = 16;           // eight rows' numbers, eight steps
    static __device__ SAR_INLINE inline void load(uint32_t* w, const int8_t* q, const uint8_t* e, int group, int rows, bool full, int c, int K)
    {
        const uint32_t stride = packed_stride(K), steps = packed_steps(K), at = (uint32_t)min(c, (int)stride - 4);
        if (full) {
            const uint32_t off = at + (uint32_t)group * 8 * stride, eoff = at / kPackBlock + (uint32_t)group * 8 * steps;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                w[k] = *reinterpret_cast<const uint32_t*>(q + (off + (uint32_t)k * stride));
                w[8 + k] = e[eoff + (uint32_t)k * steps];
            }
        } else {
            asm volatile("" : "+v"(group));
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const uint32_t r = (uint32_t)min(8 * group + k, rows - 1);
                w[k] = *reinterpret_cast<const uint32_t*>(q + (at + r * stride));
                w[8 + k] = e[at / kPackBlock + r * steps];
            }
        }
    }
    static __device__ SAR_INLINE inline void put(uint32_t* w, uint4* out, int group, int rows, bool full, bool negate)
    {
        if (!full) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (8 * group + k >= rows) w[k] = 0u, w[8 + k] = 1u;
        }
        uint32_t p[4][4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            float a[4], b[4];
            const float sa = step_of(w[8 + 2 * k]), sb = step_of(w[8 + 2 * k + 1]);
            unpack4(w[2 * k], negate ? -sa : sa, a);
            unpack4(w[2 * k + 1], negate ? -sb : sb, b);
#pragma unroll
            for (int j = 0; j < 4; ++j) p[j][k] = pack2_bf16(a[j], b[j]);        // (bf16 values: not rounded)
        }
        // columns c, c + 1, c + 2, c + 3: two even ones and two odd ones
        out[0] = make_uint4(p[0][0], p[0][1], p[0][2], p[0][3]);
        out[1] = make_uint4(p[2][0], p[2][1], p[2][2], p[2][3]);
        out[32] = make_uint4(p[1][0], p[1][1], p[1][2], p[1][3]);
        out[33] = make_uint4(p[3][0], p[3][1], p[3][2], p[3][3]);
    }
};
template <typename XR>
constexpr int kXRegs = Unit<XR>::kRegs;
template <>
constexpr int kXRegs<PackedRows> = PackedUnit::kRegs;

// WM x WN wavefronts of MT x NT tiles of 32 x 32; S products of 16 rows a chunk.
template <typename XR, typename ZR, int MT, int NT, int WM, int WN, int S, int AHEAD>
__global__ __launch_bounds__(kThreads, 2) void k_typed_dw(DwArgs a)
{
    constexpr int TK = WM * MT * 32, TF = WN * NT * 32, PX = XR::kPieces, PZ = ZR::kPieces;
    static_assert(WM * WN * 64 == kThreads, "four wavefronts");
    constexpr int kGroups = 2 * S;                                  // eight rows each
    constexpr int kXUnits = kGroups * TK / XR::kCols, kZUnits = kGroups * TF / ZR::kCols;
    constexpr int kXSlots = (kXUnits + kThreads - 1) / kThreads, kZSlots = (kZUnits + kThreads - 1) / kThreads;
    constexpr int kXSize = PX * kGroups * TK, kSize = kXSize + PZ * kGroups * TF;      // fragments a buffer
    extern __shared__ __attribute__((aligned(16))) uint4 lds[];                         // [2][kSize]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int wm = wave % WM, wn = wave / WM;
    const int k0 = blockIdx.y * TK, f0 = blockIdx.z * TF;

    // A chunk's units, columns fastest, wavefront by wavefront; X's are dealt from the last wavefront on and dZ's from the first, so that
    // few units are spread over all of them.
    struct Chunk {
        uint32_t x[kXSlots][kXRegs<XR>], z[kZSlots][Unit<ZR>::kRegs];
    };
    Chunk raw[AHEAD];
    // (a thread's places are worked out anew for every chunk: carried through the loop, their addresses are dozens of registers)
    auto anew = [](int v) SAR_INLINE {
        asm volatile("" : "+v"(v));
        return v;
    };
    auto fetch = [&](Chunk& raw, int64_t r0, int64_t end) SAR_INLINE {
        const int rows = (int)min(end - r0, (int64_t)(16 * S));
        const bool full = rows == 16 * S;
        const int lane = anew(threadIdx.x & 63);
#pragma unroll
        for (int u = 0; u < kXSlots; ++u) {
            const int first = (kWaves - 1 - wave) * 64 + u * kThreads, id = first + lane;
            if (first >= kXUnits || (kXUnits % 64 && id >= kXUnits)) continue;
            const int g = id / (TK / XR::kCols), c = k0 + id % (TK / XR::kCols) * XR::kCols;
            if constexpr (XR::kCols == 4)
                PackedUnit::load(raw.x[u], a.Xq + r0 * packed_stride(a.K), a.Xe + r0 * packed_steps(a.K), g, rows, full, c, a.K);
            else
                Unit<XR>::load(raw.x[u], static_cast<const typename XR::T*>(a.X) + r0 * a.K, g, rows, full, c, a.K);
        }
#pragma unroll
        for (int u = 0; u < kZSlots; ++u) {
            const int first = wave * 64 + u * kThreads, id = first + lane;
            if (first >= kZUnits || (kZUnits % 64 && id >= kZUnits)) continue;
            const int g = id / (TF / 2), c = f0 + id % (TF / 2) * 2;
            Unit<ZR>::load(raw.z[u], static_cast<const typename ZR::T*>(a.dZ) + r0 * a.F, g, rows, full, c, a.F);
        }
    };
    auto put = [&](Chunk& raw, int64_t r0, int64_t end, uint4* buf, bool negate) SAR_INLINE {
        const int rows = (int)min(end - r0, (int64_t)(16 * S));
        const bool full = rows == 16 * S;
        const int lane = anew(threadIdx.x & 63);
#pragma unroll
        for (int u = 0; u < kXSlots; ++u) {
            const int first = (kWaves - 1 - wave) * 64 + u * kThreads, id = first + lane;
            if (first >= kXUnits || (kXUnits % 64 && id >= kXUnits)) continue;
            const int g = id / (TK / XR::kCols), c = id % (TK / XR::kCols) * XR::kCols;
            if constexpr (XR::kCols == 4) PackedUnit::put(raw.x[u], buf + g * TK + place_of(c), g, rows, full, negate);
            else Unit<XR>::put(raw.x[u], buf + g * TK + place_of(c), kGroups * TK, g, rows, full, k0 + c, a.K, negate);
        }
#pragma unroll
        for (int u = 0; u < kZSlots; ++u) {
            const int first = wave * 64 + u * kThreads, id = first + lane;
            if (first >= kZUnits || (kZUnits % 64 && id >= kZUnits)) continue;
            const int g = id / (TF / 2), c = id % (TF / 2) * 2;
            Unit<ZR>::put(raw.z[u], buf + kXSize + g * TF + place_of(c), kGroups * TF, g, rows, full, f0 + c, a.F, false);
        }
    };

    const int64_t from = blockIdx.x * a.share, to = min(from + a.share, a.types.n);
    for (int base = 0; base < a.types.T; base += 64) {
        // the types that have rows among mine
        int64_t lo = 0, hi = 0;
        if (base + lane < a.types.T) a.types.span(base + lane, lo, hi);
        lo = max(lo, from), hi = min(hi, to);
        uint64_t mine = __ballot(lo < hi);
        while (mine) {
            const int l = __builtin_ctzll(mine);
            mine &= mine - 1;
            const int t = base + l;
            const int64_t first = __builtin_amdgcn_readfirstlane(__shfl((int)lo, l));
            const int64_t end = __builtin_amdgcn_readfirstlane(__shfl((int)hi, l));

            float16_t acc[MT][NT];
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int n = 0; n < NT; ++n) acc[m][n] = float16_t{};
            // Which sign X has in chunk i, so that what the matrix unit cuts leans to neither side.  Bf16 products, which are added to the sums
            // there: the other sign every four chunks and in every other workgroup, with the sums turned round where it changes.
            auto minus = [&](int i) SAR_INLINE { return PZ == 1 ? (((i >> 2) + (int)blockIdx.x) & 1) != 0 : (i & 1) != 0; };
            auto step = [&](int i, int64_t r0, Chunk& later, Chunk& next) SAR_INLINE {
                constexpr int kRows = 16 * S;
                if (r0 + AHEAD * kRows < end) fetch(later, r0 + AHEAD * kRows, end);
                const uint4* xb = lds + (i & 1) * kSize + wm * MT * 32 + (lane & 31);
                const uint4* zb = lds + (i & 1) * kSize + kXSize + wn * NT * 32 + (lane & 31);
                if constexpr (PZ == 1) {
                    if (i > 0 && minus(i) != minus(i - 1)) {
#pragma unroll
                        for (int n = 0; n < MT * NT; ++n) acc[n % MT][n / MT] = -acc[n % MT][n / MT];
                    }
#pragma unroll
                    for (int s = 0; s < S; ++s) {
                        uint4 x[MT];
#pragma unroll
                        for (int m = 0; m < MT; ++m) x[m] = xb[(2 * s + h) * TK + m * 32];
#pragma unroll
                        for (int n = 0; n < NT; ++n) {
                            const uint4 z = zb[(2 * s + h) * TF + n * 32];
#pragma unroll
                            for (int m = 0; m < MT; ++m)
                                acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, x[m]),
                                                                                    __builtin_bit_cast(bf16x8_t, z), acc[m][n], 0, 0, 0);
                        }
                    }
                } else {
                    constexpr float kBack = (PX == 3 ? kDown : 1.f) * kDown;
                    const float sign = minus(i) ? -kBack : kBack;
                    // one tile's products run while the sums of the one before are added; no more than these two are kept at once
                    auto add = [&](int i, const float16_t& sum) SAR_INLINE {
#pragma unroll
                        for (int r = 0; r < 16; ++r) acc[i % MT][i / MT][r] = fmaf(sum[r], sign, acc[i % MT][i / MT][r]);
                        // (here, not where the compiler would have them: behind the next chunk's way to LDS, with all tiles' sums kept until then)
                        asm volatile("" : "+v"(acc[i % MT][i / MT]));
                    };
                    float16_t last;
#pragma unroll
                    for (int s = 0; s < S; ++s) {
                        uint4 x[MT][PX], z[PZ];
#pragma unroll
                        for (int m = 0; m < MT; ++m)
#pragma unroll
                            for (int p = 0; p < PX; ++p) x[m][p] = xb[p * kGroups * TK + (2 * s + h) * TK + m * 32];
#pragma unroll
                        for (int i = 0; i < MT * NT; ++i) {
                            if (i % MT == 0) {
#pragma unroll
                                for (int p = 0; p < PZ; ++p) z[p] = zb[p * kGroups * TF + (2 * s + h) * TF + i / MT * 32];
                            }
                            float16_t sum = {};
#pragma unroll
                            for (int k = 0; k < 6; ++k)
                                if (kTerm[k][0] < PX)
                                    sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, x[i % MT][kTerm[k][0] < PX ? kTerm[k][0] : 0]),
                                                                                  __builtin_bit_cast(bf16x8_t, z[kTerm[k][1]]), sum, 0, 0, 0);
                            if (i > 0) add(i - 1, last);
                            last = sum;
                            __builtin_amdgcn_sched_barrier(0);
                        }
                        add(MT * NT - 1, last);
                    }
                }
                if (r0 + kRows < end) put(next, r0 + kRows, end, lds + ((i & 1) ^ 1) * kSize, minus(i + 1));
                __syncthreads();
            };
            fetch(raw[0], first, end);
            if (AHEAD == 2 && first + 16 * S < end) fetch(raw[1 % AHEAD], first + 16 * S, end);
            put(raw[0], first, end, lds, minus(0));
            __syncthreads();
            int chunks = 0;
            for (int64_t r0 = first; r0 < end;) {
                step(chunks, r0, raw[0], raw[1 % AHEAD]);
                ++chunks, r0 += 16 * S;
                if (AHEAD == 1 || r0 >= end) continue;
                step(chunks, r0, raw[1 % AHEAD], raw[0]);
                ++chunks, r0 += 16 * S;
            }
            if (PZ == 1 && minus(chunks - 1)) {
#pragma unroll
                for (int n = 0; n < MT * NT; ++n) acc[n % MT][n / MT] = -acc[n % MT][n / MT];
            }

            float* out = a.partial + ((int64_t)blockIdx.x + t) * a.K * a.F;
            // lane holds column f (of two neighbouring tiles: f and f + 1); register r holds the weight's row at place 8*(r/4) + 4*h + r%4.  (The
            // places are worked out here: carried through the loops they are registers that the sums need.)
            int own = lane;
            asm volatile("" : "+v"(own));
            struct __attribute__((packed, aligned(4))) Two { float x, y; };
#pragma unroll
            for (int m = 0; m < MT; ++m)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int k = k0 + column_at((wm * MT + m) * 32 + 8 * (r / 4) + 4 * (own >> 5) + r % 4);
                    if (k >= a.K) continue;
                    float* to = out + (int64_t)k * a.F;
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const int f = f0 + column_at((wn * NT + n) * 32 + (own & 31));
                        if (NT > 1 && n % 2 == 0 && f + 1 < a.F) {
                            *reinterpret_cast<Two*>(to + f) = Two{acc[m][n][r], acc[m][NT > 1 ? n + 1 : n][r]};
                        } else if ((NT == 1 || n % 2 == 0) && f < a.F) {
                            to[f] = acc[m][n][r];
                        }
                    }
                }
        }
    }
}

// What a workgroup's place w + t should hold where it holds no finite number: three pieces of bf16 are no infinity, no NaN and none of the
// numbers that are too large to be scaled up (kUp).  Summed again from the operands, by multiply-adds.
template <typename XR, typename ZR>
__device__ float sum_again(const DwArgs& a, int64_t w, int64_t lo, int64_t hi, int64_t element)
{
    const int k = (int)(element / a.F), f = (int)(element % a.F);
    float v = 0.f;
    for (int64_t r = max(lo, w * a.share); r < min(hi, (w + 1) * a.share); ++r) v = fmaf(x_value<XR>(a, r, k), z_value<ZR>(a, r, f), v);
    return v;
}

// dW[t] (+)= the places of the workgroups that have rows of type t, in order.  32 threads take 32 or, where weights are whole pieces of
// four, 128 consecutive values; eight such groups of a workgroup take every eighth place, four at a time.
template <typename XR, typename ZR, int V>
__global__ __launch_bounds__(256) void k_typed_sum(DwArgs a, int accumulate, float* dW)
{
    __shared__ float part[8][32][V];
    const int e = threadIdx.x & 31, z = threadIdx.x >> 5, t = blockIdx.y;
    const int64_t count = (int64_t)a.K * a.F;
    int64_t lo, hi;
    a.types.span(t, lo, hi);
    const int64_t w0 = lo / a.share, w1 = hi > lo ? (hi - 1) / a.share + 1 : w0;
    struct __attribute__((packed, aligned(4))) Values { float v[V]; };
    for (int64_t k0 = (int64_t)blockIdx.x * (32 * V); k0 < count; k0 += (int64_t)gridDim.x * (32 * V)) {
        const int64_t k = k0 + e * V;
        Values sum = {};
        if (k < count) {
            const float* p = a.partial + t * count + k;
            for (int64_t w = w0 + z; w < w1; w += 4 * 8) {
                Values x[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    x[u] = Values{};
                    if (w + u * 8 < w1) x[u] = *reinterpret_cast<const Values*>(p + (w + u * 8) * count);
                }
                if constexpr (ZR::kPieces == 3) {
                    float zero = 0.f;
#pragma unroll
                    for (int u = 0; u < 4 * V; ++u) zero = fmaf(x[u / V].v[u % V], 0.f, zero);
                    if (zero != 0.f) {         // (NaN)
#pragma unroll
                        for (int u = 0; u < 4 * V; ++u)
                            if (!(fabsf(x[u / V].v[u % V]) < __builtin_inff())) x[u / V].v[u % V] = sum_again<XR, ZR>(a, w + u / V * 8, lo, hi, k + u % V);
                    }
                }
#pragma unroll
                for (int j = 0; j < V; ++j) sum.v[j] += (x[0].v[j] + x[1].v[j]) + (x[2].v[j] + x[3].v[j]);
            }
        }
#pragma unroll
        for (int j = 0; j < V; ++j) part[z][e][j] = sum.v[j];
        __syncthreads();
        // the eight groups' sums, by as many threads as there are values
        for (int i = threadIdx.x; i < 32 * V; i += 256) {
            const int64_t at = k0 + i;
            if (at >= count) break;
            float total = 0.f;
#pragma unroll
            for (int s = 0; s < 8; ++s) total += part[s][i / V][i % V];
            float* out = dW + t * count + at;
            *out = accumulate ? *out + total : total;
        }
        __syncthreads();
    }
}

// The tile of sums of a workgroup, its rows, and how many workgroups share them.
struct Shape {
    int tk, tf;
    int64_t share, groups;
};
// Wide tiles read the rows fewer times, narrow ones are more workgroups for as many shares of the rows, and every share is a set of sums to write and read
// again: the widest tile whose workgroups have chunks enough.  256 x 256 by tiles of 128 x 256 / 128 x 128 / 128 x 64, us:
//   fp32, from 8 bits:  10 thousand rows 27.3 / 22.3 / 20.5, 40 thousand 43.3 / 39.3 / 40.7, 160 thousand 107 / 111 / 122
//   bf16, from 8 bits:  10 thousand rows 24.3 / 22.9 / 18.0, 80 thousand 41.5 / 37.8 / 40.7, 160 thousand 56.8 / 58.0 / 67.9
// From 8 bits rather 256 x 128 than 128 x 256, so that it is the short rows that two tiles read (867187 rows, bf16: 218 us and 226; 200 thousand, fp32: 133 and 137; of plain bf16
// rows 82 and 72).
// A compute unit holds two workgroups of 128 x 128 with fp32 rows (three asked for: 160 thousand rows 128 x 128, 60.1 us, two 50.8) and three with bf16 ones
// (256 x 256: 58.0, two 66.1), three of 64 columns or rows (256 x 47, fp32: four 61.8, three 56.3).  Four chunks are a share's least (100 x 47, fp32: two, four, eight chunks, 4
// thousand rows 10.5, 10.6, 13.6 us, 16 thousand 20.5, 15.5, 15.9).
struct Tile {
    int tk, tf, resident, least;       // weights; workgroups of a compute unit; the chunks that a share has at least
};
// The tiles that may take K x F weights, widest first, a narrow one last.
int tiles_of(int K, int F, int chunk, bool packed, Tile (&t)[3])
{
    int count = 0;
    if (F > 64 && K > 64) {
        const bool wide_K = (K + 127) / 128 % 2 == 0, wide_F = (F + 127) / 128 % 2 == 0;
        if (wide_K && (packed || !wide_F)) t[count++] = {256, 128, 2, 16};
        else if (wide_F) t[count++] = {128, 256, 2, 16};
        t[count++] = {128, 128, chunk == kChunk32 ? 2 : 3, 8};
    }
    t[count++] = K <= 64 && F > 64 ? Tile{64, 128, 3, 4} : Tile{128, 64, 3, 4};
    return count;
}
int64_t most_at_once(const Tile& t, int K, int F) { return std::max(1, 256 * t.resident / (((K + t.tk - 1) / t.tk) * ((F + t.tf - 1) / t.tf))); }

Shape shape_of(int64_t n, int K, int F, int chunk, bool packed)
{
    Tile t[3];
    const int count = tiles_of(K, F, chunk, packed, t);
    for (int i = 0;; ++i) {
        const int64_t least = 4 * chunk;
        const int64_t want = std::max<int64_t>(1, std::min<int64_t>((n + least - 1) / least, most_at_once(t[i], K, F)));
        Shape s{t[i].tk, t[i].tf, std::max<int64_t>(least, ((n + want - 1) / want + 31) / 32 * 32), 0};
        s.groups = std::max<int64_t>(1, (n + s.share - 1) / s.share);
        if (i == count - 1 || s.share >= t[i].least * chunk) return s;
    }
}

// No fewer workgroups than any call of up to n rows has: what that is grows with n, though their number need not (shares are whole 32 rows, and
// wider tiles are fewer).  Scratch for a batch's most rows then serves all of its batches.
int64_t most_groups(int64_t n, int K, int F, int chunk, bool packed)
{
    Tile t[3];
    int64_t most = 1;
    for (int i = tiles_of(K, F, chunk, packed, t) - 1; i >= 0; --i) {
        const int64_t share = t[i].least * chunk;
        most = std::max(most, std::min((n + share - 1) / share, most_at_once(t[i], K, F)));
    }
    return most;
}

template <typename XR, typename ZR, int MT, int NT, int WM, int WN, int S, int AHEAD>
int run(const DwArgs& a, const Shape& s, hipStream_t st)
{
    constexpr int TK = WM * MT * 32, TF = WN * NT * 32;
    constexpr size_t shared = (size_t)2 * (XR::kPieces * TK + ZR::kPieces * TF) * 2 * S * sizeof(uint4);
    auto* fn = k_typed_dw<XR, ZR, MT, NT, WM, WN, S, AHEAD>;
    if (shared > 65536) SAR_HIP(hipFuncSetAttribute(reinterpret_cast<const void*>(fn), hipFuncAttributeMaxDynamicSharedMemorySize, (int)shared));
    fn<<<dim3((unsigned)s.groups, (a.K + TK - 1) / TK, (a.F + TF - 1) / TF), kThreads, shared, st>>>(a);
    SAR_LAUNCH_CHECK();
    return SAR_OK;
}

// S: products of 16 rows a chunk; W: chunks under way in the wide tiles, whose sums leave fewer registers.
template <typename XR, typename ZR, int S, int W>
int run_all(const DwArgs& a, const Shape& s, int accumulate, float* dW, hipStream_t st)
{
    if (a.types.n > 0) {
        if (s.tk == 256) SAR_TRY((run<XR, ZR, 4, 2, 2, 2, S, W>(a, s, st)));
        else if (s.tf == 256) SAR_TRY((run<XR, ZR, 2, 4, 2, 2, S, W>(a, s, st)));
        else if (s.tf == 64) SAR_TRY((run<XR, ZR, 2, 1, 2, 2, S, 2>(a, s, st)));
        else if (s.tk == 64) SAR_TRY((run<XR, ZR, 1, 2, 2, 2, S, 2>(a, s, st)));
        else SAR_TRY((run<XR, ZR, 2, 2, 2, 2, S, 2>(a, s, st)));
    }
    // four values a thread where that leaves two workgroups a compute unit (100 x 256 of one type by fours 11.9 us, one by one 9.6; 200 x 47 of
    // 37 types 6.3 and 15.3)
    const int64_t count = (int64_t)a.K * a.F;
    const bool single = count % 4 != 0 || count * a.types.T < 512 * 128;
    const int64_t per = single ? 32 : 128, blocks = std::min<int64_t>((count + per - 1) / per, 1 << 20);
    if (single) k_typed_sum<XR, ZR, 1><<<dim3((unsigned)blocks, a.types.T), 256, 0, st>>>(a, accumulate, dW);
    else k_typed_sum<XR, ZR, 4><<<dim3((unsigned)blocks, a.types.T), 256, 0, st>>>(a, accumulate, dW);
    SAR_LAUNCH_CHECK();
    return SAR_OK;
}

}  // namespace

size_t typed_dw_bytes(int64_t n, int K, int F, int T)
{
    auto most = [&](int chunk) { return std::max(most_groups(n, K, F, chunk, false), most_groups(n, K, F, chunk, true)); };
    return (size_t)(std::max(most(kChunk32), most(kChunk16)) + T) * K * F * sizeof(float);
}

int typed_dw(int dtype, const TypedDw& g, hipStream_t st)
{
    if (few_rows_dw(g.types.n, g.types.T, g.K, g.F)) return few_dw(dtype, g, st);
    const Shape s = shape_of(g.types.n, g.K, g.F, dtype == SAR_F32 ? kChunk32 : kChunk16, g.Xq != nullptr);
    const DwArgs a{g.X, g.Xq, g.Xe, g.dZ, g.partial, g.types, g.K, g.F, s.share};
    if (dtype == SAR_F32)
        return g.Xq ? run_all<PackedRows, F32Rows, kChunk32 / 16, 2>(a, s, g.accumulate, g.dW, st)
                    : run_all<F32Rows, F32Rows, kChunk32 / 16, 1>(a, s, g.accumulate, g.dW, st);
    return g.Xq ? run_all<PackedRows, Bf16Rows, kChunk16 / 16, 2>(a, s, g.accumulate, g.dW, st)
                : run_all<Bf16Rows, Bf16Rows, kChunk16 / 16, 2>(a, s, g.accumulate, g.dW, st);
}

}  // namespace sar
