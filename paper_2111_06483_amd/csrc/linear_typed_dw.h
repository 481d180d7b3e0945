// The kernels of linear_typed_dw.hip, which says how they work; of linear_act_dw.hip, whose dZ is formed where it is read, or summed as well.
#pragma once

#include <algorithm>

#include "linear_act.h"
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
    static __device__ SAR_INLINE inline void load_full(uint32_t* w, const T* base, int group, int c, int width)
    {
        const uint32_t bytes = (uint32_t)width * sizeof(T);
        const char* p = reinterpret_cast<const char*>(base);
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
    }
    static __device__ SAR_INLINE inline void load(uint32_t* w, const T* base, int group, int rows, bool full, int c, int width)
    {
        if (full && width >= 2) {
            load_full(w, base, group, c, width);
        } else {
            const uint32_t bytes = (uint32_t)width * sizeof(T);
            const char* p = reinterpret_cast<const char*>(base);
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
// Bf16 rows and what they are formed with: 16 registers; two pieces.
struct FormedUnit {
    using Plain = Unit<Bf16Rows>;
    static constexpr int kRegs = 2 * Plain::kRegs;
    static __device__ SAR_INLINE inline void load_full(uint32_t* w, const bf16_t* base, const bf16_t* pre, int group, int c, int width)
    {
        Plain::load_full(w, base, group, c, width);
        Plain::load_full(w + Plain::kRegs, pre, group, c, width);
    }
    static __device__ SAR_INLINE inline void load(uint32_t* w, const bf16_t* base, const bf16_t* pre, int group, int rows, bool full, int c, int width)
    {
        Plain::load(w, base, group, rows, full, c, width);
        Plain::load(w + Plain::kRegs, pre, group, rows, full, c, width);
    }
    // `negate`: of dY's sign, which leaves X as it is (a quarter of the values to turn)
    // `formed`, `low`: WRITTEN: the chunk's rows of dA, which are written as bf16, and of what that leaves, or null (what is not there: outside of the buffer).
    template <bool WRITTEN>
    static __device__ SAR_INLINE inline void put(uint32_t* w, int act, uint4* out, int stride, int group, int rows, bool full, int c, int width, bool negate,
                                                 float (&sums)[2], bf16_t* formed, bf16_t* low, bool mine)
    {
        float v[2][8];
        const uint32_t flip = negate ? 0x80008000u : 0u;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            w[k] ^= flip;
            v[0][k] = __uint_as_float(w[k] << 16), v[1][k] = __uint_as_float(w[k] & 0xffff0000u);
        }
        with_act(act, [&](auto which) SAR_INLINE {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                v[0][k] = act_grad<decltype(which)::value>(v[0][k], __uint_as_float(w[8 + k] << 16));
                v[1][k] = act_grad<decltype(which)::value>(v[1][k], __uint_as_float(w[8 + k] & 0xffff0000u));
            }
        });
        if (!full) {
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (8 * group + k >= rows) v[0][k] = v[1][k] = 0.f;
        }
        if (c == width - 1) {          // the two values end with the row's last
#pragma unroll
            for (int k = 0; k < 8; ++k) v[0][k] = v[1][k];
        }
        uint32_t hi[2][4], lo[2][4];
        float largest = 0.f;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            float sum = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float a = v[j][2 * k], b = v[j][2 * k + 1];
                hi[j][k] = pack2_bf16(a, b);
                lo[j][k] = pack2_bf16(a - __uint_as_float(hi[j][k] << 16), b - __uint_as_float(hi[j][k] & 0xffff0000u));
                largest = fmaxf(largest, fmaxf(fabsf(a), fabsf(b)));
                sum += a + b;
            }
            sums[j] = negate ? sums[j] - sum : sums[j] + sum;
        }
        if (largest >= 0x1.fep127f) {          // an infinity (as bf16) has no second piece
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if ((hi[j][k] & 0x7fffu) == 0x7f80u) lo[j][k] &= 0xffff0000u;
                    if ((hi[j][k] & 0x7fff0000u) == 0x7f800000u) lo[j][k] &= 0xffffu;
                }
        }
        if constexpr (WRITTEN) {
            const int bytes = mine ? rows * width * (int)sizeof(bf16_t) : 0;
            const auto first = __builtin_amdgcn_make_buffer_rsrc(formed, 0, bytes, 0x00020000), second = __builtin_amdgcn_make_buffer_rsrc(low, 0, low ? bytes : 0, 0x00020000);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int place = c < width ? ((8 * group + k) * width + c) * (int)sizeof(bf16_t) : -1;
                const uint32_t which = k % 2 ? 0x07060302u : 0x05040100u;
                __builtin_amdgcn_raw_buffer_store_b32(__builtin_amdgcn_perm(hi[1][k / 2], hi[0][k / 2], which) ^ flip, first, place, 0, 0);
                __builtin_amdgcn_raw_buffer_store_b32(__builtin_amdgcn_perm(lo[1][k / 2], lo[0][k / 2], which) ^ flip, second, place, 0, 0);
            }
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            out[32 * j] = make_uint4(hi[j][0], hi[j][1], hi[j][2], hi[j][3]);
            out[stride + 32 * j] = make_uint4(lo[j][0], lo[j][1], lo[j][2], lo[j][3]);
        }
    }
};
template <typename ZR>
constexpr int kZRegs = ZTraits<ZR>::kFormed ? FormedUnit::kRegs : Unit<typename ZTraits<ZR>::Plain>::kRegs;
// The sums of a unit's two columns, of rows as they are (what is not there is zero by now).
template <typename T>
__device__ SAR_INLINE inline void add_columns(const uint32_t* w, int rows, int group, bool full, float (&sums)[2])
{
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        const bool there = full || 8 * group + k < rows;
        float a, b;
        if constexpr (sizeof(T) == 4) a = __uint_as_float(w[2 * k]), b = __uint_as_float(w[2 * k + 1]);
        else a = __uint_as_float(w[k] << 16), b = __uint_as_float(w[k] & 0xffff0000u);
        sums[0] += there ? a : 0.f;
        sums[1] += there ? b : 0.f;
    }
}
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
    using Plain = typename ZTraits<ZR>::Plain;
    constexpr int TK = WM * MT * 32, TF = WN * NT * 32, PX = XR::kPieces, PZ = ZR::kPieces;
    constexpr bool kThere = PZ < 3;        // whether products are added up in the matrix unit
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
        uint32_t x[kXSlots][kXRegs<XR>], z[kZSlots][kZRegs<ZR>];
    };
    Chunk raw[AHEAD];
    float sums[ZTraits<ZR>::kSums ? kZSlots : 1][2] = {};
    // (a thread's places are worked out anew for every chunk: carried through the loop, their addresses are dozens of registers)
    auto anew = [](int v) SAR_INLINE {
        asm volatile("" : "+v"(v));
        return v;
    };
    // (WHOLE: a full chunk of rows of at least two values)
    auto fetch = [&](auto whole, Chunk& raw, int64_t r0, int64_t end) SAR_INLINE {
        constexpr bool WHOLE = decltype(whole)::value;
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
            else if constexpr (WHOLE)
                Unit<XR>::load_full(raw.x[u], static_cast<const typename XR::T*>(a.X) + r0 * a.K, g, c, a.K);
            else
                Unit<XR>::load(raw.x[u], static_cast<const typename XR::T*>(a.X) + r0 * a.K, g, rows, full, c, a.K);
        }
#pragma unroll
        for (int u = 0; u < kZSlots; ++u) {
            const int first = wave * 64 + u * kThreads, id = first + lane;
            if (first >= kZUnits || (kZUnits % 64 && id >= kZUnits)) continue;
            const int g = id / (TF / 2), c = f0 + id % (TF / 2) * 2;
            if constexpr (ZTraits<ZR>::kFormed && WHOLE)
                FormedUnit::load_full(raw.z[u], static_cast<const bf16_t*>(a.dZ) + r0 * a.F, static_cast<const bf16_t*>(a.pre) + r0 * a.F, g, c, a.F);
            else if constexpr (WHOLE)
                Unit<Plain>::load_full(raw.z[u], static_cast<const typename ZR::T*>(a.dZ) + r0 * a.F, g, c, a.F);
            else if constexpr (ZTraits<ZR>::kFormed)
                FormedUnit::load(raw.z[u], static_cast<const bf16_t*>(a.dZ) + r0 * a.F, static_cast<const bf16_t*>(a.pre) + r0 * a.F, g, rows, full, c, a.F);
            else
                Unit<Plain>::load(raw.z[u], static_cast<const typename ZR::T*>(a.dZ) + r0 * a.F, g, rows, full, c, a.F);
        }
    };
    auto put = [&](auto whole, Chunk& raw, int64_t r0, int64_t end, uint4* buf, bool negate) SAR_INLINE {
        const int rows = decltype(whole)::value ? 16 * S : (int)min(end - r0, (int64_t)(16 * S));
        const bool full = rows == 16 * S;
        const int lane = anew(threadIdx.x & 63);
#pragma unroll
        for (int u = 0; u < kXSlots; ++u) {
            const int first = (kWaves - 1 - wave) * 64 + u * kThreads, id = first + lane;
            if (first >= kXUnits || (kXUnits % 64 && id >= kXUnits)) continue;
            const int g = id / (TK / XR::kCols), c = id % (TK / XR::kCols) * XR::kCols;
            if constexpr (XR::kCols == 4) PackedUnit::put(raw.x[u], buf + g * TK + place_of(c), g, rows, full, negate);
            else Unit<XR>::put(raw.x[u], buf + g * TK + place_of(c), kGroups * TK, g, rows, full, k0 + c, a.K, negate && !ZTraits<ZR>::kFormed);
        }
#pragma unroll
        for (int u = 0; u < kZSlots; ++u) {
            const int first = wave * 64 + u * kThreads, id = first + lane;
            if (first >= kZUnits || (kZUnits % 64 && id >= kZUnits)) continue;
            const int g = id / (TF / 2), c = id % (TF / 2) * 2;
            if constexpr (ZTraits<ZR>::kFormed) {
                FormedUnit::put<ZR::kWritten>(raw.z[u], a.act, buf + kXSize + g * TF + place_of(c), kGroups * TF, g, rows, full, f0 + c, a.F, negate, sums[u],
                                              ZR::kWritten ? static_cast<bf16_t*>(a.formed) + r0 * a.F : nullptr,
                                              ZR::kWritten && a.low ? static_cast<bf16_t*>(a.low) + r0 * a.F : nullptr, blockIdx.y == 0);
            } else {
                Unit<Plain>::put(raw.z[u], buf + kXSize + g * TF + place_of(c), kGroups * TF, g, rows, full, f0 + c, a.F, false);
                if constexpr (ZTraits<ZR>::kSums) {
                    if (blockIdx.y == 0) add_columns<typename ZR::T>(raw.z[u], rows, g, full, sums[u]);
                }
            }
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
            // there: the other sign every four chunks (of formed rows sixteen) and in every other workgroup, with the sums turned round where it changes.
            auto minus = [&](int i) SAR_INLINE { return kThere ? (((i >> (ZTraits<ZR>::kFormed ? 4 : 2)) + (int)blockIdx.x) & 1) != 0 : (i & 1) != 0; };
            constexpr std::integral_constant<bool, false> part{};
            auto step = [&](auto whole, int i, int64_t r0, Chunk& later, Chunk& next) SAR_INLINE {
                constexpr int kRows = 16 * S;
                if (decltype(whole)::value || r0 + AHEAD * kRows < end) fetch(whole, later, r0 + AHEAD * kRows, end);
                const uint4* xb = lds + (i & 1) * kSize + wm * MT * 32 + (lane & 31);
                const uint4* zb = lds + (i & 1) * kSize + kXSize + wn * NT * 32 + (lane & 31);
                if constexpr (kThere) {
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
#pragma unroll
                            for (int p = PZ - 1; p >= 0; --p) {
                                const uint4 z = zb[p * kGroups * TF + (2 * s + h) * TF + n * 32];
#pragma unroll
                                for (int m = 0; m < MT; ++m)
                                    acc[m][n] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, x[m]),
                                                                                        __builtin_bit_cast(bf16x8_t, z), acc[m][n], 0, 0, 0);
                            }
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
                if (decltype(whole)::value || r0 + kRows < end) put(whole, next, r0 + kRows, end, lds + ((i & 1) ^ 1) * kSize, minus(i + 1));
                __syncthreads();
            };
            fetch(part, raw[0], first, end);
            if (AHEAD == 2 && first + 16 * S < end) fetch(part, raw[1 % AHEAD], first + 16 * S, end);
            put(part, raw[0], first, end, lds, minus(0));
            __syncthreads();
            int chunks = 0;
            int64_t r0 = first;
            // As long as the chunks to come are full ones: loads without a branch, which would have all of them waited for (their number is not known behind it;
            // 306250 x 256 -> 256 fp32, both products, 597 us for 617, 867187 bf16 835 for 850).
            if (ZTraits<ZR>::kSums && a.K >= 2 && a.F >= 2) {
                constexpr std::integral_constant<bool, true> whole{};
                for (; r0 + (2 * AHEAD + 1) * 16 * S <= end; r0 += AHEAD * 16 * S) {
                    step(whole, chunks++, r0, raw[0], raw[1 % AHEAD]);
                    if (AHEAD == 2) step(whole, chunks++, r0 + 16 * S, raw[1 % AHEAD], raw[0]);
                }
            }
            while (r0 < end) {
                step(part, chunks, r0, raw[0], raw[1 % AHEAD]);
                ++chunks, r0 += 16 * S;
                if (AHEAD == 1 || r0 >= end) continue;
                step(part, chunks, r0, raw[1 % AHEAD], raw[0]);
                ++chunks, r0 += 16 * S;
            }
            if (kThere && minus(chunks - 1)) {
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
    if constexpr (ZTraits<ZR>::kSums) {
        if (a.sums == nullptr || blockIdx.y != 0) return;
        // a column's groups of rows, in order (the last chunk's fragments have been read: a barrier ends each)
        float* const part = reinterpret_cast<float*>(lds);
#pragma unroll
        for (int u = 0; u < kZSlots; ++u) {
            const int id = threadIdx.x + u * kThreads;
            if (kZUnits % kThreads && id >= kZUnits) continue;
            const int g = id / (TF / 2), c = id % (TF / 2) * 2;
            part[g * TF + c] = sums[u][0], part[g * TF + c + 1] = sums[u][1];
        }
        __syncthreads();
        for (int c = threadIdx.x; c < TF && f0 + c < a.F; c += kThreads) {
            float v = 0.f;
#pragma unroll
            for (int g = 0; g < kGroups; ++g) v += part[g * TF + c];
            a.sums[(int64_t)blockIdx.x * a.F + f0 + c] = v;
        }
    }
}

// What a workgroup's place w + t should hold where it holds no finite number: pieces of bf16 are no infinity and no NaN, three of them none of the
// numbers that are too large to be scaled up (kUp), and an infinity of X times a second piece of zero is NaN.  Summed again from the operands, by multiply-adds.
template <typename XR, typename ZR>
__device__ float sum_again(const DwArgs& a, int64_t w, int64_t lo, int64_t hi, int64_t element)
{
    const int k = (int)(element / a.F), f = (int)(element % a.F);
    float v = 0.f;
    for (int64_t r = max(lo, w * a.share); r < min(hi, (w + 1) * a.share); ++r) v = fmaf(x_value<XR>(a, r, k), whole_z<ZR>(a, r, f), v);
    return v;
}

// db (+)= the sums of `groups` workgroups, in order: eight columns a workgroup of 256 threads, whose 32 slices take every 32nd, four at a time.
__device__ inline void sum_columns(const float* sums, int groups, int F, int block, float* part, int accumulate, float* db)
{
    const int k = threadIdx.x & 7, slice = threadIdx.x >> 3, c = block * 8 + k;
    float v = 0.f;
    if (c < F) {
        for (int w = slice; w < groups; w += 4 * 32) {
            float x[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) x[u] = w + u * 32 < groups ? sums[(int64_t)(w + u * 32) * F + c] : 0.f;
#pragma unroll
            for (int u = 0; u < 4; ++u) v += x[u];
        }
    }
    part[threadIdx.x] = v;
    __syncthreads();
    if (slice == 0 && c < F) {
        float total = 0.f;
#pragma unroll
        for (int s = 0; s < 32; ++s) total += part[s * 8 + k];
        db[c] = accumulate ? db[c] + total : total;
    }
}

// dW[t] (+)= the places of the workgroups that have rows of type t, in order.  32 threads take 32 or, where weights are whole pieces of
// four, 128 consecutive values; eight such groups of a workgroup take every eighth place, four at a time.
// SUMS: of one type, with db (or null) in the workgroups from `blocks` on.
template <typename XR, typename ZR, int V, bool SUMS>
__global__ __launch_bounds__(256) void k_typed_sum(DwArgs a, int accumulate, float* dW, int blocks, float* db)
{
    __shared__ float part[8][32][V];
    if constexpr (SUMS) {
        if ((int)blockIdx.x >= blocks) {
            const int groups = (int)((a.types.n + a.share - 1) / a.share);
            sum_columns(a.sums, groups, a.F, (int)blockIdx.x - blocks, &part[0][0][0], accumulate, db);
            return;
        }
    }
    const int across = SUMS ? blocks : (int)gridDim.x;
    const int e = threadIdx.x & 31, z = threadIdx.x >> 5, t = blockIdx.y;
    const int64_t count = (int64_t)a.K * a.F;
    int64_t lo, hi;
    a.types.span(t, lo, hi);
    const int64_t w0 = lo / a.share, w1 = hi > lo ? (hi - 1) / a.share + 1 : w0;
    struct __attribute__((packed, aligned(4))) Values { float v[V]; };
    for (int64_t k0 = (int64_t)blockIdx.x * (32 * V); k0 < count; k0 += (int64_t)across * (32 * V)) {
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
                if constexpr (ZR::kPieces > 1) {
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
int run_all(const DwArgs& a, const Shape& s, int accumulate, float* dW, hipStream_t st, float* db = nullptr)
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
    using Rows = std::conditional_t<ZTraits<ZR>::kFormed, Bf16Formed, typename ZTraits<ZR>::Plain>;
    // (columns' sums in a launch of their own: 5 us more)
    constexpr bool kSums = ZTraits<ZR>::kSums;
    const dim3 grid((unsigned)(blocks + (db ? (a.F + 7) / 8 : 0)), a.types.T);
    if (single) k_typed_sum<XR, Rows, 1, kSums><<<grid, 256, 0, st>>>(a, accumulate, dW, (int)blocks, db);
    else k_typed_sum<XR, Rows, 4, kSums><<<grid, 256, 0, st>>>(a, accumulate, dW, (int)blocks, db);
    SAR_LAUNCH_CHECK();
    return SAR_OK;
}

}  // namespace
}  // namespace sar
