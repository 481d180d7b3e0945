// Rows kept in 8 bits (packed.hip says why in this form): what the kernels that write and read them share.
//
// A row of K values is cut into blocks of 32; a block has one step 2^(e - 127), a power of two, and every value x of it is kept as the
// whole number q = rint(x / step) of -127 to 127.  q: int8 [n, packed_stride(K)], zeros behind a row's end; e: uint8 [n, packed_steps(K)].
// A block that holds an infinity or a NaN has e = 255 and q = 0, and stands for NaN in all its places.
#pragma once

#include "linear_common.h"

namespace sar {

constexpr int kPackBlock = 32;
constexpr int kMostPackedWidth = 1 << 24;
__host__ __device__ inline int packed_stride(int K) { return (K + 15) / 16 * 16; }
__host__ __device__ inline int packed_steps(int K) { return (K + kPackBlock - 1) / kPackBlock; }

// The exponent byte of a block whose largest size has these bits: the smallest step 2^k of which that size is fewer than 127.5.  With the
// size m 2^t, 1 <= m < 2, that is k = t - 6, or t - 5 where m >= 127.5 / 64 = 2 - 2^-7: adding 2^-7 to m then carries.  Not below 2^-126, so that
// q times the step is never a subnormal number, and not above 2^121, so that it is never beyond the largest one.
constexpr uint32_t kLongestStep = 121 + 127;
__device__ inline uint32_t step_byte(uint32_t largest)
{
    if (largest >= 0x7f800000u) return 255u;
    return (uint32_t)min(max((int)((largest + (1u << 16)) >> 23) - 6, 1), (int)kLongestStep);
}

// Four values in their block's step, as bytes.  x / step is exact (a power of two; what falls below the smallest number rounds to zero either
// way), and the sum with 1.5 2^23 rounds it to the nearest whole number, ties to even, in its low bits.
__device__ inline uint32_t pack4(float a, float b, float c, float d, uint32_t byte)
{
    if (byte == kLongestStep) {            // (of sizes beyond 127.5 2^121 the number stays at 127)
        const float most = 127.f * 0x1p121f;
        a = fminf(fmaxf(a, -most), most), b = fminf(fmaxf(b, -most), most);
        c = fminf(fmaxf(c, -most), most), d = fminf(fmaxf(d, -most), most);
    }
    const float inv = __uint_as_float((254u - byte) << 23);        // (byte 255: whatever it is, the bytes are cleared)
    const float magic = 12582912.f;
    const uint32_t w0 = __float_as_uint(fmaf(a, inv, magic)), w1 = __float_as_uint(fmaf(b, inv, magic)),
                   w2 = __float_as_uint(fmaf(c, inv, magic)), w3 = __float_as_uint(fmaf(d, inv, magic));
    const uint32_t lo = __builtin_amdgcn_perm(w1, w0, 0x0c0c0400u), hi = __builtin_amdgcn_perm(w3, w2, 0x04000c0cu);
    return byte == 255u ? 0u : lo | hi;
}

// What four bytes stand for: q step, exact.  (With e = 255 the step reads as infinity, and zero times that is NaN.)
__device__ inline float step_of(uint32_t byte) { return __uint_as_float(byte << 23); }
__device__ inline void unpack4(uint32_t q, float step, float (&v)[4])
{
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = (float)((int32_t)(q << (24 - 8 * j)) >> 24) * step;
}

// The largest of the sizes that LANES consecutive lanes hold (4 or 8).
template <int LANES>
__device__ inline uint32_t lanes_max(uint32_t v)
{
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0xB1, 0xf, 0xf, false));       // lane ^ 1
    v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x4E, 0xf, 0xf, false));       // lane ^ 2
    if constexpr (LANES == 8) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x141, 0xf, 0xf, false));
    return v;
}

// A piece of 16 bytes of a row of D values, from column c on, as fp32; zeros behind the row's end.  A row's last piece may end in the next
// row; where there is none (`left`: values from the row's beginning to the tensor's end), it is read where the row ends and moved to its front, or,
// of rows of less than a piece, value by value.
template <typename T>
struct Cols {
    static constexpr int N = 16 / (int)sizeof(T);
    static __device__ inline void unpack(const uint4& r, float (&v)[N])
    {
        if constexpr (N == 4) {
            v[0] = __uint_as_float(r.x), v[1] = __uint_as_float(r.y), v[2] = __uint_as_float(r.z), v[3] = __uint_as_float(r.w);
        } else {
            Vec<bf16_t>::unpack(r, v);
        }
    }
    // (the load and what is done with it apart, so that a thread can have several under way; lanes behind the row read its first piece)
    static __device__ inline uint4 load(const T* row, int c, int D, int64_t left)
    {
        if (c >= D) c = 0;
        if (c + N <= left) return load16(row + c);
        if (D >= N) return front_of_piece<T>(load16(row + D - N), D - c);
        T one[N] = {};
#pragma unroll
        for (int j = 0; j < N; ++j)
            if (c + j < D) one[j] = row[c + j];
        return __builtin_bit_cast(uint4, one);
    }
    // What a piece's words have within the row.
    static __device__ inline uint4 within(int c, int D)
    {
        uint32_t m[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if constexpr (N == 4) m[k] = c + k < D ? 0xffffffffu : 0u;
            else m[k] = c + 2 * k + 1 < D ? 0xffffffffu : c + 2 * k < D ? 0xffffu : 0u;
        }
        return make_uint4(m[0], m[1], m[2], m[3]);
    }
    static __device__ inline void values(const uint4& r, const uint4& m, float (&v)[N])
    {
        unpack(make_uint4(r.x & m.x, r.y & m.y, r.z & m.z, r.w & m.w), v);
    }
    static __device__ inline void values(const uint4& r, int c, int D, float (&v)[N])
    {
        if (c + N <= D) unpack(r, v);
        else values(r, within(c, D), v);
    }
    static __device__ inline uint4 round(const float (&v)[N])
    {
        if constexpr (N == 4)
            return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3]));
        else
            return make_uint4(pack2_bf16(v[0], v[1]), pack2_bf16(v[2], v[3]), pack2_bf16(v[4], v[5]), pack2_bf16(v[6], v[7]));
    }
    static __device__ inline void store(T* row, int c, int D, const float (&v)[N])
    {
        const uint4 r = round(v);
        if (c + N <= D) {
            store16(row + c, r);
        } else if (c < D) {
            // the rest of a row, the same for all rows: 8, 4 and 2 bytes
            struct __attribute__((packed, aligned(2))) U2 { uint32_t x, y; };
            struct __attribute__((packed, aligned(2))) U1 { uint32_t x; };
            uint32_t w[4] = {r.x, r.y, r.z, r.w};
            const int rest = D % N;
            constexpr int kPer = 4 / (int)sizeof(T);
            T* p = row + c;
            if (rest & (2 * kPer)) {
                *reinterpret_cast<U2*>(p) = U2{w[0], w[1]};
                p += 2 * kPer, w[0] = w[2], w[1] = w[3];
            }
            if (rest & kPer) {
                reinterpret_cast<U1*>(p)->x = w[0];
                p += kPer, w[0] = w[1];
            }
            if constexpr (kPer == 2) {
                if (rest & 1) *reinterpret_cast<uint16_t*>(p) = (uint16_t)w[0];
            }
        }
    }
};

// The piece's values (zeros behind the row's end) into row q, e of packed rows; a block's lanes are neighbours, and all of them are here.
template <typename T>
__device__ inline void store_packed(int8_t* q, uint8_t* e, int c, int D, const float (&v)[Cols<T>::N])
{
    constexpr int N = Cols<T>::N, kLanes = kPackBlock / N;
    uint32_t largest = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) largest = max(largest, __float_as_uint(v[j]) & 0x7fffffffu);
    const uint32_t byte = step_byte(lanes_max<kLanes>(largest));
    if (c >= packed_stride(D)) return;
    if constexpr (N == 4) {
        *reinterpret_cast<uint32_t*>(q + c) = pack4(v[0], v[1], v[2], v[3], byte);
    } else {
        *reinterpret_cast<uint2*>(q + c) = make_uint2(pack4(v[0], v[1], v[2], v[3], byte), pack4(v[4], v[5], v[6], v[7], byte));
    }
    if (c % kPackBlock == 0) e[c / kPackBlock] = (uint8_t)byte;
}
// ... and back: what columns c.. of a packed row stand for; zeros behind its padded end.
template <int N>
struct PackedCols {
    struct Raw {
        uint32_t w[N / 4], byte;
    };
    static __device__ inline Raw load(const int8_t* q, const uint8_t* e, int c, int stride)
    {
        const int at = min(c, stride - N);
        Raw r;
        if constexpr (N == 4) {
            r.w[0] = *reinterpret_cast<const uint32_t*>(q + at);
        } else {
            const uint2 x = *reinterpret_cast<const uint2*>(q + at);
            r.w[0] = x.x, r.w[1] = x.y;
        }
        r.byte = e[at / kPackBlock];
        return r;
    }
    static __device__ inline void values(const Raw& r, int c, int stride, float (&v)[N])
    {
        const float step = step_of(r.byte);
#pragma unroll
        for (int k = 0; k < N; k += 4) {
            float x[4];
            unpack4(r.w[k / 4], step, x);
#pragma unroll
            for (int j = 0; j < 4; ++j) v[k + j] = c < stride ? x[j] : 0.f;
        }
    }
};

// Whether two ranges of memory have no byte in common (b null: so).
inline bool apart(const void* a, size_t a_bytes, const void* b, size_t b_bytes)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return !b || x + a_bytes <= y || y + b_bytes <= x;
}

// Refuses what is no packed tensor (both or neither; q in whole pieces of 16 bytes).
int check_packed(const char* what, const void* q, const void* e);

}  // namespace sar
