// What is done to a row of X W before it is stored: bias, residual, activation (linear_act.hip); the activations and their derivatives.
#pragma once

#include "linear_typed.h"
#include "packed.h"
#include "sar_internal.h"

namespace sar {

struct NoEpilogue {
    static constexpr bool kAny = false;
};
// a = X W + bias (+ res), pre = a, Y = act(a) (+ res, `after`); null where there is none.
struct Epilogue {
    static constexpr bool kAny = true;
    const float* bias;
    const void* res;
    void* pre;
    int act, after;
};

__device__ inline float value_of(float v) { return v; }
__device__ inline float value_of(bf16_t v) { return bf16_to_f32(v); }

// ---- activations, in 32 bits.  Infinities have their limits, NaN stays.

// Phi(a) and exp(-a^2 / 2).  The smaller side is t P(t) exp(-a^2 / 2) with t = 1 / (1 + 0.275 |a|), P of degree 5 fitted to it by least squares with weights
// raised where it was furthest off: Phi is off by 9e-9 at most, by fp32 operations 2e-7, of 1.  Of itself the smaller side is off by 3e-6 at 3 from zero, 5e-5 at 4,
// 5e-4 at 6 and 2e-3 at 8 (where it is 7e-16; 1 + erf(a / sqrt 2) in 32 bits has nothing left from 6 on).
__device__ inline float normal_share(float a, float& bell)
{
    const float t = __builtin_amdgcn_rcpf(fmaf(fabsf(a), 0.275f, 1.f));
    bell = __builtin_amdgcn_exp2f(a * a * -0.72134752f);
    float p = fmaf(t, -0.11485983431339264f, 0.45200487971305847f);
    p = fmaf(t, p, -0.33100342750549316f);
    p = fmaf(t, p, 0.3339403569698334f);
    p = fmaf(t, p, 0.042108260095119476f);
    p = fmaf(t, p, 0.11780976504087448f);
    const float side = p * t * bell;
    return a > 0.f ? 1.f - side : side;
}
__device__ inline float logistic(float a) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(a * -kLog2e)); }
// Between them the derivatives of what follows are still to be told from their limits.
__device__ inline float within(float a, float most) { return __builtin_amdgcn_fmed3f(a, -most, most); }
// exp(a) - 1 for a <= 0: near zero by the series (its first term left out, a^7 / 8!, is 2^-26 of the sum at most).
__device__ inline float below_one(float a)
{
    float s = fmaf(a, 1.f / 5040.f, 1.f / 720.f);
    s = fmaf(a, s, 1.f / 120.f);
    s = fmaf(a, s, 1.f / 24.f);
    s = fmaf(a, s, 1.f / 6.f);
    s = fmaf(a, s, 0.5f);
    s = fmaf(a * a, s, a);
    return a > -0.35f ? s : __builtin_amdgcn_exp2f(a * kLog2e) - 1.f;
}

template <int ACT>
__device__ inline float act_of(float a)
{
    if constexpr (ACT == SAR_ACT_RELU) return a < 0.f ? 0.f : a;
    if constexpr (ACT == SAR_ACT_GELU) {
        float bell;
        const float share = normal_share(a, bell);
        return fmaxf(a, -64.f) * share;
    }
    if constexpr (ACT == SAR_ACT_SILU) return fmaxf(a, -256.f) * logistic(a);
    if constexpr (ACT == SAR_ACT_ELU) return a > 0.f ? a : below_one(a);
    return a;
}
// d act'(a)
template <int ACT>
__device__ inline float act_grad(float d, float a)
{
    if constexpr (ACT == SAR_ACT_RELU) return a > 0.f ? d : 0.f;
    if constexpr (ACT == SAR_ACT_GELU) {
        float bell;
        const float share = normal_share(a, bell);
        return d * fmaf(within(a, 64.f) * bell, 0.39894228040143267f, share);
    }
    if constexpr (ACT == SAR_ACT_SILU) {
        const float s = logistic(a);
        return d * (s * fmaf(within(a, 256.f), 1.f - s, 1.f));
    }
    if constexpr (ACT == SAR_ACT_ELU) return a > 0.f ? d : d * __builtin_amdgcn_exp2f(a * kLog2e);
    return d;
}

// f with the activation as a constant.
template <typename F>
__device__ __attribute__((always_inline)) inline void with_act(int act, F&& f)
{
    switch (act) {
    case SAR_ACT_RELU: f(std::integral_constant<int, SAR_ACT_RELU>{}); break;
    case SAR_ACT_GELU: f(std::integral_constant<int, SAR_ACT_GELU>{}); break;
    case SAR_ACT_SILU: f(std::integral_constant<int, SAR_ACT_SILU>{}); break;
    case SAR_ACT_ELU: f(std::integral_constant<int, SAR_ACT_ELU>{}); break;
    default: break;
    }
}

// What is done to a row's values before they are multiplied: nothing; dA = dY act'(A) is formed of them; or they are the first pieces of values whose others lie
// elsewhere.  Of bf16 rows dA is multiplied as two pieces of bf16, 16 bits: of one, a result's terms would have 8 before they are added up and rounded
// (867187 x 256 -> 256, by GELU: dX is 1.66e-3 off from 64 bits, which is its own rounding; of one piece 2.35e-3).
struct NoPrologue {
    static constexpr bool kAny = false, kForms = false;
};
struct ActPrologue {
    static constexpr bool kAny = true, kForms = true;
    const void* pre;       // [n, C]: what the activation was taken of
    void* formed;          // [n, C] or null: receives dA
    int act;
};
struct LowPieces {
    static constexpr bool kAny = true, kForms = false;
    const void* low;       // [n, C] of bf16
};

// dA of a piece of dY, rounded; bf16: what the rounding left, in `low` (beside an infinity nothing).
template <typename T>
__device__ __attribute__((always_inline)) inline void form_piece(int act, uint4& d, const uint4& pre, uint4& low)
{
    constexpr int N = Cols<T>::N;
    float v[N], a[N];
    Cols<T>::unpack(d, v);
    Cols<T>::unpack(pre, a);
    with_act(act, [&](auto which) {
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = act_grad<decltype(which)::value>(v[j], a[j]);
    });
    d = Cols<T>::round(v);
    if constexpr (sizeof(T) == 2) {
        Cols<T>::unpack(d, a);
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const float left = v[j] - a[j];
            v[j] = fabsf(left) < __builtin_inff() ? left : 0.f;
        }
        low = Cols<T>::round(v);
    }
}

// One value, at place `at` of the rows, whole.
template <typename T>
__device__ inline float formed_value(const ActPrologue& p, float d, int64_t at)
{
    const float a = value_of(static_cast<const T*>(p.pre)[at]);
    with_act(p.act, [&](auto which) { d = act_grad<decltype(which)::value>(d, a); });
    return d;
}
template <typename T>
__device__ inline float formed_value(const LowPieces& p, float d, int64_t at)
{
    return d + value_of(static_cast<const T*>(p.low)[at]);
}

// One value of the product, place `at` of the rows, with its bias and residual.
template <typename T>
__device__ inline float finish_value(const Epilogue& e, float v, float bias, float res, int64_t at)
{
    v += bias;
    if (!e.after) v += res;
    if (e.pre) static_cast<T*>(e.pre)[at] = from_f32<T>(v);
    with_act(e.act, [&](auto act) { v = act_of<decltype(act)::value>(v); });
    return e.after ? v + res : v;
}

// A value of dZ, formed where ZR's rows are.
template <typename ZR>
__device__ __attribute__((always_inline)) inline float whole_z(const DwArgs& a, int64_t r, int f)
{
    float v = z_value<typename ZTraits<ZR>::Plain>(a, r, f);
    if constexpr (ZTraits<ZR>::kFormed) {
        const float pre = value_of(static_cast<const typename ZR::T*>(a.pre)[r * a.F + f]);
        with_act(a.act, [&](auto which) { v = act_grad<decltype(which)::value>(v, pre); });
    }
    return v;
}

// dW (+)= X^T dA and db (+)= the sums of dA's columns, dA = dY act'(A) formed where it is read (bf16), or dY as it is (act 0, pre null); db may be
// null.  work: act_dw_bytes.  (linear_act_dw.hip; more rows than few_rows_dw takes.)
struct ActDw {
    const void* X;         // [n, K]
    const void* dY;        // [n, F]
    const void* pre;
    int act;
    float *dW, *db;
    int64_t n;
    int K, F, accumulate;
    void* work;
    void* formed;          // receives dA, of an even F; or null
    void* low;             // ... what its rounding left; or null
};
size_t act_dw_bytes(int64_t n, int K, int F);
int act_dw(int dtype, const ActDw& g, hipStream_t st);
// db (+)= the sums [groups, F] of workgroups, in order.
int act_sum(const float* partial, int groups, int F, int accumulate, float* db, hipStream_t st);

}  // namespace sar
