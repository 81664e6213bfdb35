// Activations and their slopes, in fp32: group norm (gnorm.hpp), the short convolution (short.hip), the dense product (linear.hip).
#pragma once
#include <type_traits>

#include "common.hpp"

namespace lc {
namespace {

// The normal distribution function, and e = exp(-z^2 / 2) beside it.  erfc(x) exp(x^2) is t Q(t), t = 1 / (1 + 0.4 x), for x >= 0, Q the
// polynomial of degree eight of the least largest relative error (fitted by weighted least squares): 1.3e-7, and 2.2e-7 absolute in
// fp32.  Below zero the result is not a difference, so its relative error is that of e, 8e-7 down to z = -4.
__device__ __forceinline__ float normal_cdf(float z, float& e)
{
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.28284271247461901f, fabsf(z), 1.f));
    float q = __builtin_fmaf(0.025127103552222252f, t, -0.09143677353858948f);
    q = __builtin_fmaf(q, t, 0.08452295511960983f);
    q = __builtin_fmaf(q, t, -0.0027893988881260157f);
    q = __builtin_fmaf(q, t, 0.07071001827716827f);
    q = __builtin_fmaf(q, t, 0.08427219092845917f);
    q = __builtin_fmaf(q, t, 0.10392122715711594f);
    q = __builtin_fmaf(q, t, 0.11283480376005173f);
    q = __builtin_fmaf(q, t, 0.11283793300390244f);
    e = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);
    const float h = q * t * e;      // (half of erfc: the factor is in Q)
    return z < 0.f ? h : 1.f - h;
}

template <int ACT>
__device__ __forceinline__ float act_of(float z)
{
    if constexpr (ACT == LONGCONV_ACT_SILU) return z * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.4426950408889634f));
    if constexpr (ACT == LONGCONV_ACT_GELU) {
        float e;
        return z * normal_cdf(z, e);
    }
    if constexpr (ACT == LONGCONV_ACT_RELU) return z > 0.f ? z : z != z ? z : 0.f;
    return z;
}
template <int ACT>
__device__ __forceinline__ float slope_of(float z)
{
    if constexpr (ACT == LONGCONV_ACT_SILU) {
        const float q = __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.4426950408889634f));
        return q * (1.f + z * (1.f - q));
    }
    if constexpr (ACT == LONGCONV_ACT_GELU) {
        float e;
        const float c = normal_cdf(z, e);
        return __builtin_fmaf(z * 0.39894228040143268f, e, c);
    }
    if constexpr (ACT == LONGCONV_ACT_RELU) return z > 0.f ? 1.f : 0.f;
    return 1.f;
}

// by a value that is the same for all of a launch
__device__ __forceinline__ float act_by(int act, float z)
{
    switch (act) {
        case LONGCONV_ACT_SILU: return act_of<LONGCONV_ACT_SILU>(z);
        case LONGCONV_ACT_GELU: return act_of<LONGCONV_ACT_GELU>(z);
        case LONGCONV_ACT_RELU: return act_of<LONGCONV_ACT_RELU>(z);
        default: return z;
    }
}
__device__ __forceinline__ float slope_by(int act, float z)
{
    switch (act) {
        case LONGCONV_ACT_SILU: return slope_of<LONGCONV_ACT_SILU>(z);
        case LONGCONV_ACT_GELU: return slope_of<LONGCONV_ACT_GELU>(z);
        case LONGCONV_ACT_RELU: return slope_of<LONGCONV_ACT_RELU>(z);
        default: return 1.f;
    }
}

// of N at a time, one decision for all
template <int N>
__device__ __forceinline__ void acts_by(int act, float (&z)[N])
{
    const auto each = [&](auto which) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = act_of<decltype(which)::value>(z[i]);
    };
    if (act == LONGCONV_ACT_SILU) each(std::integral_constant<int, LONGCONV_ACT_SILU>());
    else if (act == LONGCONV_ACT_GELU) each(std::integral_constant<int, LONGCONV_ACT_GELU>());
    else if (act == LONGCONV_ACT_RELU) each(std::integral_constant<int, LONGCONV_ACT_RELU>());
}
template <int N>
__device__ __forceinline__ void slopes_by(int act, float (&z)[N])
{
    const auto each = [&](auto which) {
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = slope_of<decltype(which)::value>(z[i]);
    };
    if (act == LONGCONV_ACT_SILU) each(std::integral_constant<int, LONGCONV_ACT_SILU>());
    else if (act == LONGCONV_ACT_GELU) each(std::integral_constant<int, LONGCONV_ACT_GELU>());
    else if (act == LONGCONV_ACT_RELU) each(std::integral_constant<int, LONGCONV_ACT_RELU>());
    else each(std::integral_constant<int, LONGCONV_ACT_NONE>());
}

}  // namespace
}  // namespace lc
