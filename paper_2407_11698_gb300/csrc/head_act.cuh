// The activations of the floating-point head, act(u) and act'(u): u, max(u, 0), u s(u) with s = 1 / (1 + e^-u), and
// u Phi(u) with the normal distribution Phi.
#pragma once

#include <type_traits>

#include "head_out.cuh"

namespace nitro {
namespace {

__device__ __forceinline__ float rcp(float x) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}

// Phi(u) and its density.  For t = |u|, Phi(-t) = e^(-t^2 / 2) R(t); R falls smoothly from 1/2 like 1 / t, so with
// q = 1 / (1 + 0.35 t) it is q times a polynomial in q: nine coefficients, fitted to scipy's erfcx with equal
// relative errors over 0 <= t <= 14.5 (beyond it the exponential is 0), leave 3.2e-8, and in 32 bits 3.4e-7 at most
// (7.7e-8 in the mean square).  An erfc of the library is three times the instructions, which the
// memory-bound kernels feel, and does not give the density.
__device__ __forceinline__ void normal(float u, float* cdf, float* density) {
    const float t = fabsf(u), q = rcp(fmaf(0.35f, t, 1.0f));
    float p = -0.029158229008316994f;
    p = fmaf(p, q, 0.1440325528383255f);
    p = fmaf(p, q, -0.25584226846694946f);
    p = fmaf(p, q, 0.1593232899904251f);
    p = fmaf(p, q, -0.02321472205221653f);
    p = fmaf(p, q, 0.10555345565080643f);
    p = fmaf(p, q, 0.11982106417417526f);
    p = fmaf(p, q, 0.13986355066299438f);
    p = fmaf(p, q, 0.139621302485466f);
    const float e = ex2(u * u * (-0.5f * kLog2e)), tail = e * (p * q);
    *cdf = u < 0.0f ? tail : 1.0f - tail;
    *density = e * 0.3989422804f;
}

template <int ACT>
__device__ __forceinline__ float act_value(float u) {
    if constexpr (ACT == NITRO_ACT_RELU) return u < 0.0f ? 0.0f : u;          // (a NaN stays one)
    if constexpr (ACT == NITRO_ACT_SILU) return u * rcp(1.0f + ex2(u * -kLog2e));
    if constexpr (ACT == NITRO_ACT_GELU) {
        float c, d;
        normal(u, &c, &d);
        return u * c;
    }
    return u;
}

// (act(u), act'(u))
template <int ACT>
__device__ __forceinline__ float2 act_slope(float u) {
    if constexpr (ACT == NITRO_ACT_RELU) return make_float2(u < 0.0f ? 0.0f : u, u > 0.0f ? 1.0f : 0.0f);
    if constexpr (ACT == NITRO_ACT_SILU) {
        const float s = rcp(1.0f + ex2(u * -kLog2e));
        return make_float2(u * s, s * fmaf(u, 1.0f - s, 1.0f));
    }
    if constexpr (ACT == NITRO_ACT_GELU) {
        float c, d;
        normal(u, &c, &d);
        return make_float2(u * c, fmaf(u, d, c));
    }
    return make_float2(u, 1.0f);
}

// f(std::integral_constant<int, act>): one branch for a loop over values
template <class F>
__device__ __forceinline__ void with_act(int act, F&& f) {
    if (act == NITRO_ACT_SILU) f(std::integral_constant<int, NITRO_ACT_SILU>{});
    else if (act == NITRO_ACT_GELU) f(std::integral_constant<int, NITRO_ACT_GELU>{});
    else if (act == NITRO_ACT_RELU) f(std::integral_constant<int, NITRO_ACT_RELU>{});
    else f(std::integral_constant<int, NITRO_ACT_NONE>{});
}

inline bool act_known(int act) { return act >= NITRO_ACT_NONE && act <= NITRO_ACT_GELU; }

}  // namespace
}  // namespace nitro
