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

// Two values a register pair: one instruction issues two sums, products or both, which leaves the issue slots that
// conversions, exponentials and addresses need
__device__ __forceinline__ unsigned long long bits2(float2 v) { return *reinterpret_cast<unsigned long long*>(&v); }
__device__ __forceinline__ float2 pair(float a) { return make_float2(a, a); }
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    unsigned long long r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)));
    return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)));
    return *reinterpret_cast<float2*>(&r);
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    unsigned long long r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(bits2(a)), "l"(bits2(b)), "l"(bits2(c)));
    return *reinterpret_cast<float2*>(&r);
}
// (a - b: a fused a + (-1) b, which rounds once as well)
__device__ __forceinline__ float2 sub2(float2 a, float2 b) { return fma2(b, pair(-1.0f), a); }
__device__ __forceinline__ float2 ex2(float2 t) { return make_float2(ex2(t.x), ex2(t.y)); }
__device__ __forceinline__ float2 rcp(float2 t) { return make_float2(rcp(t.x), rcp(t.y)); }

// Phi(u) and its density.  For t = |u|, Phi(-t) = e^(-t^2 / 2) R(t); R falls smoothly from 1/2 like 1 / t, so with
// q = 1 / (1 + 0.35 t) it is q times a polynomial in q: nine coefficients, fitted to scipy's erfcx with equal
// relative errors over 0 <= t <= 14.5 (beyond it the exponential is 0), leave 3.2e-8, and in 32 bits 3.4e-7 at most
// (7.7e-8 in the mean square) of R.  Phi is 1.8e-7 off at most, but in its tail the rounding of u^2 is most of the error: 1.5e-6 of
// Phi(-5), 7.5e-6 of Phi(-12).  An erfc of the library is three times the instructions, which the
// memory-bound kernels feel, and does not give the density.
__device__ __forceinline__ void normal(float2 u, float2* cdf, float2* density) {
    const float2 t = make_float2(fabsf(u.x), fabsf(u.y)), q = rcp(fma2(t, pair(0.35f), pair(1.0f)));
    float2 p = pair(-0.029158229008316994f);
    p = fma2(p, q, pair(0.1440325528383255f));
    p = fma2(p, q, pair(-0.25584226846694946f));
    p = fma2(p, q, pair(0.1593232899904251f));
    p = fma2(p, q, pair(-0.02321472205221653f));
    p = fma2(p, q, pair(0.10555345565080643f));
    p = fma2(p, q, pair(0.11982106417417526f));
    p = fma2(p, q, pair(0.13986355066299438f));
    p = fma2(p, q, pair(0.139621302485466f));
    const float2 e = ex2(mul2(mul2(u, u), pair(-0.5f * kLog2e))), tail = mul2(e, mul2(p, q)), rest = sub2(pair(1.0f), tail);
    *cdf = make_float2(u.x < 0.0f ? tail.x : rest.x, u.y < 0.0f ? tail.y : rest.y);
    *density = mul2(e, pair(0.3989422804f));
}

template <int ACT>
__device__ __forceinline__ float2 act_value(float2 u) {
    if constexpr (ACT == NITRO_ACT_RELU) return make_float2(u.x < 0.0f ? 0.0f : u.x, u.y < 0.0f ? 0.0f : u.y);   // (a NaN stays one)
    if constexpr (ACT == NITRO_ACT_SILU) return mul2(u, rcp(add2(ex2(mul2(u, pair(-kLog2e))), pair(1.0f))));
    if constexpr (ACT == NITRO_ACT_GELU) {
        float2 c, d;
        normal(u, &c, &d);
        return mul2(u, c);
    }
    return u;
}
template <int ACT>
__device__ __forceinline__ float act_value(float u) {
    return act_value<ACT>(make_float2(u, 0.0f)).x;
}

// act(u) and act'(u)
template <int ACT>
__device__ __forceinline__ float2 act_slope(float2 u, float2* value) {
    if constexpr (ACT == NITRO_ACT_RELU) {
        *value = act_value<ACT>(u);
        return make_float2(u.x > 0.0f ? 1.0f : 0.0f, u.y > 0.0f ? 1.0f : 0.0f);
    }
    if constexpr (ACT == NITRO_ACT_SILU) {
        const float2 s = rcp(add2(ex2(mul2(u, pair(-kLog2e))), pair(1.0f)));
        *value = mul2(u, s);
        return fma2(*value, sub2(pair(1.0f), s), s);
    }
    if constexpr (ACT == NITRO_ACT_GELU) {
        float2 c, d;
        normal(u, &c, &d);
        *value = mul2(u, c);
        return fma2(u, d, c);
    }
    *value = u;
    return pair(1.0f);
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
