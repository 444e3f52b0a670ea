// fff_activations.hpp -- the activations and their derivatives where many values
// are formed beside a product or a pass over memory: fewer instructions than the layer's own
// (fff_device.hpp) at the same or half the accuracy, as each says.
#pragma once

#include "fff_device.hpp"

#include <hip/hip_runtime.h>

namespace fff {

// Phi(-a) for a = |z|, Phi the standard normal distribution, and e = exp(-a^2 / 2): e t Q(t) with
// t = 1 / (1 + 0.3 a), Q the polynomial of degree 7 nearest to Phi(-a) / (e t) over a = 0 .. 14 in relative
// error (1.5e-7, fitted for this kernel; 15 roundings of fp32 to a = 4, 130 at 13, where e carries
// that of its argument).  Twenty instructions; erfcf's are several times as many, and at 268 M values
// they took as long as the product.
__device__ __forceinline__ float normal_tail(float z, float& e) {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3f, __builtin_fabsf(z), 1.0f));
    e = __builtin_amdgcn_exp2f(z * z * -0.72134752044448170368f);
    float q = 0.03567512333393097f;
    q = __builtin_fmaf(q, t, -0.15720446407794952f);
    q = __builtin_fmaf(q, t, 0.2063557654619217f);
    q = __builtin_fmaf(q, t, -0.05368557944893837f);
    q = __builtin_fmaf(q, t, 0.1285625696182251f);
    q = __builtin_fmaf(q, t, 0.09991323202848434f);
    q = __builtin_fmaf(q, t, 0.12075399607419968f);
    q = __builtin_fmaf(q, t, 0.11962929368019104f);
    return e * t * q;
}

// Phi(z) where its result is stored in fp32 (FINE below): within |z| < 1, where the tail's roundings are largest
// beside the result, 0.5 + z R(z^2), R the polynomial of degree 5 nearest to (Phi(z) - 0.5) / z there
// (7e-10 relative, fitted for this kernel).  For z ~ N(0, 1) the root mean square errors in units of 2^-24,
// by the tail alone, by this and by the layer's own erfcf (fff_device.hpp): GELU 0.475, 0.381, 0.375; its
// derivative 0.826, 0.454, 0.465.  Time (us) in the same order: 9001 x 16 fp32, 768 -> 1000 with the
// derivative 153.7, 156.3, 162.7; 65536 x 32, bf16 1024 -> 4096 to fp32 with GELU 778, 809, 948.  Results
// stored in bf16 lose 16 bits more than either, and take the tail alone.
__device__ __forceinline__ float normal_cdf(float z, float& e) {
    const float s = z * z, p = normal_tail(z, e);
    float q = -7.654209184693173e-06f;
    q = __builtin_fmaf(q, s, 0.00011348637781338766f);
    q = __builtin_fmaf(q, s, -0.0011863299878314137f);
    q = __builtin_fmaf(q, s, 0.009973322972655296f);
    q = __builtin_fmaf(q, s, -0.06649035960435867f);
    q = __builtin_fmaf(q, s, 0.3989422917366028f);
    return s < 1.0f ? __builtin_fmaf(z, q, 0.5f) : z > 0.0f ? 1.0f - p : p;
}

// The activations and their derivatives (fff_device.hpp has their formulas).  FINE: to be stored in fp32.
template <int ACT, bool FINE>
__device__ __forceinline__ float act_value(float z) {
    if constexpr (ACT == ACT_GELU_ERF) {
        float e;
        if constexpr (FINE) return z * normal_cdf(z, e);
        const float p = normal_tail(z, e);
        return z * (z > 0.0f ? 1.0f - p : p);
    } else if constexpr (ACT == ACT_GELU_TANH) {
        const float d = 1.0f + __builtin_amdgcn_exp2f(-2.88539008177792681472f * gelu_tanh_u(z));
        const float t = __builtin_amdgcn_rcpf(d), q = z * t;
        // the quotient's own remainder once more, as a true division leaves it (0.516 -> 0.465 of the units above);
        // where d overflows, t and q are 0 and stay so, and over 1 there is none (nor a NaN of infinities)
        if constexpr (FINE) {
            const float left = __builtin_fmaf(-__builtin_fminf(d, 3.4028234663852886e38f), q, z);
            return d > 1.0f ? __builtin_fmaf(left, t, q) : q;
        }
        return q;
    } else {
        return z;
    }
}
template <int ACT, bool FINE>
__device__ __forceinline__ float act_slope(float z) {
    if constexpr (ACT == ACT_GELU_ERF) {
        float e;
        if constexpr (FINE) {
            const float c = normal_cdf(z, e);
            return __builtin_fmaf(z * 0.39894228040143267794f, e, c);
        }
        const float p = normal_tail(z, e);
        return __builtin_fmaf(z * 0.39894228040143267794f, e, z > 0.0f ? 1.0f - p : p);
    } else if constexpr (ACT == ACT_GELU_TANH) {
        const float u = 2.88539008177792681472f * gelu_tanh_u(z);
        const float up = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-u));
        const float down = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(u));
        // far out up * down is 0, and so are its products with a finite z and a square kept from overflow
        const float du = __builtin_fminf(__builtin_fmaf(0.134145f * z, z, 1.0f), 1e38f);
        return __builtin_fmaf(z * up * down, 1.59576912160573071176f * du, up);
    } else {
        return 1.0f;
    }
}

}  // namespace fff
