// The activations of the learner's layers and their derivatives, in fp32.
#pragma once

#include <hip/hip_runtime.h>

#include "malib.h"

namespace malib {

namespace {   // (each kernel file's own)

// The activations and their derivatives at z, in fp32.  relu passes a NaN on, as the
// policies' hidden layers do; its derivative at 0 is 0.
__device__ __forceinline__ float relu_f32(float z) { return z != z ? z : (z > 0.0f ? z : 0.0f); }

// e^-x^2 / 2 (`e`) and Phi(x), the normal distribution function.  With ax = |x|,
// 1 - Phi(ax) = e^(-x^2 / 2) R(ax), where R is smooth and falls like 1 / ax: a polynomial
// in t = 1 / (1 + 0.32 ax), fitted to R for the least relative error over all ax >= 0
// (3.2e-8).  To the left the exponent's rounding is the larger part: Phi is within 4e-7 of
// itself down to -2, 2e-6 at -6 (0.5 (1 + erf) in fp32: 1e-5 at -3, 5% at -5).
__device__ __forceinline__ float normal_cdf(float x, float& e)
{
    constexpr int N = 10;
    constexpr float kR[N] = {1.276615262e-01f, 1.276609451e-01f,  1.146223545e-01f,
                             8.782909811e-02f, 5.865395442e-02f,  -9.377530776e-03f,
                             6.532797217e-02f, -1.467074007e-01f, 9.540722519e-02f,
                             -2.107816003e-02f};
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.32f, __builtin_fabsf(x), 1.0f));
    float p = kR[N - 1];
#pragma unroll
    for (int i = N - 2; i >= 0; --i)
        p = __builtin_fmaf(p, t, kR[i]);
    e = __builtin_amdgcn_exp2f(-0.72134752044448170f * (x * x));
    const float tail = (p * t) * e;
    return x > 0.0f ? 1.0f - tail : tail;
}

__device__ __forceinline__ float sigmoid_f32(float z)
{
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-1.44269504088896341f * z));
}

template <int N>
__device__ __forceinline__ void activate(int act, float (&v)[N])
{
    switch (act) {
    case MALIB_ACT_RELU:
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] = relu_f32(v[i]);
        break;
    case MALIB_ACT_GELU:
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float e;
            v[i] *= normal_cdf(v[i], e);
        }
        break;
    case MALIB_ACT_SILU:
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] *= sigmoid_f32(v[i]);
        break;
    }
}

// v[i] *= act'(z[i])
template <int N>
__device__ __forceinline__ void times_slope(int act, const float (&z)[N], float (&v)[N])
{
    switch (act) {
    case MALIB_ACT_RELU:
#pragma unroll
        for (int i = 0; i < N; ++i)
            v[i] *= z[i] > 0.0f ? 1.0f : 0.0f;
        break;
    case MALIB_ACT_GELU:
#pragma unroll
        for (int i = 0; i < N; ++i) {
            float e;
            const float p = normal_cdf(z[i], e);
            v[i] *= __builtin_fmaf(z[i] * 0.39894228040143268f, e, p);
        }
        break;
    case MALIB_ACT_SILU:
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float s = sigmoid_f32(z[i]);
            v[i] *= s * __builtin_fmaf(z[i], 1.0f - s, 1.0f);
        }
        break;
    }
}

}  // namespace

}  // namespace malib
