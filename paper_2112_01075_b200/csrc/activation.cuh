// Activations of the linear layer on values in registers.
#pragma once

#include <cuda_runtime.h>

#include <cstdint>

#include "elements.cuh"
#include "product.h"

namespace redist {

__device__ __forceinline__ float reciprocal(float v)
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

__device__ __forceinline__ float exp2_fast(float v)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
    return r;
}

// Phi, the normal distribution function, below zero, where its relative accuracy counts: Phi(-x) = exp(-x^2 / 2) R(x) for x =
// |z|, with R falling slowly, from 1/2 like 1 / (x sqrt(2 pi)).  In v = 1 / (x + 5/2) R is v times a polynomial of degree 7,
// fitted on 0 <= x <= 13.3 by iterated least squares (relative error 9e-8 up to x = 4, 1.7e-6 at most beyond).  So the lower
// tail of GELU and of its slope is as accurate as 32-bit numbers reach: 5e-7 + 1.5 z^2 2^-24 of Phi (the latter from the
// exponent's rounding), where 1 + erf loses all digits towards z = -5.5.  Above zero Phi is 1 - Phi(-z).
// below[i] = Phi(-|z|), e[i] = 8 exp(-z^2 / 2) (eight times, so that what z e takes out of the subnormal numbers has not been
// flushed to zero).  Eight values are interleaved, so that the chain of one hides behind the others'.
__device__ __forceinline__ void phi8(const float *z, float *below, float *e)
{
    constexpr float kR[8] = {-7.040148735e+00f, 1.433973980e+01f, -1.063558006e+01f, 2.726462602e+00f,
                             2.835668437e-02f, 2.950876057e-01f, 1.230796501e-01f, 4.989921674e-02f};        // of R / 8
    uint64_t v[4], q[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const Pair both(z[2 * k], z[2 * k + 1]);
        fma2(mul2(both, both), Pair(-0.72134752f, -0.72134752f), Pair(3.0f, 3.0f)).get(e[2 * k], e[2 * k + 1]);
        e[2 * k] = exp2_fast(e[2 * k]);
        e[2 * k + 1] = exp2_fast(e[2 * k + 1]);
        v[k] = Pair(reciprocal(fabsf(z[2 * k]) + 2.5f), reciprocal(fabsf(z[2 * k + 1]) + 2.5f)).both;
        q[k] = Pair(kR[0], kR[0]).both;
    }
#pragma unroll
    for (int i = 1; i < 8; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) q[k] = fma2(Pair(q[k]), Pair(v[k]), Pair(kR[i], kR[i])).both;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        mul2(mul2(Pair(q[k]), Pair(v[k])), Pair(e[2 * k], e[2 * k + 1])).get(below[2 * k], below[2 * k + 1]);
}

__device__ __forceinline__ void gelu8(float *z)
{
    float below[8], e[8];
    phi8(z, below, e);
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] *= z[i] < 0.0f ? below[i] : 1.0f - below[i];
}

// v times the activation's slope at z.
__device__ __forceinline__ void times_slope8(float (&v)[8], const float (&z)[8], int act)
{
    if (act == ACT_GELU) {                                  // Phi(z) + z exp(-z^2 / 2) / sqrt(2 pi)
        float below[8], e[8];
        phi8(z, below, e);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float s = fmaf(fabsf(z[i]) * (-0.39894228f / 8), e[i], below[i]);         // of -|z|; that of |z| is 1 - s
            v[i] *= z[i] < 0.0f ? s : 1.0f - s;
        }
    } else if (act == ACT_SILU) {                           // with s = 1 / (1 + exp(-z)): s + z s (1 - s)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float s = reciprocal(1.0f + exp2_fast(z[i] * -1.44269504f));
            v[i] *= fmaf(z[i] * s, 1.0f - s, s);
        }
    } else if (act == ACT_RELU) {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = z[i] > 0.0f ? v[i] : v[i] * 0.0f;
    }
}

// N values (a multiple of eight), one branch for all.
template <int N> __device__ __forceinline__ void activate_all(float *v, int act)
{
    if (act == ACT_GELU) {
#pragma unroll
        for (int i = 0; i < N; i += 8) gelu8(v + i);
    } else if (act == ACT_SILU) {                           // (0 below z = -87.3, where it is above -1.1e-36: the reciprocal is flushed)
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] *= reciprocal(1.0f + exp2_fast(v[i] * -1.44269504f));
    } else if (act == ACT_RELU) {
#pragma unroll
        for (int i = 0; i < N; ++i) asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(v[i]));
    }
}
__device__ __forceinline__ void activate8(float (&v)[8], int act) { activate_all<8>(v, act); }
__device__ __forceinline__ void activate32(float (&v)[32], int act) { activate_all<32>(v, act); }

}  // namespace redist
