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

// z Phi(z) with Phi(z) = 1/2 + z Q(z^2), Q a polynomial of degree 13 in (z^2 - c/2) / (c/2) on z^2 <= c = 5.2^2, fitted
// to the normal distribution function by iterated least squares (least maximum of |z| times the error: 6.4e-8; with the
// rounding of 32-bit Horner 2.3e-7).  Beyond, z Q(c) passes 1/2 and saturation makes Phi exactly 0 or 1.  Ten
// instructions a value, no special functions, where erff takes thirty and branches; accurate to 2.3e-7 |z|.
// Eight values are interleaved, so that the chain of one hides behind the others'.
__device__ __forceinline__ void phi8(const float *z, float *phi)
{
    const float top = 5.2f * 5.2f;
    constexpr float kQ[14] = {-4.813592823e-04f, 1.268577063e-03f, -1.221270184e-03f, 1.799950609e-03f, -4.789268132e-03f,
                              8.560134098e-03f, -1.250501070e-02f, 1.795471460e-02f, -2.472365461e-02f, 3.198997304e-02f,
                              -3.992981836e-02f, 5.002452061e-02f, -6.774366647e-02f, 1.359499991e-01f};
    uint64_t s[4], q[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float u0, u1;
        const Pair both(z[2 * k], z[2 * k + 1]);
        mul2(both, both).get(u0, u1);
        s[k] = fma2(Pair(fminf(u0, top), fminf(u1, top)), Pair(2.0f / top, 2.0f / top), Pair(-1.0f, -1.0f)).both;
        q[k] = Pair(kQ[0], kQ[0]).both;
    }
#pragma unroll
    for (int i = 1; i < 14; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) q[k] = fma2(Pair(q[k]), Pair(s[k]), Pair(kQ[i], kQ[i])).both;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        float q0, q1;
        Pair(q[k]).get(q0, q1);
        phi[2 * k] = __saturatef(fmaf(z[2 * k], q0, 0.5f));
        phi[2 * k + 1] = __saturatef(fmaf(z[2 * k + 1], q1, 0.5f));
    }
}

__device__ __forceinline__ void gelu8(float *z)
{
    float phi[8];
    phi8(z, phi);
#pragma unroll
    for (int i = 0; i < 8; ++i) z[i] *= phi[i];
}

// v times the activation's slope at z.
__device__ __forceinline__ void times_slope8(float (&v)[8], const float (&z)[8], int act)
{
    if (act == ACT_GELU) {                                  // Phi(z) + z exp(-z^2 / 2) / sqrt(2 pi)
        float phi[8];
        phi8(z, phi);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= fmaf(z[i] * 0.39894228f, exp2_fast(z[i] * z[i] * -0.72134752f), phi[i]);
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
    } else if (act == ACT_SILU) {
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
