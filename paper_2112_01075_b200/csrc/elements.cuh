// 16- and 32-bit floating point elements: conversion, and loads of several neighbours at any alignment.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "product.h"

namespace redist {

template <int TYPE> struct Element;
template <> struct Element<T_BF16> { using type = __nv_bfloat16; };
template <> struct Element<T_F16> { using type = __half; };
template <> struct Element<T_F32> { using type = float; };

__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(float v) { return v; }

template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }

// Two neighbours in one 32-bit word, the first in the low half.
template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi)
{
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi)
{
    const __half2 v = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&v);
}
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t v);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t v)
{
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t v)
{
    return __half22float2(*reinterpret_cast<const __half2 *>(&v));
}

// Two values at a time: one instruction for both where the operation is an addition or a product.
struct Pair {
    uint64_t both;
    __device__ __forceinline__ Pair(uint64_t v) : both(v) {}
    __device__ __forceinline__ Pair(float a, float b) { asm("mov.b64 %0, {%1, %2};" : "=l"(both) : "f"(a), "f"(b)); }
    __device__ __forceinline__ void get(float &a, float &b) const { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(both)); }
    __device__ __forceinline__ float sum() const
    {
        float a, b;
        get(a, b);
        return a + b;
    }
};
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a.both), "l"(b.both), "l"(c.both));
    return Pair(r);
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b)
{
    uint64_t r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a.both), "l"(b.both));
    return Pair(r);
}

__device__ __forceinline__ Pair add2(Pair a, Pair b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a.both), "l"(b.both));
    return Pair(r);
}

// Element `i` of an array whose type is only known at run time.
__device__ __forceinline__ float load_any(const void *p, int type, int64_t i)
{
    if (type == T_F32) return static_cast<const float *>(p)[i];
    if (type == T_BF16) return to_float(static_cast<const __nv_bfloat16 *>(p)[i]);
    return to_float(static_cast<const __half *>(p)[i]);
}

// 16 bytes that start at any multiple of the element size: the one or two aligned 16-byte blocks that hold them, to be
// shifted together.  `bytes` of the 16 are wanted (1 to 16); a block that holds none of those is not touched, so nothing is
// read outside the 16-byte blocks of the array's own bytes.  Loading and shifting are two steps, so that several loads can be
// under way before the first is looked at.
struct Blocks {
    uint4 a, b;
    __device__ __forceinline__ void load(const void *p, int bytes)
    {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        const uint32_t off = uint32_t(at & 15);
        const uint4 *q = reinterpret_cast<const uint4 *>(at - off);
        a = q[0];
        b = make_uint4(0, 0, 0, 0);
        if (int(off) + bytes > 16) b = q[1];
    }
    __device__ __forceinline__ uint4 get(const void *p) const
    {
        const uint32_t off = uint32_t(reinterpret_cast<uintptr_t>(p) & 15);
        const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
        const uint32_t word = off >> 2, bit = (off & 3) * 8;
        uint32_t r[5];
#pragma unroll
        for (int i = 0; i < 5; ++i) {
            uint32_t v = w[i];
            if (word == 1) v = w[i + 1];
            if (word == 2) v = w[i + 2];
            if (word == 3) v = i + 3 < 8 ? w[i + 3] : 0;
            r[i] = v;
        }
        return make_uint4(__funnelshift_r(r[0], r[1], bit), __funnelshift_r(r[1], r[2], bit), __funnelshift_r(r[2], r[3], bit),
                          __funnelshift_r(r[3], r[4], bit));
    }
};

__device__ __forceinline__ uint4 load16_any(const void *p, int bytes)
{
    Blocks v;
    v.load(p, bytes);
    return v.get(p);
}

__device__ __forceinline__ void wait_for_previous() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void let_next_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

}  // namespace redist
