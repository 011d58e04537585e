// Element types of the reader operators: conversion to and from fp32, vector loads and stores.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace w2v {

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }

template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

// N consecutive elements as one memory access of sizeof(T) * N bytes (4, 8 or 16, or one element).
template <typename T, int N>
struct __align__(sizeof(T) * N) Pack {
    T e[N];
};

template <typename T, int N>
__device__ __forceinline__ Pack<T, N> load_pack(const T *p)
{
    return *reinterpret_cast<const Pack<T, N> *>(p);
}
template <typename T, int N>
__device__ __forceinline__ void store_pack(T *p, const Pack<T, N> &v)
{
    *reinterpret_cast<Pack<T, N> *>(p) = v;
}

// Two fp32 values rounded into one 32-bit register, the first in the low half.
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b)
{
    const __nv_bfloat162 x = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&x);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b)
{
    const __half2 x = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&x);
}

}  // namespace w2v
