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

// Elements 2 i and 2 i + 1 of a pack in fp32, and back.
template <int N> __device__ __forceinline__ float2 pair_f32(const Pack<float, N> &p, int i) { return make_float2(p.e[2 * i], p.e[2 * i + 1]); }
template <int N> __device__ __forceinline__ float2 pair_f32(const Pack<__half, N> &p, int i) { return __half22float2(*reinterpret_cast<const __half2 *>(&p.e[2 * i])); }
template <int N>
__device__ __forceinline__ float2 pair_f32(const Pack<__nv_bfloat16, N> &p, int i)
{
    const uint32_t u = *reinterpret_cast<const uint32_t *>(&p.e[2 * i]);
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
}
template <int N> __device__ __forceinline__ void set_pair(Pack<float, N> &p, int i, float2 v) { p.e[2 * i] = v.x; p.e[2 * i + 1] = v.y; }
template <typename T, int N>
__device__ __forceinline__ void set_pair(Pack<T, N> &p, int i, float2 v) { *reinterpret_cast<uint32_t *>(&p.e[2 * i]) = pack2<T>(v.x, v.y); }

}  // namespace w2v
