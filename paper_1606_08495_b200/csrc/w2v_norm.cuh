// What the forward and the backward layer-norm kernels share: how a row is laid over threads.
//
// A row is held in registers by a group of `gw` warps, at most kNormPer = 16 elements a lane: d <= 512
// takes one warp, d = 4096 eight.  A chunk is E consecutive elements of a lane (one access), chunk c of
// a row belongs to lane c mod 32 gw.  E is the widest access that row length, strides and base addresses allow.
#pragma once
#include "w2v_device.cuh"
#include "w2v_reader.h"
#include "w2v_types.cuh"

namespace w2v {

constexpr uint32_t kNormPer = 16;

// Sums K values over the `gw` warps of a row's group; `slot` is shared memory for K floats per warp, twice: `flip`
// alternates from call to call so that one barrier per call is enough.
template <int K>
__device__ __forceinline__ void group_sum(float (&a)[K], uint32_t gw, uint32_t wig, uint32_t group, uint32_t lane, float *slot,
                                          uint32_t flip)
{
#pragma unroll
    for (int k = 0; k < K; ++k) a[k] = warp_sum(a[k]);
    if (gw == 1) return;
    float *s = slot + flip * 32u * K + group * gw * K;
    if (lane == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) s[wig * K + k] = a[k];
    }
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1u), "r"(gw * 32u) : "memory");
    const uint32_t wide = 1u << (32 - __clz(gw - 1u)), from = lane & (wide - 1u);     // gw rounded up to a power of two
#pragma unroll
    for (int k = 0; k < K; ++k) a[k] = from < gw ? s[from * K + k] : 0.f;
    for (uint32_t o = wide >> 1; o > 0; o >>= 1) {
#pragma unroll
        for (int k = 0; k < K; ++k) a[k] += __shfl_xor_sync(kFullMask, a[k], o);
    }
}

// A lane's chunks of one row, zeros past its end.
template <typename T, int E, int NV>
__device__ __forceinline__ void norm_row_load(Pack<T, E> (&v)[NV], const T *row, uint32_t gl, uint32_t gw, uint32_t d)
{
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const uint32_t at = (gl + c * 32u * gw) * E;
        if (at < d) v[c] = load_pack<T, E>(row + at);
        else {
#pragma unroll
            for (int e = 0; e < E; ++e) v[c].e[e] = from_f32<T>(0.f);
        }
    }
}

// A lane's weights (zeros past the row's end), 16 bytes at a time where they are aligned.
template <int E, int NV>
__device__ __forceinline__ void norm_weights_load(float (&w)[NV * E], const float *from, uint32_t gl, uint32_t gw, uint32_t d)
{
    const bool wide = E % 4 == 0 && (reinterpret_cast<uintptr_t>(from) & 15u) == 0;
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const uint32_t at = (gl + c * 32u * gw) * E;
        if (wide) {
#pragma unroll
            for (int e = 0; e + 3 < E; e += 4) {
                const float4 t = at < d ? __ldg(reinterpret_cast<const float4 *>(from + at + e)) : make_float4(0.f, 0.f, 0.f, 0.f);
                w[c * E + e] = t.x; w[c * E + e + 1] = t.y; w[c * E + e + 2] = t.z; w[c * E + e + 3] = t.w;
            }
        } else {
#pragma unroll
            for (int e = 0; e < E; ++e) w[c * E + e] = at < d ? __ldg(from + at + e) : 0.f;
        }
    }
}

struct NormShape {
    uint32_t gw;        // warps per row
    uint32_t groups;    // rows per block
    uint32_t e;         // elements per access
    uint32_t nv;        // accesses per lane and row
};

inline uint32_t widest_access(uint32_t d, uint32_t size, uint64_t ld, const void *p, uint32_t e)
{
    while (e > 1 && (d % e || ld % e || (reinterpret_cast<uintptr_t>(p) % (e * size)))) e >>= 1;
    return e;
}

inline NormShape norm_shape(uint32_t d, uint32_t e)
{
    NormShape s;
    s.e = e == 2 ? 1 : e;
    const uint32_t chunks = (d + s.e - 1) / s.e;
    s.gw = (chunks * s.e + 32u * kNormPer - 1) / (32u * kNormPer);
    s.groups = s.gw >= 8 ? 1 : 8 / s.gw;
    s.nv = (chunks + 32u * s.gw - 1) / (32u * s.gw);
    return s;
}

}  // namespace w2v
