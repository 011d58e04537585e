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

// Sums two values over the `gw` warps of a row's group; `slot` is the group's shared memory, two
// floats per warp, and `flip` alternates from call to call so that one barrier per call is enough.
__device__ __forceinline__ float2 group_sum2(float a, float b, uint32_t gw, uint32_t wig, uint32_t group, uint32_t lane,
                                             float2 *slot, uint32_t flip)
{
    a = warp_sum(a);
    b = warp_sum(b);
    if (gw == 1) return make_float2(a, b);
    float2 *s = slot + flip * 32u;
    if (lane == 0) s[group * gw + wig] = make_float2(a, b);
    asm volatile("bar.sync %0, %1;" ::"r"(group + 1u), "r"(gw * 32u) : "memory");
    float2 t = make_float2(0.f, 0.f);
    for (uint32_t w = 0; w < gw; ++w) {
        const float2 x = s[group * gw + w];
        t.x += x.x;
        t.y += x.y;
    }
    return t;
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
