// What the forward and the backward layer-norm kernels share: how a row is laid over threads.
//
// A row is held in registers by a group of `gw` warps, at most kNormPer = 16 elements a lane: d <= 512
// takes one warp, d = 4096 eight.  A chunk is E consecutive elements of a lane (one access), chunk c of
// a row belongs to lane c mod 32 gw.  E is the widest access that row length, strides and base addresses allow.
#pragma once
#include "w2v_device.cuh"
#include "w2v_kernel_ready.h"
#include "w2v_reader.h"
#include "w2v_tc.cuh"
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

// ---- rows through a ring in shared memory ------------------------------------------------------------
// A row in registers is a row's bytes in flight only for as long as it takes to arrive, and the registers of a lane
// hold few of them.  Where rows can be copied in bulk (16-byte starts and lengths), every group of warps has a ring of
// units of kNormUnit consecutive rows that are copied in the background, and works on a unit at a time: the
// barrier and the lane sums of its rows are shared.
constexpr int kNormUnit = 2;

// How an array of rows is copied: a row at a time (row starts and lengths are multiples of 16 bytes: x always, since the
// kernels with a ring read it in 16-byte accesses), or a unit at a time (rows without gaps, whose units are; dy beside fp32 x), or not.
enum : uint32_t { kCopyRows = 0, kCopyUnits = 1, kCopyNot = 2 };
inline uint32_t norm_copy_mode(const void *p, uint64_t ld, uint32_t d, uint32_t size)
{
    if (reinterpret_cast<uintptr_t>(p) & 15u) return kCopyNot;
    if ((ld * size) % 16 == 0 && (d * size) % 16 == 0) return kCopyRows;
    return ld == d && (kNormUnit * d * size) % 16 == 0 ? kCopyUnits : kCopyNot;
}
// Bytes between the rows of a unit in shared memory.
inline __host__ __device__ uint32_t norm_pitch(uint32_t mode, uint32_t d, uint32_t size) { return mode == kCopyRows ? (d * size + 15u) & ~15u : d * size; }

__device__ __forceinline__ void norm_bulk(uint32_t dst, const void *src, uint32_t bytes, uint64_t *bar)
{
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(dst), "l"(src), "r"(bytes), "r"(smem_addr(bar)) : "memory");
}
// Rows [r, r + n) of an array to shared memory (one lane; returns the bytes to expect).  A unit that is copied whole but is
// cut off by the end of the array is left to norm_copy_tail.
__device__ __forceinline__ uint32_t norm_copy(uint32_t mode, uint32_t dst, const char *base, uint64_t ld_bytes, uint32_t row_bytes, uint32_t pitch,
                                              uint64_t r, uint32_t n, uint64_t *bar, bool issue)
{
    if (mode == kCopyUnits) {
        if (n < kNormUnit) return 0;
        if (issue) norm_bulk(dst, base + r * ld_bytes, kNormUnit * row_bytes, bar);
        return kNormUnit * row_bytes;
    }
    if (issue) for (uint32_t i = 0; i < n; ++i) norm_bulk(dst + i * pitch, base + (r + i) * ld_bytes, row_bytes, bar);
    return n * row_bytes;
}
// After a wait that ran out: what a group's first lane has issued lands (or has as long again) before the block leaves the
// ring or puts anything else there.  Unit number k of the group is in stage k mod stages.
__device__ __forceinline__ void norm_ring_drain(uint64_t *full, uint32_t issued, uint32_t stages, bool needed, int *quiet)
{
    if (!needed) return;
    for (uint32_t k = issued > stages ? issued - stages : 0; k < issued; ++k) mbar_wait(full + k % stages, (k / stages) & 1u, quiet);
}
// The cut-off unit of an array that is copied in units, by the lanes of a group.
template <typename T>
__device__ __forceinline__ void norm_copy_tail(unsigned char *dst, const T *row, uint32_t d, uint32_t n, uint32_t gl, uint32_t lanes)
{
    for (uint32_t i = gl; i < n * d; i += lanes) reinterpret_cast<T *>(dst)[i] = row[i];
}
__device__ __forceinline__ void group_barrier(uint32_t gw, uint32_t group)
{
    if (gw == 1) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(group + 1u), "r"(gw * 32u) : "memory");
}

// A ring pays from this many KB of x per SM on; less, and the registers' next row is enough and the ring's start is not.
constexpr uint64_t kNever = ~0ull;
inline bool ring_pays(uint64_t rows, uint32_t d, uint32_t size, int sms, uint64_t from_kb)
{
    return from_kb != kNever && rows * d * size >= from_kb * 1024 * (uint64_t)sms;
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
