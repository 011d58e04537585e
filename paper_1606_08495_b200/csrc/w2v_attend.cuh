// What the forward and backward attention kernels share.
//
// A block works on kAttendTile = 128 consecutive positions of the token stream, whatever sentences they
// belong to: a stream of short sessions fills the tiles as well as one long document.  The keys that the
// block's rows see are one run of positions [lo, hi) (from the least window start to the largest window end)
// plus, where the sentence of the first rows begins before lo, that sentence's sinks below lo.  Inside the
// run a row's own limits decide: [window start, window end) or [sentence start, min(start + sinks, window start)).
#pragma once
#include "w2v_device.cuh"
#include "w2v_reader.h"
#include "w2v_tc.cuh"
#include "w2v_types.cuh"

namespace w2v {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kErrAttend = 8;                    // bit of the handle's error word

// What one row sees; an empty row has all limits 0.
struct RowLimits {
    int32_t lo, hi;                              // window
    int32_t s, se;                               // sinks before the window
};

__device__ __forceinline__ RowLimits row_limits(const AttendParams &p, int64_t i)
{
    RowLimits r = {0, 0, 0, 0};
    if (i < 0 || i >= p.n) return r;
    const int2 sp = __ldg(p.spans + i);
    if (sp.y <= sp.x) return r;
    r.lo = (int32_t)max((int64_t)sp.x, i - p.left);
    r.hi = (int32_t)min((int64_t)sp.y, i + p.right + 1);
    r.s = sp.x;
    r.se = (int32_t)min((int64_t)sp.x + p.sinks, (int64_t)r.lo);
    return r;
}

// Bits [a, b) of the 32 positions from `at` on.
__device__ __forceinline__ uint32_t range_bits(int32_t a, int32_t b, int32_t at)
{
    const int32_t x = min(max(a - at, 0), 32), y = min(max(b - at, 0), 32);
    if (y <= x) return 0u;
    return (y == 32 ? 0xFFFFFFFFu : (1u << y) - 1u) & ~((1u << x) - 1u);   // x < 32 here
}

// The bias by distance, in base-2 units, for every distance that a tile can hold which is not beyond the last
// bucket's start on one side: entries -(last + 255) .. last + 255.
__host__ __device__ inline int32_t bias_last(const BucketStarts &b) { return b.n ? b.start[b.n - 1] : 0; }
constexpr int32_t kBiasPad = 255;
__host__ __device__ inline uint32_t bias_entries(const BucketStarts &b) { return b.n ? 2u * (uint32_t)(bias_last(b) + kBiasPad) + 1u : 0u; }

__device__ __forceinline__ uint32_t bucket_of(const BucketStarts &b, int32_t rel)
{
    const int32_t far = b.two_sided ? abs(rel) : max(-rel, 0);
    uint32_t lo = 0, hi = b.n - 1;
    while (lo < hi) {
        const uint32_t mid = (lo + hi + 1) >> 1;
        if (b.start[mid] <= far) lo = mid; else hi = mid - 1;
    }
    return lo + (b.two_sided && rel > 0 ? b.n : 0u);
}

// A bias in base-2 units; one of the lowest float stays finite, so that a row of nothing else is still a row.
__device__ __forceinline__ float log2_bias(float b) { return b == -INFINITY ? b : fmaxf(b, -1e30f) * kLog2e; }

__device__ __forceinline__ void fill_bias(const AttendParams &p, uint32_t h, float *lut, uint32_t tid, uint32_t threads)
{
    const int32_t off = bias_last(p.b) + kBiasPad;
    for (uint32_t e = tid; e < bias_entries(p.b); e += threads)
        lut[e] = log2_bias(__ldg(p.bias + (size_t)bucket_of(p.b, (int32_t)e - off) * p.heads + h));
}

// Rows [at, at + rows) of an operand into a tile of the 128-byte swizzle by the `threads` calling threads
// (thread number lt): zeros for rows whose bit in `vis` (one word per 32 rows) is clear and for columns past the
// head.  CH = 16-byte chunks a row has room for (8 or 16), `used` of them are written.
template <int CH>
__device__ __forceinline__ void copy_rows_sw128(uint32_t tile, uint32_t block_bytes, const void *base, uint64_t ld_bytes, int64_t at,
                                                uint32_t rows, const uint32_t (&vis)[4], uint32_t dim_chunks, uint32_t used,
                                                uint32_t lt, uint32_t threads)
{
    const uint32_t ch = lt % CH;
    if (ch >= used) return;
    const uint32_t dst0 = tile + (ch >> 3) * block_bytes;
    const char *src0 = static_cast<const char *>(base) + ch * 16u;
    for (uint32_t r = lt / CH; r < rows; r += threads / CH) {
        const uint32_t word = r < 32 ? vis[0] : r < 64 ? vis[1] : r < 96 ? vis[2] : vis[3];
        const bool real = ch < dim_chunks && ((word >> (r & 31u)) & 1u);
        copy16(dst0 + r * 128u + (((ch & 7u) ^ (r & 7u)) << 4), real ? src0 + (uint64_t)(at + r) * ld_bytes : src0, real);
    }
}

// Which of the 128 positions from `at` on are words: one word of bits per 32, the same in every lane of the warp.
__device__ __forceinline__ void visible_bits(const AttendParams &p, int64_t at, uint32_t rows, uint32_t lane, uint32_t (&vis)[4])
{
    int2 sp[4];
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const int64_t j = at + w * 32 + lane;
        sp[w] = w * 32u + lane < rows && j >= 0 && j < p.n ? __ldg(p.spans + j) : make_int2(0, 0);
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) vis[w] = __ballot_sync(kFullMask, sp[w].y > sp[w].x);
}

}  // namespace w2v
