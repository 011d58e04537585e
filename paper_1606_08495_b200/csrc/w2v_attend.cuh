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
#include "w2v_tma.h"
#include "w2v_types.cuh"

namespace w2v {

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kErrAttend = 8;                    // bit of the handle's error word

// The sentence of position i (0 <= i < n), empty for one that is not a word.  It ends with the stream; a pair that is not
// around i, which w2v_sentence_spans does not write for this position, counts as empty: nothing is read by such an index.
__device__ __forceinline__ int2 word_span(const AttendParams &p, int64_t i)
{
    const int2 sp = __ldg(p.spans + i);
    return sp.x >= 0 && sp.x <= i && sp.y > i ? make_int2(sp.x, min(sp.y, (int32_t)p.n)) : make_int2(0, 0);
}

// What one row sees; an empty row has all limits 0.
struct RowLimits {
    int32_t lo, hi;                              // window
    int32_t s, se;                               // sinks before the window
};

__device__ __forceinline__ RowLimits row_limits(const AttendParams &p, int64_t i)
{
    RowLimits r = {0, 0, 0, 0};
    if (i < 0 || i >= p.n) return r;
    const int2 sp = word_span(p, i);
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

// The bias by distance, in base-2 units, for every distance that the part of a tile which a warp works on (32 rows, up
// to 64 columns: distances that span 94) can hold unless all of it lies beyond the last bucket's start: entries
// -(last + kBiasPad) .. last + kBiasPad.
__host__ __device__ inline int32_t bias_last(const BucketStarts &b) { return b.n ? b.start[b.n - 1] : 0; }
constexpr int32_t kBiasPad = 96;
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

// A bias in base-2 units; one of the lowest float stays finite (the lowest that does is 2.35e38 below zero), so that a row of
// nothing else is still a row.
constexpr float kLowest = -2.35e38f, kLowestBias = kLowest * kLog2e;
__device__ __forceinline__ float log2_bias(float b) { return b == -INFINITY ? b : fmaxf(b, kLowest) * kLog2e; }

// Relative positions [r0, r1) (key - query, within -off .. off) whose bias is bucket b's.
__device__ __forceinline__ void bucket_range(const BucketStarts &s, uint32_t b, int32_t off, int32_t &r0, int32_t &r1)
{
    const uint32_t side = b >= s.n ? 1u : 0u, k = b - side * s.n;
    const int32_t d0 = s.start[k], d1 = k + 1 < s.n ? s.start[k + 1] : off + 1;       // distances [d0, d1) on its side
    if (side) { r0 = max(d0, 1); r1 = d1; }
    else { r0 = 1 - d1; r1 = k == 0 && !s.two_sided ? off + 1 : 1 - d0; }
}

// The table of a head by `warps` warps (this one is number `warp`).  A lane takes one distance and counts the buckets
// that start at or before it; the entries beyond the last start are the last bucket's.
__device__ __forceinline__ void fill_bias(const AttendParams &p, uint32_t h, float *lut, uint32_t warp, uint32_t warps, uint32_t lane)
{
    const int32_t last = bias_last(p.b), off = last + kBiasPad;
    const uint32_t n = p.b.n, buckets = n * (p.b.two_sided ? 2u : 1u);
    float v[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) v[i] = lane + 32u * i < buckets ? __ldg(p.bias + (size_t)(lane + 32 * i) * p.heads + h) : 0.f;
    v[0] = log2_bias(v[0]);
    v[1] = log2_bias(v[1]);
    auto value = [&](uint32_t b) {                                   // every lane its own bucket
        const float x = __shfl_sync(kFullMask, v[0], b & 31u), y = buckets > 32 ? __shfl_sync(kFullMask, v[1], b & 31u) : 0.f;
        return b < 32 ? x : y;
    };
    for (int32_t d0 = (int32_t)warp * 32; d0 <= last; d0 += (int32_t)warps * 32) {
        const int32_t d = d0 + (int32_t)lane;
        uint32_t b = 0;
#pragma unroll 8
        for (uint32_t k = 1; k < n; ++k) b += p.b.start[k] <= d ? 1u : 0u;
        const float x = value(b), y = value(p.b.two_sided ? b + n : 0u);
        if (d <= last) {
            if (d > 0) lut[off + d] = y;
            lut[off - d] = x;
        }
    }
    const float x = value(n - 1), y = value(p.b.two_sided ? 2 * n - 1 : 0u);
    for (int32_t i = last + 1 + (int32_t)(warp * 32 + lane); i <= off; i += (int32_t)warps * 32) {
        lut[off - i] = x;
        lut[off + i] = y;
    }
}

// Which of `rows` <= 64 positions from `at` on are words: a bit each in two words, the same in every lane of the warp.
__device__ __forceinline__ void word_bits(const AttendParams &p, int64_t at, uint32_t rows, uint32_t lane, uint32_t (&vis)[2])
{
    int2 sp[2];
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        const int64_t j = at + w * 32 + lane;
        sp[w] = w * 32u + lane < rows && j < p.n ? word_span(p, j) : make_int2(0, 0);
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) vis[w] = __ballot_sync(kFullMask, sp[w].y > sp[w].x);
}

// Rows of a tile that are not words are zeroed once it has landed (by one warp): their weights are zero, but what
// they hold may not be finite.  A row is NB blocks of 128 bytes, `block` bytes apart.
template <int NB>
__device__ __forceinline__ void zero_rows(uint32_t tile, uint32_t block, uint32_t rows, const uint32_t (&vis)[2], uint32_t lane)
{
#pragma unroll
    for (int w = 0; w < 2; ++w) {
        uint32_t bad = ~vis[w] & (rows >= (w + 1) * 32u ? 0xFFFFFFFFu : rows > w * 32u ? (1u << (rows - w * 32u)) - 1u : 0u);
        while (bad) {
            const uint32_t r = w * 32u + (uint32_t)__ffs(bad) - 1u;
            bad &= bad - 1u;
            if (lane < NB * 8u)
                asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(tile + (lane >> 3) * block + r * 128u + (lane & 7u) * 16u), "r"(0u) : "memory");
        }
    }
}

// ---- rows that came out not finite, once more ----
// The tensor cores multiply a masked weight, zero, with whatever lies there, and zero times an infinity or NaN is NaN: a
// value that is not finite spoils the rows of its tile, also of other sentences.  A row of finite inputs that fit is
// finite, so that a look at what leaves the kernel finds these; a warp forms each again from the pairs it sees alone.

// A row's softmax sum is known from lse.  Scores so far from zero that lse does not hold the sum's digits (beyond 1,024 in
// base-2 units it is off by 2^-14, at 2^30 by 64) make a far row: the backward pass adds up its weights and takes the rest off.
constexpr float kFarLse = 1024.f;
__device__ __forceinline__ bool far_row(float lse) { return fabsf(lse) > kFarLse && fabsf(lse) < INFINITY; }

// A pair's bias in base-2 units.
__device__ __forceinline__ float pair_bias(const AttendParams &p, uint32_t h, int32_t rel)
{
    return p.b.n ? log2_bias(__ldg(p.bias + (size_t)bucket_of(p.b, rel) * p.heads + h)) : 0.f;
}

__device__ __forceinline__ bool is_word(const AttendParams &p, int64_t i)
{
    const int2 sp = word_span(p, i);
    return sp.y > sp.x;
}

template <typename T>
__device__ __forceinline__ float row_dot(const T *a, const T *b, uint32_t dim)
{
    float x = 0.f;
#pragma unroll 1
    for (uint32_t c = 0; c < dim; c += 8) {
        const Pack<T, 8> u = load_pack<T, 8>(a + c), w = load_pack<T, 8>(b + c);
#pragma unroll
        for (int e = 0; e < 8; ++e) x = fmaf(to_f32(u.e[e]), to_f32(w.e[e]), x);
    }
    return x;
}

// acc += the lanes' weights times the lanes' rows, for the lanes in `live`; a lane holds columns lane, lane + 32, ...
template <typename T>
__device__ __forceinline__ void add_rows(float (&acc)[4], float w, uint32_t live, const T *rows, uint64_t ld, uint32_t dim, uint32_t lane)
{
#pragma unroll 1
    while (live) {
        const uint32_t e = (uint32_t)__ffs(live) - 1u;
        live &= live - 1u;
        const float by = __shfl_sync(kFullMask, w, e);
#pragma unroll
        for (int x = 0; x < 4; ++x)
            if (lane + 32u * x < dim) acc[x] = fmaf(by, to_f32(rows[e * ld + lane + 32u * x]), acc[x]);
    }
}

// Nothing finite is left to be found: more pairs change no column.
__device__ __forceinline__ bool all_nan(const float (&acc)[4], uint32_t dim, uint32_t lane)
{
    bool nan = true;
#pragma unroll
    for (int x = 0; x < 4; ++x) nan = nan && (lane + 32u * x >= dim || acc[x] != acc[x]);
    return __all_sync(kFullMask, nan);
}

// A barrier of 64 threads that says whether any of them found something.
__device__ __forceinline__ bool any_of_64(uint32_t barrier, bool found)
{
    uint32_t any;
    asm volatile("{ .reg .pred p, q; setp.ne.u32 p, %2, 0; barrier.cta.red.or.pred q, %1, 64, p; selp.u32 %0, 1, 0, q; }"
                 : "=r"(any) : "r"(barrier), "r"((uint32_t)found) : "memory");
    return any;
}

// Rows of `chunks` 16-byte chunks from a stripe of shared memory (chunk c of row r at chunk (c + r) mod chunks) to
// global memory, by `threads` threads of which this is number `at`.
__device__ __forceinline__ void store_rows(char *out, uint64_t ld_bytes, const unsigned char *stripe, uint32_t chunks, int32_t rows,
                                           uint32_t at, uint32_t threads)
{
    const uint32_t inv = (65536u + chunks - 1) / chunks;             // exact for the up to 512 chunks of 32 rows
    for (int32_t e = (int32_t)at; e < rows * (int32_t)chunks; e += (int32_t)threads) {
        const uint32_t r = ((uint32_t)e * inv) >> 16, c = (uint32_t)e - r * chunks;
        const uint32_t turned = c + r - ((r * inv) >> 16) * chunks;  // c + r mod chunks
        *reinterpret_cast<uint4 *>(out + (uint64_t)r * ld_bytes + c * 16u) =
            *reinterpret_cast<const uint4 *>(stripe + (r * chunks + (turned >= chunks ? turned - chunks : turned)) * 16u);
    }
}

}  // namespace w2v
