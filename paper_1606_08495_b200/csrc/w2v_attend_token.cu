// Attention of one new token per sequence over a ring cache: the first `sinks` positions keep their
// places, every later position p lies at place sinks + (p - sinks) mod (places - sinks).  The call
// writes the new key and value into their place and attends over the positions that the window and
// the sinks leave visible, the new one included.
//
// Bound by reading the cache once.  A block takes one key/value head of one sequence (up to 16 of the query heads
// that share it) and a part of the visible positions; the parts of one head are the blocks of a
// cluster, which join their running maxima, sums and outputs through distributed shared memory: one
// launch, a fixed order of additions.
//
// A warp takes 16 keys a step and lets the matrix units form the products (query heads as the 16 rows): on the
// other units the products, conversions and lane sums of four heads took 21 instructions per cache element, against
// the three that the copy rate leaves time for.  Which dimension lands in which k (and which column) is free as long
// as both sides agree, so that keys and values go from global memory to the operand registers in accesses of 16 bytes:
//   scores:  lane (g, t) holds chunk 4 j + t (8 dimensions) of key g, the same of query head g;
//   output:  lane (g, t) holds chunk g of keys 2t, 2t + 1, 2t + 8, 2t + 9; a byte permutation pairs the keys, and
//            column g of product e is dimension 8 g + e.
// The softmax weights enter the second product as the sum of two numbers of the cache's type, so that what is lost is at most
// 2^-16 (bf16) and not 2^-8 of them; fp16 weights are 2^15 times as large, so that one below 2^-25 of the largest is not zero beside
// the sum, in which it counts.  Each warp copies its next step's keys and values to shared memory in the background, so
// that what is under way does not have to fit in registers.  There chunk c of row r lies at c ^ turn(r), which keeps
// both ways of reading free of bank conflicts.  96 sequences, 16 heads of 128 over 4 of keys and values, windows of 4,096: 150 us,
// 4.8 TB/s = 0.75 of measured copy; with direct loads 236 us, with copies but an address per access 191 us.  A single sequence of
// 5 heads of 64 and windows of 1,001 takes 6 us.
#include <cooperative_groups.h>
#include <type_traits>

#include "w2v_attend.cuh"
#include "w2v_kernel_ready.h"

namespace cg = cooperative_groups;

namespace w2v {

constexpr int kTokWarps = 4, kTokThreads = kTokWarps * 32, kTokRows = 16;
constexpr int kTokStages = 2;                    // steps of 16 keys and values per warp

// Eight lanes read 16 bytes at once: keys in rows 2 i and 2 i + 1, chunks t = 0..3; values in rows 2 t (or 2 t + 1),
// chunks 2 i and 2 i + 1.
__device__ __forceinline__ uint32_t turn(uint32_t row) { return (row & 6u) ^ ((row & 1u) << 2); }

template <typename T>
__device__ __forceinline__ void mma_token(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1);
template <>
__device__ __forceinline__ void mma_token<__nv_bfloat16>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
template <>
__device__ __forceinline__ void mma_token<__half>(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// A weight pair as the sum of two pairs of T.
template <typename T>
__device__ __forceinline__ void split_pair(float a, float b, uint32_t &head, uint32_t &tail)
{
    const T ha = from_f32<T>(a), hb = from_f32<T>(b);
    head = pack2<T>(a, b);
    tail = pack2<T>(a - to_f32(ha), b - to_f32(hb));
}

// NB = 64-column blocks of a head; HI: more than 8 query heads share the key/value head.
template <typename T, int NB, bool HI>
__global__ void __launch_bounds__(kTokThreads, NB == 1 ? 4 : 3)
attend_token_kernel(TokenParams p, uint32_t splits, uint32_t passes)
{
    extern __shared__ __align__(128) unsigned char token_smem[];        // the warps' stages, then what is joined
    float *sm = reinterpret_cast<float *>(token_smem + kTokWarps * kTokStages * 2 * 16 * NB * 128);
    constexpr int kR = HI ? 2 : 1;                                      // rows g and g + 8 of a lane
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const uint32_t group = p.heads / p.kv_heads, chunks = p.dim >> 3;
    const uint32_t split = blockIdx.x % splits, item = blockIdx.x / splits;
    const uint32_t pass = item % passes, kvh = (item / passes) % p.kv_heads, b = item / (passes * p.kv_heads);
    const uint32_t h0 = kvh * group + pass * kTokRows, nh = min((uint32_t)kTokRows, group - pass * kTokRows);
    constexpr float kLift = std::is_same<T, __half>::value ? 15.f : 0.f;               // of the weights, base 2
    constexpr uint32_t kKeep = 8 * kR;                                  // rows of a block's results
    float *bias_s = sm;                                                 // [rows][reach + 1] bias by distance
    // what is joined lies where the stages were
    float *stat = reinterpret_cast<float *>(token_smem);                // [rows][2] maximum and sum of this block
    float *acc_s = stat + 2 * kKeep;                                    // [rows][dim] output of this block
    float *wstat = acc_s + kKeep * p.dim;                               // [warps][rows][2]
    float *wacc = wstat + kTokWarps * kKeep * 2;                        // [warps][rows][dim]
    constexpr uint32_t kRow = NB * 128, kHalf = 16 * kRow, kStage = 2 * kHalf;           // bytes: a row, 16 keys, a step
    const int32_t pos = p.pos[b];
    const int32_t reach = p.b.n ? p.b.start[p.b.n - 1] : 0;             // from here on one bucket
    if (p.b.n)
        for (uint32_t i = tid; i < (uint32_t)(reach + 1) * nh; i += kTokThreads) {
            const uint32_t r = i / (uint32_t)(reach + 1), dist = i - r * (uint32_t)(reach + 1);
            bias_s[i] = log2_bias(__ldg(p.bias + (size_t)bucket_of(p.b, -(int32_t)dist) * p.heads + h0 + r));
        }
    __syncthreads();
    float acc[NB * 8][4], mx[kR], sum[kR];
#pragma unroll
    for (int i = 0; i < NB * 8; ++i) acc[i][0] = acc[i][1] = acc[i][2] = acc[i][3] = 0.f;
#pragma unroll
    for (int r = 0; r < kR; ++r) { mx[r] = -INFINITY; sum[r] = 0.f; }
    if (pos >= 0) {
        uint4 q[kR][NB * 2];                                            // chunk 4 j + t of query heads g and g + 8
#pragma unroll
        for (int r = 0; r < kR; ++r)
#pragma unroll
            for (int j = 0; j < NB * 2; ++j) {
                const uint32_t c = 4 * j + t;
                q[r][j] = g + 8 * r < nh && c < chunks ? __ldg(reinterpret_cast<const uint4 *>(static_cast<const T *>(p.q) + ((size_t)b * p.heads + h0 + g + 8 * r) * p.dim) + c)
                                                       : make_uint4(0, 0, 0, 0);
            }
        const int32_t win = pos > p.left ? pos - p.left : 0;            // first position of the window
        const int32_t ns = min(p.sinks, win);                           // sinks before it
        const int32_t total = pos - win + 1 + ns;                       // visible positions, numbered sinks first
        const int32_t t0 = (int32_t)((int64_t)total * split / splits), t1 = (int32_t)((int64_t)total * (split + 1) / splits);
        const uint32_t ring = (uint32_t)(p.places - (uint64_t)p.sinks);
        // place of visible position number ns: the window lies in the ring with one wrap at most
        const int64_t place0 = win < p.sinks ? win : p.sinks + (int64_t)((uint32_t)(win - p.sinks) % ring);
        const size_t row = (size_t)p.kv_heads * p.dim;
        T *ck = static_cast<T *>(p.ck) + (size_t)b * p.places * row + (size_t)kvh * p.dim, *cv = static_cast<T *>(p.cv) + (size_t)b * p.places * row + (size_t)kvh * p.dim;
        const T *nk = static_cast<const T *>(p.k) + ((size_t)b * p.kv_heads + kvh) * p.dim, *nv = static_cast<const T *>(p.v) + ((size_t)b * p.kv_heads + kvh) * p.dim;
        if (t1 == total && pass == 0 && t0 < t1 && tid < 2 * chunks) {  // the part that ends with the new token stores it; nobody reads its place
            const int64_t at = pos < p.sinks ? pos : p.sinks + (int64_t)((uint32_t)(pos - p.sinks) % ring);
            const bool value = tid >= chunks;
            const uint32_t c = value ? tid - chunks : tid;
            reinterpret_cast<uint4 *>((value ? cv : ck) + (size_t)at * row)[c] = __ldg(reinterpret_cast<const uint4 *>(value ? nv : nk) + c);
        }
        // 16 keys and values from visible position number x0 on to a stage; zeros past the part's end
        const uint32_t stages = smem_addr(token_smem) + warp * (kTokStages * kStage);
        constexpr uint32_t kLanes = NB * 8, kAtOnce = 32 / kLanes;       // lanes per row, rows per request
        const uint32_t lane_row = lane / kLanes, lane_chunk = lane % kLanes;
        const bool inside = lane_chunk < chunks;
        const uint32_t row_bytes = (uint32_t)row * 2u;
        const char *kb = reinterpret_cast<const char *>(ck) + lane_chunk * 16u, *vb = reinterpret_cast<const char *>(cv) + lane_chunk * 16u;
        const uint32_t shift = (uint32_t)place0 - (uint32_t)ns, places = (uint32_t)p.places;
        auto copy_step = [&](int32_t x0, uint32_t stage) {
            const uint32_t to = stages + stage * kStage + lane_row * kRow;
            // all but the steps with a sink, the new token or the part's end in them: places in a row, but for the wrap
            const bool even = x0 >= ns && x0 + 16 < total && x0 + 16 <= t1;
#pragma unroll
            for (uint32_t i = 0; i < 16 / kAtOnce; ++i) {
                const uint32_t r = i * kAtOnce + lane_row, dst = to + i * kAtOnce * kRow + ((lane_chunk ^ turn(r)) << 4);
                const int32_t x = x0 + (int32_t)r;
                uint32_t at = (uint32_t)x + shift;
                if (at >= places) at -= ring;
                if (even) {
                    const uint64_t off = (uint64_t)at * row_bytes;
                    copy16(dst, kb + off, inside);
                    copy16(dst + kHalf, vb + off, inside);
                } else {
                    if (x < ns) at = (uint32_t)x;
                    const bool real = inside && x < t1, fresh = x >= total - 1;
                    const uint64_t off = real && !fresh ? (uint64_t)at * row_bytes : 0u;
                    copy16(dst, fresh ? reinterpret_cast<const char *>(nk) + lane_chunk * 16u : kb + off, real);
                    copy16(dst + kHalf, fresh ? reinterpret_cast<const char *>(nv) + lane_chunk * 16u : vb + off, real);
                }
            }
            copy_commit();
        };
        const int32_t first = t0 + (int32_t)warp * 16;
        if (first < t1) copy_step(first, 0);
        uint32_t stage = 0;
        for (int32_t x0 = first; x0 < t1; x0 += kTokWarps * 16, stage ^= 1u) {
            if (x0 + kTokWarps * 16 < t1) {
                copy_step(x0 + kTokWarps * 16, stage ^ 1u);
                copy_wait<1>();
            } else {
                copy_wait<0>();
            }
            __syncwarp();
            const unsigned char *keys = token_smem + warp * (kTokStages * kStage) + stage * kStage, *vals = keys + kHalf;
            uint4 key[2][NB * 2];
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < NB * 2; ++j) {
                    const uint32_t r = i * 8 + g;
                    key[i][j] = *reinterpret_cast<const uint4 *>(keys + r * kRow + (((4 * j + t) ^ turn(r)) << 4));
                }
            float sc[2][4];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                sc[i][0] = sc[i][1] = sc[i][2] = sc[i][3] = 0.f;
#pragma unroll
                for (int j = 0; j < NB * 2; ++j) {
                    mma_token<T>(sc[i], q[0][j].x, HI ? q[kR - 1][j].x : 0u, q[0][j].y, HI ? q[kR - 1][j].y : 0u, key[i][j].x, key[i][j].y);
                    mma_token<T>(sc[i], q[0][j].z, HI ? q[kR - 1][j].z : 0u, q[0][j].w, HI ? q[kR - 1][j].w : 0u, key[i][j].z, key[i][j].w);
                }
            }
            uint32_t head[2][kR], tail[2][kR];
#pragma unroll
            for (int r = 0; r < kR; ++r) {
                float s[4], top = mx[r];
                const float *near = bias_s + min(g + 8 * r, nh - 1) * (uint32_t)(reach + 1);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int32_t x = x0 + (i >> 1) * 8 + 2 * (int32_t)t + (i & 1);
                    s[i] = sc[i >> 1][2 * r + (i & 1)] * (p.scale * kLog2e);
                    if (p.b.n) s[i] += near[x < ns ? min(pos - x, reach) : min(max(total - 1 - x, 0), reach)];
                    if (x >= t1) s[i] = -INFINITY;
                    top = fmaxf(top, s[i]);
                }
                top = fmaxf(top, __shfl_xor_sync(kFullMask, top, 1));
                top = fmaxf(top, __shfl_xor_sync(kFullMask, top, 2));
                const float from = top == -INFINITY ? 0.f : top;
                if (__any_sync(kFullMask, top > mx[r])) {
                    const float keep = fast_exp2(mx[r] - from);         // 0 for the first keys
                    sum[r] *= keep;
#pragma unroll
                    for (int i = 0; i < NB * 8; ++i) { acc[i][2 * r] *= keep; acc[i][2 * r + 1] *= keep; }
                    mx[r] = top;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) { s[i] = fast_exp2(s[i] - (from - kLift)); sum[r] += s[i]; }
                split_pair<T>(s[0], s[1], head[0][r], tail[0][r]);
                split_pair<T>(s[2], s[3], head[1][r], tail[1][r]);
            }
#pragma unroll
            for (int n = 0; n < NB; ++n) {
                uint4 val[4];                                           // chunk g + 8 n of keys 2t, 2t + 1, 2t + 8, 2t + 9
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const uint32_t r = (i >> 1) * 8 + 2 * t + (i & 1);
                    val[i] = *reinterpret_cast<const uint4 *>(vals + r * kRow + (((g + 8 * n) ^ turn(r)) << 4));
                }
                const uint32_t *v0 = reinterpret_cast<const uint32_t *>(&val[0]), *v1 = reinterpret_cast<const uint32_t *>(&val[1]);
                const uint32_t *v2 = reinterpret_cast<const uint32_t *>(&val[2]), *v3 = reinterpret_cast<const uint32_t *>(&val[3]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const uint32_t pick = e & 1 ? 0x7632u : 0x5410u;    // dimension e of two keys in one register
                    const uint32_t b0 = __byte_perm(v0[e >> 1], v1[e >> 1], pick), b1 = __byte_perm(v2[e >> 1], v3[e >> 1], pick);
                    mma_token<T>(acc[n * 8 + e], tail[0][0], HI ? tail[0][kR - 1] : 0u, tail[1][0], HI ? tail[1][kR - 1] : 0u, b0, b1);
                    mma_token<T>(acc[n * 8 + e], head[0][0], HI ? head[0][kR - 1] : 0u, head[1][0], HI ? head[1][kR - 1] : 0u, b0, b1);
                }
            }
            __syncwarp();                                               // the stage may be filled again
        }
    }
    __syncthreads();                                                    // every warp is done with its stages
    // join the warps; a lane has columns 2t, 2t + 1 of every product: dimensions 64 n + 8 (2t) + e and 64 n + 8 (2t + 1) + e
#pragma unroll
    for (int r = 0; r < kR; ++r) {
        sum[r] += __shfl_xor_sync(kFullMask, sum[r], 1);
        sum[r] += __shfl_xor_sync(kFullMask, sum[r], 2);
        const uint32_t at = warp * kKeep + g + 8 * r;
        if (t == 0) { wstat[at * 2] = mx[r]; wstat[at * 2 + 1] = sum[r]; }
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const uint32_t d = 64 * n + 8 * (2 * t + c);
                if (d < p.dim) {
                    float4 *o = reinterpret_cast<float4 *>(wacc + at * p.dim + d);
                    o[0] = make_float4(acc[n * 8][2 * r + c], acc[n * 8 + 1][2 * r + c], acc[n * 8 + 2][2 * r + c], acc[n * 8 + 3][2 * r + c]);
                    o[1] = make_float4(acc[n * 8 + 4][2 * r + c], acc[n * 8 + 5][2 * r + c], acc[n * 8 + 6][2 * r + c], acc[n * 8 + 7][2 * r + c]);
                }
            }
    }
    __syncthreads();
    for (uint32_t i = tid; i < nh * p.dim; i += kTokThreads) {
        const uint32_t r = i / p.dim, c = i - r * p.dim;
        float top = -INFINITY, s = 0.f, a = 0.f;
#pragma unroll
        for (int w = 0; w < kTokWarps; ++w) top = fmaxf(top, wstat[(w * kKeep + r) * 2]);
        const float from = top == -INFINITY ? 0.f : top;                // no finite score: the sums are zeros, or NaN, which stays
#pragma unroll
        for (int w = 0; w < kTokWarps; ++w) {
            const float f = fast_exp2(wstat[(w * kKeep + r) * 2] - from);
            s = fmaf(f, wstat[(w * kKeep + r) * 2 + 1], s);
            a = fmaf(f, wacc[(w * kKeep + r) * p.dim + c], a);
        }
        acc_s[i] = a;
        if (c == 0) { stat[2 * r] = top; stat[2 * r + 1] = s; }
    }
    // join the blocks of the cluster: each writes a share of the outputs
    cg::cluster_group cluster = cg::this_cluster();
    if (splits > 1) cluster.sync(); else __syncthreads();
    T *out = static_cast<T *>(p.out) + ((size_t)b * p.heads + h0) * p.dim;
    for (uint32_t i = split * kTokThreads + tid; i < nh * p.dim; i += splits * kTokThreads) {
        const uint32_t r = i / p.dim;
        float top = -INFINITY, s = 0.f, a = 0.f;
        for (uint32_t x = 0; x < splits; ++x) top = fmaxf(top, splits > 1 ? cluster.map_shared_rank(stat, x)[2 * r] : stat[2 * r]);
        const float from = top == -INFINITY ? 0.f : top;
        for (uint32_t x = 0; x < splits; ++x) {
            const float *st = splits > 1 ? cluster.map_shared_rank(stat, x) : stat;
            const float *ac = splits > 1 ? cluster.map_shared_rank(acc_s, x) : acc_s;
            const float f = fast_exp2(st[2 * r] - from);
            s = fmaf(f, st[2 * r + 1], s);
            a = fmaf(f, ac[i], a);
        }
        out[i] = from_f32<T>(s == 0.f ? 0.f : a / s);                   // a sum that is NaN is not an empty row
    }
    if (splits > 1) cluster.sync();                                     // nobody leaves while its memory is read
}

template <typename T, int NB, bool HI>
int launch_token_shape(const TokenParams &p, int sms, cudaStream_t s)
{
    const uint32_t group = p.heads / p.kv_heads, passes = (group + kTokRows - 1) / kTokRows;
    const uint64_t items = (uint64_t)p.batch * p.kv_heads * passes;
    // parts of a head: enough blocks for several on every SM, as long as a part keeps some 64 keys (one step of its
    // warps) when blocks are few, 512 when there are plenty
    const uint64_t keys = (uint64_t)p.left + 1 + (uint64_t)p.sinks;
    uint32_t splits = 1;
    while (splits < 8 && keys / (2 * splits) >= (items * splits < 2ull * (uint64_t)sms ? 64u : 512u) && items * splits < 8ull * (uint64_t)sms) splits *= 2;
    const uint32_t reach = p.b.n ? (uint32_t)p.b.start[p.b.n - 1] + 1 : 0;
    const size_t smem = (size_t)kTokWarps * kTokStages * 2 * 16 * NB * 128 + sizeof(float) * (size_t)reach * (group < kTokRows ? group : kTokRows);
    static_assert((size_t)kTokWarps * kTokStages * 2 * 16 * NB * 128 >= sizeof(float) * (HI ? 16 : 8) * (2 + NB * 64) * (kTokWarps + 1), "joined where the stages were");
    auto kernel = attend_token_kernel<T, NB, HI>;
    if (smem > 48 * 1024 && !kernel_ready<attend_token_kernel<T, NB, HI>>()) return -1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((uint32_t)(items * splits));
    cfg.blockDim = dim3(kTokThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cudaLaunchAttribute at[1];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = splits;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = splits > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, kernel, p, splits, passes) == cudaSuccess ? 1 : -1;
}

template <typename T>
int launch_token_typed(const TokenParams &p, int sms, cudaStream_t s)
{
    const bool hi = p.heads / p.kv_heads > 8;
    if (p.dim <= 64) return hi ? launch_token_shape<T, 1, true>(p, sms, s) : launch_token_shape<T, 1, false>(p, sms, s);
    return hi ? launch_token_shape<T, 2, true>(p, sms, s) : launch_token_shape<T, 2, false>(p, sms, s);
}

int launch_attend_token(const TokenParams &p, uint32_t type, int sms, cudaStream_t s)
{
    if (p.batch == 0) return 0;
    return type == kBF16 ? launch_token_typed<__nv_bfloat16>(p, sms, s) : launch_token_typed<__half>(p, sms, s);
}

}  // namespace w2v
