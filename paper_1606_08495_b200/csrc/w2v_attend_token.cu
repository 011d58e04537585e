// Attention of one new token per sequence over a ring cache: the first `sinks` positions keep their
// places, every later position p lies at place sinks + (p - sinks) mod (places - sinks).  The call
// writes the new key and value into their place and attends over the positions that the window and
// the sinks leave visible, the new one included.
//
// Bound by reading the cache once.  A block takes one key/value head of one sequence (all query heads
// that share it) and a part of the visible positions; the parts of one head are the blocks of a
// cluster, which join their running maxima, sums and outputs through distributed shared memory: one
// launch, a fixed order of additions.  Inside a block a key is read by LPK lanes, 16 bytes each, and
// every LPK lanes run over keys of their own in steps of kTokU (that many keys and values in flight
// per lane before the first is used).
#include <cooperative_groups.h>

#include "w2v_device.cuh"
#include "w2v_reader.h"
#include "w2v_types.cuh"

namespace cg = cooperative_groups;

namespace w2v {

constexpr int kTokThreads = 256;
constexpr int kTokU = 4;
constexpr float kLog2e = 1.4426950408889634f;

template <typename T, int LPK, int GC>
__global__ void __launch_bounds__(kTokThreads)
attend_token_kernel(TokenParams p, uint32_t splits, uint32_t passes)
{
    extern __shared__ float sm[];
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    constexpr int kWarps = kTokThreads / 32, kSub = 32 / LPK;          // keys a warp reads at once
    const uint32_t group = p.heads / p.kv_heads;
    const uint32_t split = blockIdx.x % splits, item = blockIdx.x / splits;
    const uint32_t pass = item % passes, kvh = (item / passes) % p.kv_heads, b = item / (passes * p.kv_heads);
    const uint32_t h0 = kvh * group + pass * GC, nh = min((uint32_t)GC, group - pass * GC);
    float *stat = sm;                                                   // [GC][2] maximum and sum of this block
    float *acc_s = stat + 2 * GC;                                       // [GC][dim] output of this block
    float *wstat = acc_s + GC * p.dim;                                  // [warps][GC][2]
    float *wacc = wstat + kWarps * GC * 2;                              // [warps][GC][dim]
    float *bias_s = wacc + kWarps * GC * p.dim;                         // [reach + 1][GC] bias by distance
    const int32_t pos = p.pos[b];
    const int32_t reach = p.b.n ? p.b.start[p.b.n - 1] : 0;             // from here on one bucket
    if (p.b.n) {
        for (uint32_t i = tid; i < (uint32_t)(reach + 1) * GC; i += kTokThreads) {
            const int32_t dist = (int32_t)(i / GC);
            const uint32_t g = i % GC;
            uint32_t lo = 0, hi = p.b.n - 1;                            // last bucket that starts at or before dist
            while (lo < hi) {
                const uint32_t mid = (lo + hi + 1) >> 1;
                if (p.b.start[mid] <= dist) lo = mid; else hi = mid - 1;
            }
            const float v = g < nh ? p.bias[(size_t)lo * p.heads + h0 + g] : 0.f;
            bias_s[i] = v == -INFINITY ? v : fmaxf(v, -1e30f) * kLog2e;   // the lowest float stays finite
        }
    }
    __syncthreads();
    const uint32_t li = lane % LPK, sub = warp * kSub + lane / LPK;
    const bool mine = li * 8 < p.dim;
    const T *q = static_cast<const T *>(p.q) + ((size_t)b * p.heads + h0) * p.dim + li * 8;
    float qf[GC][8], acc[GC][8], mx[GC], sum[GC];
#pragma unroll
    for (int g = 0; g < GC; ++g) {
        mx[g] = -INFINITY;
        sum[g] = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            acc[g][e] = 0.f;
            qf[g][e] = mine && (uint32_t)g < nh ? to_f32(q[(size_t)g * p.dim + e]) * (p.scale * kLog2e) : 0.f;
        }
    }
    if (pos >= 0) {
        const int32_t win = pos > p.left ? pos - p.left : 0;            // first position of the window
        const int32_t ns = min(p.sinks, win);                           // sinks before it
        const int64_t total = (int64_t)pos - win + 1 + ns;
        const int64_t t0 = total * split / splits, t1 = total * (split + 1) / splits;
        const uint64_t ring = p.places - (uint64_t)p.sinks;
        const size_t row = (size_t)p.kv_heads * p.dim;
        const size_t base = (size_t)b * p.places * row + (size_t)kvh * p.dim + li * 8;
        T *ck = static_cast<T *>(p.ck) + base, *cv = static_cast<T *>(p.cv) + base;
        const T *nk = static_cast<const T *>(p.k) + ((size_t)b * p.kv_heads + kvh) * p.dim + li * 8;
        const T *nv = static_cast<const T *>(p.v) + ((size_t)b * p.kv_heads + kvh) * p.dim + li * 8;
        constexpr int kStep = kWarps * kSub;                            // keys the block reads side by side
        for (int64_t t = t0 + sub; t - sub < t1; t += kStep * kTokU) {  // all lanes of a warp take part to the end
            Pack<T, 8> kk[kTokU], vv[kTokU];
            int32_t at[kTokU];
            int64_t place[kTokU];
#pragma unroll
            for (int u = 0; u < kTokU; ++u) {
                const int64_t tu = t + (int64_t)u * kStep;
                at[u] = -1;
                place[u] = 0;
                if (tu < t1) {
                    at[u] = tu < ns ? (int32_t)tu : (int32_t)(win + (tu - ns));
                    place[u] = at[u] < p.sinks ? at[u] : p.sinks + (int64_t)((uint32_t)(at[u] - p.sinks) % (uint32_t)ring);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) kk[u].e[e] = vv[u].e[e] = from_f32<T>(0.f);
                if (tu < t1 && mine) {
                    const bool fresh = at[u] == pos;
                    kk[u] = load_pack<T, 8>(fresh ? nk : ck + (size_t)place[u] * row);
                    vv[u] = load_pack<T, 8>(fresh ? nv : cv + (size_t)place[u] * row);
                }
            }
#pragma unroll
            for (int u = 0; u < kTokU; ++u)
                if (at[u] == pos && mine && pass == 0) {
                    store_pack<T, 8>(ck + (size_t)place[u] * row, kk[u]);
                    store_pack<T, 8>(cv + (size_t)place[u] * row, vv[u]);
                }
#pragma unroll
            for (int g = 0; g < GC; ++g) {
                float sc[kTokU], top = mx[g];
#pragma unroll
                for (int u = 0; u < kTokU; ++u) {
                    float s = 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) s = fmaf(qf[g][e], to_f32(kk[u].e[e]), s);
#pragma unroll
                    for (int o = LPK / 2; o > 0; o >>= 1) s += __shfl_xor_sync(kFullMask, s, o);
                    if (p.b.n) s += bias_s[(at[u] < 0 ? 0 : min(pos - at[u], reach)) * GC + g];
                    sc[u] = at[u] < 0 ? -INFINITY : s;
                    top = fmaxf(top, sc[u]);
                }
                const float keep = top == -INFINITY ? 1.f : exp2f(mx[g] - top);
                mx[g] = top;
                sum[g] *= keep;
#pragma unroll
                for (int e = 0; e < 8; ++e) acc[g][e] *= keep;
#pragma unroll
                for (int u = 0; u < kTokU; ++u) {
                    const float w = sc[u] == -INFINITY ? 0.f : exp2f(sc[u] - top);
                    sum[g] += w;
#pragma unroll
                    for (int e = 0; e < 8; ++e) acc[g][e] = fmaf(w, to_f32(vv[u].e[e]), acc[g][e]);
                }
            }
        }
    }
    // join the keys that the lanes of a warp ran over, then the warps
#pragma unroll
    for (int g = 0; g < GC; ++g) {
        float top = mx[g];
#pragma unroll
        for (int o = LPK; o < 32; o <<= 1) top = fmaxf(top, __shfl_xor_sync(kFullMask, top, o));
        const float keep = mx[g] == -INFINITY ? 0.f : exp2f(mx[g] - top);
        sum[g] *= keep;
#pragma unroll
        for (int o = LPK; o < 32; o <<= 1) sum[g] += __shfl_xor_sync(kFullMask, sum[g], o);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            acc[g][e] *= keep;
#pragma unroll
            for (int o = LPK; o < 32; o <<= 1) acc[g][e] += __shfl_xor_sync(kFullMask, acc[g][e], o);
        }
        if (lane < LPK) {
            if (li == 0) { wstat[(warp * GC + g) * 2] = top; wstat[(warp * GC + g) * 2 + 1] = sum[g]; }
            if (mine)
#pragma unroll
                for (int e = 0; e < 8; ++e) wacc[(warp * GC + g) * p.dim + li * 8 + e] = acc[g][e];
        }
    }
    __syncthreads();
    for (uint32_t i = tid; i < GC * p.dim; i += kTokThreads) {
        const uint32_t g = i / p.dim, c = i - g * p.dim;
        float top = -INFINITY, s = 0.f, a = 0.f;
        for (int w = 0; w < kWarps; ++w) top = fmaxf(top, wstat[(w * GC + g) * 2]);
        if (top != -INFINITY)
            for (int w = 0; w < kWarps; ++w) {
                const float m = wstat[(w * GC + g) * 2], f = m == -INFINITY ? 0.f : exp2f(m - top);
                s = fmaf(f, wstat[(w * GC + g) * 2 + 1], s);
                a = fmaf(f, wacc[(w * GC + g) * p.dim + c], a);
            }
        acc_s[i] = a;
        if (c == 0) { stat[2 * g] = top; stat[2 * g + 1] = s; }
    }
    // join the blocks of the cluster: each writes a share of the outputs
    cg::cluster_group cluster = cg::this_cluster();
    if (splits > 1) cluster.sync(); else __syncthreads();
    T *out = static_cast<T *>(p.out) + ((size_t)b * p.heads + h0) * p.dim;
    for (uint32_t i = split * kTokThreads + tid; i < nh * p.dim; i += splits * kTokThreads) {
        const uint32_t g = i / p.dim;
        float top = -INFINITY, s = 0.f, a = 0.f;
        for (uint32_t r = 0; r < splits; ++r) top = fmaxf(top, splits > 1 ? cluster.map_shared_rank(stat, r)[2 * g] : stat[2 * g]);
        if (top != -INFINITY)
            for (uint32_t r = 0; r < splits; ++r) {
                const float *st = splits > 1 ? cluster.map_shared_rank(stat, r) : stat;
                const float *ac = splits > 1 ? cluster.map_shared_rank(acc_s, r) : acc_s;
                const float f = st[2 * g] == -INFINITY ? 0.f : exp2f(st[2 * g] - top);
                s = fmaf(f, st[2 * g + 1], s);
                a = fmaf(f, ac[i], a);
            }
        out[i] = from_f32<T>(s > 0.f ? a / s : 0.f);
    }
    if (splits > 1) cluster.sync();                                     // nobody leaves while its memory is read
}

template <typename T, int LPK, int GC>
int launch_token_shape(const TokenParams &p, int sms, cudaStream_t s)
{
    const uint32_t group = p.heads / p.kv_heads, passes = (group + GC - 1) / GC;
    const uint64_t items = (uint64_t)p.batch * p.kv_heads * passes;
    // parts of a head: enough blocks for two on every SM, as long as a part keeps some 64 keys
    const uint64_t keys = (uint64_t)p.left + 1 + (uint64_t)p.sinks;
    uint32_t splits = 1;
    while (splits < 8 && items * splits < 2ull * (uint64_t)sms && keys / (2 * splits) >= 64) splits *= 2;
    const uint32_t reach = p.b.n ? (uint32_t)p.b.start[p.b.n - 1] + 1 : 0;
    const size_t smem = sizeof(float) * (2 * GC + (size_t)GC * p.dim + (kTokThreads / 32) * GC * (2 + (size_t)p.dim) + (size_t)reach * GC);
    auto kernel = attend_token_kernel<T, LPK, GC>;
    if (smem > 48 * 1024 && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) != cudaSuccess) return -1;
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

template <typename T, int LPK>
int launch_token_lanes(const TokenParams &p, int sms, cudaStream_t s)
{
    const uint32_t group = p.heads / p.kv_heads;
    if (group == 1) return launch_token_shape<T, LPK, 1>(p, sms, s);
    if (group == 2) return launch_token_shape<T, LPK, 2>(p, sms, s);
    if (group <= 4) return launch_token_shape<T, LPK, 4>(p, sms, s);
    return launch_token_shape<T, LPK, 8>(p, sms, s);
}

int launch_attend_token(const TokenParams &p, uint32_t type, int sms, cudaStream_t s)
{
    if (p.batch == 0) return 0;
    if (type == kBF16)
        return p.dim <= 32 ? launch_token_lanes<__nv_bfloat16, 4>(p, sms, s)
               : p.dim <= 64 ? launch_token_lanes<__nv_bfloat16, 8>(p, sms, s) : launch_token_lanes<__nv_bfloat16, 16>(p, sms, s);
    return p.dim <= 32 ? launch_token_lanes<__half, 4>(p, sms, s)
           : p.dim <= 64 ? launch_token_lanes<__half, 8>(p, sms, s) : launch_token_lanes<__half, 16>(p, sms, s);
}

}  // namespace w2v
