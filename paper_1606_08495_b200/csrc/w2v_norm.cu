// Layer norm of rows: y = (x - mean) rstd gamma + beta, statistics in fp32 from a row that stays in
// registers (the mean first, then the centred squares: no cancellation).  Bound by memory: x is read
// once and y written once.
#include "w2v_norm.cuh"

namespace w2v {

template <typename TX, typename TY, int E, int NV>
__global__ void __launch_bounds__(512)
norm_kernel(NormParams p, uint32_t gw, uint32_t groups)
{
    __shared__ float2 slot[64];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t group = warp / gw, wig = warp - group * gw, gl = wig * 32 + lane;
    const TX *x = static_cast<const TX *>(p.x);
    TY *y = static_cast<TY *>(p.y);
    const float inv_d = 1.0f / (float)p.d;
    uint32_t flip = 0;
    for (uint64_t r = (uint64_t)blockIdx.x * groups + group; r < p.rows; r += (uint64_t)gridDim.x * groups) {
        float v[NV * E];
        float s = 0.f;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const uint32_t at = (gl + c * 32u * gw) * E;
            if (at < p.d) {
                const Pack<TX, E> t = load_pack<TX, E>(x + r * p.ldx + at);
#pragma unroll
                for (int e = 0; e < E; ++e) v[c * E + e] = to_f32(t.e[e]);
            } else {
#pragma unroll
                for (int e = 0; e < E; ++e) v[c * E + e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < E; ++e) s += v[c * E + e];
        }
        const float mean = group_sum2(s, 0.f, gw, wig, group, lane, slot, flip).x * inv_d;
        flip ^= 1u;
        float q = 0.f;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const uint32_t at = (gl + c * 32u * gw) * E;
            if (at < p.d) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    v[c * E + e] -= mean;
                    q = fmaf(v[c * E + e], v[c * E + e], q);
                }
            }
        }
        const float var = group_sum2(q, 0.f, gw, wig, group, lane, slot, flip).x * inv_d;
        flip ^= 1u;
        const float rstd = 1.0f / sqrtf(var + p.eps);
        if (gl == 0) {
            if (p.mean) p.mean[r] = mean;
            if (p.rstd) p.rstd[r] = rstd;
        }
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const uint32_t at = (gl + c * 32u * gw) * E;
            if (at < p.d) {
                Pack<TY, E> t;
#pragma unroll
                for (int e = 0; e < E; ++e)
                    t.e[e] = from_f32<TY>(fmaf(v[c * E + e] * rstd, __ldg(p.gamma + at + e), __ldg(p.beta + at + e)));
                store_pack<TY, E>(y + r * p.ldy + at, t);
            }
        }
    }
}

template <typename TX, typename TY>
int launch_norm_typed(const NormParams &p, int sms, cudaStream_t s)
{
    uint32_t e = widest_access(p.d, sizeof(TX), p.ldx, p.x, 16u / sizeof(TX));
    e = widest_access(p.d, sizeof(TY), p.ldy, p.y, e);
    const NormShape sh = norm_shape(p.d, e);
    const uint32_t threads = sh.gw * sh.groups * 32;
    const uint64_t want = (p.rows + sh.groups - 1) / sh.groups, most = (uint64_t)sms * (2048u / threads);
    const uint32_t grid = (uint32_t)(want < most ? want : most);
#define W2V_NORM(E, NV) norm_kernel<TX, TY, E, NV><<<grid, threads, 0, s>>>(p, sh.gw, sh.groups)
    if constexpr (sizeof(TX) == 2) {
        if (sh.e == 8) {
            if (sh.nv <= 1) W2V_NORM(8, 1); else W2V_NORM(8, 2);
            return cudaPeekAtLastError() == cudaSuccess ? 1 : -1;
        }
    }
    if (sh.e == 4) {
        if (sh.nv <= 1) W2V_NORM(4, 1); else if (sh.nv == 2) W2V_NORM(4, 2); else if (sh.nv == 3) W2V_NORM(4, 3); else W2V_NORM(4, 4);
    } else {
        if (sh.nv <= 4) W2V_NORM(1, 4); else W2V_NORM(1, 16);
    }
#undef W2V_NORM
    return cudaPeekAtLastError() == cudaSuccess ? 1 : -1;
}

int launch_norm(const NormParams &p, uint32_t xt, uint32_t yt, int sms, cudaStream_t s)
{
    if (p.rows == 0) return 0;
    if (xt == kBF16) return launch_norm_typed<__nv_bfloat16, __nv_bfloat16>(p, sms, s);
    if (xt == kF16) return launch_norm_typed<__half, __half>(p, sms, s);
    if (yt == kBF16) return launch_norm_typed<float, __nv_bfloat16>(p, sms, s);
    if (yt == kF16) return launch_norm_typed<float, __half>(p, sms, s);
    return launch_norm_typed<float, float>(p, sms, s);
}

}  // namespace w2v
