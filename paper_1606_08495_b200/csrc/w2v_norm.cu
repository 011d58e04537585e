// Layer norm of rows: y = (x - mean) rstd gamma + beta, statistics in fp32 from a row that stays in
// registers (the mean first, then the centred squares: no cancellation).  Bound by memory: x is read
// once and y written once.  A lane has the same columns of every row of its group, so gamma and beta stay in its
// registers too (read from L1 for every row they took more L1 time than the rows themselves), and the next row is
// under way while one is worked on.
#include "w2v_norm.cuh"

namespace w2v {

template <typename TX, typename TY, int E, int NV>
__global__ void __launch_bounds__(512)
norm_kernel(NormParams p, uint32_t gw, uint32_t groups)
{
    __shared__ float slot[64];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t group = warp / gw, wig = warp - group * gw, gl = wig * 32 + lane;
    const TX *x = static_cast<const TX *>(p.x);
    TY *y = static_cast<TY *>(p.y);
    const float inv_d = 1.0f / (float)p.d;
    const uint64_t step = (uint64_t)gridDim.x * groups;
    uint64_t r = (uint64_t)blockIdx.x * groups + group;
    Pack<TX, E> next[NV];
    if (r < p.rows) norm_row_load<TX, E, NV>(next, x + r * p.ldx, gl, gw, p.d);
    float gamma[NV * E], beta[NV * E];
    norm_weights_load<E, NV>(gamma, p.gamma, gl, gw, p.d);
    norm_weights_load<E, NV>(beta, p.beta, gl, gw, p.d);
    uint32_t flip = 0;
    for (; r < p.rows; r += step) {
        float v[NV * E];
        float s[1] = {0.f};
#pragma unroll
        for (int c = 0; c < NV; ++c)
#pragma unroll
            for (int e = 0; e < E; ++e) {
                v[c * E + e] = to_f32(next[c].e[e]);
                s[0] += v[c * E + e];
            }
        if (r + step < p.rows) norm_row_load<TX, E, NV>(next, x + (r + step) * p.ldx, gl, gw, p.d);
        group_sum<1>(s, gw, wig, group, lane, slot, flip);
        const float mean = s[0] * inv_d;
        flip ^= 1u;
        float q[1] = {0.f};
#pragma unroll
        for (int c = 0; c < NV; ++c)
            if ((gl + c * 32u * gw) * E < p.d) {
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    v[c * E + e] -= mean;
                    q[0] = fmaf(v[c * E + e], v[c * E + e], q[0]);
                }
            }
        group_sum<1>(q, gw, wig, group, lane, slot, flip);
        const float var = q[0] * inv_d;
        flip ^= 1u;
        const float rstd = rsqrtf(var + p.eps);              // 2 units in the last place
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
                for (int e = 0; e < E; ++e) t.e[e] = from_f32<TY>(fmaf(v[c * E + e] * rstd, gamma[c * E + e], beta[c * E + e]));
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
    const uint64_t want = (p.rows + sh.groups - 1) / sh.groups, most = (uint64_t)sms * (1024u / threads);
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
