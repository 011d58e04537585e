// Layer norm backwards.  With xh = (x - mean) rstd and G = dy gamma,
//   dx = rstd (G - mean(G) - xh mean(G xh)),  dgamma = sum over rows of dy xh,  dbeta = sum of dy.
// Bound by memory: x and dy are read once, dx is written once.  A lane keeps the same columns of every
// row that its group handles, so the weights' gradients stay in its registers until the end; each block
// then writes one partial row and a second kernel adds the partials in a fixed order (no atomics: the
// same inputs give the same bits).
#include "w2v_norm.cuh"

namespace w2v {

template <typename TX, typename TY, int E, int NV>
__global__ void __launch_bounds__(512)
norm_backward_kernel(NormParams p, uint32_t gw, uint32_t groups)
{
    __shared__ float slot[128];
    extern __shared__ float sums[];                     // [groups - 1][2][d], only with more than one row per block
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t group = warp / gw, wig = warp - group * gw, gl = wig * 32 + lane;
    const TX *x = static_cast<const TX *>(p.x);
    const TY *dy = static_cast<const TY *>(p.dy);
    TX *dx = static_cast<TX *>(p.dx);
    const float inv_d = 1.0f / (float)p.d;
    const uint64_t step = (uint64_t)gridDim.x * groups;
    uint64_t r = (uint64_t)blockIdx.x * groups + group;
    // the next row's x, dy and statistics are under way while one row is worked on
    Pack<TX, E> xn[NV];
    Pack<TY, E> yn[NV];
    float mean_n = 0.f, rstd_n = 0.f;
    auto fetch = [&](uint64_t row) {
        norm_row_load<TX, E, NV>(xn, x + row * p.ldx, gl, gw, p.d);
        norm_row_load<TY, E, NV>(yn, dy + row * p.ldy, gl, gw, p.d);
        mean_n = p.mean[row];
        rstd_n = p.rstd[row];
    };
    if (r < p.rows) fetch(r);
    float gamma[NV * E], dg[NV * E], db[NV * E];
    norm_weights_load<E, NV>(gamma, p.gamma, gl, gw, p.d);
#pragma unroll
    for (int i = 0; i < NV * E; ++i) dg[i] = db[i] = 0.f;
    uint32_t flip = 0;
    for (; r < p.rows; r += step) {
        const float mean = mean_n, rstd = rstd_n;
        Pack<TX, E> xc[NV];
        Pack<TY, E> yc[NV];
        float t[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            xc[c] = xn[c];
            yc[c] = yn[c];
#pragma unroll
            for (int e = 0; e < E; ++e) {               // past the row's end dy and gamma are zero
                const float h = (to_f32(xc[c].e[e]) - mean) * rstd, w = to_f32(yc[c].e[e]), g = w * gamma[c * E + e];
                dg[c * E + e] = fmaf(w, h, dg[c * E + e]);
                db[c * E + e] += w;
                t[0] += g;
                t[1] = fmaf(g, h, t[1]);
            }
        }
        if (r + step < p.rows) fetch(r + step);
        group_sum<2>(t, gw, wig, group, lane, slot, flip);
        flip ^= 1u;
        const float ma = t[0] * inv_d, mb = t[1] * inv_d;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const uint32_t at = (gl + c * 32u * gw) * E;
            if (at < p.d) {
                Pack<TX, E> o;
#pragma unroll
                for (int e = 0; e < E; ++e) {           // formed again from the packed row: fewer registers than keeping them
                    const float h = (to_f32(xc[c].e[e]) - mean) * rstd, g = to_f32(yc[c].e[e]) * gamma[c * E + e];
                    o.e[e] = from_f32<TX>(rstd * (g - ma - h * mb));
                }
                store_pack<TX, E>(dx + r * p.ld_dx + at, o);
            }
        }
    }
    // the block's groups add up in shared memory, group 0 writes the block's row
    float *out = p.part + (uint64_t)blockIdx.x * 2 * p.d;
    if (group > 0) {
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const uint32_t at = (gl + c * 32u * gw) * E;
            if (at < p.d)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    sums[(group - 1) * 2 * p.d + at + e] = dg[c * E + e];
                    sums[(group - 1) * 2 * p.d + p.d + at + e] = db[c * E + e];
                }
        }
    }
    __syncthreads();
    if (group == 0) {
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            const uint32_t at = (gl + c * 32u * gw) * E;
            if (at < p.d)
#pragma unroll
                for (int e = 0; e < E; ++e) {
                    float a = dg[c * E + e], b = db[c * E + e];
                    for (uint32_t k = 0; k + 1 < groups; ++k) {
                        a += sums[k * 2 * p.d + at + e];
                        b += sums[k * 2 * p.d + p.d + at + e];
                    }
                    out[at + e] = a;
                    out[p.d + at + e] = b;
                }
        }
    }
}

// Column sums of the partial rows: 32 columns per block, 32 threads down each column.
__global__ void __launch_bounds__(1024)
norm_weights_kernel(const float *part, uint32_t blocks, uint32_t d, float *dgamma, float *dbeta)
{
    __shared__ float t[32][33];
    const uint32_t cx = threadIdx.x & 31, ry = threadIdx.x >> 5, col = blockIdx.x * 32 + cx;
    float a = 0.f;
    if (col < 2 * d)
        for (uint32_t r = ry; r < blocks; r += 32) a += part[(uint64_t)r * 2 * d + col];
    t[ry][cx] = a;
    __syncthreads();
    a = warp_sum(t[cx][ry]);
    const uint32_t c = blockIdx.x * 32 + ry;
    if (cx == 0 && c < 2 * d) (c < d ? dgamma[c] : dbeta[c - d]) = a;
}

uint32_t norm_backward_blocks(uint64_t rows, uint32_t d, int sms)
{
    // at 128 registers a thread 16 warps are resident per SM
    const uint32_t gw = (d + 32 * kNormPer - 1) / (32 * kNormPer), groups = gw >= 8 ? 1 : 8 / gw;
    const uint32_t per_sm = 16 / (gw * groups) ? 16 / (gw * groups) : 1;
    const uint64_t want = (rows + groups - 1) / groups, most = (uint64_t)sms * per_sm;
    return (uint32_t)(want < most ? want : most);
}

template <typename TX, typename TY>
int launch_typed(const NormParams &p, uint32_t blocks, cudaStream_t s)
{
    uint32_t e = widest_access(p.d, sizeof(TX), p.ldx, p.x, 16u / sizeof(TX));
    e = widest_access(p.d, sizeof(TX), p.ld_dx, p.dx, e);
    e = widest_access(p.d, sizeof(TY), p.ldy, p.dy, e);
    const NormShape sh = norm_shape(p.d, e);
    const uint32_t threads = sh.gw * sh.groups * 32, smem = (sh.groups - 1) * 2 * p.d * sizeof(float);
#define W2V_NORM(E, NV) norm_backward_kernel<TX, TY, E, NV><<<blocks, threads, smem, s>>>(p, sh.gw, sh.groups)
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

int launch_norm_backward(const NormParams &p, uint32_t xt, uint32_t yt, float *dgamma, float *dbeta, uint32_t blocks,
                         cudaStream_t s)
{
    int k = 0;
    if (blocks) {
        k = xt == kBF16 ? launch_typed<__nv_bfloat16, __nv_bfloat16>(p, blocks, s)
            : xt == kF16 ? launch_typed<__half, __half>(p, blocks, s)
            : yt == kBF16 ? launch_typed<float, __nv_bfloat16>(p, blocks, s)
            : yt == kF16 ? launch_typed<float, __half>(p, blocks, s)
                         : launch_typed<float, float>(p, blocks, s);
        if (k < 0) return -1;
    }
    norm_weights_kernel<<<(2 * p.d + 31) / 32, 1024, 0, s>>>(p.part, blocks, p.d, dgamma, dbeta);
    return cudaPeekAtLastError() == cudaSuccess ? k + 1 : -1;
}

}  // namespace w2v
