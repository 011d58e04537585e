// Layer norm backwards.  With xh = (x - mean) rstd and G = dy gamma,
//   dx = rstd (G - mean(G) - xh mean(G xh)),  dgamma = sum over rows of dy xh,  dbeta = sum of dy.
// Bound by memory: x and dy are read once, dx is written once.  A lane keeps the same columns of every
// row that its group handles, so the weights' gradients stay in its registers until the end; each block
// then writes one partial row and a second kernel adds the partials in a fixed order (no atomics: the
// same inputs give the same bits).
//
// Many rows come through a ring in shared memory, as forwards; both sums over the row are formed from there and the second
// reading for dx costs no memory traffic.  262,144 rows of 300 (fp32, dy bf16): 149 us, 5.3 TB/s = 0.82 of measured copy; in
// registers 158 us.  9,472 rows of 4,096 bf16 62 us with the sums over blocks, 3.8 TB/s = 0.58; in registers 89 us.
#include "w2v_norm.cuh"

namespace w2v {

// The block's groups add up in shared memory ([groups - 1][2][d]), group 0 writes the block's row.
template <int E, int NV>
__device__ __forceinline__ void norm_block_sums(const NormParams &p, const float (&dg)[NV * E], const float (&db)[NV * E], float *sums,
                                                uint32_t gw, uint32_t group, uint32_t groups, uint32_t gl)
{
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
    norm_block_sums<E, NV>(p, dg, db, sums, gw, group, groups, gl);
}

// The same for rows that arrive through a ring (see w2v_norm.cuh): `stages` units of x and dy per group.  A unit is read
// twice from shared memory, for the sums and for dx.
template <typename TX, typename TY, int E, int NV>
__global__ void __launch_bounds__(512)
norm_backward_ring_kernel(NormParams p, uint32_t gw, uint32_t groups, uint32_t stages, uint32_t mode_y, int *error)
{
    extern __shared__ __align__(16) unsigned char ring[];
    __shared__ float slot[128 * kNormUnit];
    __shared__ uint64_t full[8][4];
    __shared__ int abort_flag, quiet;
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t group = warp / gw, wig = warp - group * gw, gl = wig * 32 + lane;
    const uint32_t pitch_x = p.d * sizeof(TX), pitch_y = norm_pitch(mode_y, p.d, sizeof(TY));
    const uint32_t x_bytes = kNormUnit * pitch_x, unit_bytes = x_bytes + ((kNormUnit * pitch_y + 15u) & ~15u);
    const TX *x = static_cast<const TX *>(p.x);
    const TY *dy = static_cast<const TY *>(p.dy);
    TX *dx = static_cast<TX *>(p.dx);
    unsigned char *mine = ring + group * stages * unit_bytes;
    const float inv_d = 1.0f / (float)p.d;
    const uint64_t units = (p.rows + kNormUnit - 1) / kNormUnit, step = (uint64_t)gridDim.x * groups;
    uint64_t u = (uint64_t)blockIdx.x * groups + group;
    if (threadIdx.x == 0) {
        for (uint32_t g = 0; g < groups; ++g)
            for (uint32_t s = 0; s < stages; ++s) mbar_init(&full[g][s], 1);
        abort_flag = quiet = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_proxy();
    }
    __syncthreads();
    auto issue = [&](uint64_t unit, uint32_t stage) {                 // by the group's first lane
        const uint64_t r = unit * kNormUnit;
        const uint32_t n = (uint32_t)min((uint64_t)kNormUnit, p.rows - r), dst = smem_addr(mine + stage * unit_bytes);
        uint64_t *bar = &full[group][stage];
        const char *xb = reinterpret_cast<const char *>(x), *yb = reinterpret_cast<const char *>(dy);
        auto both = [&](bool now) {
            return norm_copy(kCopyRows, dst, xb, p.ldx * sizeof(TX), p.d * sizeof(TX), pitch_x, r, n, bar, now) +
                   norm_copy(mode_y, dst + x_bytes, yb, p.ldy * sizeof(TY), p.d * sizeof(TY), pitch_y, r, n, bar, now);
        };
        mbar_expect(bar, both(false));
        both(true);
    };
    uint32_t issued = 0;                                              // the first lane's: units on their way or here
    bool live = true;                                                 // no wait of this thread has run out
    if (gl == 0)
        for (; issued < stages && u + issued * step < units; ++issued) issue(u + issued * step, issued);
    constexpr int kPairs = NV * E / 2;                                // two columns per instruction
    float gamma[NV * E];
    float2 dg2[kPairs], db2[kPairs];
    norm_weights_load<E, NV>(gamma, p.gamma, gl, gw, p.d);
#pragma unroll
    for (int i = 0; i < kPairs; ++i) dg2[i] = db2[i] = make_float2(0.f, 0.f);
    uint32_t flip = 0, stage = 0, phase = 0;
    for (; u < units; u += step) {
        const uint64_t r = u * kNormUnit;
        const uint32_t n = (uint32_t)min((uint64_t)kNormUnit, p.rows - r);
        unsigned char *rows_x = mine + stage * unit_bytes, *rows_y = rows_x + x_bytes;
        float mean[kNormUnit], rstd[kNormUnit], t[2 * kNormUnit];
#pragma unroll
        for (int i = 0; i < kNormUnit; ++i) {
            const uint64_t at = min(r + i, p.rows - 1);
            mean[i] = __ldg(p.mean + at);
            rstd[i] = (uint32_t)i < n ? __ldg(p.rstd + at) : 0.f;
            t[2 * i] = t[2 * i + 1] = 0.f;
        }
        live = mbar_wait(&full[group][stage], phase, &abort_flag) && live;     // once it has given up the rest runs through on whatever is there
        if (n < kNormUnit && mode_y == kCopyUnits) {
            norm_copy_tail<TY>(rows_y, dy + r * p.ldy, p.d, n, gl, gw * 32);
            group_barrier(gw, group);
        }
#pragma unroll
        for (int i = 0; i < kNormUnit; ++i) {
            if ((uint32_t)i >= n) break;                              // what a cut-off unit lacks is not in shared memory
            Pack<TX, E> xc[NV];
            Pack<TY, E> yc[NV];
            norm_row_load<TX, E, NV>(xc, reinterpret_cast<const TX *>(rows_x + i * pitch_x), gl, gw, p.d);
            norm_row_load<TY, E, NV>(yc, reinterpret_cast<const TY *>(rows_y + i * pitch_y), gl, gw, p.d);
            const float2 by = make_float2(rstd[i], rstd[i]), less = make_float2(-mean[i], -mean[i]);
            float2 sg = make_float2(0.f, 0.f), sh = sg;
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int e = 0; e < E / 2; ++e) {                     // past the row's end dy and gamma are zero
                    const int k = c * (E / 2) + e;
                    const float2 h = mul2(add2(pair_f32(xc[c], e), less), by), w = pair_f32(yc[c], e), g = mul2(w, make_float2(gamma[2 * k], gamma[2 * k + 1]));
                    dg2[k] = fma2(w, h, dg2[k]);
                    db2[k] = add2(db2[k], w);
                    sg = add2(sg, g);
                    sh = fma2(g, h, sh);
                }
            t[2 * i] = sg.x + sg.y;
            t[2 * i + 1] = sh.x + sh.y;
        }
        group_sum<2 * kNormUnit>(t, gw, wig, group, lane, slot, flip);
        flip ^= 1u;
#pragma unroll
        for (int i = 0; i < kNormUnit; ++i) {
            if ((uint32_t)i >= n) break;
            // dx = rstd g - rstd mean(g) - h rstd mean(g h)
            const float ma = -rstd[i] * t[2 * i] * inv_d, mb = -rstd[i] * t[2 * i + 1] * inv_d;
            const float2 by = make_float2(rstd[i], rstd[i]), less = make_float2(-mean[i], -mean[i]), ma2 = make_float2(ma, ma), mb2 = make_float2(mb, mb);
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                const uint32_t at = (gl + c * 32u * gw) * E;
                if (at < p.d) {
                    const Pack<TX, E> xc = load_pack<TX, E>(reinterpret_cast<const TX *>(rows_x + i * pitch_x) + at);
                    const Pack<TY, E> yc = load_pack<TY, E>(reinterpret_cast<const TY *>(rows_y + i * pitch_y) + at);
                    Pack<TX, E> o;
#pragma unroll
                    for (int e = 0; e < E / 2; ++e) {
                        const int k = c * (E / 2) + e;
                        const float2 h = mul2(add2(pair_f32(xc, e), less), by), g = mul2(pair_f32(yc, e), make_float2(gamma[2 * k], gamma[2 * k + 1]));
                        set_pair(o, e, fma2(g, by, fma2(h, mb2, ma2)));
                    }
                    store_pack<TX, E>(dx + (r + i) * p.ld_dx + at, o);
                }
            }
        }
        group_barrier(gw, group);                                     // everybody has read the unit
        if (gl == 0 && live && u + stages * step < units) { issue(u + stages * step, stage); ++issued; }
        if (++stage == stages) { stage = 0; phase ^= 1u; }
    }
    norm_ring_drain(full[group], issued, stages, gl == 0 && !live, &quiet);
    __syncthreads();
    if (threadIdx.x == 0 && abort_flag) atomicOr(error, kErrRing);
    float dg[NV * E], db[NV * E];
#pragma unroll
    for (int i = 0; i < kPairs; ++i) { dg[2 * i] = dg2[i].x; dg[2 * i + 1] = dg2[i].y; db[2 * i] = db2[i].x; db[2 * i + 1] = db2[i].y; }
    norm_block_sums<E, NV>(p, dg, db, reinterpret_cast<float *>(ring), gw, group, groups, gl);
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

template <typename TX, typename TY, int E, int NV>
int launch_back_ring(const NormParams &p, const NormShape &sh, uint32_t stages, uint32_t mode_y, size_t smem, uint32_t blocks,
                     int *error, cudaStream_t s)
{
    if (!kernel_ready<norm_backward_ring_kernel<TX, TY, E, NV>>()) return -1;
    norm_backward_ring_kernel<TX, TY, E, NV><<<blocks, sh.gw * sh.groups * 32, smem, s>>>(p, sh.gw, sh.groups, stages, mode_y, error);
    return cudaPeekAtLastError() == cudaSuccess ? 1 : -1;
}

template <typename TX, typename TY>
int launch_typed(const NormParams &p, uint32_t blocks, int *error, int sms, cudaStream_t s)
{
    uint32_t e = widest_access(p.d, sizeof(TX), p.ldx, p.x, 16u / sizeof(TX));
    e = widest_access(p.d, sizeof(TX), p.ld_dx, p.dx, e);
    e = widest_access(p.d, sizeof(TY), p.ldy, p.dy, e);
    const NormShape sh = norm_shape(p.d, e);
    constexpr uint32_t kE = 16 / sizeof(TX);
    const uint32_t mode_y = norm_copy_mode(p.dy, p.ldy, p.d, sizeof(TY));
    // Registers against ring, us with the sums over blocks, at KB of x per SM, by type and by accesses per lane and row (nv):
    //   16-bit:        rows of 64: 8 KB 10.5 and 10.5, 16 KB 15.9 and 14.2; of 256: 16 KB 10.0 and 10.3, 64 KB 17.4 and 16.5;
    //                  of 4,096: 8 KB 12.2 and 12.5, 16 KB 19.2 and 17.5, 512 KB 89 and 62
    //   fp32, 1:       rows of 64: 443 KB 99 and 107; of 128: 886 KB 100 and 113
    //   fp32, 2 and 3: rows of 200: 400 KB 44.1 and 43.6, 1,384 KB 132 and 127; of 300: 300 KB 30.9 and 32.6, 600 KB 53.9 and 53.5,
    //                  2,076 KB 163 and 153; of 320: 640 KB 31.5 and 34.0, 2,214 KB 167 and 163; of 768: 192 KB 18.7 and 20.2, 768 KB 61 and 54
    //   fp32, 4:       rows of 400: 25 KB 12.3 and 12.5, 50 KB 14.2 and 13.4; of 512: 32 KB 12.5 and 12.7, 256 KB 29.8 and 27.1
    const uint64_t from_kb = kE == 8 ? 16 : sh.nv <= 1 ? kNever : sh.nv <= 3 ? 700 : 48;
    if (e == kE && mode_y != kCopyNot && ring_pays(p.rows, p.d, sizeof(TX), sms, from_kb)) {
        const uint32_t per_sm = 512u / (sh.gw * sh.groups * 32) ? 512u / (sh.gw * sh.groups * 32) : 1u;
        const size_t unit = kNormUnit * p.d * sizeof(TX) + ((kNormUnit * norm_pitch(mode_y, p.d, sizeof(TY)) + 15u) & ~15u);
        const size_t most = 216 * 1024 / per_sm, add = (size_t)(sh.groups - 1) * 2 * p.d * sizeof(float);
        uint32_t stages = 4;
        while (stages > 1 && unit * sh.groups * stages > most) --stages;
        const size_t smem = unit * sh.groups * stages > add ? unit * sh.groups * stages : add;       // the ring, then the block's sums
        if (smem <= most && stages > 1) {
            if constexpr (kE == 8) return sh.nv <= 1 ? launch_back_ring<TX, TY, 8, 1>(p, sh, stages, mode_y, smem, blocks, error, s)
                                                      : launch_back_ring<TX, TY, 8, 2>(p, sh, stages, mode_y, smem, blocks, error, s);
            else return sh.nv == 2 ? launch_back_ring<TX, TY, 4, 2>(p, sh, stages, mode_y, smem, blocks, error, s)
                        : sh.nv == 3 ? launch_back_ring<TX, TY, 4, 3>(p, sh, stages, mode_y, smem, blocks, error, s)
                                     : launch_back_ring<TX, TY, 4, 4>(p, sh, stages, mode_y, smem, blocks, error, s);
        }
    }
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
                         int *error, int sms, cudaStream_t s)
{
    int k = 0;
    if (blocks) {
        k = xt == kBF16 ? launch_typed<__nv_bfloat16, __nv_bfloat16>(p, blocks, error, sms, s)
            : xt == kF16 ? launch_typed<__half, __half>(p, blocks, error, sms, s)
            : yt == kBF16 ? launch_typed<float, __nv_bfloat16>(p, blocks, error, sms, s)
            : yt == kF16 ? launch_typed<float, __half>(p, blocks, error, sms, s)
                         : launch_typed<float, float>(p, blocks, error, sms, s);
        if (k < 0) return -1;
    }
    norm_weights_kernel<<<(2 * p.d + 31) / 32, 1024, 0, s>>>(p.part, blocks, p.d, dgamma, dbeta);
    return cudaPeekAtLastError() == cudaSuccess ? k + 1 : -1;
}

}  // namespace w2v
