// Layer norm of rows: y = (x - mean) rstd gamma + beta, statistics in fp32 from a row that stays in
// registers (the mean first, then the centred squares: no cancellation).  Bound by memory: x is read
// once and y written once.  A lane has the same columns of every row of its group, so gamma and beta stay in its
// registers too (read from L1 for every row they took more L1 time than the rows themselves), and the next row is
// under way while one is worked on.
//
// With many rows a ring in shared memory, filled by bulk copies, has several units of two rows under way instead, and the
// two rows' sums go through the same shuffles.  262,144 rows of 300 (fp32 in a padded table to bf16): 76 us, 6.2 TB/s = 0.96
// of measured copy; in registers 113 us.  9,472 rows of 4,096 bf16: 32 us, 4.9 TB/s = 0.76 (two barriers of eight warps per two
// rows); in registers 60 us.
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

// The same for rows that arrive through a ring (see w2v_norm.cuh): `stages` units per group.
template <typename TX, typename TY, int E, int NV>
__global__ void __launch_bounds__(512)
norm_ring_kernel(NormParams p, uint32_t gw, uint32_t groups, uint32_t stages, int *error)
{
    extern __shared__ __align__(16) unsigned char ring[];
    __shared__ float slot[64 * kNormUnit];
    __shared__ uint64_t full[8][4];
    __shared__ int abort_flag, quiet;
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t group = warp / gw, wig = warp - group * gw, gl = wig * 32 + lane;
    const uint32_t row_bytes = p.d * sizeof(TX), unit_bytes = kNormUnit * row_bytes;
    const TX *x = static_cast<const TX *>(p.x);
    TY *y = static_cast<TY *>(p.y);
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
        mbar_expect(&full[group][stage], n * row_bytes);
        norm_copy(kCopyRows, dst, reinterpret_cast<const char *>(x), p.ldx * sizeof(TX), row_bytes, row_bytes, r, n, &full[group][stage], true);
    };
    uint32_t issued = 0;                                              // the first lane's: units on their way or here
    bool live = true;                                                 // no wait of this thread has run out
    if (gl == 0)
        for (; issued < stages && u + issued * step < units; ++issued) issue(u + issued * step, issued);
    constexpr int kPairs = NV * E / 2;                                // two columns per instruction
    float gamma[NV * E], beta[NV * E];
    norm_weights_load<E, NV>(gamma, p.gamma, gl, gw, p.d);
    norm_weights_load<E, NV>(beta, p.beta, gl, gw, p.d);
    uint32_t flip = 0, stage = 0, phase = 0;
    for (; u < units; u += step) {
        const uint64_t r = u * kNormUnit;
        const uint32_t n = (uint32_t)min((uint64_t)kNormUnit, p.rows - r);
        unsigned char *rows = mine + stage * unit_bytes;
        live = mbar_wait(&full[group][stage], phase, &abort_flag) && live;     // once it has given up the rest runs through on whatever is there
        float2 v[kNormUnit][kPairs];
        float s[kNormUnit], q[kNormUnit];
#pragma unroll
        for (int i = 0; i < kNormUnit; ++i) {
            Pack<TX, E> t[NV];
            norm_row_load<TX, E, NV>(t, reinterpret_cast<const TX *>(rows + i * row_bytes), gl, gw, p.d);
            float2 sum = make_float2(0.f, 0.f);
#pragma unroll
            for (int c = 0; c < NV; ++c)
#pragma unroll
                for (int e = 0; e < E / 2; ++e) {
                    v[i][c * (E / 2) + e] = pair_f32(t[c], e);
                    sum = add2(sum, v[i][c * (E / 2) + e]);
                }
            s[i] = sum.x + sum.y;
        }
        group_sum<kNormUnit>(s, gw, wig, group, lane, slot, flip);
        flip ^= 1u;
        if (gw == 1) __syncwarp();                                    // everybody has read the unit
        if (gl == 0 && live && u + stages * step < units) { issue(u + stages * step, stage); ++issued; }
        if (++stage == stages) { stage = 0; phase ^= 1u; }
#pragma unroll
        for (int i = 0; i < kNormUnit; ++i) {
            s[i] *= inv_d;
            const float2 less = make_float2(-s[i], -s[i]);
            float2 sum = make_float2(0.f, 0.f);
#pragma unroll
            for (int c = 0; c < NV; ++c)
                if ((gl + c * 32u * gw) * E < p.d) {
#pragma unroll
                    for (int e = c * (E / 2); e < (c + 1) * (E / 2); ++e) {
                        v[i][e] = add2(v[i][e], less);
                        sum = fma2(v[i][e], v[i][e], sum);
                    }
                }
            q[i] = sum.x + sum.y;
        }
        group_sum<kNormUnit>(q, gw, wig, group, lane, slot, flip);
        flip ^= 1u;
#pragma unroll
        for (int i = 0; i < kNormUnit; ++i) {
            if ((uint32_t)i >= n) break;
            const float rstd = rsqrtf(q[i] * inv_d + p.eps);          // 2 units in the last place
            if (gl == 0) {
                if (p.mean) p.mean[r + i] = s[i];
                if (p.rstd) p.rstd[r + i] = rstd;
            }
#pragma unroll
            for (int c = 0; c < NV; ++c) {
                const uint32_t at = (gl + c * 32u * gw) * E;
                if (at < p.d) {
                    Pack<TY, E> t;
#pragma unroll
                    for (int e = 0; e < E / 2; ++e) {
                        const int k = c * E + 2 * e;
                        set_pair(t, e, fma2(mul2(v[i][k / 2], make_float2(rstd, rstd)), make_float2(gamma[k], gamma[k + 1]), make_float2(beta[k], beta[k + 1])));
                    }
                    store_pack<TY, E>(y + (r + i) * p.ldy + at, t);
                }
            }
        }
    }
    norm_ring_drain(full[group], issued, stages, gl == 0 && !live, &quiet);
    __syncthreads();
    if (threadIdx.x == 0 && abort_flag) atomicOr(error, kErrRing);
}

template <typename TX, typename TY, int E, int NV>
int launch_norm_ring(const NormParams &p, const NormShape &sh, uint32_t stages, size_t smem, int *error, int sms, cudaStream_t s)
{
    if (!kernel_ready<norm_ring_kernel<TX, TY, E, NV>>()) return -1;
    const uint32_t threads = sh.gw * sh.groups * 32;
    const uint64_t units = (p.rows + kNormUnit - 1) / kNormUnit, want = (units + sh.groups - 1) / sh.groups, most = (uint64_t)sms * (512u / threads ? 512u / threads : 1u);
    norm_ring_kernel<TX, TY, E, NV><<<(uint32_t)(want < most ? want : most), threads, smem, s>>>(p, sh.gw, sh.groups, stages, error);
    return cudaPeekAtLastError() == cudaSuccess ? 1 : -1;
}

template <typename TX, typename TY>
int launch_norm_typed(const NormParams &p, int *error, int sms, cudaStream_t s)
{
    uint32_t e = widest_access(p.d, sizeof(TX), p.ldx, p.x, 16u / sizeof(TX));
    e = widest_access(p.d, sizeof(TY), p.ldy, p.y, e);
    const NormShape sh = norm_shape(p.d, e);
    constexpr uint32_t kE = 16 / sizeof(TX);
    // Registers against ring, us, at KB of x per SM, by type and by accesses per lane and row (nv):
    //   16-bit, 1:     rows of 256: 64 KB 6.7 and 7.6, 256 KB 21.6 and 21.2, 886 KB 73 and 66; of 128: 128 KB 20.7 and 21.3, 443 KB 68 and 66
    //   16-bit, more:  rows of 320: 10 KB 2.6 and 3.8, 20 KB 5.0 and 4.4; of 4,096: 16 KB 3.4 and 3.6, 32 KB 6.0 and 4.4, 512 KB 60 and 32
    //   fp32, 1 and 2: rows of 128: 886 KB 56 and 61; of 256: 512 KB 27.3 and 27.4, 1,771 KB 89 and 98
    //   fp32, 3:       rows of 300: 19 KB 2.9 and 4.1, 75 KB 6.5 and 6.4, 150 KB 9.9 and 9.3, 2,076 KB 113 and 78; of 768: 48 KB 5.5 and 4.7
    //   fp32, 4:       rows of 400: 200 KB 10.7 and 11.1, 400 KB 20.0 and 18.4, 2,768 KB 126 and 100
    const uint64_t from_kb = kE == 8 ? (sh.nv <= 1 ? 400 : 20) : sh.nv <= 2 ? kNever : sh.nv == 3 ? 48 : 300;
    if (e == kE && ring_pays(p.rows, p.d, sizeof(TX), sms, from_kb)) {
        const size_t unit = kNormUnit * p.d * sizeof(TX), most = 104 * 1024 / (512u / (sh.gw * sh.groups * 32) ? 512u / (sh.gw * sh.groups * 32) : 1u);
        uint32_t stages = 4;
        while (stages > 1 && unit * sh.groups * stages > most) --stages;
        const size_t smem = unit * sh.groups * stages;
        if (smem <= most && stages > 1) {
            if constexpr (kE == 8) return sh.nv <= 1 ? launch_norm_ring<TX, TY, 8, 1>(p, sh, stages, smem, error, sms, s) : launch_norm_ring<TX, TY, 8, 2>(p, sh, stages, smem, error, sms, s);
            else return sh.nv == 3 ? launch_norm_ring<TX, TY, 4, 3>(p, sh, stages, smem, error, sms, s)
                                   : launch_norm_ring<TX, TY, 4, 4>(p, sh, stages, smem, error, sms, s);
        }
    }
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

int launch_norm(const NormParams &p, uint32_t xt, uint32_t yt, int *error, int sms, cudaStream_t s)
{
    if (p.rows == 0) return 0;
    if (xt == kBF16) return launch_norm_typed<__nv_bfloat16, __nv_bfloat16>(p, error, sms, s);
    if (xt == kF16) return launch_norm_typed<__half, __half>(p, error, sms, s);
    if (yt == kBF16) return launch_norm_typed<float, __nv_bfloat16>(p, error, sms, s);
    if (yt == kF16) return launch_norm_typed<float, __half>(p, error, sms, s);
    return launch_norm_typed<float, float>(p, error, sms, s);
}

}  // namespace w2v
