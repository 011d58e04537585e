// Attention over a window of the sentence on the tensor cores.
#include <type_traits>

#include "w2v_attend.cuh"

namespace w2v {

constexpr int kFwdThreads = 256;                 // warps 0-3: one softmax row per thread; warp 4: MMA; warps 5-7: copies
constexpr int kFwdLoaders = 96;
constexpr int kSoftmaxRegs = 200, kOtherRegs = 56;      // of 128 per thread at launch: 4 x 200 + 4 x 56 warps' shares = 8 x 128
constexpr float kRescale = 8.f;                  // base-2: how far a row's scores may outgrow its reference before the output is rescaled

// NB = 64-column blocks of a head (1: head_dim <= 64, 2: up to 128).
template <int NB>
struct FwdShape {
    static constexpr int kStages = NB == 1 ? 2 : 1;                 // of keys and of values each
    static constexpr int kTileBytes = NB * kAttendTile * 128;
    static constexpr bool kOwnP = NB == 1;                          // the weights have tensor memory of their own
    static constexpr uint32_t kS = 0, kP = NB == 1 ? 128 : 0, kO = NB == 1 ? 192 : 128;   // columns
    static constexpr int kSmem = kTileBytes * (1 + 2 * kStages) + 1024;
};

struct FwdShared {
    uint64_t q_full, k_full[2], k_empty[2], v_full[2], v_empty[2], s_full, s_free, p_full, pv_done;
    uint32_t tmem;
    int abort_flag;
    int32_t limits[4][6];                        // per warp: least lo, largest hi, least s, largest lo, least hi, any row
    uint32_t vis[2][4];                          // per key stage: which keys are words
};

template <typename T, int NB>
__global__ void __launch_bounds__(kFwdThreads, 2)
attend_tc_kernel(AttendParams p, int *error)
{
    using Sh = FwdShape<NB>;
    constexpr bool kBf16 = sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value;
    extern __shared__ unsigned char smem_raw[];
    __shared__ FwdShared sh;
    unsigned char *smem = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    const uint32_t qs = smem_addr(smem), ks = qs + Sh::kTileBytes, vs = ks + Sh::kStages * Sh::kTileBytes;
    float *lut = reinterpret_cast<float *>(smem + Sh::kTileBytes * (1 + 2 * Sh::kStages));

    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t h = blockIdx.x % p.heads, kvh = h / (p.heads / p.kv_heads);
    const int32_t t0 = (int32_t)(blockIdx.x / p.heads) * kAttendTile;
    const uint32_t dim16 = (p.dim + 15u) & ~15u;

    if (tid == 0) {
        mbar_init(&sh.q_full, kFwdLoaders);
        for (int i = 0; i < 2; ++i) {
            mbar_init(&sh.k_full[i], kFwdLoaders); mbar_init(&sh.k_empty[i], 1 + kAttendTile);
            mbar_init(&sh.v_full[i], kFwdLoaders); mbar_init(&sh.v_empty[i], 1);
        }
        mbar_init(&sh.s_full, 1); mbar_init(&sh.s_free, kAttendTile);
        mbar_init(&sh.p_full, kAttendTile); mbar_init(&sh.pv_done, 1);
        sh.abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    RowLimits row = {0, 0, 0, 0};
    if (warp < 4) {
        row = row_limits(p, (int64_t)t0 + tid);
        const bool any = row.hi > row.lo;
        const int32_t lo = __reduce_min_sync(kFullMask, any ? row.lo : INT32_MAX), hi = __reduce_max_sync(kFullMask, row.hi);
        const int32_t s = __reduce_min_sync(kFullMask, any ? row.s : INT32_MAX);
        if (lane == 0) { sh.limits[warp][0] = lo; sh.limits[warp][1] = hi; sh.limits[warp][2] = s; }
    }
    if (warp == 4) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&sh.tmem)), "r"(256));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (p.b.n) fill_bias(p, h, lut, tid, kFwdThreads);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = sh.tmem;
    volatile int *abort_flag = &sh.abort_flag;
    // the run of keys [lo, hi) and the sinks [s, s_end) before it
    int32_t lo = INT32_MAX, hi = 0, s = INT32_MAX;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        lo = min(lo, sh.limits[w][0]);
        hi = max(hi, sh.limits[w][1]);
        s = min(s, sh.limits[w][2]);
    }
    const int32_t s_end = hi ? min(s + p.sinks, lo) : 0;
    const int32_t extra = s < s_end ? 1 : 0;
    const int32_t tiles = hi ? extra + (hi - lo + kAttendTile - 1) / kAttendTile : 0;
    auto tile_at = [&](int32_t t) { return extra && t == 0 ? s : lo + (t - extra) * kAttendTile; };
    auto tile_keys = [&](int32_t t) { return extra && t == 0 ? s_end - s : min(kAttendTile, hi - tile_at(t)); };

    if (warp < 4) {
        // ============ softmax: one row per thread ============
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        const int64_t i = (int64_t)t0 + tid;
        const uint32_t lanes = (warp * 32u) << 16;
        const float scale = p.scale * kLog2e;
        const int32_t last = bias_last(p.b);
        const float *near_row = lut - i + last + kBiasPad;         // + key position
        float ref = -INFINITY, sum = 0.f;
        bool ok = true;
        for (int32_t t = 0; t < tiles; ++t) {
            const int32_t k0 = tile_at(t), keys = tile_keys(t), cols = (keys + 15) & ~15;
            if (!__all_sync(kFullMask, mbar_wait(&sh.s_full, t & 1, abort_flag))) { ok = false; break; }
            tc_fence_after();
            const uint32_t stage = t % Sh::kStages;
            if (!__all_sync(kFullMask, mbar_wait(&sh.k_full[stage], (t / Sh::kStages) & 1, abort_flag))) { ok = false; break; }   // the bits of the keys
            float x[4][32];
            float top = -INFINITY;
            // far from the rows every key of the tile has the bias of the side's last bucket
            const bool far = p.b.n == 0 || k0 + cols - 1 - t0 <= -last || k0 - (t0 + kAttendTile - 1) >= last;
            const float flat = p.b.n ? lut[k0 < t0 ? 0 : bias_entries(p.b) - 1] : 0.f;
            const float *near = near_row + k0;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (c * 32 < cols) {
                    uint32_t v[32];
                    tmem_ld32(tmem + lanes + Sh::kS + c * 32, v);
                    tmem_wait_ld(v);
                    if (far) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) x[c][e] = fmaf(__uint_as_float(v[e]), scale, flat);
                    } else {
#pragma unroll
                        for (int e = 0; e < 32; ++e) x[c][e] = fmaf(__uint_as_float(v[e]), scale, near[c * 32 + e]);
                    }
                    const int32_t at = k0 + c * 32;
                    const uint32_t m = (range_bits(row.lo, row.hi, at) | range_bits(row.s, row.se, at)) & sh.vis[stage][c];
                    if (!__all_sync(kFullMask, m == 0xFFFFFFFFu)) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) x[c][e] = (m >> e) & 1u ? x[c][e] : -INFINITY;
                    }
#pragma unroll
                    for (int e = 0; e < 32; ++e) top = fmaxf(top, x[c][e]);
                }
            }
            mbar_arrive(&sh.k_empty[stage]);                         // this thread is done with the stage's bits
            if (Sh::kOwnP) {                                         // the next scores may be computed
                tc_fence_before();
                mbar_arrive(&sh.s_free);
            }
            const bool grown = top > ref + kRescale || (ref == -INFINITY && top > ref);
            if (t > 0 && !__all_sync(kFullMask, mbar_wait(&sh.pv_done, (t - 1) & 1, abort_flag))) { ok = false; break; }
            if (__any_sync(kFullMask, grown)) {
                const float to = grown ? top : ref;
                const float keep = ref == -INFINITY ? 0.f : fast_exp2(ref - to);
                ref = to;
                sum *= keep;
                if (t > 0) {
                    tc_fence_after();
                    for (uint32_t c = 0; c < dim16; c += 16) {
                        uint32_t o[16];
                        tmem_ld16(tmem + lanes + Sh::kO + c, o);
                        tmem_wait_ld(o);
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * keep);
                        tmem_st16(tmem + lanes + Sh::kO + c, o);
                    }
                }
            }
            const float from = ref == -INFINITY ? 0.f : ref;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (c * 32 < cols) {
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float a = fast_exp2(x[c][2 * e] - from), b = fast_exp2(x[c][2 * e + 1] - from);
                        sum += a + b;
                        w[e] = pack2<T>(a, b);
                    }
                    tmem_st16(tmem + lanes + Sh::kP + c * 16, w);
                }
            }
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(&sh.p_full);
        }
        ok = __all_sync(kFullMask, ok && (tiles == 0 || mbar_wait(&sh.pv_done, (tiles - 1) & 1, abort_flag)));
        tc_fence_after();
        // the output leaves through shared memory (every tile is read by now), a row of 16-byte chunks at a time
        const float inv = ok && sum > 0.f ? 1.f / sum : 0.f;
        if (p.lse && i < p.n) p.lse[(int64_t)h * p.n + i] = sum > 0.f ? ref + log2f(sum) : INFINITY;
        const uint32_t row_bytes = p.dim * 2u;
        unsigned char *mine = smem + warp * 32u * row_bytes, *line = mine + lane * row_bytes;
        const int32_t rows = (int32_t)min((int64_t)32, p.n - (t0 + (int64_t)warp * 32));
        for (uint32_t c = 0; c < dim16; c += 16) {
            uint32_t o[16];
            if (tiles) { tmem_ld16(tmem + lanes + Sh::kO + c, o); tmem_wait_ld(o); }
            else {
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = 0u;
            }
#pragma unroll
            for (int g = 0; g < 2; ++g)
                if (c + g * 8 < p.dim) {
                    uint4 w;
                    w.x = pack2<T>(__uint_as_float(o[g * 8 + 0]) * inv, __uint_as_float(o[g * 8 + 1]) * inv);
                    w.y = pack2<T>(__uint_as_float(o[g * 8 + 2]) * inv, __uint_as_float(o[g * 8 + 3]) * inv);
                    w.z = pack2<T>(__uint_as_float(o[g * 8 + 4]) * inv, __uint_as_float(o[g * 8 + 5]) * inv);
                    w.w = pack2<T>(__uint_as_float(o[g * 8 + 6]) * inv, __uint_as_float(o[g * 8 + 7]) * inv);
                    const uint32_t ch = (c >> 3) + g, chunks = p.dim >> 3;
                    *reinterpret_cast<uint4 *>(line + ((ch + lane) % chunks) * 16u) = w;       // turned by the row: fewer bank conflicts
                }
        }
        __syncwarp();
        {
            const uint32_t chunks = p.dim >> 3;
            char *out = static_cast<char *>(p.out) + ((uint64_t)(t0 + warp * 32) * p.ldo + (uint64_t)h * p.dim) * 2u;
            for (int32_t e = (int32_t)lane; e < rows * (int32_t)chunks; e += 32) {
                const uint32_t r = (uint32_t)e / chunks, ch = (uint32_t)e - r * chunks;
                *reinterpret_cast<uint4 *>(out + (uint64_t)r * p.ldo * 2u + ch * 16u) =
                    *reinterpret_cast<const uint4 *>(mine + r * row_bytes + ((ch + r) % chunks) * 16u);
            }
        }
        tc_fence_before();
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (warp == 4) {
            // ============ MMA issue: one lane ============
            if (lane == 0 && tiles) {
                const uint32_t idesc_o = umma_idesc_f16(kBf16, kAttendTile, dim16, true);
                auto scores = [&](int32_t t) {
                    const uint32_t stage = t % Sh::kStages, cols = (uint32_t)(tile_keys(t) + 15) & ~15u;
                    const uint32_t idesc = umma_idesc_f16(kBf16, kAttendTile, cols, false);
                    for (uint32_t c = 0; c < dim16; c += 16) {
                        const uint32_t off = (c >> 6) * (kAttendTile * 128) + (c & 63u) * 2u;
                        umma_f16_ss(tmem + Sh::kS, umma_desc_sw128(qs + off, 0), umma_desc_sw128(ks + stage * Sh::kTileBytes + off, 0), idesc, c > 0);
                    }
                    umma_commit(&sh.s_full);
                    umma_commit(&sh.k_empty[stage]);
                };
                bool ok = mbar_wait(&sh.q_full, 0, abort_flag) && mbar_wait(&sh.k_full[0], 0, abort_flag);
                if (ok) { tc_fence_after(); scores(0); }
                for (int32_t t = 0; t < tiles && ok; ++t) {
                    const uint32_t stage = t % Sh::kStages;
                    const int32_t n1 = t + 1;
                    if (Sh::kOwnP && n1 < tiles) {
                        ok = mbar_wait(&sh.k_full[n1 % Sh::kStages], (n1 / Sh::kStages) & 1, abort_flag) && mbar_wait(&sh.s_free, t & 1, abort_flag);
                        if (!ok) break;
                        tc_fence_after();
                        scores(n1);
                    }
                    ok = mbar_wait(&sh.v_full[stage], (t / Sh::kStages) & 1, abort_flag) && mbar_wait(&sh.p_full, t & 1, abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                    const uint32_t cols = (uint32_t)(tile_keys(t) + 15) & ~15u;
                    for (uint32_t k = 0; k < cols; k += 16)
                        umma_f16_ts(tmem + Sh::kO, tmem + Sh::kP + k / 2, umma_desc_sw128(vs + stage * Sh::kTileBytes + k * 128u, kAttendTile * 128),
                                    idesc_o, t > 0 || k > 0);
                    umma_commit(&sh.pv_done);
                    umma_commit(&sh.v_empty[stage]);
                    if (!Sh::kOwnP && n1 < tiles) {
                        ok = mbar_wait(&sh.k_full[n1 % Sh::kStages], (n1 / Sh::kStages) & 1, abort_flag);
                        if (!ok) break;
                        tc_fence_after();
                        scores(n1);
                    }
                }
            }
            __syncwarp();
        } else if (tiles) {
            // ============ copies: keys and values of one tile after the other ============
            const uint32_t lt = tid - 160u;
            constexpr int CH = NB * 8;
            const uint32_t used = dim16 >> 3, dch = p.dim >> 3;
            const T *q = static_cast<const T *>(p.q) + (uint64_t)h * p.dim, *k = static_cast<const T *>(p.k) + (uint64_t)kvh * p.dim,
                    *v = static_cast<const T *>(p.v) + (uint64_t)kvh * p.dim;
            uint64_t *pending = nullptr;
            bool ok = true;
            // waits for the slot; the copies already under way are handed over first if it is not free yet
            auto slot = [&](uint64_t *empty, uint32_t parity) {
                if (mbar_try(empty, parity)) return true;
                if (pending) { copy_wait<0>(); fence_async_proxy(); mbar_arrive(pending); pending = nullptr; }
                return mbar_wait(empty, parity, abort_flag);
            };
            auto issued = [&](uint64_t *full) {
                copy_commit();
                if (pending) { copy_wait<1>(); fence_async_proxy(); mbar_arrive(pending); }
                pending = full;
            };
            uint32_t vis[4];
            visible_bits(p, t0, kAttendTile, lane, vis);
            copy_rows_sw128<CH>(qs, kAttendTile * 128, q, p.ldq * 2, t0, kAttendTile, vis, dch, used, lt, kFwdLoaders);
            issued(&sh.q_full);
            for (int32_t t = 0; t < tiles && ok; ++t) {
                const uint32_t stage = t % Sh::kStages, round = t / Sh::kStages;
                const int32_t at = tile_at(t), keys = tile_keys(t);
                const uint32_t cols = (uint32_t)(keys + 15) & ~15u;
                visible_bits(p, at, (uint32_t)keys, lane, vis);
                if (round > 0) ok = slot(&sh.k_empty[stage], (round - 1) & 1);
                if (!ok) break;
                if (lt == 0) { sh.vis[stage][0] = vis[0]; sh.vis[stage][1] = vis[1]; sh.vis[stage][2] = vis[2]; sh.vis[stage][3] = vis[3]; }
                copy_rows_sw128<CH>(ks + stage * Sh::kTileBytes, kAttendTile * 128, k, p.ldk * 2, at, cols, vis, dch, used, lt, kFwdLoaders);
                issued(&sh.k_full[stage]);
                if (round > 0) ok = slot(&sh.v_empty[stage], (round - 1) & 1);
                if (!ok) break;
                copy_rows_sw128<CH>(vs + stage * Sh::kTileBytes, kAttendTile * 128, v, p.ldv * 2, at, cols, vis, dch, used, lt, kFwdLoaders);
                issued(&sh.v_full[stage]);
            }
            copy_wait<0>();
            if (pending && ok) { fence_async_proxy(); mbar_arrive(pending); }
        }
    }
    __syncthreads();
    tc_fence_after();
    if (warp == 4) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(256));
    if (tid == 0 && sh.abort_flag) atomicOr(error, kErrAttend);
}

template <typename T, int NB>
int launch_attend_shape(const AttendParams &p, int *error, cudaStream_t s)
{
    auto kernel = attend_tc_kernel<T, NB>;
    const int smem = FwdShape<NB>::kSmem + (int)(bias_entries(p.b) * sizeof(float));
    cudaFuncAttributes at;
    // the softmax warps take registers that the others give up: the block must have been launched with all of them
    if (cudaFuncGetAttributes(&at, kernel) != cudaSuccess || at.numRegs * 8 < 4 * (kSoftmaxRegs + kOtherRegs)) return -1;
    if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) return -1;
    const uint64_t tiles = ((uint64_t)p.n + kAttendTile - 1) / kAttendTile;
    kernel<<<(uint32_t)(tiles * p.heads), kFwdThreads, smem, s>>>(p, error);
    return cudaPeekAtLastError() == cudaSuccess ? 1 : -1;
}

int launch_attend(const AttendParams &p, uint32_t type, int *error, int, cudaStream_t s)
{
    if (p.n == 0) return 0;
    if (type == kBF16) return p.dim <= 64 ? launch_attend_shape<__nv_bfloat16, 1>(p, error, s) : launch_attend_shape<__nv_bfloat16, 2>(p, error, s);
    return p.dim <= 64 ? launch_attend_shape<__half, 1>(p, error, s) : launch_attend_shape<__half, 2>(p, error, s);
}

}  // namespace w2v
