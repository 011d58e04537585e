// Attention over a window of the sentence on the tensor cores.
//
// A block takes 128 queries of a head and streams the keys and values of its run in tiles of 64 (32) through a ring in
// shared memory.  Two warpgroups take the tiles in turn, one row per thread; each has a score buffer, a running
// reference, a sum and an output accumulator of its own in tensor memory, so that neither waits for the other; the two
// are joined at the end.  The softmax weights go back to tensor memory, over the scores, as the A side of P V; they are
// rounded to the arrays' type there, as the matrix units want them, while their sum is kept in fp32.
// A tile's scores are read twice from tensor memory instead of being held: the first pass finds the largest (and,
// where a tile has masks or differing biases, writes the scores back with both applied), the second exponentiates.
// The output is rescaled only when a row's largest score outgrows the reference by 2^8.
//
// What bounds it: latency.  The softmax warps wait for their tensor-memory reads and for the chain from there to the
// weights (issue slots 35 % busy, matrix units 24 %, heads of 128), and tensor memory holds no more of them.  A prompt of 32,768 words (fp16, 8 heads of 64,
// 2 of keys and values, windows of 4,096): 0.51 ms, 0.30 of the measured rate of matrix products; 16,381 words of long
// documents, 16 heads of 128, windows of 1,024: 0.29 ms; 131,072 words in sessions of 5 to 40, 4 heads of 80: 0.16 ms, where
// beginnings and ends of blocks are most of the time.
#include <type_traits>

#include "w2v_attend.cuh"
#include "w2v_kernel_ready.h"

namespace w2v {

constexpr int kFwdThreads = 384;                 // warps 0-7: two softmax warpgroups; warp 8: MMA; warp 9: copies; warps 10-11: rows that are not words
// Of the 80 registers a thread has at launch with two blocks per SM, the third warpgroup gives
// its share beyond 48 to the two of the softmax (96 + 96 + 48 = 3 x 80).
constexpr int kLaunchRegs = 80, kSoftmaxRegs = 96, kOtherRegs = 48;
constexpr float kRescale = 8.f;                  // base-2: how far a row's scores may outgrow its reference before the output is rescaled

// NB = 64-column blocks of a head (1: head_dim <= 64, 2: up to 128).  SMALL (up to 96): half of the tensor memory, so that
// two blocks share an SM and one's beginning and end lie under the other's middle; tiles of 32 keys where two 96-column
// outputs leave room for no more.  Against the whole of the tensor memory and one block: those sessions 240 -> 153 us, 65,536
// words in sentences of 1,000 (5 heads of 64, windows of 257) 201 -> 132 us, the prompt 708 -> 511 us (with what came since 158, 132
// and 514).
template <int NB, bool SMALL>
struct FwdShape {
    static constexpr int kBlocks = SMALL ? 2 : 1;                   // resident per SM: tensor memory is the limit
    static constexpr int kRows = SMALL && NB == 2 ? 32 : 64;        // keys per tile
    static constexpr bool kQTmem = !SMALL;                          // queries as an A side in tensor memory (read from shared memory
                                                                    // for every tile they would cost as much as keys and values)
    static constexpr int kStages = SMALL ? 4 : 3;
    static constexpr int kOperand = NB * kRows * 128, kStage = 2 * kOperand, kQBytes = kQTmem ? 0 : NB * 128 * 128;
    static constexpr uint32_t kWide = SMALL && NB == 2 ? 96 : NB * 64;                          // columns of an output
    static constexpr uint32_t kQ = 0, kS = kQTmem ? NB * 32 : 0, kO = kS + 2 * kRows, kAlloc = SMALL ? 256 : 512;
    static_assert(kO + 2 * kWide <= kAlloc, "tensor memory");
    static constexpr int kRing = kQBytes + kStages * kStage;
    static_assert(kRing >= NB * 128 * 128, "the output is staged where the ring was");
};

struct FwdShared {
    uint64_t q_full, landed[4], full[4], empty[4], s_full[2], p_full[2], done, still;
    uint32_t tmem;
    int abort_flag, quiet;
    int32_t limits[4][3];                        // per warp: least lo, largest hi, least sentence start
    uint32_t vis[4][2];                          // per stage: which keys are words
    float ref[2][128], sum[2][128];              // per warpgroup and row
};

// The output of row i by a warp, from the pairs that it sees; `ref` and `inv` are the row's reference and inverse sum.
template <typename T>
__device__ __forceinline__ void output_again(const AttendParams &p, uint32_t h, uint32_t kvh, int64_t i, float ref, float inv, uint32_t lane)
{
    const RowLimits row = row_limits(p, i);
    const T *q = static_cast<const T *>(p.q) + i * (int64_t)p.ldq + h * p.dim;
    const T *k = static_cast<const T *>(p.k) + kvh * p.dim, *v = static_cast<const T *>(p.v) + kvh * p.dim;
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int part = 0; part < 2; ++part) {
        const int32_t a = part ? row.lo : row.s, b = part ? row.hi : row.se;
#pragma unroll 1
        for (int64_t j0 = a; j0 < b && !all_nan(acc, p.dim, lane); j0 += 32) {
            const int64_t j = j0 + lane;
            const bool seen = j < b && is_word(p, j);
            float w = 0.f;
            if (seen) w = fast_exp2(fmaf(row_dot(q, k + j * (int64_t)p.ldk, p.dim), p.scale * kLog2e, pair_bias(p, h, (int32_t)(j - i))) - ref) * inv;
            add_rows(acc, w, __ballot_sync(kFullMask, seen), v + j0 * (int64_t)p.ldv, p.ldv, p.dim, lane);
        }
    }
    T *out = static_cast<T *>(p.out) + i * (int64_t)p.ldo + h * p.dim;
#pragma unroll
    for (int x = 0; x < 4; ++x)
        if (lane + 32u * x < p.dim) out[lane + 32u * x] = from_f32<T>(acc[x]);
}

template <typename T, int NB, bool SMALL>
__global__ void __launch_bounds__(kFwdThreads, FwdShape<NB, SMALL>::kBlocks)
attend_tc_kernel(const __grid_constant__ CUtensorMap map_q, const __grid_constant__ CUtensorMap map_k,
                 const __grid_constant__ CUtensorMap map_v, AttendParams p, int *error)
{
    using Sh = FwdShape<NB, SMALL>;
    constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
    extern __shared__ unsigned char smem_raw[];
    __shared__ FwdShared sh;
    unsigned char *smem = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    const uint32_t qs = smem_addr(smem), ring = qs + Sh::kQBytes;
    float *lut = reinterpret_cast<float *>(smem + Sh::kRing);

    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t h = blockIdx.x % p.heads, kvh = h / (p.heads / p.kv_heads);
    const int32_t t0 = (int32_t)(blockIdx.x / p.heads) * kAttendTile;
    const uint32_t dim16 = (p.dim + 15u) & ~15u, dch = p.dim >> 3;
    const uint32_t r = tid & 127u;                                   // this thread's row (softmax warps)
    const int64_t own = (int64_t)t0 + r;
    const T *q_head = static_cast<const T *>(p.q) + (uint64_t)h * p.dim;
    RowLimits row = {0, 0, 0, 0};
    uint4 q_row[Sh::kQTmem ? NB * 8 : 1];
    int32_t issued = 0;                                              // tiles whose copies were started (the copying lane's)

    if (warp < 8) {
        row = row_limits(p, own);
        if (warp < 4) {
            if (Sh::kQTmem) {
#pragma unroll
                for (int c = 0; c < NB * 8; ++c)
                    q_row[c] = own < p.n && (uint32_t)c < dch ? __ldg(reinterpret_cast<const uint4 *>(q_head + own * (int64_t)p.ldq) + c) : make_uint4(0, 0, 0, 0);
            }
            const bool any = row.hi > row.lo;
            const int32_t lo = __reduce_min_sync(kFullMask, any ? row.lo : INT32_MAX), hi = __reduce_max_sync(kFullMask, row.hi);
            const int32_t s = __reduce_min_sync(kFullMask, any ? row.s : INT32_MAX);
            if (lane == 0) { sh.limits[warp][0] = lo; sh.limits[warp][1] = hi; sh.limits[warp][2] = s; }
        } else if (p.b.n) {
            fill_bias(p, h, lut, warp - 4, 4, lane);
        }
    } else if (warp == 8) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&sh.tmem)), "r"(Sh::kAlloc));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    } else if (warp == 9 && lane == 0) {
        mbar_init(&sh.q_full, Sh::kQTmem ? 128 : 1);
        for (int i = 0; i < Sh::kStages; ++i) { mbar_init(&sh.landed[i], 1); mbar_init(&sh.full[i], 32); mbar_init(&sh.empty[i], 1 + 128); }
        for (int i = 0; i < 2; ++i) { mbar_init(&sh.s_full[i], 1); mbar_init(&sh.p_full[i], 128); }
        mbar_init(&sh.done, 1);
        mbar_init(&sh.still, 1);
        sh.abort_flag = sh.quiet = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_proxy();
        // a query that is not a word may hold anything: it spoils its own scores only, which are never used
        if (!Sh::kQTmem) {
            mbar_expect(&sh.q_full, Sh::kQBytes);
#pragma unroll
            for (int c = 0; c < NB; ++c) copy_box(qs + c * (128 * 128), &map_q, c * 64, (int32_t)h, t0, &sh.q_full);
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = warp_value(sh.tmem);
    volatile int *abort_flag = &sh.abort_flag;
    auto ready = [&](uint64_t *bar, uint32_t parity) { return SMALL ? mbar_wait(bar, parity, abort_flag) : mbar_nap(bar, parity, abort_flag); };
    // the run of keys [lo, hi) and the sinks [s, s_end) before it, which are the first tiles
    int32_t lo = INT32_MAX, hi = 0, s = INT32_MAX;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        lo = min(lo, sh.limits[w][0]);
        hi = max(hi, sh.limits[w][1]);
        s = min(s, sh.limits[w][2]);
    }
    lo = warp_value(lo);
    hi = warp_value(hi);
    s = warp_value(s);
    const int32_t s_end = hi ? min(s + p.sinks, lo) : 0;
    const int32_t extra = s < s_end ? (s_end - s + Sh::kRows - 1) / Sh::kRows : 0;
    const int32_t tiles = hi ? extra + (hi - lo + Sh::kRows - 1) / Sh::kRows : 0;
    auto tile_at = [&](int32_t t) { return t < extra ? s + t * Sh::kRows : lo + (t - extra) * Sh::kRows; };
    auto tile_keys = [&](int32_t t) { return min(Sh::kRows, (t < extra ? s_end : hi) - tile_at(t)); };

    if (warp < 8) {
        // ============ softmax: one row per thread, tiles in turn ============
        if (SMALL) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        const uint32_t wg = warp >> 2, lanes = ((warp & 3u) * 32u) << 16;
        const uint32_t cs = tmem + lanes + Sh::kS + wg * Sh::kRows, co = tmem + lanes + Sh::kO + wg * Sh::kWide;
        if (Sh::kQTmem && wg == 0) {
#pragma unroll
            for (int g = 0; g < NB * 2; ++g) {
                uint32_t x[16];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    const uint4 u = q_row[Sh::kQTmem ? g * 4 + c : 0];
                    x[c * 4] = u.x; x[c * 4 + 1] = u.y; x[c * 4 + 2] = u.z; x[c * 4 + 3] = u.w;
                }
                tmem_st16(tmem + lanes + Sh::kQ + g * 16, x);
            }
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(&sh.q_full);
        }
        const float scale = p.scale * kLog2e;
        const int32_t last = bias_last(p.b), w0 = t0 + (int32_t)(warp & 3u) * 32;
        const bool word = row.hi > row.lo;
        // keys that every row of the warp sees (rows that are not words do not matter)
        const int32_t all_lo = __reduce_max_sync(kFullMask, word ? row.lo : 0), all_hi = __reduce_min_sync(kFullMask, word ? row.hi : INT32_MAX);
        float ref = -INFINITY;
        float2 sum2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
        bool ok = true;
        for (int32_t t = (int32_t)wg; t < tiles; t += 2) {
            const int32_t k0 = tile_at(t), cols = tile_keys(t);
            const uint32_t stage = t % Sh::kStages;
            ok = __all_sync(kFullMask, ready(&sh.full[stage], (t / Sh::kStages) & 1) &&        // the bits of the keys
                                           ready(&sh.s_full[wg], (t >> 1) & 1));
            if (!ok) break;
            tc_fence_after();
            // far from the warp's rows every key of the tile has the bias of the side's last bucket
            const bool far_left = k0 + Sh::kRows - 1 - w0 <= -last, far = p.b.n == 0 || far_left || k0 - (w0 + 31) >= last;
            const float flat = p.b.n ? lut[far_left ? 0 : bias_entries(p.b) - 1] : 0.f;
            const uint32_t vis0 = sh.vis[stage][0], vis1 = Sh::kRows == 64 ? sh.vis[stage][1] : 0xFFFFFFFFu;
            // in a plain tile the bias joins the reference first; scores beside a bias far from zero lose their digits as in every
            // other tile, or not at all, so that only a bias that leaves nothing of them is taken there
            const bool hidden = flat <= kLowestBias;
            const bool plain = far && (fabsf(flat) <= kFarLse || hidden) && k0 >= all_lo && k0 + Sh::kRows <= all_hi && (vis0 & vis1) == 0xFFFFFFFFu;
            float top = -INFINITY, by = 1.f, add = 0.f;
            if (plain) {
                float m[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
                constexpr int kC = Sh::kRows / 32;
                uint32_t v[kC][32];
#pragma unroll
                for (int c = 0; c < kC; ++c) tmem_ld32(cs + c * 32, v[c]);
                tmem_wait_ld(v[0]);
                if (kC == 2) tmem_held(v[kC - 1]);
#pragma unroll
                for (int c = 0; c < kC; ++c)
#pragma unroll
                    for (int e = 0; e < 32; e += 2) {
                        float &x = m[(e >> 1) & 3];
                        x = fmaxf(x, fmaxf(__uint_as_float(v[c][e]), __uint_as_float(v[c][e + 1])));
                    }
                by = hidden ? 0.f : scale;
                top = fmaf(fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3])), by, flat);
                add = flat;
            } else {
#pragma unroll 1
                for (int c = 0; c < Sh::kRows / 32; ++c) {
                    if (c * 32 >= cols) break;
                    uint32_t v[32];
                    tmem_ld32(cs + c * 32, v);
                    tmem_wait_ld(v);
                    const int32_t at = k0 + c * 32;
                    const uint32_t m = (range_bits(row.lo, row.hi, at) | range_bits(row.s, row.se, at)) & (c ? vis1 : vis0);
                    if (far) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(fmaf(__uint_as_float(v[e]), scale, flat));
                    } else {
                        const float *near = lut + (at - (int32_t)own + last + kBiasPad);
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(fmaf(__uint_as_float(v[e]), scale, near[e]));
                    }
                    if (!__all_sync(kFullMask, m == 0xFFFFFFFFu)) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = m & (1u << e) ? v[e] : 0xFF800000u;      // -infinity
                    }
                    float n[4] = {top, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                    for (int e = 0; e < 32; e += 2) n[(e >> 1) & 3] = fmaxf(n[(e >> 1) & 3], fmaxf(__uint_as_float(v[e]), __uint_as_float(v[e + 1])));
                    top = fmaxf(fmaxf(n[0], n[1]), fmaxf(n[2], n[3]));
                    tmem_st32(cs + c * 32, v);
                }
                tmem_wait_st();
            }
            const bool grown = top > ref + kRescale || (ref == -INFINITY && top > ref);
            if (__any_sync(kFullMask, grown)) {
                const float to = grown ? top : ref, keep = ref == -INFINITY ? 0.f : fast_exp2(ref - to);
                ref = to;
                sum2[0].x *= keep; sum2[0].y *= keep; sum2[1].x *= keep; sum2[1].y *= keep;
                if (t >= 2) {                                        // the scores came after the warpgroup's last product with values: the output is still
                    for (uint32_t c = 0; c < dim16; c += 16) {
                        uint32_t o[16];
                        tmem_ld16(co + c, o);
                        tmem_wait_ld(o);
#pragma unroll
                        for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * keep);
                        tmem_st16(co + c, o);
                    }
                }
            }
            add -= ref == -INFINITY ? 0.f : ref;
            const float2 by2 = make_float2(by, by), add_2 = make_float2(add, add);
#pragma unroll
            for (int c = 0; c < Sh::kRows / 32; ++c) {
                if (c * 32 < cols) {
                    uint32_t v[32], w[16];
                    tmem_ld32(cs + c * 32, v);
                    tmem_wait_ld(v);
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float2 x = fma2(pair_of(v[2 * e], v[2 * e + 1]), by2, add_2);
                        x.x = fast_exp2(x.x);
                        x.y = fast_exp2(x.y);
                        sum2[e & 1] = add2(sum2[e & 1], x);
                        w[e] = pack2<T>(x.x, x.y);
                    }
                    tmem_st16(cs + c * 16, w);                       // over scores that have been read
                }
            }
            tmem_wait_st();
            tc_fence_before();
            mbar_arrive(&sh.p_full[wg]);
            mbar_arrive(&sh.empty[stage]);                           // this thread is done with the stage's bits
        }
        // the two warpgroups' rows are joined: each takes half of the columns of every row
        const float mine = (sum2[0].x + sum2[0].y) + (sum2[1].x + sum2[1].y);
        sh.ref[wg][r] = word ? ref : -INFINITY;                      // what a row that is not a word holds may be anything
        sh.sum[wg][r] = word ? mine : 0.f;
        asm volatile("bar.sync 1, 256;" ::: "memory");
        const float r0 = sh.ref[0][r], r1 = sh.ref[1][r], to = fmaxf(r0, r1);
        // a block without a word has no products, but its queries land where the output is staged
        ok = __all_sync(kFullMask, ok && (tiles ? ready(&sh.done, 0) : Sh::kQTmem || ready(&sh.q_full, 0)));
        tc_fence_after();
        float f0 = to == -INFINITY ? 0.f : fast_exp2(r0 - to), f1 = to == -INFINITY ? 0.f : fast_exp2(r1 - to);
        const float total = sh.sum[0][r] * f0 + sh.sum[1][r] * f1, inv = total == 0.f ? 0.f : 1.f / total;
        const float lse = total == 0.f ? INFINITY : to + log2f(total);      // a sum that is NaN stays one
        if (p.lse && wg == 0 && own < p.n) p.lse[(int64_t)h * p.n + own] = lse;
        f0 *= inv;
        f1 *= inv;
        // out through shared memory (every tile is read by now), a row of 16-byte chunks at a time
        const uint32_t row_bytes = p.dim * 2u, part = (warp & 3u) * 32u;
        unsigned char *stripe = smem + part * row_bytes, *line = stripe + lane * row_bytes;
        const uint32_t turn = lane % dch;                            // chunks are turned by the row: fewer bank conflicts
        float2 zero = make_float2(0.f, 0.f);                         // NaN once an output is not finite
#pragma unroll
        for (int i = 0; i < NB * 2; ++i) {
            const uint32_t c = i * 32 + wg * 16;
            if (c >= dim16) break;
            uint32_t a[16], b[16];
            tmem_ld16(tmem + lanes + Sh::kO + c, a);
            tmem_ld16(tmem + lanes + Sh::kO + Sh::kWide + c, b);
            tmem_wait_ld(a);
            tmem_wait_ld(b);
            float o[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) {                           // an accumulator that no tile was added to holds anything
                const float x = f0 == 0.f ? 0.f : __uint_as_float(a[e]) * f0;
                o[e] = f1 == 0.f ? x : fmaf(__uint_as_float(b[e]), f1, x);
            }
#pragma unroll
            for (int e = 0; e < 16; e += 2) zero = fma2(make_float2(o[e], o[e + 1]), make_float2(0.f, 0.f), zero);
#pragma unroll
            for (int g = 0; g < 2; ++g)
                if (c + g * 8 < p.dim) {
                    uint4 w;
                    w.x = pack2<T>(o[g * 8], o[g * 8 + 1]); w.y = pack2<T>(o[g * 8 + 2], o[g * 8 + 3]);
                    w.z = pack2<T>(o[g * 8 + 4], o[g * 8 + 5]); w.w = pack2<T>(o[g * 8 + 6], o[g * 8 + 7]);
                    const uint32_t ch = (c >> 3) + g + turn;
                    *reinterpret_cast<uint4 *>(line + (ch >= dch ? ch - dch : ch) * 16u) = w;
                }
        }
        uint32_t bad = __ballot_sync(kFullMask, ok && zero.x + zero.y != 0.f && own < p.n && lse == lse);
        const bool again = any_of_64(2u + (warp & 3u), bad != 0u);  // the two warps of these rows
        store_rows(static_cast<char *>(p.out) + ((uint64_t)(t0 + part) * p.ldo + (uint64_t)h * p.dim) * 2u, p.ldo * 2u, stripe, dch,
                   (int32_t)min((int64_t)32, p.n - (int64_t)(t0 + part)), wg * 32u + lane, 64u);
        if (again) {                                                 // both warps or neither
            asm volatile("bar.sync %0, 64;" ::"r"(2u + (warp & 3u)) : "memory");     // over what has been stored
#pragma unroll 1
            for (; bad; bad &= bad - 1u) {                           // a row that both warps found is written twice, the same
                const int32_t x = __ffs(bad) - 1;
                output_again<T>(p, h, kvh, (int64_t)t0 + part + x, __shfl_sync(kFullMask, to, x), __shfl_sync(kFullMask, inv, x), lane);
            }
        }
        tc_fence_before();
    } else if (warp == 8) {
        // ============ MMA issue: one lane ============
        if (SMALL) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        // The whole block waits for this warp when its code is long: everything that does not change is formed once, a
        // product costs an addition per operand, and the warp stays together, so that addresses and descriptors are
        // formed in uniform registers, where the instruction wants them; one lane issues.
        if (tiles) {
            const bool leader = elect_one();
            constexpr uint32_t kBlock = Sh::kRows * 128, kStep = Sh::kStage >> 4;
            const uint32_t idesc_o = umma_idesc_f16(kBf16, kAttendTile, dim16, true), idesc_s = umma_idesc_f16(kBf16, kAttendTile, Sh::kRows, false);
            const uint32_t q_low = umma_desc_low(qs, 0), k_low = umma_desc_low(ring, 0), v_low = umma_desc_low(ring + Sh::kOperand, kBlock);
            // keys past the tile's end are products of what lies there and are masked
            auto scores = [&](uint32_t b, uint32_t stage) {
                const uint32_t k = k_low + stage * kStep, d = tmem + Sh::kS + b * Sh::kRows;
#pragma unroll
                for (int c = 0; c < NB * 4; ++c)
                    if ((uint32_t)c * 16 < dim16) {
                        const uint32_t k_at = k + (c >> 2) * (kBlock >> 4) + (c & 3) * 2;
                        if (Sh::kQTmem) umma_f16_ts(d, tmem + Sh::kQ + c * 8, k_at, idesc_s, c > 0);
                        else umma_f16_ss(d, q_low + (c >> 2) * (kAttendTile * 128 >> 4) + (c & 3) * 2, k_at, idesc_s, c > 0);
                    }
                umma_commit(&sh.s_full[b]);
            };
            auto wait = [&](uint64_t *bar, uint32_t parity) {
                const bool got = __all_sync(kFullMask, ready(bar, parity));
                tc_fence_after();
                return got;
            };
            bool ok = wait(&sh.q_full, 0);
            uint32_t ahead = 0, ahead_phase = 0;                     // stage and phase of the next scores, two tiles ahead of the products with values
            for (int32_t t = 0; t < 2 && t < tiles && ok; ++t) {
                ok = wait(&sh.full[ahead], 0);
                if (ok && leader) scores((uint32_t)t, ahead);
                __syncwarp();
                ++ahead;
            }
            uint32_t stage = 0;
            for (int32_t t = 0; t < tiles && ok; ++t) {
                const uint32_t b = t & 1, v = v_low + stage * kStep, w = tmem + Sh::kS + b * Sh::kRows, d = tmem + Sh::kO + b * Sh::kWide;
                const int32_t keys = tile_keys(t);
                ok = wait(&sh.p_full[b], (t >> 1) & 1);
                if (!ok) break;
                if (leader) {
#pragma unroll
                    for (int k = 0; k < Sh::kRows / 16; ++k)
                        if (k * 16 < keys) umma_f16_ts(d, w + k * 8, v + k * 128, idesc_o, t > 1 || k > 0);
                    umma_commit(&sh.empty[stage]);
                    if (t + 1 == tiles) umma_commit(&sh.done);
                }
                __syncwarp();
                if (++stage == Sh::kStages) stage = 0;
                if (t + 2 < tiles) {
                    ok = wait(&sh.full[ahead], ahead_phase);
                    if (!ok) break;
                    if (leader) scores(b, ahead);
                    __syncwarp();
                    if (++ahead == Sh::kStages) { ahead = 0; ahead_phase ^= 1u; }
                }
            }
        }
        __syncwarp();
    } else if (warp == 9) {
        // ============ copies: one lane ============
        if (SMALL) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (lane == 0) {
            int32_t t = 0;
            for (; t < tiles; ++t) {
                const uint32_t stage = t % Sh::kStages, round = t / Sh::kStages, base = ring + stage * Sh::kStage;
                if (round > 0 && !mbar_nap(&sh.empty[stage], (round - 1) & 1, abort_flag)) break;
                mbar_expect(&sh.landed[stage], Sh::kStage);
#pragma unroll
                for (int c = 0; c < NB; ++c) {
                    copy_box(base + c * Sh::kRows * 128, &map_k, c * 64, (int32_t)kvh, tile_at(t), &sh.landed[stage]);
                    copy_box(base + Sh::kOperand + c * Sh::kRows * 128, &map_v, c * 64, (int32_t)kvh, tile_at(t), &sh.landed[stage]);
                }
            }
            issued = t;
        }
        __syncwarp();
    } else {
        // ============ rows that are not words: a warp per tile, in turn ============
        if (SMALL) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        int32_t t = (int32_t)warp - 10;
        uint32_t vis[2] = {0u, 0u};
        if (t < tiles) word_bits(p, tile_at(t), (uint32_t)tile_keys(t), lane, vis);
        for (; t < tiles; t += 2) {
            const uint32_t stage = t % Sh::kStages;
            if (!__all_sync(kFullMask, mbar_nap(&sh.landed[stage], (t / Sh::kStages) & 1, abort_flag))) break;
            if (lane < 2) sh.vis[stage][lane] = lane ? vis[1] : vis[0];
            // values only: the scores of such a key are masked
            zero_rows<NB>(ring + stage * Sh::kStage + Sh::kOperand, Sh::kRows * 128, (uint32_t)(tile_keys(t) + 15) & ~15u, vis, lane);
            fence_async_proxy();
            mbar_arrive(&sh.full[stage]);
            if (t + 2 < tiles) word_bits(p, tile_at(t + 2), (uint32_t)tile_keys(t + 2), lane, vis);
        }
    }
    __syncthreads();
    tc_fence_after();
    if (sh.abort_flag) {
        // a wait ran out: the copies and products under way end (or have as long again) before the block leaves what they use
        if (warp == 9 && lane == 0) {
            if (!Sh::kQTmem) mbar_wait(&sh.q_full, 0, &sh.quiet);
            for (int32_t u = max(0, issued - Sh::kStages); u < issued; ++u) mbar_wait(&sh.landed[u % Sh::kStages], (u / Sh::kStages) & 1, &sh.quiet);
        } else if (warp == 8) {
            if (elect_one()) umma_commit(&sh.still);
            __syncwarp();
            mbar_wait(&sh.still, 0, &sh.quiet);
        }
        __syncthreads();
    }
    if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(Sh::kAlloc));
    if (tid == 0 && sh.abort_flag) atomicOr(error, kErrAttend);
}

template <typename T, int NB, bool SMALL>
int launch_attend_shape(const AttendParams &p, int *error, cudaStream_t s)
{
    auto kernel = attend_tc_kernel<T, NB, SMALL>;
    using Sh = FwdShape<NB, SMALL>;
    int smem = Sh::kRing + 1024 + (int)(bias_entries(p.b) * sizeof(float));
    if (Sh::kBlocks == 1 && smem < 116 * 1024) smem = 116 * 1024;      // a second block would only wait for tensor memory
    if (!kernel_ready<attend_tc_kernel<T, NB, SMALL>>(SMALL ? kLaunchRegs : 0)) return -1;
    const uint64_t tiles = ((uint64_t)p.n + kAttendTile - 1) / kAttendTile;
    CUtensorMap q, k, v;
    const bool bf16 = std::is_same<T, __nv_bfloat16>::value;
    if (!make_rows_map(&q, bf16, p.q, p.dim, p.heads, (uint64_t)p.n, p.ldq, kAttendTile) ||
        !make_rows_map(&k, bf16, p.k, p.dim, p.kv_heads, (uint64_t)p.n, p.ldk, Sh::kRows) ||
        !make_rows_map(&v, bf16, p.v, p.dim, p.kv_heads, (uint64_t)p.n, p.ldv, Sh::kRows))
        return -1;
    kernel<<<(uint32_t)(tiles * p.heads), kFwdThreads, smem, s>>>(q, k, v, p, error);
    return cudaPeekAtLastError() == cudaSuccess ? 1 : -1;
}

int launch_attend(const AttendParams &p, uint32_t type, int *error, int, cudaStream_t s)
{
    if (p.n == 0) return 0;
    auto shape = [&](auto element) {
        using T = decltype(element);
        return p.dim <= 64 ? launch_attend_shape<T, 1, true>(p, error, s)
               : p.dim <= 96 ? launch_attend_shape<T, 2, true>(p, error, s) : launch_attend_shape<T, 2, false>(p, error, s);
    };
    return type == kBF16 ? shape(__nv_bfloat16()) : shape(__half());
}

}  // namespace w2v
