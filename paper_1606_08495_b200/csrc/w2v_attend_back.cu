// Attention backwards on the tensor cores.
//
// With P = exp2(S - lse) and dP = dO V^T:  dS = P (dP - delta), delta = rowsum(P dP) = rowsum(dO o),
//   dQ = scale dS K,  dK = scale dS^T Q,  dV = P^T dO,  dbias[b] = sum of dS over the pairs of bucket b.
// (A far row, whose lse cannot hold its sum's digits, has weights that are all off by one factor; role 0 adds them up and puts
// its own results right, role 1 takes the factor from there.)
// Two passes over the scores, so that nothing is added up with atomics and the same inputs give the same bits:
//   role 0, a block per 128 queries: dQ and delta.  The rounded o gives a first delta; the row's sum of dS, which is
//           zero for an exact one, says how far it is off, and dQ is put right with the product P K that is formed
//           beside dS K.  The delta kept for role 1 is so good to fp32: dbias sums cancel so far that they need it.
//   role 1, a block per 128 keys and key/value head: dK, dV (all query heads that share them) and dbias.
// Both keep two operands of their 128 rows in tensor memory (A sides), stream the other two through shared memory
// and form both score products of a tile; a warpgroup turns them into P and dS, one row per thread, and puts those
// back into tensor memory as the A sides of the gradient products, whose B sides are the streamed tiles again, read
// with rows as the summed side.  Keys that are sinks of queries far behind them get what those add from role 0, as
// sums over its 128 queries (the tile of the sinks is there anyway), which a small kernel adds up for role 1.
//
// P and dS are rounded to the arrays' type as A sides of the gradient products; dbias, delta and the sinks' sums take them in
// fp32.  Bound by latency in the warpgroups (issue slots 40 %, matrix units 35 % busy): 16,381 words, 16 heads of 128 (4 of
// keys and values), windows of 1,024: 420 us (role 0) and 427 us (role 1).
#include <type_traits>

#include "w2v_attend.cuh"
#include "w2v_kernel_ready.h"

namespace w2v {

// Two layouts of a block.
//   SMALL (heads of up to 96): 256 columns of tensor memory and half of the shared memory, so that two blocks share an SM
//          and one's beginning and end lie under the other's middle; the A sides stay in shared memory; the two softmax
//          warpgroups take half of the columns of every tile.  Against the other, role 1 and role 0: 131,072
//          words in sessions of 5 to 40, 4 heads of 80, 370 -> 284 us and 270 -> 220 us; 65,536 words in sentences of 1,000, 5
//          heads of 64, windows of 257, 312 -> 217 us and 262 -> 201 us (with what came since 290, 229, 227 and 208).
//   else:  all of the tensor memory; the A sides in tensor memory; the warpgroups take the tiles in turn.
template <int NB, bool SMALL>
struct BackShape {
    static constexpr int kTile = SMALL ? 256 : 128;                  // softmax threads that share a tile
    static constexpr int kBuf = SMALL && NB == 2 ? 1 : 2;            // score buffers
    static constexpr int kRows = 32;                                 // streamed rows per tile
    static constexpr int kChunk = SMALL ? kRows / 2 : kRows;         // columns of a tile that a thread takes
    static_assert(SMALL || NB == 2, "heads of up to 64 are SMALL");
    static constexpr int kStages = SMALL && NB == 2 ? 2 : 4;
    static constexpr uint32_t kWide = !SMALL ? NB * 64 : NB == 1 ? 64 : 96;              // columns of a gradient
    static constexpr uint32_t kA0 = 0, kA1 = NB * 32, kG0 = SMALL ? 0 : NB * 64, kG1 = kG0 + kWide;      // tensor-memory columns
    static constexpr uint32_t kScores = kG1 + kWide, kAlloc = SMALL ? 256 : 512;
    static_assert(kScores + kBuf * 2 * kRows <= kAlloc, "tensor memory");
    static constexpr int kOperand = NB * kRows * 128, kStage = 2 * kOperand, kRing = kStages * kStage;
    static constexpr int kOwn = NB * 128 * 128;                      // bytes of one operand of the block's own rows
    static constexpr int kSoft = 256, kThreads = kSoft + 128, kBlocks = 512 / (int)kAlloc;
    static_assert(kRing + 2 * kOwn >= 2 * NB * 128 * 128, "the outputs are staged where the ring and the own rows were");
};
// SMALL: of the 80 registers a thread has at launch, the helpers' warpgroup gives what it has beyond 48 to the two of
// the softmax (96 + 96 + 48 = 3 x 80).
constexpr int kBackLaunchRegs = 80, kBackSoftRegs = 96, kBackOtherRegs = 48;

template <typename Sh>
struct BackShared {
    uint64_t own_landed, own_full, landed[Sh::kStages], full[Sh::kStages], empty[Sh::kStages], s_full[2], p_full[2], done, still;
    uint32_t tmem;
    int abort_flag, quiet;
    int32_t limits[4][3];
    uint32_t vis[Sh::kStages];                       // which streamed rows of the stage are words
    int32_t run_lo[Sh::kStages];                     // role 1: where the run of the stage's query tile begins
    __align__(16) float lse[Sh::kStages][Sh::kRows], delta[Sh::kStages][Sh::kRows], extra[Sh::kStages][Sh::kRows];       // role 1: of the stage's queries, negated
    int far[Sh::kStages];                            // role 1: there are far rows among them
    float far_sum[8][2];
};

__device__ __forceinline__ void soft_barrier(int threads) { asm volatile("bar.sync 1, %0;" ::"r"(threads) : "memory"); }

// Sums per distance (`off` on either side of 0) and the warps' far sums over the distances of each bucket; warp w of
// `warps` takes buckets w, w + warps, ...
__device__ __forceinline__ void write_bucket_sums(const AttendParams &p, const float *sums, int32_t off, const float (*far_sum)[2],
                                                  uint32_t warp, uint32_t warps, uint32_t lane, float *out)
{
    const uint32_t n = p.b.n, buckets = n * (p.b.two_sided ? 2u : 1u);
    const float far_l = lane < warps ? far_sum[lane][0] : 0.f, far_r = lane < warps ? far_sum[lane][1] : 0.f;
    for (uint32_t b = warp; b < buckets; b += warps) {
        const uint32_t side = b >= n ? 1u : 0u, k = b - side * n;
        int32_t r0, r1;
        bucket_range(p.b, b, off, r0, r1);
        float a[4] = {0.f, 0.f, 0.f, 0.f};
        for (int32_t r = r0 + (int32_t)lane; r < r1; r += 128) {
#pragma unroll
            for (int i = 0; i < 4; ++i) if (r + i * 32 < r1) a[i] += sums[r + i * 32 + off];
        }
        float t = (a[0] + a[1]) + (a[2] + a[3]);
        if (side == 0 && k == n - 1) t += far_l;
        if (p.b.two_sided ? side == 1 && k == n - 1 : k == 0) t += far_r;
        t = warp_sum(t);
        if (lane == 0) out[b] = t;
    }
}

// What this block's queries add to the sinks before its run: dK (before the scale) and dV of each, and the bias' sums,
// by the softmax threads.  sink_d holds dS for the first delta, which eps puts right, sink_p the weights; `by` puts a far row
// right.  A thread takes two columns
// and a part of the rows, four sinks at a time; `red` is 16 KB for joining the parts.
template <typename T, int NB, int kSoft>
__device__ __forceinline__ void sink_sums(const AttendParams &p, unsigned char *own_rows, float *sink_p, float *sink_d,
                                       RowLimits row, float eps, float by, float *red, int32_t sinks, int32_t s, int32_t t0, uint32_t wg, uint32_t r,
                                       uint32_t tid, float *out, float *bias_out)
{
    constexpr int kPairs = 32 * NB, kParts = kSoft / kPairs, kPartRows = 128 / kParts, kOwn = NB * 128 * 128;
    // a row of another sentence, or one that has all these sinks in its window, takes no part, whatever it holds
    const bool part_of = row.s == s && row.s < row.se;
    for (int32_t k = (int32_t)wg; k < sinks; k += kSoft / 128) {
        const int32_t at = k * 128 + (int32_t)r;
        // nor does any with a sink that is not a word: its weight is zero, but eps may not be finite
        sink_d[at] = part_of && is_word(p, s + k) ? fmaf(-eps, sink_p[at], sink_d[at]) * by : 0.f;
        if (by != 1.f) sink_p[at] *= by;
    }
    if (!part_of)
#pragma unroll
        for (int c = 0; c < NB * 8; ++c)
            *reinterpret_cast<uint4 *>(own_rows + wg * kOwn + (c >> 3) * (128 * 128) + r * 128u + ((c & 7) << 4)) = make_uint4(0, 0, 0, 0);
    soft_barrier(kSoft);
    const uint32_t pair = tid % kPairs, part = tid / kPairs, width = 2 * p.dim;
    for (int32_t k0 = 0; k0 < sinks; k0 += 4) {
        float2 a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) a[i] = b[i] = make_float2(0.f, 0.f);
        if (2 * pair < p.dim) {
#pragma unroll 2
            for (uint32_t x0 = part * kPartRows; x0 < (part + 1) * kPartRows; x0 += 4) {
                float2 q[4], g[4];
#pragma unroll
                for (uint32_t y = 0; y < 4; ++y) {
                    const uint32_t x = x0 + y, at = (pair >> 5) * (128 * 128) + x * 128u + (((((pair & 31u) >> 2) ^ (x & 7u)) << 4) | ((pair & 3u) << 2));
                    const Pack<T, 2> u = *reinterpret_cast<const Pack<T, 2> *>(own_rows + at), w = *reinterpret_cast<const Pack<T, 2> *>(own_rows + kOwn + at);
                    q[y] = make_float2(to_f32(u.e[0]), to_f32(u.e[1]));
                    g[y] = make_float2(to_f32(w.e[0]), to_f32(w.e[1]));
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (k0 + i < sinks) {
                        const float4 d = *reinterpret_cast<const float4 *>(sink_d + (k0 + i) * 128 + x0), w = *reinterpret_cast<const float4 *>(sink_p + (k0 + i) * 128 + x0);
                        a[i] = fma2(make_float2(d.x, d.x), q[0], a[i]); a[i] = fma2(make_float2(d.y, d.y), q[1], a[i]);
                        a[i] = fma2(make_float2(d.z, d.z), q[2], a[i]); a[i] = fma2(make_float2(d.w, d.w), q[3], a[i]);
                        b[i] = fma2(make_float2(w.x, w.x), g[0], b[i]); b[i] = fma2(make_float2(w.y, w.y), g[1], b[i]);
                        b[i] = fma2(make_float2(w.z, w.z), g[2], b[i]); b[i] = fma2(make_float2(w.w, w.w), g[3], b[i]);
                    }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                *reinterpret_cast<float2 *>(red + (part * 4 + i) * width + 2 * pair) = a[i];
                *reinterpret_cast<float2 *>(red + (part * 4 + i) * width + p.dim + 2 * pair) = b[i];
            }
        }
        soft_barrier(kSoft);
        for (uint32_t i = tid; i < 4 * width; i += kSoft) {
            float x = 0.f;
#pragma unroll
            for (int y = 0; y < kParts; ++y) x += red[y * 4 * width + i];
            if (k0 * width + i < (uint32_t)p.sinks * width) out[k0 * width + i] = x;       // sinks that the tile does not have: zeros
        }
        soft_barrier(kSoft);
    }
    for (uint32_t i = tid + (((uint32_t)sinks + 3u) & ~3u) * width; i < (uint32_t)p.sinks * width; i += kSoft) out[i] = 0.f;
    if (!bias_out) return;
    // sums by distance first: key - query runs over sinks + 127 values; then by bucket
    uint32_t *of = reinterpret_cast<uint32_t *>(red + 256);
    const int32_t least = s - (t0 + 127), count = sinks + 127;
    for (int32_t i = (int32_t)tid; i < count; i += kSoft) {
        float x = 0.f;
        for (int32_t k = 0; k < sinks; ++k) {
            const int32_t q = s + k - (least + i) - t0;              // the query of this key at this distance
            if (q >= 0 && q < 128) x += sink_d[k * 128 + q];
        }
        red[i] = x;
        of[i] = bucket_of(p.b, least + i);
    }
    soft_barrier(kSoft);
    const uint32_t lane = tid & 31u, buckets = p.b.n * (p.b.two_sided ? 2u : 1u);
    for (uint32_t b = tid >> 5; b < buckets; b += kSoft / 32) {
        float x = 0.f;
        for (int32_t i = (int32_t)lane; i < count; i += 32) if (of[i] == b) x += red[i];
        x = warp_sum(x);
        if (lane == 0) bias_out[b] = x;
    }
}

// Where the run of keys of the query tile that begins at q0 begins; by a warp.
__device__ __forceinline__ int32_t run_begin(const AttendParams &p, int32_t q0, uint32_t lane)
{
    uint32_t a[2], b[2];
    word_bits(p, q0, 64, lane, a);
    word_bits(p, (int64_t)q0 + 64, 64, lane, b);
    const int32_t first = a[0] ? __ffs(a[0]) - 1 : a[1] ? 31 + __ffs(a[1]) : b[0] ? 63 + __ffs(b[0]) : 95 + __ffs(b[1]);
    return (a[0] | a[1] | b[0] | b[1]) ? row_limits(p, q0 + first).lo : INT32_MAX;
}

// dQ of row i by a warp, from the pairs that it sees.
template <typename T>
__device__ __forceinline__ void dq_again(const AttendParams &p, uint32_t h, uint32_t kvh, int64_t i, float lse, float by, float delta, uint32_t lane)
{
    const RowLimits row = row_limits(p, i);
    const T *q = static_cast<const T *>(p.q) + i * (int64_t)p.ldq + h * p.dim, *d_o = static_cast<const T *>(p.d_o) + i * (int64_t)p.ld_do + h * p.dim;
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
            if (seen) {
                w = fast_exp2(fmaf(row_dot(q, k + j * (int64_t)p.ldk, p.dim), p.scale * kLog2e, pair_bias(p, h, (int32_t)(j - i))) - lse) * by;
                w *= row_dot(d_o, v + j * (int64_t)p.ldv, p.dim) - delta;
            }
            add_rows(acc, w, __ballot_sync(kFullMask, seen), k + j0 * (int64_t)p.ldk, p.ldk, p.dim, lane);
        }
    }
    T *out = static_cast<T *>(p.dq) + i * (int64_t)p.ld_dq + h * p.dim;
#pragma unroll
    for (int x = 0; x < 4; ++x)
        if (lane + 32u * x < p.dim) out[lane + 32u * x] = from_f32<T>(acc[x] * p.scale);
}

// dK (which = 0) or dV of key j by a warp, from the queries that see it; `sink`: what queries far behind add.
template <typename T>
__device__ __forceinline__ void dkv_again(const AttendParams &p, uint32_t which, uint32_t kvh, int64_t j, const float *sink, uint32_t lane)
{
    const int2 sp = word_span(p, j);
    const uint32_t group = p.heads / p.kv_heads;
    const T *k = static_cast<const T *>(p.k) + j * (int64_t)p.ldk + kvh * p.dim, *v = static_cast<const T *>(p.v) + j * (int64_t)p.ldv + kvh * p.dim;
    const int64_t lo = max((int64_t)sp.x, j - p.right), hi = min((int64_t)sp.y, j + p.left + 1), tile = (j + p.left) / kAttendTile;
    int64_t end = hi;                                                // and as a sink up to here, as in the tiles
    if (j - sp.x < p.sinks && hi < sp.y && run_begin(p, (int32_t)(tile * kAttendTile), lane) <= j) end = max(hi, min((int64_t)sp.y, (tile + 1) * kAttendTile));
    float acc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (uint32_t h = kvh * group; h < (kvh + 1) * group; ++h) {
        const T *q = static_cast<const T *>(p.q) + h * p.dim, *d_o = static_cast<const T *>(p.d_o) + h * p.dim;
#pragma unroll 1
        for (int64_t i0 = lo; i0 < end && !all_nan(acc, p.dim, lane); i0 += 32) {
            const int64_t i = i0 + lane;
            const bool seen = i < end && is_word(p, i);
            float w = 0.f;
            if (seen) {
                w = fast_exp2(fmaf(row_dot(q + i * (int64_t)p.ldq, k, p.dim), p.scale * kLog2e, pair_bias(p, h, (int32_t)(j - i))) - __ldg(p.lse + (int64_t)h * p.n + i) - p.extra[(int64_t)h * p.n + i]);
                if (which == 0) w *= row_dot(d_o + i * (int64_t)p.ld_do, v, p.dim) - p.delta[(int64_t)h * p.n + i];
            }
            const uint32_t live = __ballot_sync(kFullMask, seen);
            if (which == 0) add_rows(acc, w, live, q + i0 * (int64_t)p.ldq, p.ldq, p.dim, lane);
            else add_rows(acc, w, live, d_o + i0 * (int64_t)p.ld_do, p.ld_do, p.dim, lane);
        }
    }
    T *out = which == 0 ? static_cast<T *>(p.dk) + j * (int64_t)p.ld_dk + kvh * p.dim : static_cast<T *>(p.dv) + j * (int64_t)p.ld_dv + kvh * p.dim;
#pragma unroll
    for (int x = 0; x < 4; ++x)
        if (lane + 32u * x < p.dim) out[lane + 32u * x] = from_f32<T>((acc[x] + (sink ? sink[lane + 32u * x] : 0.f)) * (which == 0 ? p.scale : 1.f));
}

template <typename T, int NB, int ROLE, bool SMALL>
__global__ void __launch_bounds__(BackShape<NB, SMALL>::kThreads, BackShape<NB, SMALL>::kBlocks)
attend_back_kernel(const __grid_constant__ CUtensorMap map_x, const __grid_constant__ CUtensorMap map_y,
                   const __grid_constant__ CUtensorMap map_a0, const __grid_constant__ CUtensorMap map_a1,
                   const __grid_constant__ CUtensorMap map_o, AttendParams p, int *error)
{
    using Sh = BackShape<NB, SMALL>;
    constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
    extern __shared__ unsigned char smem_raw[];
    __shared__ BackShared<Sh> sh;
    unsigned char *smem = smem_raw + ((1024u - (smem_addr(smem_raw) & 1023u)) & 1023u);
    const uint32_t ring = smem_addr(smem);
    unsigned char *own_rows = smem + Sh::kRing;                      // the two A sides, and o in role 0 (not SMALL), as they land
    float *lut = reinterpret_cast<float *>(smem + Sh::kRing + 2 * Sh::kOwn + (ROLE == 0 ? max(SMALL ? 0 : Sh::kOwn, p.sinks * 1024) : 0));
    const uint32_t entries = bias_entries(p.b);
    float *rel_sums = lut + ((entries + 3u) & ~3u);                  // role 1: [softmax warps][entries]; role 0: [2][warpgroups][rows], parts of what is added up

    const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const uint32_t group = p.heads / p.kv_heads, across = ROLE == 0 ? p.heads : p.kv_heads;
    const uint32_t h_own = blockIdx.x % across, kvh = ROLE == 0 ? h_own / group : h_own;
    const int32_t tile = (int32_t)(blockIdx.x / across), t0 = tile * kAttendTile;
    const uint32_t heads_here = ROLE == 0 ? 1u : group, h0 = ROLE == 0 ? h_own : kvh * group;
    const uint32_t dim16 = (p.dim + 15u) & ~15u;
    constexpr uint32_t kSoftWarps = Sh::kSoft / 32, kMmaWarp = kSoftWarps;
    int32_t issued = 0;                                              // tiles whose copies were started (the copying lane's)

    if (warp == kMmaWarp + 1 && lane == 0) {
        mbar_init(&sh.own_landed, 1);
        mbar_init(&sh.own_full, SMALL ? 64 : 256);
        for (int i = 0; i < Sh::kStages; ++i) { mbar_init(&sh.landed[i], 1); mbar_init(&sh.full[i], 32); mbar_init(&sh.empty[i], 1 + Sh::kTile); }
        for (int i = 0; i < 2; ++i) { mbar_init(&sh.s_full[i], 1); mbar_init(&sh.p_full[i], Sh::kTile); }
        mbar_init(&sh.done, 1);
        mbar_init(&sh.still, 1);
        sh.abort_flag = sh.quiet = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        fence_async_proxy();
        mbar_expect(&sh.own_landed, (ROLE == 0 && !SMALL ? 3 : 2) * Sh::kOwn);
#pragma unroll
        for (int c = 0; c < NB; ++c) {
            const uint32_t to = ring + Sh::kRing + c * (128 * 128);
            copy_box(to, &map_a0, c * 64, (int32_t)h_own, t0, &sh.own_landed);
            copy_box(to + Sh::kOwn, &map_a1, c * 64, (int32_t)h_own, t0, &sh.own_landed);
            if (ROLE == 0 && !SMALL) copy_box(to + 2 * Sh::kOwn, &map_o, c * 64, (int32_t)h_own, t0, &sh.own_landed);
        }
    }
    const uint32_t r = tid & 127u;                                   // this thread's row (softmax warps)
    const int64_t own = (int64_t)t0 + r;
    RowLimits row = {0, 0, 0, 0};                                    // role 0: what the query sees
    int32_t q_lo = 0, q_hi = 0, far_lo = 0, far_hi = 0, sent = 0;    // role 1: queries that see the key; far: as a sink
    if (warp < kSoftWarps) {
        int32_t least = INT32_MAX, most = 0, s = INT32_MAX;
        if (ROLE == 0) {
            row = row_limits(p, own);
            if (row.hi > row.lo) { least = row.lo; most = row.hi; s = row.s; }
        } else if (own < p.n) {
            const int2 sp = word_span(p, own);
            if (sp.y > sp.x) {
                sent = sp.x;
                q_lo = (int32_t)max((int64_t)sp.x, own - p.right);
                q_hi = (int32_t)min((int64_t)sp.y, own + p.left + 1);
                least = q_lo; most = q_hi;
                if (own - sp.x < p.sinks) {
                    // as a sink it is also seen from beyond the window; of those queries, this block takes the ones whose
                    // tile's run reaches back to the key, all in the tile of the last query of the window
                    far_lo = q_hi;
                    far_hi = (int32_t)min((int64_t)sp.y, ((own + p.left) / kAttendTile + 1) * kAttendTile);
                    far_hi = max(far_hi, far_lo);
                    most = far_hi;
                }
            }
        }
        if (warp < 4) {
            least = __reduce_min_sync(kFullMask, least);
            most = __reduce_max_sync(kFullMask, most);
            s = __reduce_min_sync(kFullMask, s);
            if (lane == 0) { sh.limits[warp][0] = least; sh.limits[warp][1] = most; sh.limits[warp][2] = s; }
        }
    }
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&sh.tmem)), "r"(Sh::kAlloc));
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    uint32_t own_words[4];
    if (SMALL && warp >= kMmaWarp + 2) {
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            const int64_t i = (int64_t)t0 + w * 32 + lane;
            const int2 sp = i < p.n ? word_span(p, i) : make_int2(0, 0);
            own_words[w] = __ballot_sync(kFullMask, sp.y > sp.x);
        }
    }
    // the table by warps that have nothing else to begin with, the zeros by the others
    if (p.b.n) {
        if (warp >= 4 && warp < 8) fill_bias(p, h0, lut, warp - 4, 4, lane);
        if (ROLE == 1 && warp < 4)
            for (uint32_t e = tid; e < kSoftWarps * entries; e += 128) rel_sums[e] = 0.f;
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = warp_value(sh.tmem);
    volatile int *abort_flag = &sh.abort_flag;
    int32_t lo = INT32_MAX, hi = 0, s_lo = INT32_MAX;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        lo = min(lo, sh.limits[w][0]);
        hi = max(hi, sh.limits[w][1]);
        s_lo = min(s_lo, sh.limits[w][2]);
    }
    lo = warp_value(lo);
    hi = warp_value(hi);
    s_lo = warp_value(s_lo);
    // tiles of one head: role 0 the run of keys and then the sinks before it, role 1 the queries, on a grid of kRows
    if (ROLE == 1) lo = hi ? lo / Sh::kRows * Sh::kRows : 0;
    const int32_t s_end = ROLE == 0 && hi ? min(s_lo + p.sinks, lo) : 0, extra = ROLE == 0 && hi && s_lo < s_end ? (s_end - s_lo + Sh::kRows - 1) / Sh::kRows : 0;
    const int32_t sinks = extra ? s_end - s_lo : 0;
    float *sink_p = reinterpret_cast<float *>(smem + Sh::kRing + 2 * Sh::kOwn), *sink_d = sink_p + sinks * 128;      // [sink][row]; where o was, if it was
    const int32_t run = hi ? (hi - lo + Sh::kRows - 1) / Sh::kRows : 0, per_head = run + extra;
    const int32_t total = per_head * (int32_t)heads_here;
    auto tile_at = [&](int32_t k) { return ROLE == 0 && k >= run ? s_lo + (k - run) * Sh::kRows : lo + k * Sh::kRows; };
    auto tile_rows = [&](int32_t k) { return ROLE == 1 ? Sh::kRows : min((int32_t)Sh::kRows, (k >= run ? s_end : hi) - tile_at(k)); };

    if (warp < kSoftWarps) {
        // ============ softmax warpgroups ============
        if (SMALL) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kBackSoftRegs));
        const uint32_t wg = tid >> 7, lanes = ((warp & 3u) * 32u) << 16;
        const float scale = p.scale * kLog2e;
        const int32_t last = bias_last(p.b), off = last + kBiasPad;
        const int32_t w0 = t0 + (int32_t)(warp & 3u) * 32;           // first row of the warp
        const bool word = ROLE == 0 ? row.hi > row.lo : q_hi > q_lo;
        float lse = INFINITY, delta = 0.f;
        if (ROLE == 0 && word) lse = __ldg(p.lse + (int64_t)h_own * p.n + own);
        bool ok = __all_sync(kFullMask, mbar_nap(&sh.own_landed, 0, abort_flag));
        {
            auto chunk = [&](int operand, int c) {                   // 8 columns of this thread's row, from the 128-byte swizzle
                return *reinterpret_cast<const uint4 *>(own_rows + operand * Sh::kOwn + (c >> 3) * (128 * 128) + r * 128u + (((c & 7) ^ (r & 7u)) << 4));
            };
            auto first_delta = [&](uint4 d4, uint4 o4) {
                const Pack<T, 8> dd = reinterpret_cast<const Pack<T, 8> &>(d4), oo = reinterpret_cast<const Pack<T, 8> &>(o4);
#pragma unroll
                for (int e = 0; e < 8; ++e) delta = fmaf(to_f32(oo.e[e]), to_f32(dd.e[e]), delta);
            };
            if (SMALL) {
                const uint4 *o = reinterpret_cast<const uint4 *>(static_cast<const T *>(p.o) + own * (int64_t)p.ldo + (int64_t)h_own * p.dim);
                if (ROLE == 0) {                                     // each warpgroup half of the row
                    if (word)
#pragma unroll
                        for (int c = 0; c < NB * 4; ++c) {
                            const uint32_t x = 2 * c + wg;
                            if (x * 8 < p.dim) first_delta(chunk(1, (int)x), __ldg(o + x));
                        }
                    rel_sums[wg * 128 + r] = delta;
                    soft_barrier(Sh::kSoft);
                    delta = rel_sums[r] + rel_sums[128 + r];
                }
            } else {
                // the two operands of the block's rows go to tensor memory (a warpgroup each), zeros for rows that are not words
#pragma unroll
                for (int g = 0; g < NB * 2; ++g) {
                    uint32_t x[16];
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        const int at = g * 4 + c;
                        uint4 u = chunk((int)wg, at);
                        if (!word) u = make_uint4(0, 0, 0, 0);
                        if (ROLE == 0) first_delta(chunk(1, at), chunk(2, at));      // both warpgroups need it
                        x[c * 4] = u.x; x[c * 4 + 1] = u.y; x[c * 4 + 2] = u.z; x[c * 4 + 3] = u.w;
                    }
                    tmem_st16(tmem + lanes + (wg == 0 ? Sh::kA0 : Sh::kA1) + g * 16, x);
                }
                if (!word) delta = 0.f;
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(&sh.own_full);
            }
        }
        float2 eps2 = make_float2(0.f, 0.f);
        float weights = 0.f;                                         // role 0: their sum, for far rows
        const bool far_rows = ROLE == 0 && __any_sync(kFullMask, far_row(lse));
        for (uint32_t g = 0; g < heads_here; ++g) {
            if (ROLE == 1 && p.b.n && g > 0) {
                soft_barrier(Sh::kSoft);                             // the sums of the head before are written
                fill_bias(p, h0 + g, lut, warp, kSoftWarps, lane);
                for (uint32_t e = tid; e < kSoftWarps * entries; e += Sh::kSoft) rel_sums[e] = 0.f;
                soft_barrier(Sh::kSoft);
            }
            float far_l = 0.f, far_r = 0.f;
            for (int32_t k = 0; k < per_head && ok; ++k) {
                const int32_t t = (int32_t)g * per_head + k;
                const uint32_t b = t % Sh::kBuf, stage = t % Sh::kStages;
                if (!SMALL && b != wg) continue;
                const int32_t at0 = tile_at(k), cols = (tile_rows(k) + 15) & ~15;
                ok = __all_sync(kFullMask, mbar_nap(&sh.full[stage], (t / Sh::kStages) & 1, abort_flag) &&
                                               mbar_nap(&sh.s_full[b], (t / Sh::kBuf) & 1, abort_flag));
                if (!ok) break;
                tc_fence_after();
                const uint32_t cs = tmem + lanes + Sh::kScores + b * 2 * Sh::kRows, cd = cs + Sh::kRows;
                // which side of the diagonal the warp's part of the tile lies on: distances key - query
                const int32_t rel0 = ROLE == 0 ? at0 - (w0 + 31) : w0 - (at0 + Sh::kRows - 1);
                const int32_t rel1 = ROLE == 0 ? at0 + Sh::kRows - 1 - w0 : w0 + 31 - at0;
                const bool far_left = rel1 <= -last, far = p.b.n == 0 || far_left || rel0 >= last;
                const float flat = p.b.n ? lut[far_left ? 0 : entries - 1] : 0.f;
                const bool reach = ROLE == 1 && p.sinks && sh.run_lo[stage] <= own;
                constexpr int kC = Sh::kChunk;
                constexpr uint32_t kAll = kC == 32 ? 0xFFFFFFFFu : (1u << kC) - 1u;
                const int32_t c0 = SMALL ? (int32_t)wg * kC : 0;     // first column
                if (c0 < cols) {
                    uint32_t sv[kC], dv[kC];
                    tmem_ld(cs + c0, sv);
                    tmem_ld(cd + c0, dv);
                    const int32_t at = at0 + c0;
                    uint32_t m;
                    if (ROLE == 0) m = range_bits(row.lo, row.hi, at) | range_bits(row.s, row.se, at);
                    else {
                        m = range_bits(q_lo, q_hi, at);
                        if (reach) m |= range_bits(far_lo, far_hi, at);
                    }
                    m &= sh.vis[stage] >> c0;
                    tmem_wait_ld(sv);
                    tmem_held(dv);
                    // a row or column that sees nothing has lse +infinity
                    float x[kC];
                    if (far) {
                        const float2 scale2 = make_float2(scale, scale), flat2 = make_float2(flat, flat);
#pragma unroll
                        for (int e = 0; e < kC; e += 2) {
                            const float2 y = fma2(pair_of(sv[e], sv[e + 1]), scale2, flat2);
                            x[e] = y.x;
                            x[e + 1] = y.y;
                        }
                    } else {
                        // key - query grows with the column in role 0 and falls with it in role 1
                        const float *near = ROLE == 0 ? lut + (at - (int32_t)own + off) : lut + ((int32_t)own - at + off);
#pragma unroll
                        for (int e = 0; e < kC; ++e) x[e] = fmaf(__uint_as_float(sv[e]), scale, ROLE == 0 ? near[e] : near[-e]);
                    }
                    const bool masked = !__all_sync(kFullMask, (m | ~kAll) == 0xFFFFFFFFu);
                    uint32_t ws[kC / 2], wp[kC / 2];
                    // masked pairs are taken out of the weights and of dS, not of the scores: a delta, lse or product
                    // of such a pair may not be finite
                    auto take_out = [&](float *w, float *d) {
                        if (masked)
#pragma unroll
                            for (int e = 0; e < kC; ++e) {
                                w[e] = m & (1u << e) ? w[e] : 0.f;
                                d[e] = m & (1u << e) ? d[e] : 0.f;
                            }
                    };
                    float ds[kC];
                    if (ROLE == 0) {
                        const float2 lse2 = make_float2(-lse, -lse), delta2 = make_float2(-delta, -delta);
#pragma unroll
                        for (int e = 0; e < kC; e += 2) {
                            float2 w = add2(make_float2(x[e], x[e + 1]), lse2);
                            w.x = fast_exp2(w.x);
                            w.y = fast_exp2(w.y);
                            const float2 d = mul2(w, add2(pair_of(dv[e], dv[e + 1]), delta2));
                            x[e] = w.x; x[e + 1] = w.y;
                            ds[e] = d.x; ds[e + 1] = d.y;
                        }
                        take_out(x, ds);
#pragma unroll
                        for (int e = 0; e < kC; e += 2) {
                            eps2 = add2(eps2, make_float2(ds[e], ds[e + 1]));
                            wp[e / 2] = pack2<T>(x[e], x[e + 1]);
                            ws[e / 2] = pack2<T>(ds[e], ds[e + 1]);
                        }
                        tmem_st(cs + (SMALL ? c0 : c0 / 2), wp);
                        tmem_st(cd + (SMALL ? c0 : c0 / 2), ws);
                        if (far_rows) {
#pragma unroll
                            for (int e = 0; e < kC; ++e) weights += x[e];
                        }
                        if (k >= run) {                          // sinks: kept in fp32 for their own sums
#pragma unroll
                            for (int e = 0; e < kC; ++e) {
                                const int32_t i = (k - run) * Sh::kRows + c0 + e;
                                if (i < sinks) {
                                    sink_p[i * 128 + (int32_t)r] = x[e];
                                    sink_d[i * 128 + (int32_t)r] = ds[e];
                                }
                            }
                        }
                    } else {
                        const float *less = sh.lse[stage];       // negated, as delta and extra
                        if (sh.far[stage]) {
#pragma unroll
                            for (int e = 0; e < kC; ++e) x[e] += less[c0 + e];
                            less = sh.extra[stage];
                        }
#pragma unroll
                        for (int e = 0; e < kC; e += 4) {
                            const float4 l4 = *reinterpret_cast<const float4 *>(less + c0 + e);
                            const float4 d4 = *reinterpret_cast<const float4 *>(&sh.delta[stage][c0 + e]);
                            float2 p0 = add2(make_float2(x[e], x[e + 1]), make_float2(l4.x, l4.y));
                            float2 p1 = add2(make_float2(x[e + 2], x[e + 3]), make_float2(l4.z, l4.w));
                            p0.x = fast_exp2(p0.x); p0.y = fast_exp2(p0.y); p1.x = fast_exp2(p1.x); p1.y = fast_exp2(p1.y);
                            x[e] = p0.x; x[e + 1] = p0.y; x[e + 2] = p1.x; x[e + 3] = p1.y;
                            p0 = mul2(p0, add2(pair_of(dv[e], dv[e + 1]), make_float2(d4.x, d4.y)));
                            p1 = mul2(p1, add2(pair_of(dv[e + 2], dv[e + 3]), make_float2(d4.z, d4.w)));
                            ds[e] = p0.x; ds[e + 1] = p0.y; ds[e + 2] = p1.x; ds[e + 3] = p1.y;
                        }
                        take_out(x, ds);
#pragma unroll
                        for (int e = 0; e < kC; e += 2) {
                            wp[e / 2] = pack2<T>(x[e], x[e + 1]);
                            ws[e / 2] = pack2<T>(ds[e], ds[e + 1]);
                        }
                        tmem_st(cs + (SMALL ? c0 : c0 / 2), wp);
                        tmem_st(cd + (SMALL ? c0 : c0 / 2), ws);
                        if (p.dbias) {
                            if (far) {
                                float a[4] = {ds[0], ds[1], ds[2], ds[3]};
#pragma unroll
                                for (int e = 4; e < kC; ++e) a[e & 3] += ds[e];
                                if (far_left) far_l += (a[0] + a[1]) + (a[2] + a[3]); else far_r += (a[0] + a[1]) + (a[2] + a[3]);
                            } else {
                                // over 32 columns lane l gathers the diagonal key - query = base + l (acc_p) and the one 32 below (acc_n)
                                const int32_t base = w0 - at0;
                                float acc_p = 0.f, acc_n = 0.f;
#pragma unroll
                                for (int e = 0; e < kC; ++e) {
                                    const uint32_t from = lane + (uint32_t)c0 + e;
                                    const float y = __shfl_sync(kFullMask, ds[e], from & 31u);
                                    if (from < 32u) acc_p += y; else acc_n += y;
                                }
                                float *mine = rel_sums + warp * entries + base + off + (int32_t)lane;
                                mine[0] += acc_p;
                                __syncwarp();
                                mine[-32] += acc_n;
                                __syncwarp();
                            }
                        }
                    }
                }
                tmem_wait_st();
                tc_fence_before();
                mbar_arrive(&sh.p_full[b]);
                mbar_arrive(&sh.empty[stage]);
            }
            if (ROLE == 1 && p.dbias) {
                far_l = warp_sum(far_l);
                far_r = warp_sum(far_r);
                if (lane == 0) { sh.far_sum[warp][0] = far_l; sh.far_sum[warp][1] = far_r; }
                soft_barrier(Sh::kSoft);
                for (uint32_t e = tid; e < entries; e += Sh::kSoft) {        // the warps' sums
                    float a = 0.f;
#pragma unroll
                    for (uint32_t w = 0; w < kSoftWarps; ++w) a += rel_sums[w * entries + e];
                    rel_sums[e] = a;
                }
                soft_barrier(Sh::kSoft);
                const uint32_t buckets = p.b.n * (p.b.two_sided ? 2u : 1u);
                write_bucket_sums(p, rel_sums, off, sh.far_sum, warp, kSoftWarps, lane, p.dbias_part + ((size_t)tile * p.heads + h0 + g) * buckets);
            }
        }
        float eps = 0.f, far_by = 1.f;                               // far_by: what a far row's weights are to be multiplied by
        if (ROLE == 0) {
            eps = eps2.x + eps2.y;
            if (SMALL) soft_barrier(Sh::kSoft);                      // everybody has read the first delta's parts
            rel_sums[wg * 128 + r] = eps;
            rel_sums[256 + wg * 128 + r] = weights;
            soft_barrier(Sh::kSoft);
            eps = rel_sums[r] + rel_sums[128 + r];
            weights = far_row(lse) ? rel_sums[256 + r] + rel_sums[384 + r] : 1.f;
            far_by = 1.f / weights;
            eps *= far_by;
            if (wg == 0 && own < p.n) {
                p.delta[(int64_t)h_own * p.n + own] = word ? delta + eps : 0.f;
                p.extra[(int64_t)h_own * p.n + own] = weights == 1.f ? 0.f : log2f(weights);
            }
        }
        ok = __all_sync(kFullMask, ok && (total == 0 || mbar_nap(&sh.done, 0, abort_flag)));
        tc_fence_after();
        if (ROLE == 0 && p.sink_rec) {
            if (h_own == 0 && tid == 0) {
                p.sink_rec[tile] = !hi ? -1 : s_lo >= t0 ? -2 : sinks ? s_lo : -1;
                p.sink_used[tile] = -1;
            }
            const uint32_t buckets = p.b.n * (p.b.two_sided ? 2u : 1u);
            float *bias_out = p.dbias ? p.dbias_part + ((size_t)((uint32_t)((p.n + kAttendTile - 1) / kAttendTile) + tile) * p.heads + h_own) * buckets : nullptr;
            if (sinks) sink_sums<T, NB, Sh::kSoft>(p, own_rows, sink_p, sink_d, row, eps, far_by, reinterpret_cast<float *>(smem), sinks, s_lo, t0, wg, r, tid,
                                                   p.sink_part + ((size_t)tile * p.heads + h_own) * p.sinks * 2 * p.dim, bias_out);
            else if (bias_out) for (uint32_t b = tid; b < buckets; b += Sh::kSoft) bias_out[b] = 0.f;
            soft_barrier(Sh::kSoft);
        }
        // outputs leave through shared memory: dQ (half of its columns by each warpgroup), or dK and dV (one each)
        constexpr bool kHalf = ROLE == 0;
        const uint32_t which = ROLE == 0 ? 0u : wg;              // 0: dQ or dK, 1: dV
        const float by = (which == 0 ? p.scale : 1.f) * far_by;
        const float *sink = nullptr;
        if (ROLE == 1 && p.sink_used && word && own - sent < p.sinks && p.sink_used[sent / kAttendTile] == sent)
            sink = p.sink_sum + ((((size_t)(sent / kAttendTile) * p.kv_heads + kvh) * p.sinks + (size_t)(own - sent)) * 2 + which) * p.dim;
        const uint32_t row_bytes = p.dim * 2u, chunks = p.dim >> 3, turn = lane % chunks, part = ((warp & 3u) + which * 4u) * 32u;
        unsigned char *mine = smem + part * row_bytes, *line = mine + lane * row_bytes;
        constexpr int kCols = kHalf ? NB * 2 : NB * 4;           // steps of 16 columns
        float2 zero = make_float2(0.f, 0.f);                     // NaN once a value is not finite
#pragma unroll
        for (int i = 0; i < kCols; ++i) {
            const uint32_t c = kHalf ? i * 32 + wg * 16 : i * 16;
            if (c >= dim16) break;
            float f[16];
            if (total) {
                uint32_t o[16];
                tmem_ld16(tmem + lanes + (which == 0 ? Sh::kG0 : Sh::kG1) + c, o);
                if (ROLE == 0) {                                 // the correction of the first delta
                    uint32_t pk[16];
                    tmem_ld16(tmem + lanes + Sh::kG1 + c, pk);
                    tmem_wait_ld(o);
                    tmem_wait_ld(pk);
#pragma unroll
                    for (int e = 0; e < 16; ++e) f[e] = word ? fmaf(-eps, __uint_as_float(pk[e]), __uint_as_float(o[e])) : 0.f;
                } else {
                    tmem_wait_ld(o);
#pragma unroll
                    for (int e = 0; e < 16; ++e) f[e] = word ? __uint_as_float(o[e]) : 0.f;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 16; ++e) f[e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < 16; e += 2) zero = fma2(make_float2(f[e], f[e + 1]), make_float2(0.f, 0.f), zero);
#pragma unroll
            for (int q = 0; q < 2; ++q)
                if (c + q * 8 < p.dim) {
                    if (sink) {
#pragma unroll
                        for (int e = 0; e < 8; ++e) f[q * 8 + e] += sink[c + q * 8 + e];
                    }
                    uint4 w;
                    w.x = pack2<T>(f[q * 8] * by, f[q * 8 + 1] * by); w.y = pack2<T>(f[q * 8 + 2] * by, f[q * 8 + 3] * by);
                    w.z = pack2<T>(f[q * 8 + 4] * by, f[q * 8 + 5] * by); w.w = pack2<T>(f[q * 8 + 6] * by, f[q * 8 + 7] * by);
                    const uint32_t ch = (c >> 3) + q + turn;
                    *reinterpret_cast<uint4 *>(line + (ch >= chunks ? ch - chunks : ch) * 16u) = w;
                }
        }
        const int32_t rows = (int32_t)min((int64_t)32, p.n - (int64_t)w0);
        const uint64_t ld = ROLE == 0 ? p.ld_dq : which == 0 ? p.ld_dk : p.ld_dv;
        char *out = static_cast<char *>(ROLE == 0 ? p.dq : which == 0 ? p.dk : p.dv) + ((uint64_t)w0 * ld + (uint64_t)h_own * p.dim) * 2u;
        const bool nan = ROLE == 0 && (lse != lse || delta + eps != delta + eps);        // of its own: nothing to be found
        uint32_t bad = __ballot_sync(kFullMask, ok && zero.x + zero.y != 0.f && word && !nan);
        bool again = bad != 0u;
        if (kHalf) {
            again = any_of_64(2u + (warp & 3u), again);          // the two warps of these rows
            store_rows(out, ld * 2u, mine, chunks, rows, wg * 32u + lane, 64u);
        } else {
            __syncwarp();
            store_rows(out, ld * 2u, mine, chunks, rows, lane, 32u);
        }
        if (again) {                                             // both warps or neither; over what has been stored
            if (kHalf) asm volatile("bar.sync %0, 64;" ::"r"(2u + (warp & 3u)) : "memory");
            else __syncwarp();
#pragma unroll 1
            for (; bad; bad &= bad - 1u) {
                const int32_t x = __ffs(bad) - 1;
                if (ROLE == 0) dq_again<T>(p, h_own, kvh, (int64_t)w0 + x, __shfl_sync(kFullMask, lse, x), __shfl_sync(kFullMask, far_by, x), __shfl_sync(kFullMask, delta + eps, x), lane);
                else dkv_again<T>(p, which, kvh, (int64_t)w0 + x, reinterpret_cast<const float *>(__shfl_sync(kFullMask, reinterpret_cast<unsigned long long>(sink), x)), lane);
            }
        }
        tc_fence_before();
    } else if (warp == kMmaWarp) {
        // ============ MMA issue: one lane ============
        if (SMALL) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kBackOtherRegs));
        // everything that does not change is formed once, in a warp that stays together: the block waits for it when its
        // code is long
        if (total) {
            const bool leader = elect_one();
            constexpr uint32_t kBlock = Sh::kRows * 128, kStep = Sh::kStage >> 4;
            const uint32_t idesc_g = umma_idesc_f16(kBf16, kAttendTile, dim16, true), idesc_s = umma_idesc_f16(kBf16, kAttendTile, Sh::kRows, false);
            // the streamed operands with columns as the summed side (scores) and with rows as the summed side (gradients)
            const uint32_t xs = umma_desc_low(ring, 0), ys = umma_desc_low(ring + Sh::kOperand, 0);
            const uint32_t xg = umma_desc_low(ring, kBlock), yg = umma_desc_low(ring + (ROLE == 0 ? 0 : Sh::kOperand), kBlock);
            const uint32_t own_low = umma_desc_low(ring + Sh::kRing, 0);
            auto scores = [&](uint32_t b, uint32_t stage) {
                const uint32_t x = xs + stage * kStep, y = ys + stage * kStep, d = tmem + Sh::kScores + b * 2 * Sh::kRows;
#pragma unroll
                for (int c = 0; c < NB * 4; ++c)
                    if ((uint32_t)c * 16 < dim16) {
                        const uint32_t at = (c >> 2) * (kBlock >> 4) + (c & 3) * 2;
                        if (SMALL) {
                            const uint32_t a_at = (c >> 2) * (128 * 128 >> 4) + (c & 3) * 2;
                            umma_f16_ss(d, own_low + a_at, x + at, idesc_s, c > 0);
                            umma_f16_ss(d + Sh::kRows, own_low + (Sh::kOwn >> 4) + a_at, y + at, idesc_s, c > 0);
                        } else {
                            umma_f16_ts(d, tmem + Sh::kA0 + c * 8, x + at, idesc_s, c > 0);
                            umma_f16_ts(d + Sh::kRows, tmem + Sh::kA1 + c * 8, y + at, idesc_s, c > 0);
                        }
                    }
                umma_commit(&sh.s_full[b]);
            };
            auto wait = [&](uint64_t *bar, uint32_t parity) {
                const bool got = __all_sync(kFullMask, mbar_nap(bar, parity, abort_flag));
                tc_fence_after();
                return got;
            };
            bool ok = wait(&sh.own_full, 0);
            uint32_t ahead = 0, ahead_phase = 0, stage = 0;          // stage and phase of the next scores, two tiles ahead of the gradients
            for (int32_t t = 0; t < Sh::kBuf && t < total && ok; ++t) {
                ok = wait(&sh.full[ahead], 0);
                if (ok && leader) scores((uint32_t)t, ahead);
                __syncwarp();
                ++ahead;
            }
            int32_t k = 0;                                           // number of the tile within its head
            for (int32_t t = 0; t < total && ok; ++t) {
                const uint32_t b = t % Sh::kBuf, x = xg + stage * kStep, y = yg + stage * kStep, d = tmem + Sh::kScores + b * 2 * Sh::kRows;
                const int32_t rows = tile_rows(k);
                if (++k == per_head) k = 0;
                ok = wait(&sh.p_full[b], (t / Sh::kBuf) & 1);
                if (!ok) break;
                if (leader) {
#pragma unroll
                    for (int c = 0; c < Sh::kRows / 16; ++c)
                        if (c * 16 < rows) {
                            // each thread has put its weights over its own scores: SMALL, the second half of a tile's lie 16 columns on
                            umma_f16_ts(tmem + Sh::kG1, d + c * (SMALL ? 16 : 8), y + c * 128, idesc_g, t > 0 || c > 0);
                            umma_f16_ts(tmem + Sh::kG0, d + Sh::kRows + c * (SMALL ? 16 : 8), x + c * 128, idesc_g, t > 0 || c > 0);
                        }
                    umma_commit(&sh.empty[stage]);
                    if (t + 1 == total) umma_commit(&sh.done);
                }
                __syncwarp();
                if (++stage == Sh::kStages) stage = 0;
                if (t + Sh::kBuf < total) {
                    ok = wait(&sh.full[ahead], ahead_phase);
                    if (!ok) break;
                    if (leader) scores(b, ahead);
                    __syncwarp();
                    if (++ahead == Sh::kStages) { ahead = 0; ahead_phase ^= 1u; }
                }
            }
        }
        __syncwarp();
    } else if (warp == kMmaWarp + 1) {
        // ============ copies: one lane ============
        if (SMALL) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kBackOtherRegs));
        if (lane == 0) {
            int32_t t = 0;
            for (; t < total; ++t) {
                const uint32_t stage = t % Sh::kStages, round = t / Sh::kStages, base = ring + stage * Sh::kStage;
                if (round > 0 && !mbar_nap(&sh.empty[stage], (round - 1) & 1, abort_flag)) break;
                const int32_t head = ROLE == 0 ? (int32_t)kvh : (int32_t)h0 + t / per_head, at = tile_at(t % per_head);
                mbar_expect(&sh.landed[stage], Sh::kStage);
#pragma unroll
                for (int c = 0; c < NB; ++c) {
                    copy_box(base + c * Sh::kRows * 128, &map_x, c * 64, head, at, &sh.landed[stage]);
                    copy_box(base + Sh::kOperand + c * Sh::kRows * 128, &map_y, c * 64, head, at, &sh.landed[stage]);
                }
            }
            issued = t;
        }
        __syncwarp();
    } else {
        // ============ rows that are not words, and what goes with the rows: a warp per tile, in turn ============
        if (SMALL) {
            asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kBackOtherRegs));
            // the block's own rows: one operand each
            if (__all_sync(kFullMask, mbar_nap(&sh.own_landed, 0, abort_flag))) {
                const uint32_t a = ring + Sh::kRing + (warp - kMmaWarp - 2) * Sh::kOwn, top[2] = {own_words[0], own_words[1]}, low[2] = {own_words[2], own_words[3]};
                zero_rows<NB>(a, 128 * 128, 64, top, lane);
                zero_rows<NB>(a + 64 * 128, 128 * 128, 64, low, lane);
                fence_async_proxy();
                mbar_arrive(&sh.own_full);
            }
        }
        for (int32_t t = (int32_t)(warp - kMmaWarp) - 2; t < total; t += 2) {
            const uint32_t stage = t % Sh::kStages, h = h0 + (uint32_t)(t / per_head);
            const int32_t k = t % per_head, at = tile_at(k), rows = tile_rows(k);
            uint32_t vis[2];
            word_bits(p, at, (uint32_t)rows, lane, vis);
            float lse = 0.f, delta = 0.f, extra = 0.f;
            int32_t run_lo = 0;
            if (ROLE == 1) {
                const int64_t i = (int64_t)at + lane;
                lse = i < p.n ? __ldg(p.lse + (int64_t)h * p.n + i) : INFINITY;
                delta = i < p.n ? p.delta[(int64_t)h * p.n + i] : 0.f;
                extra = i < p.n ? p.extra[(int64_t)h * p.n + i] : 0.f;
                if (p.sinks) run_lo = run_begin(p, at / kAttendTile * kAttendTile, lane);
            }
            if (!__all_sync(kFullMask, mbar_nap(&sh.landed[stage], (t / Sh::kStages) & 1, abort_flag))) break;
            if (lane == 0) sh.vis[stage] = vis[0];
            if (ROLE == 1) {
                sh.lse[stage][lane] = -lse;
                sh.delta[stage][lane] = -delta;
                sh.extra[stage][lane] = -extra;
                const bool far = __any_sync(kFullMask, extra != 0.f);
                if (lane == 0) { sh.run_lo[stage] = run_lo; sh.far[stage] = far; }
            }
            const uint32_t x = ring + stage * Sh::kStage, cols = (uint32_t)(rows + 15) & ~15u;
            zero_rows<NB>(x, Sh::kRows * 128, cols, vis, lane);
            zero_rows<NB>(x + Sh::kOperand, Sh::kRows * 128, cols, vis, lane);
            fence_async_proxy();
            mbar_arrive(&sh.full[stage]);
        }
    }
    __syncthreads();
    tc_fence_after();
    if (sh.abort_flag) {
        // a wait ran out: the copies and products under way end (or have as long again) before the block leaves what they use
        if (warp == kMmaWarp + 1 && lane == 0) {
            mbar_nap(&sh.own_landed, 0, &sh.quiet);
            for (int32_t u = max(0, issued - Sh::kStages); u < issued; ++u) mbar_nap(&sh.landed[u % Sh::kStages], (u / Sh::kStages) & 1, &sh.quiet);
        } else if (warp == kMmaWarp) {
            if (elect_one()) umma_commit(&sh.still);
            __syncwarp();
            mbar_nap(&sh.still, 0, &sh.quiet);
        }
        __syncthreads();
    }
    if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(Sh::kAlloc));
    if (tid == 0 && sh.abort_flag) atomicOr(error, kErrAttend);
}

// The first word of a tile that has one.
__device__ __forceinline__ int64_t first_word(const AttendParams &p, int32_t tile)
{
    int64_t i = (int64_t)tile * kAttendTile;
    while (i + 1 < p.n && !is_word(p, i)) ++i;
    return i;
}

// Slot a holds the sums for the sentence that begins in tile a and reaches into a later one (there is at most one):
// over its query tiles and the query heads of a key/value head, in a fixed order, 32 elements at a time.
__global__ void __launch_bounds__(256)
attend_sink_sum_kernel(AttendParams p, int32_t tiles)
{
    __shared__ float part[8][32];
    const uint32_t kvh = blockIdx.x % p.kv_heads, group = p.heads / p.kv_heads, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const size_t width = (size_t)p.sinks * 2 * p.dim, e = (size_t)(blockIdx.x / p.kv_heads) * 32 + lane;
    // a sentence is added up from the first tile that has sums for it; most tiles have none or are not the first, which takes
    // one look to see: a block goes over many.  (Looking ahead from where a sentence begins took 182 ms for 2,000 words in a
    // buffer of 2,000,000 positions, 15,600 tiles of nothing.)
    for (int32_t first = (int32_t)blockIdx.y; first < tiles; first += (int32_t)gridDim.y) {
        const int32_t s = p.sink_rec[first];
        if (s < 0) continue;
        const int32_t a = s / kAttendTile, least = (int32_t)max((int64_t)a + 1, ((int64_t)s + p.left) / kAttendTile);     // none before that
        int32_t before = first - 1;                                  // over tiles of the sentence without a word
        while (before >= least && p.sink_rec[before] == -1) --before;
        if (before >= least) continue;
        if (blockIdx.x == 0 && threadIdx.x == 0) p.sink_used[a] = s;
        // the sentence's last tile is that of its last word; tiles without words in between have nothing
        const int32_t end = min(tiles, (word_span(p, first_word(p, first)).y - 1) / kAttendTile + 1);
        const int32_t items = (end - first) * (int32_t)group;
        float x[4] = {0.f, 0.f, 0.f, 0.f};
        if (e < width)
            for (int32_t i = (int32_t)warp; i < items; i += 32) {
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const int32_t j = i + u * 8, t = first + j / (int32_t)group;
                    if (j < items && p.sink_rec[t] == s) x[u] += p.sink_part[((size_t)t * p.heads + kvh * group + (uint32_t)j % group) * width + e];
                }
            }
        part[warp][lane] = (x[0] + x[1]) + (x[2] + x[3]);
        __syncthreads();
        if (warp == 0 && e < width) {
            float y = 0.f;
#pragma unroll
            for (int w = 0; w < 8; ++w) y += part[w][lane];
            p.sink_sum[((size_t)a * p.kv_heads + kvh) * width + e] = y;
        }
        __syncthreads();
    }
}

__global__ void __launch_bounds__(256)
attend_dbias_kernel(const float *part, uint64_t rows, uint32_t columns, uint32_t heads, uint32_t buckets, float *dbias)
{
    __shared__ float t[8];
    const uint32_t c = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float a = 0.f;
    for (uint64_t r = threadIdx.x; r < rows; r += blockDim.x) a += part[r * columns + c];
    a = warp_sum(a);
    if (lane == 0) t[warp] = a;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 8; ++w) a += t[w];
        dbias[(c % buckets) * heads + c / buckets] = a;
    }
}

namespace {

struct BackWs {
    uint64_t delta, extra, part, sink_part, sink_sum, rec, used, bytes;
};

bool far_sinks(const AttendParams &p) { return p.sinks > 0 && p.n > (int64_t)p.left + 1; }

BackWs back_ws(const AttendParams &p, bool want_dbias)
{
    const uint64_t tiles = ((uint64_t)p.n + kAttendTile - 1) / kAttendTile, buckets = p.b.n * (p.b.two_sided ? 2u : 1u);
    const bool sinks = far_sinks(p);
    BackWs w;
    uint64_t at = 0;
    auto take = [&](uint64_t floats) { const uint64_t x = at; at += (floats * 4 + 15) & ~15ull; return x; };
    w.delta = take((uint64_t)p.n * p.heads);
    w.extra = take((uint64_t)p.n * p.heads);
    w.part = take(want_dbias ? (sinks ? 2 : 1) * tiles * p.heads * buckets : 0);
    w.sink_part = take(sinks ? tiles * p.heads * p.sinks * 2 * p.dim : 0);
    w.sink_sum = take(sinks ? tiles * p.kv_heads * p.sinks * 2 * p.dim : 0);
    w.rec = take(sinks ? tiles : 0);
    w.used = take(sinks ? tiles : 0);
    w.bytes = at + 16;
    return w;
}

template <typename T, int NB, int ROLE, bool SMALL>
int launch_role(const AttendParams &p, uint32_t tiles, int *error, cudaStream_t s)
{
    using Sh = BackShape<NB, SMALL>;
    auto kernel = attend_back_kernel<T, NB, ROLE, SMALL>;
    const uint32_t entries = bias_entries(p.b);
    const int o_bytes = SMALL ? 0 : Sh::kOwn, sink_bytes = p.sinks * 1024;
    int smem = Sh::kRing + 2 * Sh::kOwn + (ROLE == 0 ? (sink_bytes > o_bytes ? sink_bytes : o_bytes) : 0) + 1024 +
               (int)(4 * (((entries + 3u) & ~3u) + (ROLE == 1 ? Sh::kSoft / 32 * entries : 512u)));
    if (!SMALL && smem < 116 * 1024) smem = 116 * 1024;              // a second block would only wait for tensor memory
    if (!kernel_ready<attend_back_kernel<T, NB, ROLE, SMALL>>(SMALL ? kBackLaunchRegs : 0)) return -1;
    CUtensorMap x, y, a0, a1, o;
    const bool bf16 = std::is_same<T, __nv_bfloat16>::value;
    const uint64_t n = (uint64_t)p.n;
    auto queries = [&](CUtensorMap *m, const void *at, uint64_t ld, uint32_t rows) { return make_rows_map(m, bf16, at, p.dim, p.heads, n, ld, rows); };
    auto keys = [&](CUtensorMap *m, const void *at, uint64_t ld, uint32_t rows) { return make_rows_map(m, bf16, at, p.dim, p.kv_heads, n, ld, rows); };
    if (ROLE == 0) {
        if (!keys(&x, p.k, p.ldk, Sh::kRows) || !keys(&y, p.v, p.ldv, Sh::kRows) || !queries(&a0, p.q, p.ldq, 128) ||
            !queries(&a1, p.d_o, p.ld_do, 128) || !queries(&o, p.o, p.ldo, 128))
            return -1;
    } else {
        if (!queries(&x, p.q, p.ldq, Sh::kRows) || !queries(&y, p.d_o, p.ld_do, Sh::kRows) || !keys(&a0, p.k, p.ldk, 128) || !keys(&a1, p.v, p.ldv, 128))
            return -1;
        o = a0;
    }
    kernel<<<tiles * (ROLE == 0 ? p.heads : p.kv_heads), Sh::kThreads, smem, s>>>(x, y, a0, a1, o, p, error);
    return cudaPeekAtLastError() == cudaSuccess ? 1 : -1;
}

template <typename T>
int launch_back_typed(const AttendParams &p, uint32_t tiles, int *error, cudaStream_t s)
{
    auto role = [&](auto which) {
        constexpr int R = decltype(which)::value;
        return p.dim <= 64 ? launch_role<T, 1, R, true>(p, tiles, error, s)
               : p.dim <= 96 ? launch_role<T, 2, R, true>(p, tiles, error, s) : launch_role<T, 2, R, false>(p, tiles, error, s);
    };
    int k = role(std::integral_constant<int, 0>());
    if (k < 0) return -1;
    if (far_sinks(p)) {
        const uint32_t columns = (2 * (uint32_t)p.sinks * p.dim + 31) / 32 * p.kv_heads, some = 2048 / columns + 1;
        attend_sink_sum_kernel<<<dim3(columns, tiles < some ? tiles : some), 256, 0, s>>>(p, (int32_t)tiles);
        ++k;
    }
    const int j = role(std::integral_constant<int, 1>());
    return j < 0 ? -1 : k + j;
}

}  // namespace

uint64_t attend_backward_ws(const AttendParams &p, bool want_dbias) { return back_ws(p, want_dbias).bytes; }

int launch_attend_backward(AttendParams &p, uint32_t type, unsigned char *ws, int *error, int, cudaStream_t s)
{
    const uint32_t buckets = p.b.n * (p.b.two_sided ? 2 : 1);
    const uint32_t tiles = (uint32_t)((p.n + kAttendTile - 1) / kAttendTile);
    const BackWs w = back_ws(p, p.dbias != nullptr);
    int k = 0;
    if (p.n) {
        p.delta = reinterpret_cast<float *>(ws + w.delta);
        p.extra = reinterpret_cast<float *>(ws + w.extra);
        p.dbias_part = reinterpret_cast<float *>(ws + w.part);
        if (far_sinks(p)) {
            p.sink_part = reinterpret_cast<float *>(ws + w.sink_part);
            p.sink_sum = reinterpret_cast<float *>(ws + w.sink_sum);
            p.sink_rec = reinterpret_cast<int32_t *>(ws + w.rec);
            p.sink_used = reinterpret_cast<int32_t *>(ws + w.used);
        }
        k = type == kBF16 ? launch_back_typed<__nv_bfloat16>(p, tiles, error, s) : launch_back_typed<__half>(p, tiles, error, s);
        if (k < 0) return -1;
    }
    if (p.dbias) {
        attend_dbias_kernel<<<p.heads * buckets, 256, 0, s>>>(reinterpret_cast<const float *>(ws + w.part), (far_sinks(p) ? 2ull : 1ull) * tiles,
                                                             p.heads * buckets, p.heads, buckets, p.dbias);
        ++k;
    }
    return cudaPeekAtLastError() == cudaSuccess ? k : -1;
}

}  // namespace w2v
