// Attention over a window of the word's sentence, forwards and backwards, and the sentence bounds.
#include "w2v_device.cuh"
#include "w2v_reader.h"
#include "w2v_types.cuh"

namespace w2v {

// ---- sentence bounds ----------------------------------------------------------------------------
// spans[t] = (first position of t's sentence, one past its last); a separator or a word that the
// vocabulary does not have gets the empty span (t, t).  Two passes: the last and the first separator
// of every tile, then every tile looks back and ahead for the nearest tile that has one.
constexpr int kSpanThreads = 256, kSpanPer = 8, kSpanTile = kSpanThreads * kSpanPer;

uint64_t spans_tiles(uint64_t n) { return (n + kSpanTile - 1) / kSpanTile; }

__global__ void __launch_bounds__(kSpanThreads)
span_tiles_kernel(const int32_t *tokens, uint64_t n, int2 *tile_ends)
{
    __shared__ int first, last;
    if (threadIdx.x == 0) { first = INT32_MAX; last = -1; }
    __syncthreads();
    const uint64_t t0 = (uint64_t)blockIdx.x * kSpanTile;
    for (int i = 0; i < kSpanPer; ++i) {
        const uint64_t t = t0 + i * kSpanThreads + threadIdx.x;
        if (t < n && tokens[t] == -1) { atomicMin(&first, (int)t); atomicMax(&last, (int)t); }
    }
    __syncthreads();
    if (threadIdx.x == 0) tile_ends[blockIdx.x] = make_int2(first, last);
}

__global__ void __launch_bounds__(kSpanThreads)
span_fill_kernel(const int32_t *tokens, uint64_t n, uint32_t vocab, const int2 *tile_ends, uint32_t tiles, int2 *spans)
{
    __shared__ int before, after, sh[kSpanThreads];
    const uint32_t tid = threadIdx.x;
    if (tid == 0) { before = -1; after = (int)n; }
    __syncthreads();
    for (int64_t c = (int64_t)blockIdx.x; c > 0; c -= kSpanThreads) {           // nearest separator before the tile
        const int64_t j = c - 1 - (int64_t)tid;
        if (j >= 0 && tile_ends[j].y >= 0) atomicMax(&before, tile_ends[j].y);
        __syncthreads();
        if (before >= 0) break;
        __syncthreads();
    }
    for (int64_t c = (int64_t)blockIdx.x + 1; c < (int64_t)tiles; c += kSpanThreads) {
        const int64_t j = c + (int64_t)tid;
        if (j < (int64_t)tiles && tile_ends[j].x < (int)n) atomicMin(&after, tile_ends[j].x);
        __syncthreads();
        if (after < (int)n) break;
        __syncthreads();
    }
    __syncthreads();
    const uint64_t t0 = (uint64_t)blockIdx.x * kSpanTile + (uint64_t)tid * kSpanPer;
    int tok[kSpanPer], lo[kSpanPer], hi[kSpanPer];
    int run = -1;
#pragma unroll
    for (int i = 0; i < kSpanPer; ++i) {
        tok[i] = t0 + i < n ? tokens[t0 + i] : -2;
        if (tok[i] == -1) run = (int)(t0 + i);
        lo[i] = run;
    }
    sh[tid] = run;                                                               // last separator of the thread's tokens
    __syncthreads();
    for (int o = 1; o < kSpanThreads; o <<= 1) {
        const int x = tid >= (uint32_t)o ? sh[tid - o] : -1;
        __syncthreads();
        sh[tid] = max(sh[tid], x);
        __syncthreads();
    }
    const int back = max(before, tid ? sh[tid - 1] : -1);
    __syncthreads();
    run = INT32_MAX;
#pragma unroll
    for (int i = kSpanPer - 1; i >= 0; --i) {
        if (tok[i] == -1) run = (int)(t0 + i);
        hi[i] = run;
    }
    sh[tid] = run;
    __syncthreads();
    for (int o = 1; o < kSpanThreads; o <<= 1) {
        const int x = tid + o < kSpanThreads ? sh[tid + o] : INT32_MAX;
        __syncthreads();
        sh[tid] = min(sh[tid], x);
        __syncthreads();
    }
    const int ahead = min(after, tid + 1 < kSpanThreads ? sh[tid + 1] : INT32_MAX);
#pragma unroll
    for (int i = 0; i < kSpanPer; ++i)
        if (t0 + i < n) {
            const int t = (int)(t0 + i);
            const bool word = tok[i] >= 0 && (uint32_t)tok[i] < vocab;
            spans[t0 + i] = word ? make_int2(max(lo[i], back) + 1, min(hi[i], ahead)) : make_int2(t, t);
        }
}

int launch_spans(const int32_t *tokens, uint64_t n, uint32_t vocab, int32_t *tile_ends, int2 *spans, cudaStream_t s)
{
    if (n == 0) return 0;
    const uint32_t tiles = (uint32_t)spans_tiles(n);
    int2 *ends = reinterpret_cast<int2 *>(tile_ends);
    span_tiles_kernel<<<tiles, kSpanThreads, 0, s>>>(tokens, n, ends);
    span_fill_kernel<<<tiles, kSpanThreads, 0, s>>>(tokens, n, vocab, ends, tiles, spans);
    return cudaPeekAtLastError() == cudaSuccess ? 2 : -1;
}

// ---- attention, the simple form: one warp per row --------------------------------------------------
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ uint32_t bucket_of(const BucketStarts &b, int32_t rel)
{
    const int32_t far = b.two_sided ? abs(rel) : max(-rel, 0);
    uint32_t lo = 0, hi = b.n - 1;
    while (lo < hi) {
        const uint32_t mid = (lo + hi + 1) >> 1;
        if (b.start[mid] <= far) lo = mid; else hi = mid - 1;
    }
    return lo + (b.two_sided && rel > 0 ? b.n : 0u);
}

// A score in base-2 units; a bias of the lowest float stays finite there.
__device__ __forceinline__ float log2_score(float s) { return s == -INFINITY ? s : fmaxf(s, -1e30f) * kLog2e; }
template <typename T>
__device__ __forceinline__ void row_read(float (&x)[4], const T *p, uint32_t dim, uint32_t lane)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = lane + 32u * i < dim ? to_f32(p[lane + 32 * i]) : 0.f;
}
__device__ __forceinline__ float row_dot(const float (&a)[4], const float (&b)[4])
{
    return warp_sum(a[0] * b[0] + a[1] * b[1] + a[2] * b[2] + a[3] * b[3]);
}
template <typename T>
__device__ __forceinline__ void row_write(T *p, const float (&x)[4], uint32_t dim, uint32_t lane)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) if (lane + 32u * i < dim) p[lane + 32 * i] = from_f32<T>(x[i]);
}

// Calls f(j) for every key that query i sees.
template <typename F>
__device__ __forceinline__ void each_key(const AttendParams &p, int64_t i, F f)
{
    const int2 sp = p.spans[i];
    if (sp.y <= sp.x) return;
    const int64_t lo = max((int64_t)sp.x, i - p.left), hi = min((int64_t)sp.y, i + p.right + 1);
    for (int64_t j = sp.x; j < min((int64_t)sp.x + p.sinks, lo); ++j)
        if (p.spans[j].y > p.spans[j].x) f(j);
    for (int64_t j = lo; j < hi; ++j)
        if (p.spans[j].y > p.spans[j].x) f(j);
}

template <typename T>
__global__ void attend_kernel(AttendParams p)
{
    const uint32_t lane = threadIdx.x & 31, h = blockIdx.y, kvh = h / (p.heads / p.kv_heads);
    const int64_t i = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    if (i >= p.n) return;
    float q[4], acc[4] = {0.f, 0.f, 0.f, 0.f};
    row_read(q, static_cast<const T *>(p.q) + i * p.ldq + h * p.dim, p.dim, lane);
    float top = -INFINITY, sum = 0.f;
    each_key(p, i, [&](int64_t j) {
        float k[4], v[4];
        row_read(k, static_cast<const T *>(p.k) + j * p.ldk + kvh * p.dim, p.dim, lane);
        row_read(v, static_cast<const T *>(p.v) + j * p.ldv + kvh * p.dim, p.dim, lane);
        float s = row_dot(q, k) * p.scale;
        if (p.b.n) s += p.bias[(size_t)bucket_of(p.b, (int32_t)(j - i)) * p.heads + h];
        s = log2_score(s);
        const float m = fmaxf(top, s), from = m == -INFINITY ? 0.f : m, keep = exp2f(top - from), w = exp2f(s - from);
        top = m;
        sum = sum * keep + w;
        for (int e = 0; e < 4; ++e) acc[e] = acc[e] * keep + w * v[e];
    });
    for (int e = 0; e < 4; ++e) acc[e] = sum > 0.f ? acc[e] / sum : 0.f;
    row_write(static_cast<T *>(p.out) + i * p.ldo + h * p.dim, acc, p.dim, lane);
    if (p.out_full) row_write(p.out_full + (i * p.heads + h) * p.dim, acc, p.dim, lane);
    if (p.lse && lane == 0) p.lse[(int64_t)h * p.n + i] = sum > 0.f ? top + log2f(sum) : INFINITY;
}

// dQ, delta and the bias' gradient: one block per (128 queries, head).
template <typename T>
__global__ void attend_dq_kernel(AttendParams p)
{
    __shared__ float db[4][kMaxBuckets];
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, h = blockIdx.y, kvh = h / (p.heads / p.kv_heads);
    for (uint32_t b = lane; b < kMaxBuckets; b += 32) db[warp][b] = 0.f;
    __syncwarp();
    const uint32_t buckets = p.b.n * (p.b.two_sided ? 2 : 1);
    for (int r = warp; r < kAttendTile; r += 4) {
        const int64_t i = (int64_t)blockIdx.x * kAttendTile + r;
        if (i >= p.n) break;
        float q[4], o[4], go[4], dq[4] = {0.f, 0.f, 0.f, 0.f};
        row_read(q, static_cast<const T *>(p.q) + i * p.ldq + h * p.dim, p.dim, lane);
        if (p.o_full) row_read(o, p.o_full + (i * p.heads + h) * p.dim, p.dim, lane);
        else row_read(o, static_cast<const T *>(p.o) + i * p.ldo + h * p.dim, p.dim, lane);
        row_read(go, static_cast<const T *>(p.d_o) + i * p.ld_do + h * p.dim, p.dim, lane);
        const float delta = row_dot(o, go), lse = p.lse[(int64_t)h * p.n + i];
        if (lane == 0) p.delta[(int64_t)h * p.n + i] = delta;
        each_key(p, i, [&](int64_t j) {
            float k[4], v[4];
            row_read(k, static_cast<const T *>(p.k) + j * p.ldk + kvh * p.dim, p.dim, lane);
            row_read(v, static_cast<const T *>(p.v) + j * p.ldv + kvh * p.dim, p.dim, lane);
            float s = row_dot(q, k) * p.scale;
            uint32_t b = 0;
            if (p.b.n) { b = bucket_of(p.b, (int32_t)(j - i)); s += p.bias[(size_t)b * p.heads + h]; }
            const float ds = exp2f(log2_score(s) - lse) * (row_dot(go, v) - delta);
            if (p.b.n && lane == 0) db[warp][b] += ds;
            for (int e = 0; e < 4; ++e) dq[e] += ds * p.scale * k[e];
        });
        row_write(static_cast<T *>(p.dq) + i * p.ld_dq + h * p.dim, dq, p.dim, lane);
    }
    __syncthreads();
    if (p.dbias_part && threadIdx.x < buckets)
        p.dbias_part[((size_t)blockIdx.x * p.heads + h) * buckets + threadIdx.x] =
            db[0][threadIdx.x] + db[1][threadIdx.x] + db[2][threadIdx.x] + db[3][threadIdx.x];
}

template <typename T>
__global__ void attend_dkv_kernel(AttendParams p)
{
    const uint32_t lane = threadIdx.x & 31, kvh = blockIdx.y, group = p.heads / p.kv_heads;
    const int64_t j = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
    if (j >= p.n) return;
    const int2 sp = p.spans[j];
    float k[4], v[4], dk[4] = {0.f, 0.f, 0.f, 0.f}, dv[4] = {0.f, 0.f, 0.f, 0.f};
    row_read(k, static_cast<const T *>(p.k) + j * p.ldk + kvh * p.dim, p.dim, lane);
    row_read(v, static_cast<const T *>(p.v) + j * p.ldv + kvh * p.dim, p.dim, lane);
    if (sp.y > sp.x) {
        const int64_t lo = max((int64_t)sp.x, j - p.right);
        const int64_t hi = j - sp.x < p.sinks ? sp.y : min((int64_t)sp.y, j + p.left + 1);
        for (int64_t i = lo; i < hi; ++i) {
            const int2 si = p.spans[i];
            if (si.y <= si.x) continue;
            for (uint32_t h = kvh * group; h < (kvh + 1) * group; ++h) {
                float q[4], go[4];
                row_read(q, static_cast<const T *>(p.q) + i * p.ldq + h * p.dim, p.dim, lane);
                row_read(go, static_cast<const T *>(p.d_o) + i * p.ld_do + h * p.dim, p.dim, lane);
                float s = row_dot(q, k) * p.scale;
                if (p.b.n) s += p.bias[(size_t)bucket_of(p.b, (int32_t)(j - i)) * p.heads + h];
                const float w = exp2f(log2_score(s) - p.lse[(int64_t)h * p.n + i]);
                const float ds = w * (row_dot(go, v) - p.delta[(int64_t)h * p.n + i]) * p.scale;
                for (int e = 0; e < 4; ++e) { dv[e] += w * go[e]; dk[e] += ds * q[e]; }
            }
        }
    }
    row_write(static_cast<T *>(p.dk) + j * p.ld_dk + kvh * p.dim, dk, p.dim, lane);
    row_write(static_cast<T *>(p.dv) + j * p.ld_dv + kvh * p.dim, dv, p.dim, lane);
}

__global__ void attend_dbias_kernel(const float *part, uint64_t tiles, uint32_t columns, uint32_t heads, uint32_t buckets, float *dbias)
{
    __shared__ float t[8];
    const uint32_t c = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    float a = 0.f;
    for (uint64_t r = threadIdx.x; r < tiles; r += blockDim.x) a += part[r * columns + c];
    a = warp_sum(a);
    if (lane == 0) t[warp] = a;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 8; ++w) a += t[w];
        dbias[(c % buckets) * heads + c / buckets] = a;
    }
}

int launch_attend(const AttendParams &p, uint32_t type, int *, int, cudaStream_t s)
{
    if (p.n == 0) return 0;
    const dim3 grid((uint32_t)((p.n + 3) / 4), p.heads);
    if (type == kBF16) attend_kernel<__nv_bfloat16><<<grid, 128, 0, s>>>(p);
    else attend_kernel<__half><<<grid, 128, 0, s>>>(p);
    return cudaPeekAtLastError() == cudaSuccess ? 1 : -1;
}

uint64_t attend_backward_ws(const AttendParams &p, bool want_dbias)
{
    const uint64_t tiles = ((uint64_t)p.n + kAttendTile - 1) / kAttendTile;
    return 4 * (uint64_t)p.n * p.heads + (want_dbias ? 4 * tiles * p.heads * p.b.n * 2 : 0) + 256;
}

int launch_attend_backward(AttendParams &p, uint32_t type, unsigned char *ws, int *, int, cudaStream_t s)
{
    const uint32_t buckets = p.b.n * (p.b.two_sided ? 2 : 1);
    const uint32_t tiles = (uint32_t)((p.n + kAttendTile - 1) / kAttendTile);
    int k = 0;
    if (p.n) {
        p.delta = reinterpret_cast<float *>(ws);
        p.dbias_part = p.dbias ? p.delta + (uint64_t)p.n * p.heads : nullptr;
        const dim3 gq(tiles, p.heads), gk((uint32_t)((p.n + 3) / 4), p.kv_heads);
        if (type == kBF16) {
            attend_dq_kernel<__nv_bfloat16><<<gq, 128, 0, s>>>(p);
            attend_dkv_kernel<__nv_bfloat16><<<gk, 128, 0, s>>>(p);
        } else {
            attend_dq_kernel<__half><<<gq, 128, 0, s>>>(p);
            attend_dkv_kernel<__half><<<gk, 128, 0, s>>>(p);
        }
        k = 2;
    }
    if (p.dbias) {
        attend_dbias_kernel<<<p.heads * buckets, 256, 0, s>>>(p.dbias_part, tiles, p.heads * buckets, p.heads, buckets, p.dbias);
        ++k;
    }
    return cudaPeekAtLastError() == cudaSuccess ? k : -1;
}

}  // namespace w2v
