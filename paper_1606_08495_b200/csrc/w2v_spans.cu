// Sentence bounds of a token stream.
#include "w2v_device.cuh"
#include "w2v_reader.h"

namespace w2v {

// spans[t] = (first position of t's sentence, one past its last); a separator or a word that the
// vocabulary does not have gets the empty span (t, t).  Two passes: the last and the first separator
// of every tile, then every tile looks back and ahead for the nearest tile that has one.  131,072 tokens: 5.8 and 4.5 us, the two launches' own time.
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
    if (tiles > 1) span_tiles_kernel<<<tiles, kSpanThreads, 0, s>>>(tokens, n, ends);       // a single tile looks at no other
    span_fill_kernel<<<tiles, kSpanThreads, 0, s>>>(tokens, n, vocab, ends, tiles, spans);
    return cudaPeekAtLastError() == cudaSuccess ? (tiles > 1 ? 2 : 1) : -1;
}

}  // namespace w2v
