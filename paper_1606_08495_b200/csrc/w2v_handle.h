// The handle behind the C ABI and the helpers that every file of entry points shares: error texts,
// the device guard, scratch that only grows.
#pragma once
#include <cstdio>
#include <vector>

#include "../../include/w2v.h"
#include "w2v_internal.h"

struct w2v_handle {
    uint64_t vocab = 0;
    uint32_t d = 0;
    uint32_t ld = 0;                 // row stride of U and V in floats (>= d, a multiple of 4)
    uint32_t d_full = 0;             // columns of the whole vectors (== d unless this is a column shard)
    uint32_t col_lo = 0;             // first column held (0 unless this is a column shard)
    bool is_shard = false;
    // state between w2v_shard_dots and w2v_shard_adjust
    bool shard_pending = false;
    int32_t *l_centre = nullptr, *l_context = nullptr, *l_negs = nullptr;   // pair list of a narrow shard's step
    uint64_t l_cap_pairs = 0, l_cap_context = 0, l_cap_negs = 0;
    float *inv_norm = nullptr; uint64_t inv_norm_cap = 0;                      // retrieval scratch
    float *part_cos = nullptr; long long *part_ids = nullptr; uint64_t part_cap = 0;
    uint32_t retrieval_kernel = 2;       // 0: fp32 on the CUDA cores, 1: tensor cores (3 x TF32), 2: tensor-core screen + exact fp32, 3: the screen on pairs of SMs
    int *tc_error = nullptr;             // device word raised by a tensor-core block whose wait ran out
    unsigned char *qsplit = nullptr; uint64_t qsplit_cap = 0;   // query rows split into TF32 head and tail
    unsigned char *ctiles = nullptr; uint64_t ctiles_cap = 0;   // candidate rows packed as bf16 operand blocks (screening kernel)
    unsigned int *floor_q = nullptr; uint64_t floor_cap = 0;    // per query: best K-th cosine reached by any block (screening kernel)
    uint32_t pend_window = 0, pend_negatives = 0;
    uint64_t pend_n = 0, pend_pairs = 0;
    uint64_t seed = 0;
    uint64_t step_id = 0;
    uint32_t il_phase = 0, il_stride = 1;   // interleaved minibatches: which tokens are input words
    int device = 0;
    int sms = 148;
    cudaStream_t stream = nullptr;
    float *U = nullptr, *V = nullptr;
    bool owns_tables = false;
    // sampling tables
    uint32_t *keep_thr = nullptr;
    uint2 *alias = nullptr;
    bool have_tables = false;
    // scratch
    w2v::Scratch sc;
    w2v::DevState *st = nullptr;          // device
    w2v::DevState *st_host = nullptr;     // pinned mirror
    float *G = nullptr;
    uint64_t G_cap = 0;
    float *DU = nullptr;
    uint64_t DU_cap = 0;             // floats
    double *DV = nullptr;            // fp64 sums for the most-hit output rows (snapshot mode), kept zero between steps
    uint64_t DV_cap = 0;             // doubles
    uint32_t hot_rows = 0;
    int32_t *tok_stage = nullptr;
    uint64_t tok_stage_cap = 0;
    unsigned char *reader_ws = nullptr; uint64_t reader_ws_cap = 0;   // scratch of the reader operators (sums of gradients, split caches)
    // tuning / accounting
    uint32_t rows_in_flight = 0, blocks_per_sm = 0;
    uint64_t launches = 0;
    bool profiling = false;
    std::vector<cudaEvent_t> ev;     // pairs (start, stop)
    size_t ev_used = 0;
    double prof_ms = 0.0;
    uint64_t prof_launches = 0;
    char err[256] = "no error";
};

namespace w2v {

inline int32_t fail(w2v_handle *h, int32_t code, const char *what, cudaError_t ce = cudaSuccess)
{
    if (h) {
        if (ce != cudaSuccess)
            std::snprintf(h->err, sizeof(h->err), "%s: %s", what, cudaGetErrorString(ce));
        else
            std::snprintf(h->err, sizeof(h->err), "%s", what);
    }
    return code;
}

#define W2V_CUDA(h, call)                                                     \
    do {                                                                      \
        cudaError_t ce_ = (call);                                             \
        if (ce_ != cudaSuccess)                                               \
            return fail(h, ce_ == cudaErrorMemoryAllocation ? W2V_ERR_NOMEM : W2V_ERR_CUDA, #call, ce_); \
    } while (0)

struct DeviceGuard {
    int prev = -1;
    explicit DeviceGuard(int dev) { cudaGetDevice(&prev); if (prev != dev) cudaSetDevice(dev); else prev = -1; }
    ~DeviceGuard() { if (prev >= 0) cudaSetDevice(prev); }
};

template <typename T>
cudaError_t dev_alloc(T **p, uint64_t count)
{
    return cudaMalloc(reinterpret_cast<void **>(p), (count ? count : 1) * sizeof(T));
}

// Makes *p hold at least `need` elements.  When it does not, the stream is drained (it may still
// use the old array), the array is freed and a new one allocated; with `slack`, a quarter more than
// asked for, so that chunks of slightly different sizes do not re-allocate every time.
template <typename T>
int32_t grow(w2v_handle *h, T **p, uint64_t *cap, uint64_t need, bool slack)
{
    if (need <= *cap) return W2V_OK;
    W2V_CUDA(h, cudaStreamSynchronize(h->stream));
    cudaFree(*p); *p = nullptr; *cap = 0;
    const uint64_t want = slack ? need + need / 4 + 1024 : need;
    W2V_CUDA(h, dev_alloc(p, want));
    *cap = want;
    return W2V_OK;
}

// The device word that kernels with bounded waits raise when a wait runs out (read by w2v_sync).
inline int32_t ensure_error_word(w2v_handle *h)
{
    if (h->tc_error) return W2V_OK;
    W2V_CUDA(h, dev_alloc(&h->tc_error, 1));
    W2V_CUDA(h, cudaMemsetAsync(h->tc_error, 0, sizeof(int), h->stream));
    return W2V_OK;
}

}  // namespace w2v
