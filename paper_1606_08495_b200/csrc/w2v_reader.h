// Internal declarations of the reader operators (layer norm, windowed attention, 4-bit table
// products): parameter blocks and launchers.  Every launcher returns the number of kernels it
// launched, or -1 after a launch error.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace w2v {

// Element types as the C ABI numbers them (W2V_F32 and so on).
enum : uint32_t { kF32 = 0, kBF16 = 1, kF16 = 2 };
inline uint32_t type_size(uint32_t t) { return t == kF32 ? 4u : 2u; }

// ---- layer norm (w2v_norm.cu) ----
struct NormParams {
    const void *x, *dy;
    void *y, *dx;
    const float *gamma, *beta;
    float *mean, *rstd;             // forward: written; backward: read
    float *part;                    // backward: [blocks][2][d] partial sums of the weights' gradients
    uint64_t rows, ldx, ldy, ld_dx; // strides in elements
    uint32_t d;
    float eps;
};
constexpr uint32_t kNormMaxD = 8192;
// Blocks of the backward kernel (and so rows of `part`).
uint32_t norm_backward_blocks(uint64_t rows, uint32_t d, int sms);
constexpr int kErrRing = 16;            // bit of the handle's error word: a ring of rows gave up waiting
int launch_norm(const NormParams &p, uint32_t x_type, uint32_t y_type, int *error, int sms, cudaStream_t s);
int launch_norm_backward(const NormParams &p, uint32_t x_type, uint32_t y_type, float *dgamma, float *dbeta,
                         uint32_t blocks, int *error, int sms, cudaStream_t s);

// ---- attention over a window of the sentence (w2v_attend*.cu) ----
constexpr uint32_t kMaxBuckets = 64, kMaxReach = 1024, kMaxSinks = 64, kMaxHeadDim = 128;

// First distance of every bucket of one side.
struct BucketStarts {
    uint32_t n;                     // buckets of a side, 0 = no bias
    uint32_t two_sided;
    int32_t start[kMaxBuckets];
};

struct AttendParams {
    const int2 *spans;              // [n] first position of the sentence, one past its last; empty = the row sees nothing
    const void *q, *k, *v, *o, *d_o;
    void *out, *dq, *dk, *dv;
    const float *bias;              // [buckets][heads]
    float *lse;                     // [heads][n] base-2 logarithm of the softmax sum (scores scaled by log2 e), +inf for an empty row
    float *delta;                   // [heads][n] backward: rowsum(dO o)
    float *extra;                   // [heads][n] backward: base-2 logarithm of what a row's weights sum to with lse as it is, for far rows; else 0
    float *dbias, *dbias_part;      // [buckets][heads]; [key tiles, then query tiles with sinks][heads][buckets]
    float *sink_part;               // [query tiles][heads][sinks][dk, dv][dim] sums over one query tile
    int32_t *sink_rec;              // [query tiles] start of the sentence that reaches into the tile, -1: no word, -2: none
    int32_t *sink_used;             // [query tiles] start of the sentence whose sums lie in the slot, -1: none
    float *sink_sum;                // [query tiles][kv heads][sinks][dk, dv][dim]
    uint64_t ldq, ldk, ldv, ldo, ld_do, ld_dq, ld_dk, ld_dv;   // elements between tokens
    int64_t n;
    uint32_t heads, kv_heads, dim;
    int32_t left, right, sinks;
    float scale;
    BucketStarts b;
};
constexpr int kAttendTile = 128;    // queries of a tile

int launch_spans(const int32_t *tokens, uint64_t n, uint32_t vocab, int32_t *tile_ends, int2 *spans, cudaStream_t s);
uint64_t spans_tiles(uint64_t n);   // tile_ends holds two int32 per tile
int launch_attend(const AttendParams &p, uint32_t type, int *error, int sms, cudaStream_t s);
uint64_t attend_backward_ws(const AttendParams &p, bool want_dbias);       // bytes of scratch
int launch_attend_backward(AttendParams &p, uint32_t type, unsigned char *ws, int *error, int sms, cudaStream_t s);

// ---- one new token per sequence over a ring cache (w2v_attend_token.cu) ----
struct TokenParams {
    const void *q, *k, *v;          // [batch][heads][dim], [batch][kv][dim] twice
    void *ck, *cv;                  // [batch][places][kv][dim]
    void *out;                      // [batch][heads][dim]
    const int32_t *pos;             // [batch] position of the new token, negative = nothing there
    const float *bias;
    uint64_t places;
    uint32_t batch, heads, kv_heads, dim;
    int32_t left, sinks;
    float scale;
    BucketStarts b;
};
int launch_attend_token(const TokenParams &p, uint32_t type, int sms, cudaStream_t s);

// ---- tables in 4 bits (w2v_fourbit.cu) ----
int launch_fourbit_pack(const float *rows, uint64_t n, uint32_t d, uint64_t ld, uint32_t group, unsigned char *packed,
                        void *scales, int sms, cudaStream_t s);
int launch_fourbit_scores(const float *x, uint32_t m, uint64_t ldx, const unsigned char *packed, const void *scales, uint64_t rows,
                          uint32_t d, uint32_t group, float *out, uint64_t ld_out, int sms, cudaStream_t s);

}  // namespace w2v
