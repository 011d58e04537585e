// Tables held in 4 bits with group scales, and the product of a few vectors with a whole table.
//
// Layout: row r is 16 ceil(d/32) bytes; byte b holds columns 2b (low half) and 2b + 1 (high half) as
// value + 8; columns past d hold value 0.  Group g of `group` columns has one bf16 scale (bf16 for its
// range: trained vectors are of the order 1e-3 to 1, a sum of squares less); scales are [rows][ceil(d/group)].
#include "w2v_device.cuh"
#include "w2v_reader.h"
#include "w2v_kernel_ready.h"
#include "w2v_tc.cuh"
#include "w2v_types.cuh"

namespace w2v {

// One warp per row: lane l reads columns l, l + 32, ... of a group; scale = max |x| / 7 rounded to bf16,
// value = x / scale rounded to the nearest whole number (ties to even) and held to -7..7.  One pass over the rows, but bound by
// latency: a group's loads, its maximum over the lanes, a division and the store follow one another.  4,000,001 rows of 300 out of
// a padded table: 8.1 ms with groups of 32 (0.11 of measured copy), 3.6 ms with groups of 128 (0.24).
__global__ void __launch_bounds__(256)
fourbit_pack_kernel(const float *rows, uint64_t n, uint32_t d, uint64_t ld, uint32_t group, unsigned char *packed, __nv_bfloat16 *scales)
{
    const uint32_t lane = threadIdx.x & 31, groups = (d + group - 1) / group;
    const uint64_t warps = (uint64_t)gridDim.x * (blockDim.x >> 5);
    const uint64_t row_bytes = 16ull * ((d + 31) / 32);
    for (uint64_t r = (uint64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5); r < n; r += warps)
        for (uint32_t g = 0; g < groups; ++g) {
            float x[4], top = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t c = g * group + i * 32 + lane;
                x[i] = i * 32u < group && c < d ? rows[r * ld + c] : 0.f;
                top = fmaxf(top, fabsf(x[i]));
            }
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(kFullMask, top, o));
            const __nv_bfloat16 sb = __float2bfloat16_rn(top / 7.0f);
            const float scale = __bfloat162float(sb);
            if (lane == 0) scales[r * groups + g] = sb;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t c0 = g * group + i * 32;
                if (i * 32u < group && c0 < (uint32_t)(2 * row_bytes)) {
                    const float v = scale > 0.f ? fminf(7.f, fmaxf(-7.f, rintf(x[i] / scale))) : 0.f;
                    const int nib = (int)v + 8;
                    const int other = __shfl_down_sync(kFullMask, nib, 1);
                    if (!(lane & 1)) packed[r * row_bytes + (c0 + lane) / 2] = (unsigned char)(nib | (other << 4));
                }
            }
        }
}

int launch_fourbit_pack(const float *rows, uint64_t n, uint32_t d, uint64_t ld, uint32_t group, unsigned char *packed,
                        void *scales, int sms, cudaStream_t s)
{
    if (n == 0) return 0;
    const uint64_t want = (n + 7) / 8, most = (uint64_t)sms * 8;
    fourbit_pack_kernel<<<(uint32_t)(want < most ? want : most), 256, 0, s>>>(rows, n, d, ld, group, packed,
                                                                          static_cast<__nv_bfloat16 *>(scales));
    return cudaPeekAtLastError() == cudaSuccess ? 1 : -1;
}

// out[v][r] = sum over the groups of scale times the sum of value x.
//
// Bound by reading the table, 0.56 bytes a column (d = 300, group 32); at the copy rate that leaves an SM some three
// thread instructions per column, which unpacking, converting and multiplying one column at a time exceeds.  So the
// products run on the matrix units: the values are whole numbers and exact in fp16, and every x, after its vector has
// been scaled by a power of two, is the sum of two fp16 numbers (what is lost is below 2^-22 of it, less than fp32
// sums lose over a row, and below 2^-40 of the vector's largest where x is less than 2^-18 of that); they take two of the
// eight columns of the B side, four vectors per mma.  The fp32 sums of a group are scaled and added to the row's.  Unpacking a
// word of 8 values costs 9 instructions: fields of 4 bits are put under the exponent of 1024 (fp16 1024 + n, or 1024 + 16 n) and
// brought to n - 8 by one exact operation a pair, as Kim, Henry, Fahim and Hassan Awadalla describe for integer weights ("Who
// Says Elephants Can't Run", 2022).
// Which column lands in which k is free as long as both sides agree, so a thread's word is used as it lies in memory
// and x is arranged to match, once per block.
//
// Rows are too short and too many for direct loads (8 rows a request, 16 bytes each: the L1's tag rate bounds
// them).  Each warp copies units of up to kQWords words of its 32 rows to shared memory in the background, 512
// contiguous bytes a request, one unit ahead of the one it works on, and reads them as matrices of 8 rows x 16 bytes.
// The rows' pitch there is odd in units of 16 bytes: no bank conflicts.
//
// 4,000,001 rows of 300, 4 vectors: 193 us, 4.0 TB/s = 0.63 of measured copy; what is left is the unpacking's instructions (one
// logic operation per pair of fields instead of two: 202 -> 193 us).  Kernel alone: 164 us for 1 to 4 vectors, 255 us for 5 to 8.
constexpr int kQWords = 10;             // most words of 32 columns per unit
constexpr int kQFragBytes = 64 * 1024;  // most shared memory for the B side; longer rows are taken in pieces
constexpr int kQWarps = 8;
constexpr uint32_t kQRows = 32;         // rows of a warp's tile: two A sides share one reading of the B side

// c = a b (first) or c += a b.
__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint2 b, bool first)
{
    if (first)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
                     : "=f"(c[0]), "=f"(c[1]), "=f"(c[2]), "=f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b.x), "r"(b.y), "f"(0.f));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                     : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                     : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b.x), "r"(b.y));
}

// Fields i and i + 4 (i = 0..3) of a word as four registers of two fp16 numbers, 8 taken off.
__device__ __forceinline__ void unpack8(uint32_t w, uint32_t (&h)[4])
{
    const uint32_t u = w >> 8;
    const __half2 off = __floats2half2_rn(-1032.f, -1032.f), by = __floats2half2_rn(0.0625f, 0.0625f), off16 = __floats2half2_rn(-72.f, -72.f);
    uint32_t t[4];
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(t[0]) : "r"(w), "r"(0x000F000Fu), "r"(0x64006400u));      // (a & b) | c
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(t[1]) : "r"(w), "r"(0x00F000F0u), "r"(0x64006400u));
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(t[2]) : "r"(u), "r"(0x000F000Fu), "r"(0x64006400u));
    asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(t[3]) : "r"(u), "r"(0x00F000F0u), "r"(0x64006400u));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __half2 x = *reinterpret_cast<const __half2 *>(&t[i]);
        const __half2 y = i & 1 ? __hfma2(x, by, off16) : __hadd2(x, off);
        h[i] = *reinterpret_cast<const uint32_t *>(&y);
    }
}

// PER = words of 32 columns per group, NT = tiles of 4 vectors.
template <int NT, int PER>
__global__ void __launch_bounds__(kQWarps * 32, 2)
fourbit_scores_kernel(const float *x, uint32_t m, uint64_t ldx, const unsigned char *packed, const __nv_bfloat16 *scales,
                      uint64_t rows, uint32_t d, float *out, uint64_t ld_out, uint32_t piece, uint32_t unit)
{
    extern __shared__ __align__(16) unsigned char smem[];               // frag: [words of 32 columns][2][NT][lane]; then the warps' stages
    __shared__ uint32_t expo[8];                                        // exponent field of the power of two that scales each vector
    uint2 *frag = reinterpret_cast<uint2 *>(smem);
    const uint32_t tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
    const uint32_t words = (d + 31) / 32, groups = (words + PER - 1) / PER;
    const uint32_t pitch = unit | 1u, stage_bytes = kQRows * pitch * 16;
    unsigned char *mine = smem + piece * 512 * NT + warp * (2 * stage_bytes + kQRows * kQWords * 4);
    float *sc = reinterpret_cast<float *>(mine + 2 * stage_bytes) ;     // [group of the unit][row]: of the unit worked on
    const uint64_t tiles = (rows + kQRows - 1) / kQRows;
    if (warp < m) {
        float top = 0.f;
        for (uint32_t c = lane; c < d; c += 32) top = fmaxf(top, fabsf(__ldg(x + warp * ldx + c)));
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(kFullMask, top, o));
        const uint32_t e = __float_as_uint(top) >> 23;                  // the largest goes to [2^14, 2^15)
        if (lane == 0) expo[warp] = e == 255 ? 127u : e < 15 ? 253u : 268u - e;
    }
    __syncthreads();
    auto fill = [&](uint32_t w0, uint32_t n) {
        for (uint32_t e = tid; e < n * 2 * NT * 32; e += blockDim.x) {
            const uint32_t l = e & 31, nt = (e >> 5) % NT, j = ((e >> 5) / NT) & 1, w = (e >> 5) / (2 * NT);
            const uint32_t col = l >> 2, v = nt * 4 + (col >> 1);                   // column 2 v + part of a vector
            const uint32_t c0 = (w0 + w) * 32 + (l & 3) * 8 + 2 * j;
            float y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t c = c0 + (i & 1) * 4 + (i >> 1);                     // c0, c0 + 4, c0 + 1, c0 + 5
                y[i] = v < m && c < d ? __ldg(x + v * ldx + c) * __uint_as_float(expo[v] << 23) : 0.f;
                if (col & 1) y[i] -= __half2float(__float2half_rn(y[i]));
            }
            frag[e] = make_uint2(pack2<__half>(y[0], y[1]), pack2<__half>(y[2], y[3]));
        }
    };
    const bool once = piece >= words;
    // A unit: words [w, w + n) of the rows of a tile.  Which chunk of 16 bytes and which scales a lane copies is the same for
    // every full unit of a full tile.
    uint32_t from_off[kQWords], to_off[kQWords];
    const uint32_t ng_full = (unit + PER - 1) / PER;
#pragma unroll
    for (int i = 0; i < kQWords; ++i) {
        const uint32_t e = lane + i * 32, r = e / unit, c = e - r * unit;
        from_off[i] = (r * words + c) * 16;
        to_off[i] = (r * pitch + c) * 16;
    }
    uint16_t sreg[kQWords];                                             // scales of the unit under way
    const uint16_t *scale_bits = reinterpret_cast<const uint16_t *>(scales);
    auto fetch = [&](uint64_t tile, uint32_t w, uint32_t n, uint32_t stage) {
        const uint64_t r0 = tile * kQRows;
        const uint32_t dst = smem_addr(mine + stage * stage_bytes), gr = w / PER;
        if (n == unit && r0 + kQRows <= rows) {
            const unsigned char *src = packed + (r0 * words + w) * 16;
            const uint16_t *ss = scale_bits + (r0 + lane) * groups + gr;
#pragma unroll
            for (int i = 0; i < kQWords; ++i) {
                if ((uint32_t)i < unit) copy16(dst + to_off[i], src + from_off[i], true);
                if ((uint32_t)i < ng_full) sreg[i] = __ldg(ss + i);
            }
        } else {
            const uint32_t ng = (n + PER - 1) / PER;
#pragma unroll
            for (int i = 0; i < kQWords; ++i) {                         // rows past the end are read again, not written
                const uint32_t e = lane + i * 32, r = e / n, c = e - r * n;
                if (r < kQRows) copy16(dst + (r * pitch + c) * 16, packed + (min(r0 + r, rows - 1) * words + w + c) * 16, true);
                if ((uint32_t)i < ng) sreg[i] = __ldg(scale_bits + min(r0 + lane, rows - 1) * groups + gr + i);
            }
        }
        copy_commit();
    };
    if (once) {
        fill(0, words);
        __syncthreads();
    }
    const uint64_t stride = (uint64_t)gridDim.x * kQWarps;
    uint64_t tile = (uint64_t)blockIdx.x * kQWarps + warp;
    uint32_t stage = 0;
    if (once && tile < tiles) fetch(tile, 0, min(unit, words), 0);
    // with pieces every warp of a block makes the same number of rounds, since the block refills frag together
    for (; once ? tile < tiles : tile - warp < tiles; tile += stride) {
        float tot[2][NT][4], c[2][NT][4];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int e = 0; e < 4; ++e) tot[i][n][e] = 0.f;
        for (uint32_t w0 = 0; w0 < words; w0 += piece) {
            const uint32_t w_end = min(words, w0 + piece);
            if (!once) {
                __syncthreads();
                fill(w0, w_end - w0);
                __syncthreads();
                fetch(tile, w0, min(unit, w_end - w0), stage);
            }
            for (uint32_t w = w0; w < w_end; w += unit) {
                const uint32_t n = min(unit, w_end - w), ng = (n + PER - 1) / PER;
                unsigned char *st = mine + stage * stage_bytes;
#pragma unroll
                for (int i = 0; i < kQWords; ++i) if ((uint32_t)i < ng) sc[lane + i * 32] = __uint_as_float((uint32_t)sreg[i] << 16);
                const bool more = w + unit < w_end, cross = once && !more && tile + stride < tiles;
                if (more) fetch(tile, w + unit, min(unit, w_end - w - unit), stage ^ 1u);
                else if (cross) fetch(tile + stride, 0, min(unit, words), stage ^ 1u);
                if (more || cross) copy_wait<1>(); else copy_wait<0>();
                __syncwarp();
                uint32_t from = smem_addr(st) + lane * pitch * 16;
                const uint2 *f = frag + (size_t)(w - w0) * 2 * NT * 32 + lane;
                const float *sg = sc + g;
                #pragma unroll(PER == 1 ? 2 : 1)
                for (uint32_t a = 0; a < n; a += PER, sg += kQRows) {
#pragma unroll
                    for (int sub = 0; sub < PER; ++sub, from += 16, f += 2 * NT * 32) {
                        if (sub > 0 && a + sub >= n) break;                         // the last group of a row may be shorter
                        uint32_t q[4];
                        asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
                                     : "=r"(q[0]), "=r"(q[1]), "=r"(q[2]), "=r"(q[3]) : "r"(from) : "memory");
                        uint32_t h[4][4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) unpack8(q[i], h[i]);
#pragma unroll
                        for (int j = 0; j < 2; ++j)
#pragma unroll
                            for (int k = 0; k < NT; ++k) {
                                const uint2 b = f[(j * NT + k) * 32];
#pragma unroll
                                for (int i = 0; i < 2; ++i) {
                                    const uint32_t av[4] = {h[2 * i][2 * j], h[2 * i + 1][2 * j], h[2 * i][2 * j + 1], h[2 * i + 1][2 * j + 1]};
                                    mma_f16(c[i][k], av, b, sub == 0 && j == 0);
                                }
                            }
                    }
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float s0 = sg[i * 16], s1 = sg[i * 16 + 8];
#pragma unroll
                        for (int k = 0; k < NT; ++k) {
                            tot[i][k][0] = fmaf(s0, c[i][k][0], tot[i][k][0]);
                            tot[i][k][1] = fmaf(s0, c[i][k][1], tot[i][k][1]);
                            tot[i][k][2] = fmaf(s1, c[i][k][2], tot[i][k][2]);
                            tot[i][k][3] = fmaf(s1, c[i][k][3], tot[i][k][3]);
                        }
                    }
                }
                __syncwarp();                                           // the stage may be filled again
                stage ^= 1u;
            }
        }
        // thread t has both parts of vectors t, 4 + t
#pragma unroll
        for (int k = 0; k < NT; ++k)
            if ((uint32_t)(4 * k) + t < m) {
                const float back = __uint_as_float((254u - expo[4 * k + t]) << 23);
                float *o = out + (4 * k + t) * ld_out + tile * kQRows + g;
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (tile * kQRows + i * 8 + g < rows) o[i * 8] = (tot[i >> 1][k][2 * (i & 1)] + tot[i >> 1][k][2 * (i & 1) + 1]) * back;
            }
    }
}

template <int NT, int PER>
int launch_scores(const float *x, uint32_t m, uint64_t ldx, const unsigned char *packed, const __nv_bfloat16 *scales, uint64_t rows,
                  uint32_t d, float *out, uint64_t ld_out, int sms, cudaStream_t s)
{
    auto kernel = fourbit_scores_kernel<NT, PER>;
    const uint32_t words = (d + 31) / 32;
    // units of equal length, whole groups of at most kQWords words; pieces of whole units
    const uint32_t longest = kQWords / PER * PER, parts = (words + longest - 1) / longest;
    const uint32_t unit = ((words + parts - 1) / parts + PER - 1) / PER * PER;
    const uint32_t most = kQFragBytes / (512 * NT) / unit * unit, piece = words <= most ? words : most;
    const int smem = (int)(piece * 512 * NT + kQWarps * 2 * kQRows * (unit | 1u) * 16 + kQWarps * kQRows * kQWords * 4);
    if (smem > 48 * 1024 && !kernel_ready<fourbit_scores_kernel<NT, PER>>()) return -1;
    const uint64_t want = (rows + kQRows * kQWarps - 1) / (kQRows * kQWarps), full = (uint64_t)sms * (smem <= 112 * 1024 ? 2 : 1);
    kernel<<<(uint32_t)(want < full ? want : full), kQWarps * 32, smem, s>>>(x, m, ldx, packed, scales, rows, d, out, ld_out, piece, unit);
    return cudaPeekAtLastError() == cudaSuccess ? 1 : -1;
}

int launch_fourbit_scores(const float *x, uint32_t m, uint64_t ldx, const unsigned char *packed, const void *scales, uint64_t rows,
                          uint32_t d, uint32_t group, float *out, uint64_t ld_out, int sms, cudaStream_t s)
{
    if (rows == 0 || m == 0) return 0;
    const __nv_bfloat16 *sc = static_cast<const __nv_bfloat16 *>(scales);
#define W2V_SCORES(PER) (m <= 4 ? launch_scores<1, PER>(x, m, ldx, packed, sc, rows, d, out, ld_out, sms, s) \
                                : launch_scores<2, PER>(x, m, ldx, packed, sc, rows, d, out, ld_out, sms, s))
    return group == 32 ? W2V_SCORES(1) : group == 64 ? W2V_SCORES(2) : W2V_SCORES(4);
#undef W2V_SCORES
}

}  // namespace w2v
