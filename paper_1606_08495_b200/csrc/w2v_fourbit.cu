// Tables held in 4 bits with group scales, and the product of a few vectors with a whole table.
//
// Layout: row r is 16 ceil(d/32) bytes; byte b holds columns 2b (low half) and 2b + 1 (high half) as
// value + 8; columns past d hold value 0.  Group g of `group` columns has one bf16 scale (bf16 for its
// range: trained vectors are of the order 1e-3 to 1, a sum of squares less); scales are [rows][ceil(d/group)].
#include "w2v_device.cuh"
#include "w2v_reader.h"
#include "w2v_types.cuh"

namespace w2v {

// One warp per row: lane l reads columns l, l + 32, ... of a group; scale = max |x| / 7 rounded to bf16,
// value = x / scale rounded to the nearest whole number (ties to even) and held to -7..7.
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

// out[v][r] = sum over groups of scale times the group's products, in fp32.  One warp per row; a lane
// takes words of 8 columns.
template <int M>
__global__ void __launch_bounds__(256)
fourbit_scores_kernel(const float *x, uint32_t m, uint64_t ldx, const unsigned char *packed, const __nv_bfloat16 *scales,
                      uint64_t rows, uint32_t d, uint32_t group, float *out, uint64_t ld_out)
{
    const uint32_t lane = threadIdx.x & 31, groups = (d + group - 1) / group, words = 4 * ((d + 31) / 32);
    const uint64_t warps = (uint64_t)gridDim.x * (blockDim.x >> 5);
    for (uint64_t r = (uint64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5); r < rows; r += warps) {
        const uint32_t *w = reinterpret_cast<const uint32_t *>(packed) + r * words;
        float acc[M];
#pragma unroll
        for (int v = 0; v < M; ++v) acc[v] = 0.f;
        for (uint32_t k = lane; k < words; k += 32) {
            const uint32_t c0 = k * 8;
            if (c0 >= d) break;
            const uint32_t nib = w[k];
            const float scale = __bfloat162float(scales[r * groups + c0 / group]);
#pragma unroll
            for (int v = 0; v < M; ++v) {
                float a = 0.f;
                if ((uint32_t)v < m)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (c0 + e < d) a = fmaf((float)((int)((nib >> (4 * e)) & 15u) - 8), x[v * ldx + c0 + e], a);
                acc[v] = fmaf(a, scale, acc[v]);
            }
        }
#pragma unroll
        for (int v = 0; v < M; ++v) {
            const float a = warp_sum(acc[v]);
            if (lane == 0 && (uint32_t)v < m) out[v * ld_out + r] = a;
        }
    }
}

int launch_fourbit_scores(const float *x, uint32_t m, uint64_t ldx, const unsigned char *packed, const void *scales, uint64_t rows,
                          uint32_t d, uint32_t group, float *out, uint64_t ld_out, int sms, cudaStream_t s)
{
    if (rows == 0 || m == 0) return 0;
    const __nv_bfloat16 *sc = static_cast<const __nv_bfloat16 *>(scales);
    const uint64_t want = (rows + 7) / 8, most = (uint64_t)sms * 8;
    const uint32_t grid = (uint32_t)(want < most ? want : most);
    if (m <= 1) fourbit_scores_kernel<1><<<grid, 256, 0, s>>>(x, m, ldx, packed, sc, rows, d, group, out, ld_out);
    else if (m <= 2) fourbit_scores_kernel<2><<<grid, 256, 0, s>>>(x, m, ldx, packed, sc, rows, d, group, out, ld_out);
    else if (m <= 4) fourbit_scores_kernel<4><<<grid, 256, 0, s>>>(x, m, ldx, packed, sc, rows, d, group, out, ld_out);
    else fourbit_scores_kernel<8><<<grid, 256, 0, s>>>(x, m, ldx, packed, sc, rows, d, group, out, ld_out);
    return cudaPeekAtLastError() == cudaSuccess ? 1 : -1;
}

}  // namespace w2v
