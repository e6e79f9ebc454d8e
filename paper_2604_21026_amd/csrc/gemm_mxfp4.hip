// nvq_gemm_mxfp4: both operands microscaled 4-bit floating point, for prompts.  The matrix cores take codes and
// scales as they are: one 16x16x128 scaled MFMA multiplies four blocks of 16 rows with those of 16 tokens, lane
// (i, kb) = (lane % 16, lane / 16) holding the 16 bytes of codes of one block of row or token i and that block's scale
// byte.  Sums in fp32.
#include "mfma_act.h"

namespace nvq {

namespace {

typedef int int8v __attribute__((ext_vector_type(8)));

__device__ __forceinline__ int8v fp4_operand(const uint4v &c) {
    return int8v{(int)c.x, (int)c.y, (int)c.z, (int)c.w, 0, 0, 0, 0};
}

// A wave of 64 x 64 results: weights are the first operand, so that a lane's four registers of a 16x16 tile are
// four neighbouring rows (columns of y) of one token.
__global__ __launch_bounds__(64) void gemm_mxfp4_simple_kernel(const uint4 *__restrict__ wq,
                                                               const uint8_t *__restrict__ ws, int64_t N, int G,
                                                               const uint4 *__restrict__ xq,
                                                               const uint8_t *__restrict__ xs, int64_t M,
                                                               void *__restrict__ y, int y_dtype) {
    const int lane = threadIdx.x, i = lane & 15, kb = lane >> 4;
    const int64_t n0 = (int64_t)blockIdx.x * 64, m0 = (int64_t)blockIdx.y * 64;
    float4v sum[4][4] = {};
    int64_t wr[4], xr[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int64_t n = n0 + 16 * t + i, m = m0 + 16 * t + i;
        wr[t] = (n < N ? n : N - 1) * G;
        xr[t] = (m < M ? m : M - 1) * G;
    }
    for (int g0 = 0; g0 < G; g0 += 4) {
        const int g = g0 + kb;
        const bool in = g < G;
        uint4v a[4], b[4];
        int sa[4], sb[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            const int64_t at = in ? g : G - 1;
            a[t] = load_stream(wq + wr[t] + at);
            b[t] = load_stream(xq + xr[t] + at);
            sa[t] = ws[wr[t] + at];
            sb[t] = xs[xr[t] + at];
            if (!in) {
                a[t] = b[t] = uint4v{0, 0, 0, 0};
                sa[t] = sb[t] = 127;
            }
        }
#pragma unroll
        for (int p = 0; p < 4; ++p)
#pragma unroll
            for (int t = 0; t < 4; ++t)
                sum[p][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fp4_operand(a[p]), fp4_operand(b[t]), sum[p][t],
                                                                             4, 4, 0, sa[p], 0, sb[t]);
    }
#pragma unroll
    for (int p = 0; p < 4; ++p)
#pragma unroll
        for (int t = 0; t < 4; ++t) {
            asm volatile("s_nop 7\n\ts_nop 7" : "+v"(sum[p][t]));
            const int64_t m = m0 + 16 * t + i;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int64_t n = n0 + 16 * p + 4 * kb + j;
                if (m < M && n < N) store_global(y, y_dtype, m * N + n, sum[p][t][j]);
            }
        }
}

}  // namespace

}  // namespace nvq

extern "C" int nvq_gemm_mxfp4(const uint8_t *qweight, const uint8_t *scales, int64_t N, int64_t K, const uint8_t *xq,
                              const uint8_t *xscale, int64_t M, void *y, int y_dtype, void *stream) {
    using namespace nvq;
    if (!qweight || !scales || !xq || !xscale || !y || (y_dtype != NVQ_F32 && y_dtype != NVQ_BF16))
        return NVQ_ERR_INVALID_ARG;
    if (N <= 0 || M <= 0 || K <= 0 || K % 32 || K > NVQ_MAX_K || N > INT32_MAX || M > INT32_MAX) return NVQ_ERR_SHAPE;
    if (!aligned(qweight, 16) || !aligned(xq, 16) || !aligned(y, y_dtype == NVQ_F32 ? 4 : 2)) return NVQ_ERR_ALIGN;
    const dim3 grid((unsigned)((N + 63) / 64), (unsigned)((M + 63) / 64));
    hipLaunchKernelGGL(gemm_mxfp4_simple_kernel, grid, dim3(64), 0, (hipStream_t)stream,
                       reinterpret_cast<const uint4 *>(qweight), scales, N, (int)(K / 32),
                       reinterpret_cast<const uint4 *>(xq), xscale, M, y, y_dtype);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}
