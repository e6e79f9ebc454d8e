// nvq_gemv_mxfp4: microscaled 4-bit weights times the bf16 activations of 1 to 32 tokens.  y[m][n] = sum over the
// blocks g of 2^(scale - 127) * sum_j code[n][32g + j] * x[m][32g + j], weights and activations unrounded, sums in
// fp32.
//
// Bound by reading the weights once (17 bits per 32 of them... see mx_rows.h for the product): a workgroup owns 16 * R
// rows, its W waves take the columns of 128 inputs in turn, and the partial tiles are added through LDS in wave
// order.
#include "mx_rows.h"

namespace nvq {

namespace {

template <int R, int T, int W, int B>
__global__ __launch_bounds__(64 * W) void gemv_mxfp4_kernel(const uint8_t *__restrict__ q,
                                                            const uint8_t *__restrict__ scales, int N, int G,
                                                            const uint16_t *__restrict__ x, int M,
                                                            void *__restrict__ y, int y_dtype) {
    __shared__ float red[W][R * T * 4][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int n = lane & 15, kb = lane >> 4;
    const int row0 = blockIdx.x * (16 * R);

    RowAt at[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const int row = row0 + 16 * r + n;  // (rows past the end read the last one, their results go nowhere)
        at[r] = row_at<NVQ_FMT_MXFP4>(q, scales, row < N ? row : N - 1, G);
    }
    const char *xt[T];
#pragma unroll
    for (int t = 0; t < T; ++t) {
        const int m = 16 * t + n;  // (tokens past the end read token 0: a product keeps tokens apart)
        xt[t] = reinterpret_cast<const char *>(x) + (size_t)(m < M ? m : 0) * G * 64 + kb * 16;
    }
    float4v sum[R][T];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < T; ++t) sum[r][t] = float4v{0.0f, 0.0f, 0.0f, 0.0f};
    rows_times_tokens<NVQ_FMT_MXFP4, R, T, B>(at, xt, G, w, W, sum);
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int t = 0; t < T; ++t)
#pragma unroll
            for (int j = 0; j < 4; ++j) red[w][(r * T + t) * 4 + j][lane] = sum[r][t][j];
    __syncthreads();
    // result i: lane-position i % 64 of register i / 64
    for (int i = threadIdx.x; i < R * T * 4 * 64; i += 64 * W) {
        const int reg = i >> 6, l = i & 63;
        const int t = (reg >> 2) % T, r = (reg >> 2) / T;
        const int m = 16 * t + 4 * (l >> 4) + (reg & 3), row = row0 + 16 * r + (l & 15);
        float v = red[0][reg][l];
#pragma unroll
        for (int k = 1; k < W; ++k) v += red[k][reg][l];
        if (m < M && row < N) store_global(y, y_dtype, (int64_t)m * N + row, v);
    }
}

}  // namespace

}  // namespace nvq

extern "C" int nvq_gemv_mxfp4(const uint8_t *qweight, const uint8_t *scales, int N, int K, const uint16_t *x_bf16,
                              int M, void *y, int y_dtype, void *stream) {
    using namespace nvq;
    if (!qweight || !scales || !x_bf16 || !y || (y_dtype != NVQ_F32 && y_dtype != NVQ_BF16))
        return NVQ_ERR_INVALID_ARG;
    if (N <= 0 || M < 1 || M > NVQ_MAX_M || K <= 0 || K % 32 || K > NVQ_MAX_K) return NVQ_ERR_SHAPE;
    if (!aligned(qweight, 16) || !aligned(x_bf16, 16) || !aligned(y, y_dtype == NVQ_F32 ? 4 : 2)) return NVQ_ERR_ALIGN;
    const hipStream_t st = (hipStream_t)stream;
    constexpr int R = 1, W = 4, B = 4;
    const dim3 grid((unsigned)(((int64_t)N + 16 * R - 1) / (16 * R))), block(64 * W);
    if (M <= 16)
        hipLaunchKernelGGL((gemv_mxfp4_kernel<R, 1, W, B>), grid, block, 0, st, qweight, scales, N, K / 32, x_bf16, M, y,
                           y_dtype);
    else
        hipLaunchKernelGGL((gemv_mxfp4_kernel<R, 2, W, B>), grid, block, 0, st, qweight, scales, N, K / 32, x_bf16, M, y,
                           y_dtype);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}
