// nvq_adapters_add: low-rank adapters beside a layer, each token its own.
//
// Two launches, h = A x and y + scale * B h, both on the matrix cores in tiles of sixteen tokens.  A tile goes through
// the distinct adapters of its tokens one after the other and keeps of each product the rows of that adapter's own
// tokens: an adapter's weights are read once per tile however many of its tokens use it, and sixteen tokens with
// sixteen adapters read what they have to.  h stays fp32 between the launches; it enters the second product as three
// bf16 values whose sum it is, so nothing of it is lost.
#include "mfma_act.h"

namespace nvq {

namespace {

constexpr int kTile = 16, kDownWaves = 4, kUpWaves = 4;

struct AdaptersArgs {
    const uint16_t *a, *b, *x;
    const float *scales;
    const int32_t *ids;
    const void *y;
    void *out;
    int dtype;
    int n, K, N, R, M;
    float *h;  // workspace, [M][R]
};

// The adapter of a lane's token (lane & 15 of a tile), -1: none.
__device__ __forceinline__ int adapter_of(const AdaptersArgs &g, int m0) {
    const int m = m0 + (threadIdx.x & 15);
    const int e = m < g.M ? g.ids[m] : -1;
    return (unsigned)e < (unsigned)g.n ? e : -1;
}

// The distinct adapters of a tile one after the other: `left` has a bit per token that has not had its turn.
__device__ __forceinline__ uint32_t turn(int mine, uint32_t *left, int *e) {
    const int first = __builtin_ctz(*left);
    *e = __builtin_amdgcn_readlane(mine, first);
    const uint32_t with = (uint32_t)__ballot(mine == *e) & 0xffffu;
    *left &= ~with;
    return with;
}

// h[m0 ..][r0 ..]: K split over the waves.
__global__ __launch_bounds__(64 * kDownWaves) void adapters_down_kernel(AdaptersArgs g) {
    __shared__ float red[kDownWaves][4][64];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, kb = lane >> 4;
    const int m0 = blockIdx.y * kTile, r0 = blockIdx.x * 16;
    const int mine = adapter_of(g, m0);
    uint32_t left = (uint32_t)__ballot(mine >= 0) & 0xffffu;
    const uint16_t *const x = g.x + (int64_t)(m0 + n < g.M ? m0 + n : m0) * g.K + 8 * kb;
    const int r = r0 + n < g.R ? r0 + n : g.R - 1;
    while (left) {
        int e;
        const uint32_t with = turn(mine, &left, &e);
        const uint16_t *const a = g.a + ((int64_t)e * g.R + r) * g.K + 8 * kb;
        float4v sum = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int c = w; c < g.K / 32; c += kDownWaves)
            sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, *as_global<uint4v>(x + 32 * c)),
                                                         __builtin_bit_cast(bf16x8, *as_global<uint4v>(a + 32 * c)), sum, 0, 0, 0);
        wait_written(sum);
        __syncthreads();
#pragma unroll
        for (int j = 0; j < 4; ++j) red[w][j][lane] = sum[j];
        __syncthreads();
        if (w == 0) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = 4 * kb + j;
                float v = red[0][j][lane];
#pragma unroll
                for (int k = 1; k < kDownWaves; ++k) v += red[k][j][lane];
                if ((with >> row & 1) && r0 + n < g.R) g.h[(int64_t)(m0 + row) * g.R + r0 + n] = v;
            }
        }
    }
}

// A value as three whose sum it is, each with eight bits (cut off, so that nothing grows to infinity).
__device__ __forceinline__ void split(float v, uint32_t *hi, uint32_t *mid, uint32_t *lo) {
    const uint32_t b = __float_as_uint(v) & 0xffff0000u;
    const float rest = __builtin_isfinite(v) ? v - __uint_as_float(b) : 0.0f;
    const uint32_t c = __float_as_uint(rest) & 0xffff0000u;
    *hi = b >> 16;
    *mid = c >> 16;
    *lo = __float_as_uint(rest - __uint_as_float(c)) >> 16;
}

// out[m0 ..][n0 ..], a wave per sixteen outputs.
__global__ __launch_bounds__(64 * kUpWaves) void adapters_up_kernel(AdaptersArgs g) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, n = lane & 15, kb = lane >> 4;
    const int m0 = blockIdx.y * kTile, n0 = (blockIdx.x * kUpWaves + w) * 16;
    const int mine = adapter_of(g, m0);
    uint32_t left = (uint32_t)__ballot(mine >= 0) & 0xffffu;
    const int o = n0 + n < g.N ? n0 + n : g.N - 1;
    const float *const h = g.h + (int64_t)(m0 + n < g.M ? m0 + n : m0) * g.R + 8 * kb;
    float add[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    while (left) {
        int e;
        const uint32_t with = turn(mine, &left, &e);
        const uint16_t *const b = g.b + ((int64_t)e * g.N + o) * g.R + 8 * kb;
        float4v sum = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int c = 0; c < g.R; c += 32) {
            uint4v hw[3] = {}, bw = {};
            if (c + 8 * kb < g.R) {
                bw = *as_global<uint4v>(b + c);
                if (with >> n & 1) {  // (what h holds of other tokens may be anything)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        uint32_t lo[3], hi[3];
                        split(h[c + 2 * j], &lo[0], &lo[1], &lo[2]);
                        split(h[c + 2 * j + 1], &hi[0], &hi[1], &hi[2]);
#pragma unroll
                        for (int k = 0; k < 3; ++k) hw[k][j] = lo[k] | hi[k] << 16;
                    }
                }
            }
#pragma unroll
            for (int k = 0; k < 3; ++k)
                sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, hw[k]), __builtin_bit_cast(bf16x8, bw), sum,
                                                             0, 0, 0);
        }
        wait_written(sum);
        const float scale = g.scales ? g.scales[e] : 1.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (with >> (4 * kb + j) & 1) add[j] = sum[j] * scale;
    }
    const uint32_t has = (uint32_t)__ballot(mine >= 0) & 0xffffu;
    if (n0 + n >= g.N) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int m = m0 + 4 * kb + j;
        if (m >= g.M) continue;
        const int64_t at = (int64_t)m * g.N + n0 + n;
        if (has >> (4 * kb + j) & 1) {
            const float y = g.dtype == NVQ_F32 ? static_cast<const float *>(g.y)[at]
                                               : bf16_bits_to_float(static_cast<const uint16_t *>(g.y)[at]);
            store_global(g.out, g.dtype, at, y + add[j]);
        } else if (g.out != g.y) {  // (as it is)
            if (g.dtype == NVQ_F32)
                static_cast<uint32_t *>(g.out)[at] = static_cast<const uint32_t *>(g.y)[at];
            else
                static_cast<uint16_t *>(g.out)[at] = static_cast<const uint16_t *>(g.y)[at];
        }
    }
}

bool adapters_shape(const nvq_adapters *s, int M) {
    return s && s->n >= 1 && s->n <= 1 << 16 && s->K >= 32 && s->K % 32 == 0 && s->K <= NVQ_MAX_K && s->N >= 1 && s->N <= 1 << 24 &&
           s->R >= 8 && s->R % 8 == 0 && s->R <= NVQ_MAX_RANK && M >= 1 && M <= 1 << 16;
}

}  // namespace

}  // namespace nvq

extern "C" size_t nvq_adapters_workspace_bytes(const nvq_adapters *adapters, int M) {
    using namespace nvq;
    return adapters_shape(adapters, M) ? (size_t)M * adapters->R * sizeof(float) : 0;
}

extern "C" int nvq_adapters_add(const nvq_adapters *adapters, const uint16_t *x_bf16, const int32_t *ids, int M, const void *y,
                                void *out, int dtype, void *workspace, size_t workspace_bytes, void *stream) {
    using namespace nvq;
    if (!adapters || !adapters->a || !adapters->b || !x_bf16 || !ids || !y || !out || (dtype != NVQ_F32 && dtype != NVQ_BF16))
        return NVQ_ERR_INVALID_ARG;
    if (!adapters_shape(adapters, M)) return NVQ_ERR_SHAPE;
    if (!aligned(adapters->a, 16) || !aligned(adapters->b, 16) || !aligned(adapters->scales, 4) || !aligned(x_bf16, 16) ||
        !aligned(ids, 4) || !aligned(y, 16) || !aligned(out, 16))
        return NVQ_ERR_ALIGN;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < nvq_adapters_workspace_bytes(adapters, M))
        return NVQ_ERR_WORKSPACE;
    AdaptersArgs g;
    g.a = adapters->a;
    g.b = adapters->b;
    g.scales = adapters->scales;
    g.x = x_bf16;
    g.ids = ids;
    g.y = y;
    g.out = out;
    g.dtype = dtype;
    g.n = adapters->n;
    g.K = adapters->K;
    g.N = adapters->N;
    g.R = adapters->R;
    g.M = M;
    g.h = static_cast<float *>(workspace);
    const hipStream_t st = (hipStream_t)stream;
    const unsigned tiles = (unsigned)((M + kTile - 1) / kTile);
    hipLaunchKernelGGL(adapters_down_kernel, dim3((unsigned)((g.R + 15) / 16), tiles), dim3(64 * kDownWaves), 0, st, g);
    NVQ_HIP_TRY(hipGetLastError());
    hipLaunchKernelGGL(adapters_up_kernel, dim3((unsigned)((g.N + 16 * kUpWaves - 1) / (16 * kUpWaves)), tiles), dim3(64 * kUpWaves), 0, st,
                       g);
    NVQ_HIP_TRY(hipGetLastError());
    return NVQ_OK;
}
